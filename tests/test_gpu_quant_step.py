"""A decoder's attention block as the operators are used together: a fused q | k | v projection in binary bases
(fluxbin_lut_gemm_smallbatch) or in 4 bits, its rows into the cache as slices, attention, and the output projection in 4
bits; prompts of different lengths, then single tokens, eager and as a captured graph. Every stage is checked against
plain definitions on the inputs that it got."""
import numpy as np
import pytest

from oracle import quant_oracle as qo
from synth import LayerSpec, make_layer

from conftest import gpu_available
from gpu_util import log, pack_layer

pytestmark = pytest.mark.gpu

HIDDEN, HQ, H, D, P, B, BLOCKS = 512, 8, 2, 64, 32, 3, 5
WIDE = (HQ + 2 * H) * D


@pytest.fixture(scope="module", autouse=True)
def fb():
    if not gpu_available():
        pytest.skip("no GPU")
    from paper_2608_15602_amd import fluxbin
    fluxbin.lib()
    return fluxbin


class Block:
    def __init__(self, fb, binary):
        import torch
        self.fb, self.binary, self.torch = fb, binary, torch
        rng = np.random.default_rng(31)
        weight = lambda m, n: torch.from_numpy((rng.standard_normal((m, n)) / np.sqrt(n)).astype(np.float16)).cuda()
        self.q_w4 = [fb.fluxbin_w4_quantize(weight(*s), 64, values=True) for s in ((WIDE, HIDDEN), (HIDDEN, HQ * D))]
        self.w4 = [fb.fluxbin_w4_pack(*q[:3], n, 64) for q, n in zip(self.q_w4, (HIDDEN, HQ * D))]
        if binary:
            self.qkv = pack_layer(make_layer(LayerSpec("step", M=WIDE, N=HIDDEN, Kb=2, Ks=1, mu=8, S=20, g_r=128, g_s=20,
                                                       seed=32)))
        self.cache = fb.make_kv8_cache(B * BLOCKS + 2, P, H, D)
        table = rng.permutation(B * BLOCKS + 2)[:B * BLOCKS].reshape(B, BLOCKS).astype(np.int32)
        self.table_np, self.table = table, torch.from_numpy(table).cuda()
        self.plain = qo.Kv8(B * BLOCKS + 2, P, H, D)

    def project(self, x, out):
        if self.binary:
            self.fb.fluxbin_lut_gemm_smallbatch(self.qkv, x, y=out, workspace=self.ws_qkv)
        else:
            self.fb.fluxbin_w4_gemm(self.w4[0], x, y=out, workspace=self.ws_qkv)

    def buffers(self, T):
        torch, fb = self.torch, self.fb
        new = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")
        self.x, self.fused, self.attn, self.y = new(T, HIDDEN), new(T, WIDE), new(T, HQ, D), new(T, HIDDEN)
        self.ws_qkv = fb.make_workspace(self.qkv, T) if self.binary else fb.make_w4_workspace(self.w4[0], T)
        self.ws_o, self.ws_a = fb.make_w4_workspace(self.w4[1], T), fb.make_kv8_workspace(self.cache, T, B, HQ)

    def step(self, offsets, context):
        q, k, v = (t.unflatten(1, (-1, D)) for t in self.fused.split([HQ * D, H * D, H * D], dim=1))
        self.project(self.x, self.fused)
        self.fb.fluxbin_kv8_append(self.cache, k, v, offsets, context, self.table)
        self.fb.fluxbin_kv8_attention(self.cache, q, offsets, context, self.table, out=self.attn, workspace=self.ws_a)
        self.fb.fluxbin_w4_gemm(self.w4[1], self.attn.flatten(1), y=self.y, workspace=self.ws_o)

    def check(self, offsets, context):
        fused = self.fused.cpu().numpy()
        q, k, v = (t.reshape(len(fused), -1, D) for t in np.split(fused, [HQ * D, (HQ + H) * D], axis=1))
        if not self.binary:
            self.product(0, self.x.cpu().numpy(), fused)
        self.plain.append(k, v, offsets, context, self.table_np)
        ref, mag, big, peak, _ = self.plain.attention(q, offsets, context, self.table_np, D ** -0.5)
        got = self.attn.cpu().double().numpy()
        assert (np.abs(got - ref) <= qo.attention_bound(ref, mag, big, peak, int(max(context)))).all()
        self.product(1, got.reshape(len(got), -1), self.y.cpu().numpy())

    def product(self, which, x, y):
        codes, scales, zeros, _ = (t.cpu().numpy() for t in self.q_w4[which])
        q = (codes.view(np.uint32)[..., None] >> (4 * np.arange(8, dtype=np.uint32))) & 15
        W = qo.w4_dense(q.reshape(codes.shape[0], -1)[:, :x.shape[1]], scales, zeros, 64)
        x = x.astype(np.float64)
        assert (np.abs(y - x @ W.T) <= qo.w4_bound(W, x, True)).all()


@pytest.mark.parametrize("binary", [True, False])
def test_prompts_then_tokens(fb, binary):
    import torch
    log(f"case decoder step binary={binary}")
    blk = Block(fb, binary)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    lengths = np.array([70, 1, 33])
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    blk.buffers(int(offsets[-1]))
    blk.x.copy_(torch.randn_like(blk.x))
    blk.step(ints(offsets), ints(lengths))
    blk.check(offsets, lengths)

    blk.buffers(B)
    one, context = ints([0, 1, 2, 3]), ints(lengths)
    for i in range(3):   # eager
        context += 1
        lengths += 1
        blk.x.copy_(torch.randn_like(blk.x))
        blk.step(one, context)
        blk.check(np.arange(B + 1), lengths)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        context += 1
        blk.step(one, context)
    for i in range(30):
        lengths += 1
        blk.x.copy_(torch.randn_like(blk.x))
        graph.replay()
        torch.cuda.synchronize()
        blk.check(np.arange(B + 1), lengths)


def test_memory_of_the_null_stream(fb):
    """The null stream's handle is 0: what a call on it allocates belongs to that stream, and not to one from torch's pool."""
    import torch
    log("case memory of the null stream")
    n = 1 << 20
    W = torch.zeros(n, 32, dtype=torch.float16, device="cuda")
    codes, scales, zeros, values = fb.fluxbin_w4_quantize(W, 32, values=True, stream=0)
    cache = fb.make_kv8_cache(4, 16, 1, 64)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    k, v = fb.fluxbin_kv8_read(cache, ints([0, n]), ints([0]), ints([[0]]), n, stream=0)
    torch.cuda.synchronize()
    segments = torch.cuda.memory_snapshot()
    for t in (codes, scales, zeros, values, k, v):
        where = [s for s in segments if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
        assert len(where) == 1 and where[0]["stream"] == 0
    assert not values.any() and not k.any() and not v.any()
