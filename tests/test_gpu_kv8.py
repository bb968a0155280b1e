"""The paged 8-bit key/value cache (fluxbin_kv8_*) against the plain definitions in oracle/quant_oracle.py: stored values bit
for bit, attention within the bound of its fp32 arithmetic and one rounding to fp16."""
import numpy as np
import pytest

from oracle import quant_oracle as qo

from conftest import gpu_available
from gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def fb():
    if not gpu_available():
        pytest.skip("no GPU")
    from paper_2608_15602_amd import fluxbin
    fluxbin.lib()
    return fluxbin


class Setup:
    """A cache of the library and the plain one side by side. ctx: tokens per sequence, all with room for `room` more."""

    def __init__(self, fb, B, H, D, P, room, seed, spare=3):
        import torch
        self.fb, self.H, self.D, self.P, self.B = fb, H, D, P, B
        self.rng = np.random.default_rng(seed)
        blocks = -(-room // P)
        self.pages = B * blocks + spare
        self.table = self.rng.permutation(self.pages)[:B * blocks].reshape(B, blocks).astype(np.int32)
        self.plain = qo.Kv8(self.pages, P, H, D)
        self.cache = fb.make_kv8_cache(self.pages, P, H, D)
        self.cache.buf.fill_(0xFF)   # scales that nobody has written are NaN
        self.length = np.zeros(B, np.int64)
        self.torch = torch

    def dev(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def ints(self, x):
        return self.dev(np.asarray(x, np.int32))

    def arrays(self, offsets, context):
        return self.ints(offsets), self.ints(context), self.ints(self.table)

    def rows(self, T, scale=1.0):
        k = self.rng.standard_normal((T, self.H, self.D)) * np.exp(self.rng.standard_normal((1, self.H, self.D)) * 0.5) * scale
        return k.astype(np.float16), (self.rng.standard_normal((T, self.H, self.D)) * scale).astype(np.float16)

    def append(self, new, scale=1.0, edit=None):
        """new[b] tokens to every sequence, as slices of fused rows of odd stride, with rows of nobody behind them."""
        offsets = np.concatenate([[0], np.cumsum(new)])
        T = int(offsets[-1])
        k, v = self.rows(T, scale)
        if edit:
            edit(k, v)
        self.length += new
        fused = self.torch.full((T + 2, 2 * self.H * self.D + 5), float("nan"), dtype=self.torch.float16, device="cuda")
        n = self.H * self.D
        kt, vt = fused[:, 1:1 + n].unflatten(1, (self.H, self.D)), fused[:, 2 + n:2 + 2 * n].unflatten(1, (self.H, self.D))
        kt[:T], vt[:T] = self.dev(k), self.dev(v)
        self.fb.fluxbin_kv8_append(self.cache, kt, vt, *self.arrays(offsets, self.length))
        self.plain.append(k, v, offsets, self.length, self.table)

    def check(self):
        """Every cached value, bit for bit."""
        offsets = np.concatenate([[0], np.cumsum(self.length)])
        T = int(offsets[-1])
        k, v = self.fb.fluxbin_kv8_read(self.cache, *self.arrays(offsets, self.length), T)
        pk, pv, _ = self.plain.read(offsets, self.length, self.table, T)
        assert np.array_equal(k.cpu().numpy(), pk) and np.array_equal(v.cpu().numpy(), pv)

    def attend(self, new, G, causal=True, window=0, scale=None, q=None, ws=None, chunk=False):
        """Queries of the newest new[b] tokens, as slices of longer rows; rows of nobody stay as they were."""
        offsets = np.concatenate([[0], np.cumsum(new)])
        T, Hq = int(offsets[-1]), self.H * G
        if q is None:
            q = (self.rng.standard_normal((T, Hq, self.D)) * 1.5).astype(np.float16)
        wide = self.torch.full((T + 1, Hq * self.D + 3), float("nan"), dtype=self.torch.float16, device="cuda")
        qt = wide[:, 3:].unflatten(1, (Hq, self.D))
        qt[:T] = self.dev(q)
        back = self.torch.full((T + 1, Hq * self.D + 1), 7.0, dtype=self.torch.float16, device="cuda")
        out = back[:, 1:].unflatten(1, (Hq, self.D))
        self.fb.fluxbin_kv8_attention(self.cache, qt, *self.arrays(offsets, self.length), out=out, causal=causal,
                                      window=window, scale=scale, workspace=ws)
        got = back.cpu().double().numpy()
        assert (got[T] == 7).all() and (got[:, 0] == 7).all()
        got = got[:T, 1:].reshape(T, Hq, self.D)
        ref, mag, big, peak, written = self.plain.attention(q, offsets, self.length, self.table,
                                                      self.D ** -0.5 if scale is None else scale, causal, window)
        assert written.all()
        bound = qo.attention_bound(ref, mag, big, peak, max(1, int(self.length.max())), chunk)
        far = np.abs(got - ref) / bound
        log(f"  worst {far.max():.3f} of the bound")
        assert (far <= 1).all()
        return got


# ---------------------------------------------------------------------------------------------- storing

@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("H,D", [(1, 64), (3, 128), (2, 256)])
def test_append_in_pieces(fb, H, D, P):
    """Prompts of odd lengths, then one token at a time and a few at a time, over page borders; growing values make the
    scales of partly filled pages grow."""
    log(f"case append H={H} D={D} P={P}")
    s = Setup(fb, 4, H, D, P, 2 * P + 60, seed=P + D)
    s.append([P + 3, 1, 0, 2 * P])
    s.check()
    for scale in (0.5, 2.0, 2.0, 30.0):
        s.append([1, 1, 1, 1], scale)
        s.check()
    s.append([5, 0, 17, 3], 100.0)
    s.check()
    s.append([30, P, 1, 2], 0.01)
    s.check()


def test_append_special_values(fb):
    """Zeros, subnormals, the largest fp16, infinities and NaN, in a page that holds earlier tokens of each kind."""
    log("case append special values")

    def special(k, v):
        k[0, 0], v[0, 0, ::2] = 0, 6e-8
        if len(k) > 1:
            k[1, 0, :4] = [np.nan, np.inf, -np.inf, 65504]
            v[1, 1, 3] = np.nan

    s = Setup(fb, 2, 2, 64, 16, 64, seed=9)
    s.append([1, 2], 0.0)
    s.check()
    s.append([2, 3], 1e-6, special)
    s.check()
    s.append([2, 1], 1.0, special)
    s.check()


def test_append_rewrites_positions(fb):
    """A sequence that goes back and stores other tokens at the same positions, and the same call twice."""
    log("case append again")
    s = Setup(fb, 1, 2, 128, 32, 128, seed=10)
    s.append([50])
    s.length -= 13
    s.append([9])
    s.check()
    k, v = s.rows(5)
    for _ in range(2):
        a = s.arrays([0, 5], s.length)
        fb.fluxbin_kv8_append(s.cache, s.dev(k), s.dev(v), *a)
        s.plain.append(k, v, [0, 5], s.length, s.table)
        s.check()


def test_bad_pages_and_lengths(fb):
    """Entries that are no pages, positions past the table or before 0, huge and negative lengths, ranges of rows outside the
    call: left out, and the rest of the cache stays."""
    log("case bad pages")
    s = Setup(fb, 5, 2, 64, 16, 64, seed=11)
    s.append([40, 64, 20, 33, 64])   # every position that a length below counts has been stored
    good = s.table.copy()
    s.table[0, 1], s.table[1, 3], s.table[1, 0] = -1, s.pages, 2 ** 31 - 1
    context = np.array([42, 70, 3, -5, 2 ** 31 - 1], np.int32)   # past the table, fewer than its rows, negative, huge
    near = np.array([42, 70, 3, 0, 94])                          # the same to a plain form that writes positions out
    k, v = s.rows(20, 3.0)
    q = (s.rng.standard_normal((20, 4, 64))).astype(np.float16)
    for offs in ([0, 4, 10, 16, 18, 20], [-3, 4, 10, 16, 18, 25]):
        a = s.arrays(offs, context)
        fb.fluxbin_kv8_append(s.cache, s.dev(k), s.dev(v), *a)
        s.plain.append(k, v, offs, near, s.table)
        kt, vt = fb.fluxbin_kv8_read(s.cache, *a, 20)
        pk, pv, written = s.plain.read(offs, near, s.table, 20)
        assert np.array_equal(kt.cpu().numpy()[written], pk[written]) and np.array_equal(vt.cpu().numpy()[written], pv[written])
        out = s.torch.full((20, 4, 64), 7.0, dtype=s.torch.float16, device="cuda")
        fb.fluxbin_kv8_attention(s.cache, s.dev(q), *a, out=out)
        ref, mag, big, peak, _ = s.plain.attention(q, offs, near, s.table, 0.125)
        got = out.cpu().double().numpy()
        assert (np.abs(got - ref)[written] <= qo.attention_bound(ref, mag, big, peak, 128)[written]).all()
        assert (got[~written] == 7).all()
    s.table = good
    s.length[:] = [36, 60, 0, 0, 0]
    s.check()
    # offsets that fall: nothing outside the call's tensors and the sequences' pages is touched
    a = s.arrays([0, 10, 4, 20, 9, 20], context)
    fb.fluxbin_kv8_append(s.cache, s.dev(k), s.dev(v), *a)
    fb.fluxbin_kv8_read(s.cache, *a, 20)
    fb.fluxbin_kv8_attention(s.cache, s.dev(q), *a)
    s.torch.cuda.synchronize()


def test_workspace_refusals(fb):
    log("case workspace refusals")
    s = Setup(fb, 1, 2, 64, 16, 64, seed=19)
    s.append([20])
    q = s.dev(s.rng.standard_normal((1, 4, 64)).astype(np.float16))
    a, n = s.arrays([0, 1], s.length), fb.fluxbin_kv8_workspace_query(s.cache, 1, 1, 4)
    for ws in (s.torch.empty(n - 1, dtype=s.torch.uint8, device="cuda"), s.torch.empty(n + 8, dtype=s.torch.uint8, device="cuda")[8:],
               s.torch.empty(n, dtype=s.torch.uint8), s.cache.buf):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_attention(s.cache, q, *a, workspace=ws)
    for bad in (q.float(), q[:, :3], q[:, :, :32], q.cpu(), q.transpose(1, 2)):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_attention(s.cache, bad, *a)
    with pytest.raises(fb.FluxbinError):
        fb.fluxbin_kv8_attention(s.cache, q, *a, out=q)
    for i, bad in ((0, a[0].long()), (0, a[0][:1]), (1, a[1].cpu()), (2, a[2].t()), (2, a[2][0])):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_attention(s.cache, q, *(bad if j == i else x for j, x in enumerate(a)))


# ---------------------------------------------------------------------------------------------- attention

@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,G", [(1, 1), (2, 4), (1, 7), (3, 8), (1, 16), (1, 40)])
def test_single_tokens(fb, H, G, D):
    """One new token of sequences of 1 to 700 tokens."""
    log(f"case decode H={H} G={G} D={D}")
    s = Setup(fb, 6, H, D, 32, 700, seed=H + G + D)
    s.append([1, 15, 64, 65, 300, 700])
    s.attend([1] * 6, G)


@pytest.mark.parametrize("P", [16, 64, 128, 256])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 40), (False, 70), (True, 10 ** 9)])
def test_rows_and_masks(fb, P, causal, window):
    """Several new tokens, causal or not, with and without a window; a sequence without rows, one that is all new."""
    log(f"case masks P={P} causal={causal} window={window}")
    s = Setup(fb, 5, 2, 64, P, 300, seed=P)
    s.append([200, 0, 50, 257, 90])
    s.length[1] = 0
    s.attend([3, 0, 50, 1, 33], 4, causal, window)


def test_empty_rows(fb):
    """Rows before position 0, a sequence of no tokens, a page that is missing: rows without a key are 0."""
    log("case empty rows")
    s = Setup(fb, 3, 2, 64, 16, 64, seed=12)
    s.append([5, 0, 16])
    s.table[2, 0] = -1
    got = s.attend([9, 2, 3], 2)
    assert (got[:4] == 0).all() and (got[4:9] != 0).any() and (got[9:] == 0).all()


@pytest.mark.parametrize("B,H,G,D,ctx", [(1, 1, 1, 64, 20000), (2, 1, 8, 128, 9000), (300, 1, 2, 64, 40)])
def test_split_and_many(fb, B, H, G, D, ctx):
    """A long context over many workgroups; more sequences than lanes."""
    log(f"case split B={B} ctx={ctx}")
    s = Setup(fb, B, H, D, 64, ctx, seed=13)
    s.append([max(1, ctx - 17 * (b % 5)) if ctx > 100 else 1 + (b * 7) % ctx for b in range(B)])
    ws = fb.make_kv8_workspace(s.cache, B, B, H * G)
    ws.fill_(0xFF)   # NaN wherever a call would read what it has not written
    a = s.attend([1] * B, G, ws=ws)
    s.attend([2] + [1] * (B - 1), G, ws=ws)
    assert np.isfinite(a).all()


@pytest.mark.parametrize("new,ctx", [([257], [257]), ([130, 1, 64], [400, 90, 64]), ([600, 3], [640, 1000])])
def test_prompt_chunks(fb, new, ctx):
    """Chunks of prompts, over what is cached of them."""
    log(f"case chunk new={new} ctx={ctx}")
    for H, G, D in ((2, 1, 128), (1, 8, 64), (1, 5, 256)):
        s = Setup(fb, len(new), H, D, 64, max(ctx), seed=14)
        s.append([c - n for c, n in zip(ctx, new)])
        s.append(new)
        s.attend(new, G)
        s.attend(new, G, window=100)


@pytest.mark.parametrize("H,G,D,P,new,ctx", [
    (8, 8, 64, 16, [301, 211], [301, 500]), (8, 8, 128, 64, [300, 1, 230], [333, 90, 700]), (8, 8, 256, 32, [270], [400]),
    (32, 1, 128, 128, [1030], [1030]), (7, 5, 64, 256, [500, 471], [500, 2000])])
def test_many_rows(fb, H, G, D, P, new, ctx):
    """Enough rows for the prompt chunks' own kernel, ragged, masked and not."""
    log(f"case many rows H={H} G={G} D={D} P={P} new={new} ctx={ctx}")
    assert sum(new) * G // (64 if D == 256 else 128) * H >= 256   # where that kernel takes over on 256 CUs
    s = Setup(fb, len(new), H, D, P, max(ctx), seed=20)
    s.append([c - n for c, n in zip(ctx, new)])
    s.append(new)
    s.attend(new, G, chunk=True)
    s.attend(new, G, window=77, chunk=True)
    s.attend(new, G, causal=False, chunk=True)
    s.length[0] -= 40                           # rows before position 0 (or fewer tokens)
    s.table[-1, 1] = -1                         # a page that is missing
    got = s.attend(new, G, chunk=True)
    if ctx[0] == new[0]:
        assert (got[:40] == 0).all()


def test_single_tokens_among_many_rows(fb):
    """Single tokens of long and short contexts, sequences without rows, and prompts in one call."""
    log("case mixed batch")
    s = Setup(fb, 7, 8, 128, 64, 5000, seed=24)
    new, ctx = [1, 600, 0, 3, 1, 16, 2], [5000, 600, 40, 900, 1, 77, 2]
    s.append([c - n for c, n in zip(ctx, new)])
    s.append(new)
    assert sum(new) * 8 // 128 * 8 >= 256
    s.attend(new, 8, chunk=True)
    s.attend(new, 8, window=700, chunk=True)


def test_many_rows_scales_far_apart(fb):
    log("case many rows, scales far apart")
    s = Setup(fb, 1, 16, 64, 16, 512, seed=22)
    for i in range(32):
        s.append([16], 1.0, lambda k, v, i=i: v.__imul__(np.float16([1e-7, 1e3, 1.0, 0.0, 1e-3][i % 5])))
    q = (s.rng.standard_normal((512, 64, 64)) * 3).astype(np.float16)
    s.attend([512], 4, q=q, chunk=True)
    s.attend([512], 4, causal=False, q=q, scale=0.5, chunk=True)


def test_scales_far_apart(fb):
    """Pages whose scales differ by ten orders of magnitude, the weight on any of them; values that are all zero."""
    log("case scales far apart")
    s = Setup(fb, 1, 1, 64, 16, 256, seed=15)
    for scale in (1e-7, 6e4, 1.0, 0.0, 1e-3, 6e4, 1e-7, 1.0):
        s.append([16], 1.0, lambda k, v, scale=scale: v.__imul__(np.float16(scale)))
    q = (s.rng.standard_normal((8, 4, 64)) * 0.5).astype(np.float16)
    k, _ = s.plain.values(0, 0, 128, s.table)
    for i in range(8):
        q[i, 0] = (k[16 * i + 3, 0] * 8).astype(np.float16)      # nearly all weight on one token of page i
        q[i, 1] = (k[16 * i, 0] * 0.1).astype(np.float16)
    for i in range(8):
        s.attend([1], 4, causal=False, q=q[i:i + 1])
    s.attend([8], 4, causal=False, q=q)
    s.attend([8], 4, causal=False, q=q * np.float16(20), scale=0.3)
    s.attend([8], 4, causal=False, q=q, scale=0.0)
    s.attend([8], 4, causal=False, q=q, scale=-0.1)


def test_queries_not_finite(fb):
    """Infinities and NaN in a query stay in its own row and head."""
    log("case queries not finite")
    s = Setup(fb, 2, 1, 128, 32, 100, seed=16)
    s.append([100, 30])
    q = s.rng.standard_normal((2, 8, 128)).astype(np.float16)
    a = s.arrays([0, 1, 2], s.length)
    good = fb.fluxbin_kv8_attention(s.cache, s.dev(q), *a).cpu().numpy()
    q[0, 3, 7], q[1, 0, 0] = np.nan, np.inf
    bad = fb.fluxbin_kv8_attention(s.cache, s.dev(q), *a).cpu().numpy()
    assert np.isnan(bad[0, 3]).all() and not np.isfinite(bad[1, 0]).any()
    good[0, 3], good[1, 0] = bad[0, 3], bad[1, 0]
    assert np.array_equal(good, bad, equal_nan=True)


def test_graph_with_growing_lengths(fb):
    """A captured step (append, attention) replayed while the lengths on the device grow, with eager calls between."""
    import torch
    log("case graph")
    s, t = (Setup(fb, 3, 2, 64, 16, 200, seed=17) for _ in range(2))
    s.append([5, 100, 31])
    t.append([5, 100, 31])
    G = 4
    k, v, q = (torch.zeros(3, h, 64, dtype=torch.float16, device="cuda") for h in (2, 2, 2 * G))
    offsets, context, table = s.arrays([0, 1, 2, 3], s.length)
    ws, out = fb.make_kv8_workspace(s.cache, 3, 3, 2 * G), torch.zeros_like(q)

    def step(cache, out, ws):
        fb.fluxbin_kv8_append(cache, k, v, offsets, context, table)
        fb.fluxbin_kv8_attention(cache, q, offsets, context, table, out=out, workspace=ws)

    context += 1
    step(s.cache, out, ws)
    step(t.cache, out, None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s.cache, out, ws)
    for i in range(40):
        context += 1
        for x in (k, v, q):
            x.copy_(torch.randn_like(x))
        graph.replay()
        eager = torch.zeros_like(out)
        step(t.cache, eager, None)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i
    n = fb.fluxbin_kv8_cache_query(s.pages, 16, 2, 64) // 2 // 256 * 256   # the codes of keys, at least
    assert torch.isfinite(out).all() and n > 0


def test_cache_past_32_bits(fb):
    """Pages whose codes lie past 2^32 bytes, and scales far into their sections."""
    import torch
    log("case large cache")
    H, D, P, pages = 8, 128, 64, 70000
    assert pages * H * D * P > 2 ** 32
    s = Setup(fb, 2, H, D, P, 3 * P, seed=23)
    del s.cache
    s.cache = fb.make_kv8_cache(pages, P, H, D)
    low = s.table
    high = np.array([[pages - 1, 0, pages - 2], [pages // 2, pages - 3, 65536]], np.int32)
    q = s.rng.standard_normal((2, 16, D)).astype(np.float16)
    k, v = s.rows(250)
    offsets, lengths = [0, 150, 250], np.array([150, 100])
    a = s.ints(offsets), s.ints(lengths), s.ints(high)
    fb.fluxbin_kv8_append(s.cache, s.dev(k), s.dev(v), *a)
    s.plain.append(k, v, offsets, lengths, low)
    kt, vt = fb.fluxbin_kv8_read(s.cache, *a, 250)
    pk, pv, _ = s.plain.read(offsets, lengths, low, 250)
    assert np.array_equal(kt.cpu().numpy(), pk) and np.array_equal(vt.cpu().numpy(), pv)
    out = fb.fluxbin_kv8_attention(s.cache, s.dev(q), s.ints([0, 1, 2]), a[1], a[2]).cpu().double().numpy()
    ref, mag, big, peak, _ = s.plain.attention(q, [0, 1, 2], lengths, low, D ** -0.5)
    assert (np.abs(out - ref) <= qo.attention_bound(ref, mag, big, peak, 150)).all()
    del kt, vt
    s.cache = None
    torch.cuda.empty_cache()


def test_another_stream(fb):
    import torch
    log("case stream")
    s = Setup(fb, 2, 2, 128, 64, 300, seed=18)
    s.append([300, 7])
    q = s.dev(s.rng.standard_normal((2, 16, 128)).astype(np.float16))
    a = s.arrays([0, 1, 2], s.length)
    ref = fb.fluxbin_kv8_attention(s.cache, q, *a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, ws = torch.zeros_like(ref), fb.make_kv8_workspace(s.cache, 2, 2, 16)
    fb.fluxbin_kv8_attention(s.cache, q, *a, out=out, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, ref)
    side.wait_stream(torch.cuda.current_stream())
    for handle in (side, side.cuda_stream):   # outputs and workspaces of the call's own, on its stream
        out = fb.fluxbin_kv8_attention(s.cache, q, *a, stream=handle)
        k, v = fb.fluxbin_kv8_read(s.cache, *a, 2, stream=handle)
        side.synchronize()
        assert torch.equal(out, ref)
        assert all(torch.equal(x, y) for x, y in zip((k, v), fb.fluxbin_kv8_read(s.cache, *a, 2)))


@pytest.mark.parametrize("new,G,H,D", [([2, 1, 3], 4, 2, 64), ([270, 260, 300], 8, 8, 128), ([270, 260, 300], 8, 8, 256)])
def test_queries_not_finite_without_pages(fb, new, G, H, D):
    """NaN and infinities in a query do not come out of blocks without a page: a row whose positions have none is 0, and one
    beside it with some is as if its own query were alone. Few rows, and as many as the prompt chunks' kernel takes."""
    import torch
    log(f"case queries not finite, pages missing, new={new} D={D}")
    s = Setup(fb, 3, H, D, 32, 320, seed=45)
    s.append([310, 305, 300])
    s.table[1, :], s.table[2, :9] = -1, s.pages     # no page; one page of ten
    offsets = np.concatenate([[0], np.cumsum(new)])
    q = s.rng.standard_normal((int(offsets[-1]), H * G, D)).astype(np.float16)
    a = s.arrays(offsets, s.length)
    good = fb.fluxbin_kv8_attention(s.cache, s.dev(q), *a, causal=False)
    at = int(offsets[1])
    assert not good[at:at + new[1]].any() and torch.isfinite(good).all()
    q[at, 1, 5], q[at, 2, 0], q[at, 3] = np.nan, np.inf, -np.inf
    bad = fb.fluxbin_kv8_attention(s.cache, s.dev(q), *a, causal=False)
    assert torch.equal(good, bad)
    q[int(offsets[2]), 0, 7] = np.nan
    bad = fb.fluxbin_kv8_attention(s.cache, s.dev(q), *a, causal=False)
    assert torch.isnan(bad[int(offsets[2]), 0]).all()
    bad[int(offsets[2]), 0] = good[int(offsets[2]), 0]
    assert torch.equal(good, bad)


def test_shared_pages(fb):
    """Sequences that share their first pages, and one that has a page twice: read and attended by each, while new tokens go
    to pages of their own."""
    import torch
    log("case shared pages")
    s = Setup(fb, 3, 2, 128, 32, 160, seed=46)
    s.append([96, 0, 0])
    s.table[1, :3] = s.table[0, :3]
    s.table[2, :3] = s.table[0, 1]
    s.length[:] = 96
    s.append([20, 1, 40])
    s.check()
    s.attend([20, 1, 40], 4)
    s.attend([1, 1, 1], 4, window=50)


def test_two_streams_at_once(fb):
    """Appends to and attention over different pages of one cache on two streams, each with its workspace, the same captured
    graphs replayed beside each other, and one replayed twice with other inputs."""
    import torch
    log("case two streams")
    s = Setup(fb, 2, 2, 64, 16, 3000, seed=47)
    s.append([2900, 2000])
    q = [s.dev(s.rng.standard_normal((1, 8, 64)).astype(np.float16)) for _ in range(2)]
    k = [s.dev(s.rng.standard_normal((1, 2, 64)).astype(np.float16)) for _ in range(2)]
    offsets = s.ints([0, 1])
    s.length += 1
    lengths, tables = [s.ints([n]) for n in s.length], [s.ints(s.table[b:b + 1]) for b in range(2)]
    ws, out = [fb.make_kv8_workspace(s.cache, 1, 1, 8) for _ in range(2)], [torch.zeros_like(x) for x in q]

    def step(b, stream=None):
        fb.fluxbin_kv8_append(s.cache, k[b], k[b], offsets, lengths[b], tables[b], stream=stream)
        fb.fluxbin_kv8_attention(s.cache, q[b], offsets, lengths[b], tables[b], out=out[b], workspace=ws[b], stream=stream)

    for b in range(2):
        step(b)
    ref = [x.clone() for x in out]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    for i in range(5):
        for x in out:
            x.zero_()
        torch.cuda.synchronize()
        for b in range(2):
            step(b, sides[b])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, ref))
    graphs = []
    for b in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[b]):
            step(b)
    for i in range(5):
        for x in out:
            x.zero_()
        torch.cuda.synchronize()
        for g, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, ref))
    q[0].neg_()
    for i in range(3):
        torch.cuda.synchronize()
        graphs[0].replay()
        torch.cuda.synchronize()
        got = out[0].clone()
        step(0)
        torch.cuda.synchronize()
        assert torch.equal(out[0], got) and not torch.equal(got, ref[0])


@pytest.mark.parametrize("H,P,new", [
    (8, 64, [700]), (2, 16, [333, 1000]), (8, 32, [1] * 7 + [500] + [1] * 8), (3, 128, [5] * 40), (8, 64, [17] * 30),
    (1, 256, [1] * 20 + [3000, 0, 0] + [2] * 9), (40, 16, [9] * 12 + [250]), (1, 64, [1, 900, 1, 800])])
def test_append_windows(fb, H, P, new):
    """Calls of every number of rows per window between one and a page's: one prompt, several, single tokens beside one."""
    log(f"case windows H={H} P={P} new={new}")
    s = Setup(fb, len(new), H, 64, P, max(new) + 40, seed=48)
    s.append([b % 37 for b in range(len(new))])
    s.append(new, 2.0)
    s.check()
    s.append([n % 3 for n in new], 3.0)
    s.check()
