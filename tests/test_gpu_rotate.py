"""Norms and rotation of queries and keys (fluxbin_qk_rotate) against fp64."""
import numpy as np
import pytest

from oracle import serve_oracle as so

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


class Case:
    """Queries and keys as slices of fused rows of odd stride, with rows and columns of nobody around them."""

    def __init__(self, fb, T, Hq, Hk, D, R, inter=False, norms="qk", far=100000, seed=0, magnitude=1.0, eps=1e-6):
        import torch
        self.fb, self.torch, self.Hq, self.Hk, self.D, self.T = fb, torch, Hq, Hk, D, T
        rng = self.rng = np.random.default_rng(seed)
        self.magnitude, self.inter, self.eps = magnitude, inter, eps
        self.positions = rng.integers(0, far, T).astype(np.int32)
        self.frequencies = (10000.0 ** (-np.arange(R // 2) / max(1, R // 2))).astype(np.float32)
        self.weights = [(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if s in norms else None for s in "qk"]
        self.q, self.k = ((rng.standard_normal((T, h, D)) * np.exp(rng.standard_normal((1, h, 1)))).astype(np.float16) for h in (Hq, Hk))
        dev = self.dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.plan = fb.make_rotary(D, dev(self.frequencies), dev(self.weights[0]), dev(self.weights[1]), eps, magnitude, inter)

    def fused(self):
        n = (self.Hq + self.Hk) * self.D
        wide = self.torch.full((self.T + 2, n + 7), 7.0, dtype=self.torch.float16, device="cuda")
        q = wide[1:-1, 1:1 + self.Hq * self.D].unflatten(1, (self.Hq, self.D))
        k = wide[1:-1, 3 + self.Hq * self.D:3 + n].unflatten(1, (self.Hk, self.D)) if self.Hk else None
        q.copy_(self.dev(self.q))
        if self.Hk:
            k.copy_(self.dev(self.k))
        return wide, q, k

    def check(self, q, k):
        for x, got, w in ((self.q, q, self.weights[0]), (self.k, k, self.weights[1])):
            if got is None:
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                y, size = so.rotate(x, self.positions, self.frequencies, w, self.eps, self.magnitude, self.inter)
                far = np.abs(got.cpu().double().numpy() - y) / so.rotate_bound(y, size)
            log(f"  worst {far.max():.3f} of the bound")
            assert (far <= 1).all()

    def run(self, stream=None):
        wide, q, k = self.fused()
        pos = self.dev(self.positions)
        before = wide.clone()
        qo, ko = self.fb.fluxbin_qk_rotate(self.plan, q, k, pos)
        assert self.torch.equal(wide, before)
        self.check(qo, ko)
        # in place, in the fused rows; what belongs to nobody stays
        q2, k2 = self.fb.fluxbin_qk_rotate(self.plan, q, k, pos, q_out=q, k_out=k)
        assert q2 is q and self.torch.equal(q, qo) and (k is None or self.torch.equal(k, ko))
        n = self.Hq * self.D
        rest = [wide[0], wide[-1], wide[:, 0], wide[:, 1 + n:3 + n], wide[:, 3 + n + self.Hk * self.D:]]
        assert all((r == 7).all() for r in rest)
        return qo, ko


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,R", [(64, 64), (64, 16), (128, 128), (128, 48), (128, 112), (256, 256), (256, 64), (128, 0)])
def test_sizes(fb, D, R, inter):
    log(f"case rotate D={D} R={R} inter={inter}")
    for T, Hq, Hk in ((1, 1, 0), (1, 32, 8), (3, 5, 1), (37, 7, 7), (300, 1, 0)):
        Case(fb, T, Hq, Hk, D, R, inter, seed=T + R).run()


@pytest.mark.parametrize("norms", ["", "q", "k", "qk"])
def test_norms(fb, norms):
    log(f"case rotate norms={norms}")
    Case(fb, 19, 6, 2, 128, 64, norms=norms, seed=3).run()


@pytest.mark.parametrize("D,Hq,Hk,inter", [(64, 16, 4, False), (128, 64, 8, False), (128, 3, 2, True), (256, 8, 1, True)])
def test_many_rows(fb, D, Hq, Hk, inter):
    """Outputs past 32 MB, which are streamed."""
    T = (32 << 20) // (2 * (Hq + Hk) * D) + 5
    log(f"case rotate T={T} D={D}")
    Case(fb, T, Hq, Hk, D, D, inter, seed=5).run()


@pytest.mark.parametrize("D,Hq,Hk,inter,R", [(64, 6, 2, True, 32), (256, 4, 2, False, 192)])
def test_many_rows_partly_rotated(fb, D, Hq, Hk, inter, R):
    """Streamed outputs of which elements are not rotated, in the forms that whole heads do not take."""
    T = (32 << 20) // (2 * (Hq + Hk) * D) + 3
    log(f"case rotate T={T} D={D} R={R}")
    Case(fb, T, Hq, Hk, D, R, inter, seed=11).run()


def test_far_and_odd_positions(fb):
    """Positions up to 2^31 - 1, negative ones, and a magnitude."""
    log("case rotate far")
    for far in (2 ** 20, 2 ** 31 - 1):
        Case(fb, 64, 4, 2, 128, 128, far=far, seed=6, magnitude=1.19).run()
    c = Case(fb, 8, 2, 1, 64, 64, seed=7)
    c.positions[:] = [0, -1, -5, -2 ** 31, 2 ** 31 - 1, 1, 2, 3]
    c.run()


def test_special_values(fb):
    """Zeros (with eps 0 a norm of them is NaN), subnormals, the largest fp16, infinities and NaN stay in their head."""
    log("case rotate special")
    c = Case(fb, 6, 3, 1, 64, 64, norms="q", seed=8)
    c.q[0, 0], c.q[1, 0] = 0, 6e-8
    c.q[2, 0], c.k[2, 0, ::2] = 60000, 6e-8
    c.run()
    c.q[3, 1, 5], c.q[4, 2, 7], c.k[5, 0, 3] = np.nan, np.inf, np.inf
    _, q, k = c.fused()
    qo, ko = c.fb.fluxbin_qk_rotate(c.plan, q, k, c.dev(c.positions))
    qo, ko = qo.cpu().numpy(), ko.cpu().numpy()
    assert np.isnan(qo[3, 1]).all() and np.isnan(qo[4, 2][[7, 39]]).all() and not np.isfinite(ko[5, 0][[3, 35]]).any()
    bad = ~np.isfinite(qo)
    bad[3, 1], bad[4, 2] = False, False
    ko[5, 0, [3, 35]] = 0
    assert not bad.any() and np.isfinite(ko).all()
    zero = fb.make_rotary(64, c.plan.tensors[0], c.plan.tensors[1], eps=0.0)
    qo, _ = fb.fluxbin_qk_rotate(zero, q, None, c.dev(c.positions))
    assert qo[0, 0].isnan().all() and qo[0, 1].isfinite().all()


def test_refusals(fb):
    log("case rotate refusals")
    import torch
    c = Case(fb, 4, 2, 1, 64, 32, seed=9)
    _, q, k = c.fused()
    pos = c.dev(c.positions)
    for bad in (dict(q=q.float()), dict(q=q[..., :32]), dict(k=k[:3]), dict(k=k.cpu()), dict(positions=pos.long()), dict(positions=pos[:3]),
                dict(positions=pos.cpu()), dict(q_out=q[:, :1]), dict(k_out=q[:, :1]), dict(q_out=q.transpose(1, 2)),
                dict(q_out=c.fused()[1].expand(4, 2, 64)[:, :1].expand(4, 2, 64))):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_qk_rotate(c.plan, **dict(dict(q=q, k=k, positions=pos), **bad))
    with pytest.raises(fb.FluxbinError):
        fb.make_rotary(128, c.dev(c.frequencies), torch.ones(64, device="cuda"))
    with pytest.raises(fb.FluxbinError):
        fb.make_rotary(64, c.dev(c.frequencies).double())
    empty = fb.fluxbin_qk_rotate(c.plan, q[:0], k[:0], pos[:0])
    assert empty[0].shape == (0, 2, 64)


def test_stream_and_graph(fb):
    """On another stream, and captured: each replay rotates what is there then."""
    import torch
    log("case rotate graph")
    c = Case(fb, 33, 8, 2, 128, 128, seed=10)
    want = c.run()
    _, q, k = c.fused()
    pos = c.dev(c.positions)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    qo, ko = fb.fluxbin_qk_rotate(c.plan, q, k, pos, stream=side)
    side.synchronize()
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qo, ko = fb.fluxbin_qk_rotate(c.plan, q, k, pos)
    for i in range(4):
        q.mul_(0.5 + i)
        pos.add_(i)
        eager = fb.fluxbin_qk_rotate(c.plan, q, k, pos)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, eager[0]) and torch.equal(ko, eager[1])
