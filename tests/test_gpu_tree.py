"""Trees of drafted tokens (fluxbin_tree_masks, fluxbin_kv8_tree_attention, fluxbin_kv8_keep) against the plain definitions:
masks and kept rows exactly, attention within the bound of its fp32 arithmetic and one rounding to fp16."""
import numpy as np
import pytest

from oracle import quant_oracle as qo
from oracle import serve_oracle as so

from conftest import gpu_available
from gpu_util import log
from test_gpu_kv8 import Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def fb():
    if not gpu_available():
        pytest.skip("no GPU")
    from paper_2608_15602_amd import fluxbin
    fluxbin.lib()
    return fluxbin


class Trees(Setup):
    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.plain = so.Kv8(self.pages, self.P, self.H, self.D)

    def parents(self, new):
        return np.concatenate([np.floor(self.rng.random(n) * (np.arange(n) + 1)).astype(np.int32) - 1 for n in new] or [[]]).astype(np.int32)

    def masks(self, new, words, parents=None):
        offsets = np.concatenate([[0], np.cumsum(new)])
        return so.tree_masks(self.parents(new) if parents is None else parents, offsets, self.length, words, int(offsets[-1]))[0]

    def verify(self, new, G, masks=None, words=None, window=0, scale=None, q=None, ws=None):
        """Queries of the newest new[b] tokens, as slices of longer rows; rows of nobody stay as they were."""
        offsets = np.concatenate([[0], np.cumsum(new)])
        T, Hq = int(offsets[-1]), self.H * G
        words = words or max(1, -(-max(new) // 64))
        if masks is None:
            masks = self.masks(new, words)
        if q is None:
            q = (self.rng.standard_normal((T, Hq, self.D)) * 1.5).astype(np.float16)
        wide = self.torch.full((T + 1, Hq * self.D + 3), float("nan"), dtype=self.torch.float16, device="cuda")
        qt = wide[:T, 3:].unflatten(1, (Hq, self.D))
        qt.copy_(self.dev(q))
        back = self.torch.full((T + 1, Hq * self.D + 1), 7.0, dtype=self.torch.float16, device="cuda")
        out = back[:T, 1:].unflatten(1, (Hq, self.D))
        self.fb.fluxbin_kv8_tree_attention(self.cache, qt, self.dev(so.packed(masks)), *self.arrays(offsets, self.length), out=out,
                                           window=window, scale=scale, workspace=ws)
        got = back.cpu().double().numpy()
        assert (got[T] == 7).all() and (got[:, 0] == 7).all()
        got = got[:T, 1:].reshape(T, Hq, self.D)
        ref, mag, big, peak, written = self.plain.tree_attention(q, masks, offsets, self.length, self.table,
                                                           self.D ** -0.5 if scale is None else scale, window)
        far = np.abs(got - ref) / qo.attention_bound(ref, mag, big, peak, max(1, int(self.length.max())))
        log(f"  worst {far[written].max(initial=0):.3f} of the bound")
        assert (far[written] <= 1).all() and (got[~written] == 7).all()
        return got


# ---------------------------------------------------------------------------------------------- masks

@pytest.mark.parametrize("new,words", [([1], 1), ([64, 0, 3], 1), ([65, 64, 1, 128], 2), ([300, 7, 1024], 16), ([20] * 200, 1)])
def test_masks(fb, new, words):
    import torch
    log(f"case masks {new[:5]} words={words}")
    rng = np.random.default_rng(sum(new))
    parents = np.concatenate([np.floor(rng.random(n) * (np.arange(n) + 1)).astype(np.int32) - 1 for n in new]).astype(np.int32)
    chain = np.concatenate([np.arange(-1, n - 1) for n in new]).astype(np.int32)
    odd = rng.integers(-3, 40, len(parents)).astype(np.int32)      # parents that are not before their node are none
    offsets = np.concatenate([[0], np.cumsum(new)])
    context = rng.integers(0, 5000, len(new)).astype(np.int32)
    T = len(parents)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    for p in (parents, chain, odd):
        masks, positions, _ = so.tree_masks(p, offsets, context, words, T)
        got = fb.fluxbin_tree_masks(dev(p), dev(offsets.astype(np.int32)), dev(context), words)
        assert np.array_equal(got[0].cpu().numpy(), so.packed(masks)) and np.array_equal(got[1].cpu().numpy(), positions)


def test_masks_left_out(fb):
    """Trees of more nodes than the words hold, ranges outside the rows: not written. Lengths below the tree's size."""
    import torch
    log("case masks left out")
    parents = torch.arange(-1, 99, dtype=torch.int32, device="cuda") % 60
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for offs, ctx in (([0, 10, 75, 100], [3, 100, 50]), ([-2, 10, 90, 101], [5, 5, 5]), ([10, 74, 74, 80], [2 ** 31 - 1, -9, 0])):
        masks, positions, written = so.tree_masks(parents.cpu().numpy(), offs, ctx, 1, 100)
        m, p = torch.full((100, 1), 7, dtype=torch.int64, device="cuda"), torch.full((100,), 7, dtype=torch.int32, device="cuda")
        fb.fluxbin_tree_masks(parents, ints(offs), ints(ctx), 1, masks=m, positions=p)
        m, p = m.cpu().numpy(), p.cpu().numpy()
        assert np.array_equal(m[written], so.packed(masks)[written]) and np.array_equal(p[written], positions[written])
        assert (m[~written] == 7).all() and (p[~written] == 7).all()


# ---------------------------------------------------------------------------------------------- attention

@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,G", [(1, 1), (2, 4), (1, 7), (3, 8), (1, 40)])
def test_trees(fb, H, G, D):
    """Trees of one node to many, over histories of none to many tokens."""
    log(f"case tree H={H} G={G} D={D}")
    s = Trees(fb, 6, H, D, 32, 500, seed=H + G + D)
    s.append([0, 15, 64, 65, 300, 400])
    new = [3, 1, 64, 33, 17, 70]
    s.append(new)
    s.verify(new, G)


@pytest.mark.parametrize("P", [16, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 5, 40, 10 ** 9])
def test_windows(fb, P, window):
    log(f"case tree P={P} window={window}")
    s = Trees(fb, 5, 2, 64, P, 300, seed=P)
    new = [3, 0, 50, 1, 90]
    s.append([140, 0, 20, 150, 61])
    s.append(new)
    s.verify(new, 4, window=window)
    s.verify(new, 4, window=window, masks=s.rng.random((sum(new), 128)) < 0.3, words=2)   # any mask, also of later rows


@pytest.mark.parametrize("window", [0, 7])
def test_empty_rows(fb, window):
    """Masks that leave a row nothing, rows at positions before 0, a missing page, a sequence of no tokens."""
    log(f"case tree empty rows window={window}")
    s = Trees(fb, 4, 2, 64, 16, 64, seed=12)
    s.append([9, 3, 16, 0])
    s.table[2, 0] = -1
    new = [9, 6, 16, 2]
    masks = s.masks(new, 1)
    masks[2], masks[9:12], masks[20] = False, False, True   # bits behind the tree name nobody
    got = s.verify(new, 2, masks=masks, window=window)
    assert (got[2] == 0).all() and (got[9:12] == 0).all() and (got[15:] == 0).all() and (got[0] != 0).any()


def test_left_out(fb):
    """A tree of more rows than the masks hold is left out; its rows stay as they were."""
    log("case tree left out")
    s = Trees(fb, 3, 1, 64, 16, 200, seed=13)
    s.append([20, 10, 5])
    new = [10, 70, 64]
    s.append(new)
    s.verify(new, 2, masks=s.rng.random((144, 64)) < 0.5, words=1)


@pytest.mark.parametrize("H,G,D,P,new,ctx", [
    (1, 8, 128, 64, [16, 13], [20000, 9000]), (2, 8, 64, 16, [200, 1, 64], [3000, 900, 64]), (8, 8, 128, 64, [64] * 4, [700, 1500, 64, 300]),
    (2, 1, 256, 32, [130], [1700]), (8, 4, 256, 64, [100, 40, 9], [1200, 50, 900]), (40, 1, 128, 128, [128, 33], [400, 2100]),
    (1, 2, 64, 64, [8] * 300, [40] * 300), (1, 1, 128, 64, [1024], [1500]),
    (2, 8, 128, 64, [4, 3], [5000, 1000]), (2, 8, 64, 16, [1, 5], [3000, 1300]),            # two columns tiles or fewer
    (2, 8, 128, 64, [6, 7], [3000, 1200]), (2, 8, 64, 32, [5, 8, 0], [2500, 1100, 40]),     # up to 64 columns
    (8, 8, 128, 16, [5] * 40, [100] * 40), (8, 4, 64, 32, [12] * 39 + [3], [200] * 40),     # short tables, many items
    (8, 8, 128, 64, [16] * 40, [90] * 40), (8, 16, 64, 16, [9] * 40, [70] * 40), (8, 4, 256, 64, [9] * 40, [120] * 40),
    (1, 4, 256, 64, [20], [9000]), (1, 8, 64, 64, [10], [9000]), (1, 8, 64, 32, [6], [9000]), (1, 8, 128, 64, [6], [9000]),   # parts
    (2, 4, 256, 64, [4] * 3, [5000, 1000, 300]), (8, 4, 256, 64, [3] * 4, [4096, 1000, 20, 3]),     # up to 16 columns of 256
    (8, 2, 256, 64, [2] * 64, [4100] + [70] * 63), (8, 8, 128, 64, [3] * 40, [3000] + [90] * 39), (8, 8, 64, 64, [3] * 40, [3000] + [90] * 39)])
def test_large(fb, H, G, D, P, new, ctx):
    """Long histories over many workgroups, many columns, many sequences; the workspace holds NaN where nothing was written."""
    log(f"case tree large H={H} G={G} D={D} new={new[:4]} ctx={ctx[:4]}")
    s = Trees(fb, len(new), H, D, P, max(ctx), seed=14)
    s.append([c - n for c, n in zip(ctx, new)])
    s.append(new)
    ws = fb.make_kv8_tree_workspace(s.cache, sum(new), len(new), H * G)
    ws.fill_(0xFF)
    assert np.isfinite(s.verify(new, G, ws=ws)).all()
    ws.fill_(0xFF)
    s.verify(new, G, ws=ws, window=60)


@pytest.mark.parametrize("H,G,D,P,new,ctx", [
    (1, 8, 64, 64, [6, 7], [17000, 900]), (1, 8, 64, 32, [16, 10], [17000, 3000]),          # 64 and 128 columns a workgroup
    (1, 8, 128, 64, [5, 8], [17000, 16600]), (1, 16, 128, 128, [40], [18000]),
    (1, 4, 256, 64, [20, 6], [17000, 400]), (2, 4, 256, 32, [3, 4], [17000, 3000])])        # one kernel of 256, up to 16 columns too
def test_many_parts(fb, H, G, D, P, new, ctx):
    """Few items of long histories, with a hundred parts and more, which 16 wavefronts join; a window that leaves as many, one
    that leaves few."""
    log(f"case tree many parts H={H} G={G} D={D} new={new} ctx={ctx}")
    s = Trees(fb, len(new), H, D, P, max(ctx), seed=49)
    s.append([c - n for c, n in zip(ctx, new)])
    s.append(new)
    ws = fb.make_kv8_tree_workspace(s.cache, sum(new), len(new), H * G)
    for window in (0, 16900, 60):
        ws.fill_(0xFF)
        assert np.isfinite(s.verify(new, G, ws=ws, window=window)).all()


def test_bad_pages_and_lengths(fb):
    log("case tree bad pages")
    s = Trees(fb, 5, 2, 64, 16, 64, seed=11)
    s.append([40, 64, 20, 33, 64])
    s.table[0, 1], s.table[1, 3], s.table[1, 0] = -1, s.pages, 2 ** 31 - 1
    context = np.array([42, 70, 3, -5, 2 ** 31 - 1], np.int32)
    near = np.array([42, 70, 3, 0, 94])
    q = (s.rng.standard_normal((20, 4, 64))).astype(np.float16)
    k, v = s.rows(20, 3.0)
    masks = s.rng.random((20, 64)) < 0.6
    for offs in ([0, 4, 10, 16, 18, 20], [-3, 4, 10, 16, 18, 25]):
        fb.fluxbin_kv8_append(s.cache, s.dev(k), s.dev(v), *s.arrays(offs, context))
        s.plain.append(k, v, offs, near, s.table)
        for window in (0, 9):
            out = s.torch.full((20, 4, 64), 7.0, dtype=s.torch.float16, device="cuda")
            fb.fluxbin_kv8_tree_attention(s.cache, s.dev(q), s.dev(so.packed(masks)), *s.arrays(offs, context), out=out, window=window)
            # a length past what a plain form writes out: nothing there has a page, with the tree behind it
            ref, mag, big, peak, written = s.plain.tree_attention(q, masks, offs, near, s.table, 0.125, window)
            got = out.cpu().double().numpy()
            assert (got[~written] == 7).all()
            some = written.copy()
            if window:
                some[offs[4]:min(offs[5], 20)] = False
            assert (np.abs(got - ref)[some] <= qo.attention_bound(ref, mag, big, peak, 128)[some]).all()
    fb.fluxbin_kv8_tree_attention(s.cache, s.dev(q), s.dev(so.packed(masks)), *s.arrays([0, 10, 4, 20, 9, 20], context))
    s.torch.cuda.synchronize()


def test_chain_is_causal(fb):
    """A chain's masks give what causal attention gives."""
    log("case tree chain")
    s = Trees(fb, 3, 2, 128, 64, 400, seed=21)
    new = [5, 64, 100]
    s.append([300, 0, 77])
    s.append(new)
    chain = np.concatenate([np.arange(-1, n - 1) for n in new]).astype(np.int32)
    q = (s.rng.standard_normal((sum(new), 8, 128)) * 1.5).astype(np.float16)
    for window in (0, 3, 90):
        a = s.verify(new, 4, masks=s.masks(new, 2, chain), words=2, q=q, window=window)
        b = s.attend(new, 4, q=q, window=window)
        assert qo.attention_apart(a, b) <= qo.APART


def test_precision(fb):
    """As precise as fp32 arithmetic with weights of two fp16 numbers is, with few columns and with many."""
    log("case tree precision")
    for H, G, new in ((8, 1, [9, 16]), (8, 8, [64, 40])):
        s = Trees(fb, 2, H, 128, 64, 1500, seed=22)
        s.append([1400, 900])
        s.append(new)
        masks = s.masks(new, 1)
        q = (s.rng.standard_normal((sum(new), H * G, 128)) * 1.5).astype(np.float16)
        got = s.verify(new, G, masks=masks, q=q)
        offsets = np.concatenate([[0], np.cumsum(new)])
        ref = s.plain.tree_attention(q, masks, offsets, s.length, s.table, 128 ** -0.5)[0]
        apart = qo.attention_apart(got, ref)
        log(f"  apart {apart:.2e}, may be {qo.APART:.2e}")
        assert apart <= qo.APART


def test_scales_far_apart(fb):
    log("case tree, scales far apart")
    s = Trees(fb, 1, 1, 64, 16, 256, seed=15)
    for scale in (1e-7, 6e4, 1.0, 0.0, 1e-3, 6e4, 1e-7, 1.0):
        s.append([16], 1.0, lambda k, v, scale=scale: v.__imul__(np.float16(scale)))
    for n in (8, 40):
        q = (s.rng.standard_normal((n, 4, 64)) * 0.5).astype(np.float16)
        k, _ = s.plain.values(0, 0, 128, s.table)
        for i in range(8):
            q[i, 0] = (k[16 * i + 3, 0] * 8).astype(np.float16)
            q[i, 1] = (k[16 * i, 0] * 0.1).astype(np.float16)
        for scale in (None, 0.0, -0.1):
            s.verify([n], 4, q=q, scale=scale)
        s.verify([n], 4, q=q * np.float16(20), scale=0.3)


@pytest.mark.parametrize("H,G,D,new,ctx", [(2, 4, 64, [5, 9, 3], [300, 20, 77]), (8, 8, 128, [40, 33, 64], [1400, 1200, 1000]),
                                           (2, 8, 128, [7, 6, 5], [1400, 1200, 1000]), (4, 4, 256, [20, 30, 9], [1100, 1000, 20])])
def test_queries_not_finite(fb, H, G, D, new, ctx):
    """NaN and infinities in a query stay in its row and head, with pages missing and masks that leave rows nothing."""
    log(f"case tree queries not finite H={H} G={G} D={D}")
    s = Trees(fb, 3, H, D, 32, max(ctx), seed=46)
    s.append([c - n for c, n in zip(ctx, new)])
    s.append(new)
    s.table[1, :] = -1
    masks = s.masks(new, 1)
    masks[1] = False
    q = (s.rng.standard_normal((sum(new), H * G, D))).astype(np.float16)
    clean = s.verify(new, G, masks=masks, q=q, words=1)
    bad = q.copy()
    rows = [0, new[0], sum(new) - 1]
    bad[rows[0], 0, 3], bad[rows[1], 1, :] = np.nan, np.inf
    bad[rows[2], H * G - 1, 5] = -np.inf
    offsets = np.concatenate([[0], np.cumsum(new)])
    got = fb.fluxbin_kv8_tree_attention(s.cache, s.dev(bad), s.dev(so.packed(masks)), *s.arrays(offsets, s.length)).cpu().double().numpy()
    assert np.isnan(got[rows[0], 0]).all() and not np.isfinite(got[rows[2], H * G - 1]).any()
    assert (got[new[0]:new[0] + new[1]] == 0).all()      # no page: nothing is attended, whatever the query
    for r, h in ((rows[0], 0), (rows[2], H * G - 1)):
        got[r, h] = clean[r, h]
    assert np.array_equal(got, clean)


@pytest.mark.parametrize("H,G,D,n", [(2, 2, 64, 12), (8, 8, 128, 40), (2, 8, 128, 6), (4, 4, 256, 30)])
def test_captured(fb, H, G, D, n):
    """A captured step over lengths and trees that change between replays, on a workspace that an eager call uses too; each
    replay is what the eager call gives. Then on another stream."""
    import torch
    log(f"case tree captured H={H} G={G} D={D} n={n}")
    s = Trees(fb, 3, H, D, 64, 2000, seed=47)
    s.append([2000, 2000, 2000])      # every position that a replay may read is stored
    T, context = 3 * n, s.ints([0, 0, 0])
    offsets, _, table = s.arrays(np.arange(0, T + 1, n), s.length)
    q, k, v = (torch.zeros(T, h, D, dtype=torch.float16, device="cuda") for h in (H * G, H, H))
    masks, ws = torch.zeros(T, 1, dtype=torch.int64, device="cuda"), fb.make_kv8_tree_workspace(s.cache, T, 3, H * G)
    step = lambda out, stream=None: fb.fluxbin_kv8_tree_attention(s.cache, q, masks, offsets, context, table, out=out, workspace=ws, stream=stream)
    out = torch.zeros_like(q)
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fb.fluxbin_kv8_append(s.cache, k, v, offsets, context, table)
        step(out)
    for i in range(5):
        new = np.array([n] * 3)
        s.length = np.array([[1500, 200, 900], [64, 1800, 0], [700, 700, 1900], [1, 1, 1], [1300, 0, 30]][i]) + n
        context.copy_(s.ints(s.length))
        m = s.masks(new, 1)
        masks.copy_(s.dev(so.packed(m)))
        for x in (q, k, v):
            x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        captured = out.clone()
        eager = step(torch.full_like(q, 9.0))
        torch.cuda.synchronize()
        assert torch.equal(captured, eager), i
    side = torch.cuda.Stream()
    other = torch.full_like(q, 9.0)
    torch.cuda.synchronize()
    step(other, side)
    side.synchronize()
    assert torch.equal(other, eager)


def test_cache_past_32_bits(fb):
    """Pages whose codes lie past 2^32 bytes: attention of trees with few columns and many, kept rows, copies."""
    import torch
    log("case tree large cache")
    H, D, P, pages = 8, 128, 64, 70000
    assert pages * H * D * P > 2 ** 32
    s = Trees(fb, 2, H, D, P, 3 * P, seed=48)
    s.cache = None
    s.cache = fb.make_kv8_cache(pages, P, H, D)
    low = s.table
    high = np.array([[pages - 1, 0, pages - 2], [pages // 2, pages - 3, 65536]], np.int32)
    k, v = s.rows(250)
    offs, lengths, new = [0, 150, 250], np.array([150, 100]), np.array([40, 40])
    a = s.ints(offs), s.ints(lengths), s.ints(high)
    fb.fluxbin_kv8_append(s.cache, s.dev(k), s.dev(v), *a)
    s.plain.append(k, v, offs, lengths, low)
    rows = np.array([0, 40, 80])
    s.length = lengths
    for G in (1, 8):
        q = s.rng.standard_normal((80, H * G, D)).astype(np.float16)
        masks = s.masks(new, 1)
        out = fb.fluxbin_kv8_tree_attention(s.cache, s.dev(q), s.dev(so.packed(masks)), s.ints(rows), a[1], a[2]).cpu().double().numpy()
        ref, mag, big, peak, _ = s.plain.tree_attention(q, masks, rows, lengths, low, D ** -0.5)
        assert (np.abs(out - ref) <= qo.attention_bound(ref, mag, big, peak, 150)).all()
    keep = np.concatenate([np.arange(1, 41, 3), np.zeros(26), np.arange(40)]).astype(np.int32)
    fb.fluxbin_kv8_keep(s.cache, s.dev(keep), s.ints([14, 40]), s.ints(rows), a[1], a[2])
    s.plain.keep(keep, [14, 40], rows, lengths, low, 80)
    lengths = np.array([124, 100])
    for copy in (False, True):
        if copy:   # the first sequence's pages to others, and its table with them
            fb.fluxbin_kv8_copy_pages(s.cache, s.ints([[pages - 1, 1], [0, pages - 5]]))
            high[0, :2] = 1, pages - 5
        kt, vt = fb.fluxbin_kv8_read(s.cache, s.ints([0, 124, 224]), s.ints(lengths), s.ints(high), 224)
        pk, pv, _ = s.plain.read([0, 124, 224], lengths, low, 224)
        assert np.array_equal(kt.cpu().numpy(), pk) and np.array_equal(vt.cpu().numpy(), pv)
    s.cache = None
    torch.cuda.empty_cache()


def test_attention_refusals(fb):
    log("case tree refusals")
    s = Trees(fb, 1, 2, 64, 16, 64, seed=19)
    s.append([20])
    q = s.dev(s.rng.standard_normal((3, 4, 64)).astype(np.float16))
    a, n = s.arrays([0, 3], s.length), fb.fluxbin_kv8_tree_workspace_query(s.cache, 3, 1, 4)
    m = s.torch.ones(3, 1, dtype=s.torch.int64, device="cuda")
    for ws in (s.torch.empty(n - 1, dtype=s.torch.uint8, device="cuda"), s.torch.empty(n + 8, dtype=s.torch.uint8, device="cuda")[8:],
               s.torch.empty(n, dtype=s.torch.uint8), s.cache.buf):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_tree_attention(s.cache, q, m, *a, workspace=ws)
    for bad in (m.int(), m[:2], m.cpu(), m[:, 0], m.expand(3, 17).contiguous(), m.expand(3, 2), m[:, :0]):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_tree_attention(s.cache, q, bad, *a)
    for kw in (dict(window=-1), dict(out=q), dict(out=q[:2]), dict(scale=float("nan"))):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_tree_attention(s.cache, q, m, *a, **kw)
    assert fb.fluxbin_kv8_tree_attention(s.cache, q[:0], m[:0], *s.arrays([0, 0], s.length)).shape == (0, 4, 64)


# ---------------------------------------------------------------------------------------------- kept rows

def _keep(s, new, kept_rows):
    """kept_rows[b]: the indices that sequence b keeps."""
    offsets = np.concatenate([[0], np.cumsum(new)])
    keep = np.full(int(offsets[-1]), -7, np.int32)
    for b, rows in enumerate(kept_rows):
        keep[offsets[b]:offsets[b] + len(rows)] = rows
    kept = np.array([len(r) for r in kept_rows], np.int32)
    s.fb.fluxbin_kv8_keep(s.cache, s.dev(keep), s.dev(kept), *s.arrays(offsets, s.length))
    s.plain.keep(keep, kept, offsets, s.length, s.table, int(offsets[-1]))
    s.length = s.length - np.array(new) + kept


@pytest.mark.parametrize("P", [16, 32, 64, 256])
@pytest.mark.parametrize("H,D", [(1, 64), (3, 128), (2, 256)])
def test_keep(fb, H, D, P):
    """Paths of trees over page borders, pages whose scales are larger or smaller than those of the rows that come, all rows,
    none; then more rows behind them."""
    log(f"case keep H={H} D={D} P={P}")
    s = Trees(fb, 6, H, D, P, 8 * P + 700, seed=P + D)
    s.append([0, 5, P - 3, P, 2 * P + 1, P + P // 2])
    for scale in (1.0, 3.0, 0.2, 50.0):
        new = [2 * P + 3, 20, 30, 1, 3 * P, 60]
        s.append(new, scale, lambda k, v: (k.__imul__(s.rng.random((len(k), 1, 1)).astype(np.float16) * 4)))
        path = lambda n, p: np.flatnonzero(s.rng.random(n) < p)
        _keep(s, new, [path(new[0], 0.6), path(20, 0.2), [], [0], path(3 * P, 0.9), range(60)])
        s.check()
    s.append([1, 3, 2, 1, 0, 5])
    s.check()


@pytest.mark.parametrize("P", [16, 128, 256])
def test_keep_many_sequences(fb, P):
    """As many workgroups as no longer run at a time."""
    log(f"case keep of many sequences P={P}")
    B = 700
    s = Trees(fb, B, 2, 64, P, P + 60, seed=P)
    s.append(s.rng.integers(0, P, B))
    new = s.rng.integers(0, 50, B)
    s.append(new, 2.0, lambda k, v: (k.__imul__(s.rng.random((len(k), 1, 1)).astype(np.float16) * 4)))
    _keep(s, new, [np.flatnonzero(s.rng.random(n) < 0.4) for n in new])
    s.check()


@pytest.mark.parametrize("D", [128, 256])
def test_keep_many_sequences_of_larger_heads(fb, D):
    log(f"case keep of many sequences D={D}")
    B = 530
    s = Trees(fb, B, 2, D, 32, 90, seed=D)
    s.append(s.rng.integers(0, 32, B))
    new = s.rng.integers(0, 50, B)
    s.append(new, 2.0, lambda k, v: (k.__imul__(s.rng.random((len(k), 1, 1)).astype(np.float16) * 4)))
    _keep(s, new, [np.flatnonzero(s.rng.random(n) < 0.4) for n in new])
    s.check()


def test_keep_special(fb):
    """Rows at positions before 0, missing pages on either side, counts past the rows, zero scales, ranges left out."""
    log("case keep special")
    s = Trees(fb, 5, 2, 64, 16, 100, seed=31)
    s.append([40, 40, 40, 40, 40], 0.0)
    s.append([30, 30, 30, 30, 30])
    s.table[1, 3], s.table[2, 4] = -1, s.pages + 5
    good = s.table
    kept = np.array([40, 5, 6, -3, 9], np.int32)
    for offs in ([0, 20, 40, 60, 80, 100], [-1, 20, 40, 60, 80, 101]):
        keep = np.concatenate([np.sort(s.rng.permutation(20)[:20]) if b == 0 else np.concatenate([np.sort(s.rng.permutation(20)[:10]), np.full(10, 99)])
                               for b in range(5)]).astype(np.int32)
        context = np.array([15, 70, 70, 70, 70], np.int32)
        s.fb.fluxbin_kv8_keep(s.cache, s.dev(keep), s.dev(kept), *s.arrays(offs, context))
        s.plain.keep(keep, kept, offs, context, good, 100)
        s.length = np.array([0, 48, 56, 50, 59])
        s.check()


def test_keep_bad_entries(fb):
    """Entries that fall, repeat or are no rows: only their own sequence's positions are touched."""
    log("case keep bad entries")
    s = Trees(fb, 3, 2, 128, 16, 100, seed=32)
    s.append([33, 33, 33])
    s.append([40, 40, 40])
    keep = np.zeros(120, np.int32)
    keep[:40], keep[40:80], keep[80:] = np.arange(40), s.rng.integers(-50, 90, 40), np.arange(0, 80, 2)
    s.fb.fluxbin_kv8_keep(s.cache, s.dev(keep), s.dev(np.array([40, 40, 20], np.int32)), *s.arrays([0, 40, 80, 120], s.length))
    s.plain.keep(keep, [40, 0, 20], [0, 40, 80, 120], s.length, s.table, 120)
    s.length = np.array([73, 0, 53])
    s.check()


def test_keep_refusals(fb):
    log("case keep refusals")
    s = Trees(fb, 2, 2, 64, 16, 64, seed=33)
    s.append([20, 20])
    keep, kept, a = s.ints([0, 1, 0, 1]), s.ints([2, 2]), s.arrays([0, 2, 4], s.length)
    for bad in ((keep.long(), kept), (keep.cpu(), kept), (keep[None], kept), (keep, kept[:1]), (keep, kept.cpu()), (keep[::2], kept)):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_keep(s.cache, *bad, *a)
    fb.fluxbin_kv8_keep(s.cache, keep[:0], kept, *s.arrays([0, 0, 0], s.length))
    s.check()
