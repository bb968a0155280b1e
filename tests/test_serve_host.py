"""Host-side checks of include/fluxbin_serve.h: entry points, sizes and refusals, before any launch, and the oracle's own
pins. CPU only."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import serve_oracle as so

fb = pytest.importorskip("paper_2608_15602_amd.fluxbin")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INV, UNS, SMALL = fb.FLUXBIN_ERR_INVALID_ARG, fb.FLUXBIN_ERR_UNSUPPORTED, fb.FLUXBIN_ERR_BUFFER_TOO_SMALL
A = [(i + 1) << 32 for i in range(8)]   # addresses that no launch ever sees


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fb.LIB_PATH):
        pytest.fail("libfluxbin.so is not built; run `python -m paper_2608_15602_amd.build`")
    return fb.lib()


def test_exports_every_declared_function(L):
    with open(os.path.join(ROOT, "include", "fluxbin_serve.h")) as f:
        names = set(re.findall(r"^fluxbin_status (fluxbin_\w+)\(", f.read(), re.M))
    assert names == set(fb.SERVE_EXPORTS)
    for n in names:
        assert hasattr(L, n), n


# ---------------------------------------------------------------------------------------------- rotation

def _rotate(L, rotary={}, **kw):
    r = fb.Rotary(128, 64, 0, 0, 1e-6, 1.0, A[0], A[0] + 4096, A[0] + 8192)
    for k, v in rotary.items():
        setattr(r, k, v)
    a = dict(rows=10, pos=A[0] + 16384, qh=8, q=A[1], qts=8 * 128, qhs=128, qo=A[2], qots=8 * 128, qohs=128, kh=2, k=A[3], kts=256,
             khs=128, ko=A[4], kots=256, kohs=128)
    a.update(kw)
    return L.fluxbin_qk_rotate(ctypes.byref(r), a["rows"], a["pos"], a["qh"], a["q"], a["qts"], a["qhs"], a["qo"], a["qots"],
                               a["qohs"], a["kh"], a["k"], a["kts"], a["khs"], a["ko"], a["kots"], a["kohs"], None)


FUSED = dict(q=A[1], qts=1536, k=A[1] + 2048, kts=1536)   # rows of 8 + 2 + 2 heads of 128


@pytest.mark.parametrize("kw,status", [
    (dict(rotary=dict(head_dim=0)), INV), (dict(rotary=dict(head_dim=80)), UNS), (dict(rotary=dict(rotary_dim=-16)), INV),
    (dict(rotary=dict(rotary_dim=144)), INV), (dict(rotary=dict(rotary_dim=24)), UNS), (dict(rotary=dict(interleaved=2)), INV),
    (dict(rotary=dict(eps=-1.0)), INV), (dict(rotary=dict(eps=float("nan"))), INV), (dict(rotary=dict(magnitude=float("inf"))), INV),
    (dict(rotary=dict(d_frequencies=None)), INV), (dict(rotary=dict(d_frequencies=A[0] + 2)), INV),
    (dict(rotary=dict(d_k_weight=A[0] + 1)), INV), (dict(rows=-1), INV), (dict(rows=(1 << 22) + 1), INV), (dict(qh=0), INV),
    (dict(qh=1025), INV), (dict(kh=-1), INV), (dict(kh=1025), INV), (dict(rows=1 << 22, qh=512), UNS), (dict(pos=None), INV),
    (dict(pos=A[0] + 1), INV), (dict(q=None), INV), (dict(qo=None), INV), (dict(k=None), INV), (dict(ko=A[4] + 1), INV),
    (dict(qhs=100), INV), (dict(qots=1000), INV), (dict(kots=0), INV),
    (dict(qo=A[1] + 2), INV), (dict(qo=A[1], qots=1280), INV), (dict(ko=A[2]), INV), (dict(qo=A[3]), INV), (dict(ko=A[1] + 256), INV),
    (dict(qo=A[0]), INV), (dict(ko=A[0] + 8192), INV), (dict(qo=A[0] + 16384 - 4), INV),
    # fused rows: an output that reaches into the other side's columns
    (dict(FUSED, qo=A[1] + 256, qots=1536), INV), (dict(FUSED, ko=A[1] + 2046, kots=1536), INV),
    (dict(FUSED, qo=A[1] + 2304, qots=1536), INV)])
def test_rotate_refused(L, kw, status):
    assert _rotate(L, **kw) == status
    assert L.fluxbin_last_error_message()


def test_rotate_no_rows(L):
    assert _rotate(L, rows=0, q=None, k=None, qo=None, ko=None, pos=None) == 0
    assert L.fluxbin_qk_rotate(None, 0, None, 1, None, 0, 0, None, 0, 0, 0, None, 0, 0, None, 0, 0, None) == INV


# ---------------------------------------------------------------------------------------------- trees

def _masks(L, **kw):
    a = dict(rows=10, B=2, off=A[0], ctx=A[0] + 4096, par=A[1], words=2, masks=A[2], pos=A[3])
    a.update(kw)
    return L.fluxbin_tree_masks(a["rows"], a["B"], a["off"], a["ctx"], a["par"], a["words"], a["masks"], a["pos"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INV), (dict(rows=(1 << 22) + 1), INV), (dict(B=0), INV), (dict(B=65536), INV), (dict(off=None), INV),
    (dict(ctx=None), INV), (dict(par=None), INV), (dict(masks=None), INV), (dict(words=0), INV), (dict(words=17), UNS),
    (dict(masks=A[2] + 4), INV), (dict(pos=A[3] + 2), INV), (dict(par=A[1] + 1), INV), (dict(pos=A[1]), INV), (dict(masks=A[0]), INV),
    (dict(pos=A[2] + 156), INV)])
def test_masks_refused(L, kw, status):
    assert _masks(L, **kw) == status
    assert L.fluxbin_last_error_message()


def _cache(**kw):
    d = fb.Kv8CacheDesc(100, 64, 8, 128, 1, 1 << 30, 1 << 26)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _batch(**kw):
    b = fb.Kv8Batch(10, 2, 5, 5, A[0], A[0] + 4096, A[0] + 8192)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


BAD = [(dict(cache=dict(format_version=0)), INV), (dict(cache=dict(d_base=None)), INV), (dict(cache=dict(bytes=1000)), SMALL),
       (dict(batch=dict(rows=-1)), INV), (dict(batch=dict(sequences=0)), INV), (dict(batch=dict(block_table_stride=4)), INV),
       (dict(batch=dict(d_offsets=None)), INV)]


def _tree(L, cache={}, batch={}, **kw):
    a = dict(heads=64, q=A[1], qt=8192, qh=128, out=A[2], ot=8192, oh=128, scale=0.1, masks=A[4], words=2, window=0, ws=A[3],
             bytes=1 << 30)
    a.update(kw)
    return L.fluxbin_kv8_tree_attention(ctypes.byref(_cache(**cache)), ctypes.byref(_batch(**batch)), a["heads"], a["q"], a["qt"],
                                        a["qh"], a["out"], a["ot"], a["oh"], a["scale"], a["masks"], a["words"], a["window"],
                                        a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(heads=0), INV), (dict(heads=63), INV), (dict(heads=1032), INV), (dict(scale=float("nan")), INV), (dict(words=0), INV),
    (dict(words=17), UNS), (dict(window=-1), INV), (dict(masks=None), INV), (dict(masks=A[4] + 4), INV), (dict(q=None), INV),
    (dict(out=None), INV), (dict(ot=0), INV), (dict(heads=1024, batch=dict(rows=1 << 22), cache=dict(kv_heads=1)), UNS)])
def test_tree_attention_refused(L, kw, status):
    assert _tree(L, **kw) == status
    assert L.fluxbin_last_error_message()


def _keep(L, cache={}, batch={}, keep=A[1], kept=A[2]):
    return L.fluxbin_kv8_keep(ctypes.byref(_cache(**cache)), ctypes.byref(_batch(**batch)), keep, kept, None)


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(keep=None), INV), (dict(kept=None), INV), (dict(keep=A[1] + 2), INV), (dict(kept=A[2] + 1), INV), (dict(keep=1 << 30), INV),
    (dict(kept=(1 << 30) + 64), INV)])
def test_keep_refused(L, kw, status):
    assert _keep(L, **kw) == status
    assert L.fluxbin_last_error_message()


def test_no_rows(L):
    assert _masks(L, rows=0, par=None, masks=None, pos=None) == 0
    assert _keep(L, batch=dict(rows=0), keep=None) == 0


# ---------------------------------------------------------------------------------------------- pages

def _pool(**kw):
    p = fb.PagePoolDesc(1000, 64, 0, A[5])
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_POOL = [(dict(pool=dict(pages=0)), INV), (dict(pool=dict(pages=(1 << 24) + 1)), INV), (dict(pool=dict(page_size=0)), INV),
            (dict(pool=dict(page_size=48)), UNS), (dict(pool=dict(d_state=None)), INV), (dict(pool=dict(d_state=A[5] + 8)), INV),
            (dict(B=0), INV), (dict(B=65536), INV), (dict(blocks=0), INV), (dict(blocks=(1 << 24) + 1), INV), (dict(stride=9), INV),
            (dict(table=None), INV), (dict(table=A[0] + 2), INV)]


def _resize(L, pool={}, **kw):
    a = dict(B=3, blocks=10, table=A[0], stride=10, tokens=A[1])
    a.update(kw)
    return L.fluxbin_pages_resize(ctypes.byref(_pool(**pool)), a["B"], a["blocks"], a["table"], a["stride"], a["tokens"], None)


@pytest.mark.parametrize("kw,status", BAD_POOL + [
    (dict(tokens=None), INV), (dict(tokens=A[1] + 1), INV), (dict(tokens=A[0] + 116), INV), (dict(table=A[5] + 4012), INV)])
def test_resize_refused(L, kw, status):
    assert _resize(L, **kw) == status
    assert L.fluxbin_last_error_message()


def _fork(L, pool={}, **kw):
    a = dict(B=3, blocks=10, table=A[0], stride=10, ctx=A[1], C=4, cblocks=12, child=A[2], cstride=12, source=A[3], copies=A[4])
    a.update(kw)
    return L.fluxbin_pages_fork(ctypes.byref(_pool(**pool)), a["B"], a["blocks"], a["table"], a["stride"], a["ctx"], a["C"],
                                a["cblocks"], a["child"], a["cstride"], a["source"], a["copies"], None)


@pytest.mark.parametrize("kw,status", BAD_POOL + [
    (dict(C=0), INV), (dict(C=65536), INV), (dict(cblocks=0), INV), (dict(cstride=11), INV), (dict(child=None), INV), (dict(ctx=None), INV),
    (dict(source=None), INV), (dict(copies=None), INV), (dict(copies=A[4] + 4), INV), (dict(child=A[0]), INV), (dict(child=A[3]), INV),
    (dict(copies=A[2] + 184), INV), (dict(child=A[5]), INV), (dict(ctx=A[2] + 188), INV)])
def test_fork_refused(L, kw, status):
    assert _fork(L, **kw) == status
    assert L.fluxbin_last_error_message()


def _copy(L, to={}, source={}, n=5, copies=A[1]):
    return L.fluxbin_kv8_copy_pages(ctypes.byref(_cache(**to)), ctypes.byref(_cache(**source)), n, copies, None)


@pytest.mark.parametrize("kw,status", [
    (dict(to=dict(format_version=2)), INV), (dict(source=dict(d_base=None)), INV), (dict(to=dict(page_size=32)), INV),
    (dict(source=dict(kv_heads=4)), INV), (dict(to=dict(head_dim=64)), INV), (dict(n=-1), INV), (dict(n=(1 << 22) + 1), INV),
    (dict(copies=None), INV), (dict(copies=A[1] + 4), INV), (dict(copies=1 << 30), INV), (dict(to=dict(pages=50)), INV),
    (dict(to=dict(d_base=(1 << 30) + 4096)), INV)])
def test_copy_refused(L, kw, status):
    assert _copy(L, **kw) == status
    assert L.fluxbin_last_error_message()


def test_copy_nothing(L):
    assert _copy(L, n=0, copies=None) == 0
    assert _copy(L, n=0, to=dict(d_base=A[6], pages=50)) == 0


# ---------------------------------------------------------------------------------------------- binding

def test_binding_refuses_what_does_not_fit():
    """No device here: every refusal comes before a launch."""
    import torch
    from types import SimpleNamespace
    meta = lambda *size, dtype=torch.int32: torch.empty(size, dtype=dtype, device="meta")
    for call in (lambda: fb.make_page_pool((1 << 32) + 5, 64, "cpu"), lambda: fb.make_page_pool(0, 64, "cpu"),
                 lambda: fb.make_page_pool(9, 1 << 40, "cpu"),
                 lambda: fb.make_rotary(128, torch.zeros(64)), lambda: fb.make_rotary(1 << 40, torch.zeros(64)),
                 lambda: fb.fluxbin_tree_masks(torch.zeros(4, dtype=torch.int32), None, None, 1)):
        with pytest.raises(fb.FluxbinError) as e:
            call()
        assert e.value.status == INV
    pool = SimpleNamespace(index=-1, use=SimpleNamespace(int32=torch.int32, current_device=lambda: -1), device="meta")
    for table in (meta(4, 5, dtype=torch.int64), meta(4), meta(5, 4).t(), meta((1 << 32) + 1, 1), meta(1, (1 << 32) + 5)):
        with pytest.raises(fb.FluxbinError):
            fb._page_table(pool, "table", table)
    assert fb._page_table(pool, "table", meta(1, 5)) == (1, 5, 5) and fb._page_table(pool, "table", meta(6, 9)[::2, :5]) == (3, 5, 18)
    plan = SimpleNamespace(index=-1, head_dim=64, device="meta", use=SimpleNamespace(half=torch.float16))
    for q in (meta(2, 8, 64), meta(2, 8, 128, dtype=torch.float16), meta(2, 64, 8, dtype=torch.float16).transpose(1, 2),
              meta(8, 64, dtype=torch.float16)):
        with pytest.raises(fb.FluxbinError):
            fb._heads(plan, "q", q)


# ---------------------------------------------------------------------------------------------- the oracle's pins

def test_oracle_rotation():
    """A quarter turn, by hand; turning keeps a pair's length; positions add up."""
    x = np.arange(1, 65, dtype=np.float16).reshape(1, 1, 64)
    y, _ = so.rotate(x, np.array([1]), np.full(32, np.pi / 2), interleaved=True)
    assert np.allclose(y[0, 0, :4], [-2, 1, -4, 3])
    y, _ = so.rotate(x, np.array([1]), np.full(16, np.pi / 2))
    assert np.allclose(y[0, 0, :2], [-17, -18]) and np.allclose(y[0, 0, 16:18], [1, 2]) and (y[0, 0, 32:] == x[0, 0, 32:]).all()
    y, _ = so.rotate(x, np.array([7]), np.zeros(0), weight=np.full(64, 2.0), eps=0.0)
    assert np.allclose((y / 2) ** 2 @ np.ones(64) / 64, 1)


def test_oracle_tree():
    masks, positions, _ = so.tree_masks([-1, 0, 0, 2, -1, 5, 9], [0, 7], [107], 1, 7)
    assert [list(np.flatnonzero(m)) for m in masks] == [[0], [0, 1], [0, 2], [0, 2, 3], [4], [5], [6]]
    assert positions.tolist() == [100, 101, 101, 102, 100, 100, 100]
    assert so.packed(masks)[3, 0] == 0b1101


def test_oracle_chain_is_causal():
    """The mask of a chain is the causal mask, with and without a window."""
    rng = np.random.default_rng(3)
    c = so.Kv8(6, 16, 1, 8)
    table = np.array([[3, 1, 4]])
    k, v, q = (rng.standard_normal((40, 1, 8)).astype(np.float16) for _ in range(3))
    c.append(k, v, [0, 40], [40], table)
    masks, _, _ = so.tree_masks(np.arange(-1, 6), [0, 7], [40], 1, 7)
    for window in (0, 1, 3, 9, 1000):
        a = c.tree_attention(q[:7], masks, [0, 7], [40], table, 0.3, window)
        b = c.attention(q[:7], [0, 7], [40], table, 0.3, True, window)
        assert all(np.allclose(x, y) for x, y in zip(a, b))


def test_oracle_keep():
    """Kept rows are the ones appended alone, up to the codes' steps; inside a page they keep their codes."""
    rng = np.random.default_rng(4)
    c = so.Kv8(6, 16, 2, 8)
    table = np.array([[3, 1, 4]])
    k, v = (rng.standard_normal((30, 2, 8)).astype(np.float16) for _ in range(2))
    c.append(k, v, [0, 30], [30], table)
    before, _ = c.values(0, 0, 30, table)
    c.keep(np.array([1, 4, 9] + 17 * [0]), [3], [0, 20], [30], table, 20)   # rows 10 .. 29: 11, 14, 19 to 10, 11, 12
    after, _ = c.values(0, 0, 30, table)
    step = c.scales[0, 3].max()
    assert np.abs(after[:13] - before[[*range(10), 11, 14, 19]]).max() <= step / 2
    same = so.Kv8(6, 16, 2, 8)
    same.append(k[:16], v[:16], [0, 16], [16], table)
    codes = same.codes[0, 3].copy()
    same.keep(np.array([2, 3, 0, 0]), [2], [0, 4], [16], table, 4)
    assert (same.codes[0, 3, 12:14] == codes[14:16]).all() and (same.codes[0, 3, :12] == codes[:12]).all()


def test_oracle_pool():
    p = so.Pool(8, 16)
    table = np.full((2, 4), -1, np.int32)
    p.resize(table, [33, 16])
    assert table.tolist() == [[0, 1, 2, -1], [3, -1, -1, -1]]
    children = np.full((3, 4), 7, np.int32)
    copies = p.fork(table, [33, 16], [0, 1, 0], children)
    assert children.tolist() == [[0, 1, 4, -1], [3, -1, -1, -1], [0, 1, 5, -1]]
    assert copies.tolist() == [[2, 4], [-1, -1], [2, 5]] and p.refs.tolist() == [3, 3, 1, 2, 1, 1, 0, 0]
    p.resize(table, [0, 64])
    assert p.refs.tolist() == [2, 2, 1, 2, 1, 1, 1, 1] and p.missing == 0 and table.tolist() == [[-1] * 4, [3, 2, 6, 7]]
    p.resize(table, [20, -1])
    assert p.missing == 2
