"""Host-side checks of include/fluxbin_quant.h: entry points, sizes and refusals, before any launch. CPU only."""
import ctypes
import os
import re

import pytest

fb = pytest.importorskip("paper_2608_15602_amd.fluxbin")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INV, UNS, SMALL = fb.FLUXBIN_ERR_INVALID_ARG, fb.FLUXBIN_ERR_UNSUPPORTED, fb.FLUXBIN_ERR_BUFFER_TOO_SMALL


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fb.LIB_PATH):
        pytest.fail("libfluxbin.so is not built; run `python -m paper_2608_15602_amd.build`")
    return fb.lib()


def test_exports_every_declared_function(L):
    with open(os.path.join(ROOT, "include", "fluxbin_quant.h")) as f:
        names = set(re.findall(r"^fluxbin_status (fluxbin_\w+)\(", f.read(), re.M))
    assert names == set(fb.QUANT_EXPORTS)
    for n in names:
        assert hasattr(L, n), n


def _w4(**kw):
    d = dict(M=300, N=1000, g=128, has_zeros=1)
    d.update(kw)
    return fb.W4Shape(d["M"], d["N"], d["g"], d["has_zeros"], 0)


def _up(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("kw", [{}, dict(M=1, N=1, g=1), dict(g=32), dict(g=64, has_zeros=0), dict(N=129, g=5000),
                                dict(M=28672, N=8192), dict(N=1 << 20, M=1 << 14, g=256)])
def test_w4_pack_query(L, kw):
    s = _w4(**kw)
    Mt, Nc = -(-s.M // 16), -(-s.N // 128)
    gc = 128 // s.g if s.g < 128 and s.g < s.N else 1
    Nq = -(-Nc * gc // 4)
    assert fb.fluxbin_w4_pack_query(s) == _up(Mt * Nc * 1024) + _up(Mt * Nq * 128) + (_up(Mt * Nq * 64) if s.has_zeros else 0)


@pytest.mark.parametrize("kw,status", [
    (dict(M=0), INV), (dict(M=-1), INV), (dict(M=(1 << 24) + 1), INV), (dict(N=0), INV), (dict(N=(1 << 20) + 1), INV),
    (dict(M=1 << 24, N=1025), UNS), (dict(g=0), INV), (dict(g=-128), INV), (dict(g=16), UNS), (dict(g=96), UNS),
    (dict(g=200), UNS), (dict(has_zeros=2), INV)])
def test_w4_shape_refused(L, kw, status):
    n = ctypes.c_size_t(7)
    assert L.fluxbin_w4_pack_query(ctypes.byref(_w4(**kw)), ctypes.byref(n)) == status
    assert L.fluxbin_last_error_message() and n.value == 7


def test_w4_null_pointers(L):
    s, n = _w4(), ctypes.c_size_t(0)
    assert L.fluxbin_w4_pack_query(None, ctypes.byref(n)) == INV
    assert L.fluxbin_w4_pack_query(ctypes.byref(s), None) == INV
    assert L.fluxbin_w4_workspace_query(None, 1, ctypes.byref(n)) == INV


A = [1 << 20, 2 << 20, 4 << 20, 6 << 20, 8 << 20]   # addresses for calls that are refused before any launch


def _quantize(L, **kw):
    a = dict(shape=_w4(), W=A[0], fp32=0, ldw=1000, codes=A[1], scales=A[2], zeros=A[3], values=None, ldv=0)
    a.update(kw)
    return L.fluxbin_w4_quantize(ctypes.byref(a["shape"]), a["W"], a["fp32"], a["ldw"], a["codes"], a["scales"], a["zeros"],
                                 a["values"], a["ldv"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(W=None), INV), (dict(codes=None), INV), (dict(scales=None), INV), (dict(zeros=None), INV),
    (dict(shape=_w4(has_zeros=0)), INV), (dict(fp32=2), INV), (dict(ldw=999), INV), (dict(ldw=-1000), INV),
    (dict(W=A[0] + 1), INV), (dict(W=A[0] + 2, fp32=1), INV), (dict(codes=A[1] + 2), INV), (dict(scales=A[2] + 1), INV),
    (dict(values=A[4], ldv=999), INV), (dict(values=A[4] + 1, ldv=1000), INV), (dict(codes=A[0] + 4), INV),
    (dict(scales=A[1] + 8), INV), (dict(zeros=A[2] + 2), INV), (dict(values=A[0] + 300 * 2000 - 2, ldv=1000), INV),
    (dict(shape=_w4(g=48)), UNS)])
def test_w4_quantize_refused(L, kw, status):
    assert _quantize(L, **kw) == status
    assert L.fluxbin_last_error_message()


def _pack(L, **kw):
    s = kw.pop("shape", _w4())
    a = dict(codes=A[0], scales=A[1], zeros=A[2], packed=A[3], bytes=1 << 20)
    a.update(kw)
    out = fb.W4Layer()
    return L.fluxbin_w4_pack(ctypes.byref(s), a["codes"], a["scales"], a["zeros"], a["packed"], a["bytes"],
                             ctypes.byref(out), None)


@pytest.mark.parametrize("kw,status", [
    (dict(codes=None), INV), (dict(scales=None), INV), (dict(zeros=None), INV), (dict(packed=None), INV),
    (dict(shape=_w4(has_zeros=0)), INV), (dict(bytes=1000), SMALL), (dict(packed=A[3] + 8), INV), (dict(codes=A[0] + 1), INV),
    (dict(packed=A[0] + 16), INV), (dict(zeros=A[3] + 64), INV)])
def test_w4_pack_refused(L, kw, status):
    assert _pack(L, **kw) == status


def _layer(**kw):
    layer = fb.W4Layer(_w4(**kw.pop("shape", {})), A[0], 1 << 20, 1, 0)
    for k, v in kw.items():
        setattr(layer, k, v)
    return layer


@pytest.mark.parametrize("kw,status", [
    (dict(layer=dict(format_version=2)), INV), (dict(layer=dict(d_base=None)), INV), (dict(layer=dict(bytes=1000)), SMALL),
    (dict(layer=dict(d_base=A[0] + 4)), INV), (dict(layer=dict(shape=dict(g=48))), UNS), (dict(B=0), INV), (dict(B=8193), INV),
    (dict(x=None), INV), (dict(y=None), INV), (dict(fp32=3), INV), (dict(B=2, ldx=999), INV), (dict(B=2, ldy=299), INV),
    (dict(x=A[2] + 1), INV), (dict(y=A[3] + 2, fp32=1), INV)])
def test_w4_gemm_refused(L, kw, status):
    a = dict(layer={}, B=1, x=A[2], ldx=1000, y=A[3], ldy=300, fp32=0, ws=A[4], bytes=1 << 20)
    a.update(kw)
    assert L.fluxbin_w4_gemm(ctypes.byref(_layer(**a["layer"])), a["B"], a["x"], a["ldx"], a["y"], a["ldy"], a["fp32"],
                             a["ws"], a["bytes"], None) == status
    assert L.fluxbin_last_error_message()


def test_w4_binding_refusals():
    """Shapes, types and devices are checked by the binding, before the library's raw pointers."""
    import torch
    h = torch.float16
    for W, g in ((torch.zeros(4, 8, dtype=torch.bfloat16), 8), (torch.zeros(8, dtype=h), 8),
                 (torch.zeros(4, 8, dtype=h).t(), 4), (torch.zeros(4, 8, dtype=h), 8)):   # the last: not on a GPU
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_w4_quantize(W, g)
    with pytest.raises(fb.FluxbinError):
        fb.fluxbin_w4_pack(torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 1, dtype=h), None, 8, 8)


# ---------------------------------------------------------------------------------------------- 8-bit cache

@pytest.mark.parametrize("pages,P,H,D", [(1, 16, 1, 64), (1000, 64, 8, 128), (77, 256, 3, 256)])
def test_kv8_cache_query(L, pages, P, H, D):
    assert fb.fluxbin_kv8_cache_query(pages, P, H, D) == 2 * pages * P * H * D + 2 * _up(pages * H * 4)


@pytest.mark.parametrize("args,status", [
    ((0, 64, 8, 128), INV), ((-1, 64, 8, 128), INV), (((1 << 24) + 1, 16, 1, 64), INV), ((9, 0, 8, 128), INV),
    ((9, 48, 8, 128), UNS), ((9, 512, 8, 128), UNS), ((9, 8, 8, 128), UNS), ((9, 64, 0, 128), INV), ((9, 64, 1025, 128), INV),
    ((9, 64, 8, 0), INV), ((9, 64, 8, 96), UNS), ((9, 64, 8, 512), UNS), ((1 << 24, 256, 1024, 256), UNS)])
def test_kv8_cache_refused(L, args, status):
    n = ctypes.c_size_t(7)
    assert L.fluxbin_kv8_cache_query(*args, ctypes.byref(n)) == status
    assert L.fluxbin_last_error_message() and n.value == 7


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


BAD_CALLS = [
    (dict(cache=dict(format_version=0)), INV), (dict(cache=dict(d_base=None)), INV), (dict(cache=dict(d_base=(1 << 30) + 16)), INV),
    (dict(cache=dict(bytes=1000)), SMALL), (dict(cache=dict(page_size=24)), UNS), (dict(batch=dict(rows=-1)), INV),
    (dict(batch=dict(rows=(1 << 22) + 1)), INV), (dict(batch=dict(sequences=0)), INV), (dict(batch=dict(sequences=65536)), INV),
    (dict(batch=dict(max_blocks=0)), INV), (dict(batch=dict(max_blocks=1 << 24, block_table_stride=1 << 24),
                                             cache=dict(page_size=128)), UNS),
    (dict(batch=dict(block_table_stride=4)), INV), (dict(batch=dict(d_offsets=None)), INV), (dict(batch=dict(d_context=None)), INV),
    (dict(batch=dict(d_block_table=None)), INV), (dict(batch=dict(d_block_table=A[0] + 8194)), INV),
    (dict(batch=dict(d_context=(1 << 30) + 64)), INV)]


def _append(L, cache={}, batch={}, **kw):
    a = dict(k=A[1], kt=1024, kh=128, v=A[2], vt=1024, vh=128)
    a.update(kw)
    return L.fluxbin_kv8_append(ctypes.byref(_cache(**cache)), ctypes.byref(_batch(**batch)), a["k"], a["kt"], a["kh"], a["v"],
                                a["vt"], a["vh"], None)


@pytest.mark.parametrize("kw,status", BAD_CALLS + [
    (dict(k=None), INV), (dict(v=None), INV), (dict(k=A[1] + 1), INV), (dict(kt=-1), INV), (dict(vh=127), INV),
    (dict(vh=-128), INV), (dict(k=(1 << 30) - 128), INV), (dict(kt=(1 << 36) + 1), INV)])
def test_kv8_append_refused(L, kw, status):
    assert _append(L, **kw) == status
    assert L.fluxbin_last_error_message()


def _read(L, cache={}, batch={}, k=A[1], v=A[2]):
    return L.fluxbin_kv8_read(ctypes.byref(_cache(**cache)), ctypes.byref(_batch(**batch)), k, v, None)


@pytest.mark.parametrize("kw,status", BAD_CALLS[:-1] + [
    (dict(k=None), INV), (dict(v=None), INV), (dict(k=A[1] + 2), INV), (dict(v=A[1]), INV), (dict(k=1 << 30), INV),
    (dict(v=A[0] - 64), INV)])
def test_kv8_read_refused(L, kw, status):
    assert _read(L, **kw) == status


def _attention(L, cache={}, batch={}, **kw):
    a = dict(heads=64, q=A[1], qt=8192, qh=128, out=A[2], ot=8192, oh=128, scale=0.1, causal=1, window=0, ws=A[3], bytes=1 << 40)
    a.update(kw)
    return L.fluxbin_kv8_attention(ctypes.byref(_cache(**cache)), ctypes.byref(_batch(**batch)), a["heads"], a["q"], a["qt"],
                                   a["qh"], a["out"], a["ot"], a["oh"], a["scale"], a["causal"], a["window"], a["ws"],
                                   a["bytes"], None)


@pytest.mark.parametrize("kw,status", BAD_CALLS[:-1] + [
    (dict(heads=0), INV), (dict(heads=63), INV), (dict(heads=1024, batch=dict(rows=1 << 22), cache=dict(kv_heads=1)), UNS), (dict(heads=1032), INV), (dict(scale=float("nan")), INV),
    (dict(scale=float("inf")), INV), (dict(causal=2), INV), (dict(window=-1), INV), (dict(q=None), INV), (dict(out=None), INV),
    (dict(out=A[2] + 1), INV), (dict(qh=100), INV), (dict(ot=0), INV), (dict(ot=8191), INV)])
def test_kv8_attention_refused(L, kw, status):
    assert _attention(L, **kw) == status
    assert L.fluxbin_last_error_message()


def test_kv8_null_structs(L):
    assert L.fluxbin_kv8_append(None, ctypes.byref(_batch()), A[1], 1024, 128, A[2], 1024, 128, None) == INV
    assert L.fluxbin_kv8_append(ctypes.byref(_cache()), None, A[1], 1024, 128, A[2], 1024, 128, None) == INV
    assert L.fluxbin_kv8_cache_query(9, 64, 8, 128, None) == INV


def test_kv8_no_rows(L):
    """A call without rows is valid and launches nothing."""
    assert _append(L, batch=dict(rows=0), k=None, v=None) == 0
    assert _read(L, batch=dict(rows=0), k=None, v=None) == 0


# ---------------------------------------------------------------------------------------------- groups past a row

@pytest.mark.parametrize("g", [1000, 5000, 1 << 40, (1 << 63) - 1])
def test_w4_one_group_per_row(L, g):
    """Any g >= N is one group per row, up to the largest number that its type holds: sizes and overlaps count that group."""
    assert fb.fluxbin_w4_pack_query(_w4(g=g)) == fb.fluxbin_w4_pack_query(_w4(g=1000))
    assert _quantize(L, shape=_w4(g=g), zeros=A[2] + 599) == INV   # the last scale's second byte
    assert _pack(L, shape=_w4(g=g), scales=A[3] - 599) == INV


# ---------------------------------------------------------------------------------------------- numbers past the C types

def test_binding_refuses_numbers_that_do_not_fit():
    """ctypes keeps the low bits of a number: 2^64 + 32 would be 32, with buffers sized for one group per row."""
    import torch
    from types import SimpleNamespace
    h = torch.float16
    with pytest.raises(fb.FluxbinError, match="g = "):
        fb.fluxbin_w4_quantize(torch.zeros(4, 64, dtype=h), (1 << 64) + 32)
    codes, scales = torch.zeros(4, 8, dtype=torch.int32), torch.zeros(4, 1, dtype=h)
    with pytest.raises(fb.FluxbinError, match="g = "):
        fb.fluxbin_w4_pack(codes, scales, None, 64, (1 << 64) + 32)
    with pytest.raises(fb.FluxbinError, match="N = "):
        fb.fluxbin_w4_pack(codes, scales, None, (1 << 64) + 64, 64)
    layer = SimpleNamespace(ref=ctypes.byref(_layer()))
    cache = SimpleNamespace(ref=ctypes.byref(_cache()), index=-1, use=SimpleNamespace(int32=torch.int32, current_device=lambda: -1),
                            device="meta")
    for call in (lambda: fb.fluxbin_w4_workspace_query(layer, (1 << 32) + 1),
                 lambda: fb.fluxbin_kv8_cache_query((1 << 64) + 9, 64, 8, 128), lambda: fb.fluxbin_kv8_cache_query(9, (1 << 32) + 64, 8, 128),
                 lambda: fb.fluxbin_kv8_cache_query(9, 64, 8 - (1 << 32), 128), lambda: fb.fluxbin_kv8_cache_query(9, 64, 8, 128 + (1 << 40)),
                 lambda: fb.fluxbin_kv8_workspace_query(cache, 10, (1 << 32) + 1, 8),
                 lambda: fb.fluxbin_kv8_workspace_query(cache, 10, 1, (1 << 32) + 8),
                 lambda: fb.fluxbin_kv8_read(cache, None, None, None, (1 << 64) + 1), lambda: fb.fluxbin_kv8_read(cache, None, None, None, -1)):
        with pytest.raises(fb.FluxbinError) as e:
            call()
        assert e.value.status == INV
    meta = lambda *size: torch.empty(size, dtype=torch.int32, device="meta")   # shapes without memory
    for B, blocks in (((1 << 32) + 1, 1), (1, (1 << 32) + 5)):
        with pytest.raises(fb.FluxbinError):
            fb._kv8_batch(cache, 1, meta(B + 1), meta(B), meta(B, blocks))


def test_binding_refuses_windows_that_do_not_fit(monkeypatch):
    """A negative window is refused however small it is; one past the type is the whole context."""
    import torch
    from types import SimpleNamespace
    seen = []
    lib = SimpleNamespace(fluxbin_kv8_attention=lambda *a: seen.append(ctypes.c_int32(a[11]).value) or 0)
    monkeypatch.setattr(fb, "_kv8_rows", lambda cache, name, t, heads: t.size(0))
    monkeypatch.setattr(fb, "_kv8_batch", lambda *a: fb.Kv8Batch())
    q = torch.zeros(2, 8, 64)
    cache = SimpleNamespace(use=SimpleNamespace(lib=lib, stream=lambda *a: None), ref=None, head_dim=64, index=-1, device="cpu")
    for window in (5, 5 + (1 << 32), -(1 << 32) + 5, -1):
        fb.fluxbin_kv8_attention(cache, q, None, None, None, out=q, window=window, workspace=torch.zeros(1))
    assert seen[0] == 5 and seen[1] == (1 << 31) - 1 and seen[2] < 0 and seen[3] < 0


def test_binding_refuses_scalars():
    """A tensor without dimensions is refused as one of a wrong shape is."""
    import torch
    from types import SimpleNamespace
    layer = SimpleNamespace(M=300, N=1000, index=-1, device="cpu", use=SimpleNamespace(half=torch.float16, single=torch.float32))
    with pytest.raises(fb.FluxbinError):
        fb.fluxbin_w4_gemm(layer, torch.tensor(1.0, dtype=torch.float16))
    with pytest.raises(fb.FluxbinError):
        fb.fluxbin_w4_gemm(layer, torch.zeros(1000, dtype=torch.float16), y=torch.tensor(1.0, dtype=torch.float16))
