"""4-bit linears (fluxbin_w4_*) against the plain definitions in oracle/quant_oracle.py: the quantizer's scales, zero points
and codes bit for bit, products within the bound of their fp32 sums."""
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


def weights(M, N, seed, scale=0.02):
    rng = np.random.default_rng(seed)
    W = rng.standard_normal((M, N)) * scale
    W[:, rng.choice(N, max(1, N // 100), replace=False)] *= 10
    return W


def canonical(M, N, g, asym, seed):
    rng = np.random.default_rng(seed)
    G = -(-N // g)
    codes = rng.integers(0, 16, (M, N)).astype(np.uint8)
    scales = np.exp(rng.standard_normal((M, G)) * 0.5 - 5).astype(np.float16)
    zeros = rng.integers(0, 16, (M, G)).astype(np.uint8) if asym else np.full((M, G), 8, np.uint8)
    return codes, scales, zeros


def pack(fb, codes, scales, zeros, g, asym):
    import torch
    M, N = codes.shape
    words = torch.from_numpy(qo.w4_words(codes).view(np.int32)).cuda()
    return fb.fluxbin_w4_pack(words, torch.from_numpy(scales).cuda(), torch.from_numpy(zeros).cuda() if asym else None, N, g)


# ---------------------------------------------------------------------------------------------- quantizer

@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("M,N,g", [(1, 1, 1), (3, 5, 32), (17, 31, 31), (5, 64, 32), (9, 100, 64), (4, 1000, 128), (33, 513, 32),
                                   (2, 1029, 256), (6, 1536, 512), (7, 1153, 384), (5, 2049, 1024), (3, 777, 777),
                                   (2, 4097, 5000), (1, 9001, 9001)])
def test_quantize(fb, M, N, g, asym, fp32):
    import torch
    log(f"case quantize M={M} N={N} g={g} asym={asym} fp32={fp32}")
    W = weights(M, N, seed=M * 7 + N)
    W[0, : min(N, 40)] = 0                      # a group of zeros where it is that short
    if M > 1:
        W[1] = np.abs(W[1]) + 0.01              # one sign only
    if M > 2:
        W[2] *= 1e-6                            # scales that round to a subnormal or to zero
    W = W.astype(np.float32 if fp32 else np.float16)
    wide = torch.full((M, N + 3), 9.0, dtype=torch.float32 if fp32 else torch.float16, device="cuda")
    wide[:, 1:N + 1] = torch.from_numpy(W).cuda()
    codes, scales, zeros, values = fb.fluxbin_w4_quantize(wide[:, 1:N + 1], g, asymmetric=asym, values=True)
    q, s, z = qo.w4_quantize(W, g, asym)
    assert np.array_equal(scales.cpu().numpy().view(np.uint16), s.view(np.uint16))
    assert zeros is None if not asym else np.array_equal(zeros.cpu().numpy(), z)
    assert np.array_equal(codes.cpu().numpy().view(np.uint32), qo.w4_words(q))
    dense = np.clip(qo.w4_dense(q, s, z, g), -65504, 65504)
    assert np.array_equal(values.cpu().numpy(), dense.astype(np.float16))


def test_quantize_scale_rounds_twice(fb):
    """The scale is the fp32 product rounded to fp16: over many groups some differ from the exact product rounded once."""
    import torch
    log("case quantize many scales")
    W = weights(4000, 1600, seed=21).astype(np.float32)
    for asym in (False, True):
        codes, scales, zeros, _ = fb.fluxbin_w4_quantize(torch.from_numpy(W).cuda(), 32, asymmetric=asym)
        q, s, z = qo.w4_quantize(W, 32, asym)
        assert np.array_equal(scales.cpu().numpy().view(np.uint16), s.view(np.uint16))
        assert np.array_equal(codes.cpu().numpy().view(np.uint32), qo.w4_words(q))


def test_quantize_not_finite(fb):
    """NaN counts as 0, infinities and fp32 values past fp16's range as its largest number."""
    import torch
    log("case quantize values that are not finite")
    W = weights(4, 200, seed=5).astype(np.float32)
    W[0, 3], W[0, 77], W[1, 5], W[2, 199], W[3, 0] = np.nan, np.inf, -np.inf, 1e30, -3e38
    for asym in (False, True):
        codes, scales, zeros, values = fb.fluxbin_w4_quantize(torch.from_numpy(W).cuda(), 64, asymmetric=asym, values=True)
        q, s, z = qo.w4_quantize(W, 64, asym)
        assert np.array_equal(scales.cpu().numpy(), s) and np.isfinite(s).all()
        assert np.array_equal(codes.cpu().numpy().view(np.uint32), qo.w4_words(q))
        assert np.array_equal(values.cpu().numpy(), np.clip(qo.w4_dense(q, s, z, 64), -65504, 65504).astype(np.float16))


# ---------------------------------------------------------------------------------------------- product

SHAPES = [(1, 1, 1), (15, 7, 32), (16, 128, 128), (17, 129, 32), (40, 300, 64), (130, 1000, 128), (513, 257, 256),
          (64, 4100, 128), (33, 2500, 2500), (1000, 640, 64), (48, 20000, 32), (2080, 1100, 128)]
BATCHES = [1, 2, 16, 17, 33, 65, 130]


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("M,N,g", SHAPES)
def test_gemm(fb, M, N, g, asym):
    import torch
    codes, scales, zeros = canonical(M, N, g, asym, seed=M + N)
    layer = pack(fb, codes, scales, zeros, g, asym)
    W = qo.w4_dense(codes, scales, zeros, g)
    ws = fb.make_w4_workspace(layer, max(BATCHES))
    rng = np.random.default_rng(N)
    for B in BATCHES:
        for fp32 in (False, True):
            log(f"case gemm M={M} N={N} g={g} asym={asym} B={B} fp32={fp32}")
            x = (rng.standard_normal((B, N)) * np.where(rng.random(N) < 0.01, 20, 1)).astype(np.float16)
            dt = torch.float32 if fp32 else torch.float16
            # rows at odd strides and offsets; what is between the rows of y stays
            xt = torch.full((B, N + 5), float("nan"), dtype=torch.float16, device="cuda")
            xt[:, 3:N + 3] = torch.from_numpy(x).cuda()
            yt = torch.full((B + 1, M + 3), 7.0, dtype=dt, device="cuda")
            ws.fill_(0xFF)   # NaN wherever a call would read what it has not written
            fb.fluxbin_w4_gemm(layer, xt[:, 3:N + 3], y=yt[:B, 1:M + 1], out_fp32=fp32, workspace=ws)
            y = yt.cpu().double().numpy()
            ref = x.astype(np.float64) @ W.T
            assert (np.abs(y[:B, 1:M + 1] - ref) <= qo.w4_bound(W, x.astype(np.float64), not fp32)).all()
            y[:B, 1:M + 1] = 7
            assert (y == 7).all()


# layers tall enough for two row tiles a workgroup, with and without chunks after the last whole step; long enough for every
# number of wavefronts and for the many-row kernel's parts
LARGE = [(8200, 600, 64, True), (4100, 2050, 128, False), (8200, 2112, 32, True), (8210, 4224, 128, True), (2000, 9000, 256, True),
         (16400, 520, 64, False)]


@pytest.mark.parametrize("M,N,g,asym", LARGE)
def test_gemm_large(fb, M, N, g, asym):
    import torch
    codes, scales, zeros = canonical(M, N, g, asym, seed=M + N)
    layer = pack(fb, codes, scales, zeros, g, asym)
    W = qo.w4_dense(codes, scales, zeros, g)
    x = (np.random.default_rng(N).standard_normal((256, N))).astype(np.float16)
    ref, bound = x.astype(np.float64) @ W.T, qo.w4_bound(W, x.astype(np.float64), False)
    xt, ws = torch.from_numpy(x).cuda(), fb.make_w4_workspace(layer, 256)
    for B in (1, 4, 5, 16, 17, 32, 40, 48, 64, 100, 256):
        log(f"case gemm M={M} N={N} g={g} asym={asym} B={B}")
        ws.fill_(0xFF)
        y = fb.fluxbin_w4_gemm(layer, xt[:B], out_fp32=True, workspace=ws).cpu().double().numpy()
        assert (np.abs(y - ref[:B]) <= bound[:B]).all()


def test_workspace_refusals(fb):
    import torch
    log("case gemm refusals")
    codes, scales, zeros = canonical(48, 20000, 128, True, seed=9)
    layer = pack(fb, codes, scales, zeros, 128, True)
    x = torch.randn(16, 20000, device="cuda").half()
    n = fb.fluxbin_w4_workspace_query(layer, 16)
    assert n > 0
    for ws in (torch.empty(256, dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.uint8), layer.buf,
               torch.empty(n + 8, dtype=torch.uint8, device="cuda")[8:]):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_w4_gemm(layer, x, workspace=ws)
    for bad in (x.float(), x[:, :-1], x.cpu(), x.t(), x[None], x.repeat(1, 2)[:, ::2]):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_w4_gemm(layer, bad)
    for bad in (x[:, :48], torch.empty(16, 48, device="cuda"), torch.empty(15, 48, dtype=torch.float16, device="cuda"),
                torch.empty(16, 49, dtype=torch.float16, device="cuda")):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_w4_gemm(layer, x, y=bad)


def test_gemv_is_the_first_row(fb):
    """A vector gives what a batch of one gives, with and without given outputs and workspaces, twice the same bits."""
    import torch
    log("case gemv")
    codes, scales, zeros = canonical(300, 900, 128, True, seed=3)
    layer = pack(fb, codes, scales, zeros, 128, True)
    x = torch.randn(1, 900, device="cuda").half()
    a = fb.fluxbin_w4_gemm(layer, x)
    b = fb.fluxbin_w4_gemm(layer, x[0], workspace=fb.make_w4_workspace(layer))
    assert torch.equal(a[0], b) and torch.equal(fb.fluxbin_w4_gemm(layer, x[0], out_fp32=True).half(), b)


def test_rows_are_independent(fb):
    """Infinities and NaN in one activation row stay in that row of the result; an inf times a zero weight is NaN there."""
    import torch
    log("case gemm rows with inf and nan")
    codes, scales, zeros = canonical(100, 500, 64, True, seed=4)
    layer = pack(fb, codes, scales, zeros, 64, True)
    for B in (3, 40, 100):
        x = torch.randn(B, 500, device="cuda").half()
        y = fb.fluxbin_w4_gemm(layer, x)
        x2 = x.clone()
        x2[1, 7], x2[2, 499] = float("inf"), float("nan")
        y2 = fb.fluxbin_w4_gemm(layer, x2)
        keep = [b for b in range(B) if b not in (1, 2)]
        assert torch.equal(y[keep], y2[keep])
        assert not torch.isfinite(y2[1]).any() and torch.isnan(y2[2]).all()


def test_streams_and_graph(fb):
    """A call on another stream, and a captured one replayed between eager calls, give the eager call's bits."""
    import torch
    log("case gemm stream and graph")
    codes, scales, zeros = canonical(48, 20000, 128, True, seed=6)
    layer = pack(fb, codes, scales, zeros, 128, True)
    for B in (1, 5, 100):
        x = torch.randn(B, 20000, device="cuda").half()
        ref = fb.fluxbin_w4_gemm(layer, x)
        ws, y = fb.make_w4_workspace(layer, B), torch.zeros_like(ref)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        fb.fluxbin_w4_gemm(layer, x, y=y, workspace=ws, stream=side)
        side.synchronize()
        assert torch.equal(y, ref)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fb.fluxbin_w4_gemm(layer, x, y=y, workspace=ws)
        for i in range(4):
            x.copy_(torch.randn(B, 20000, device="cuda"))
            ref = fb.fluxbin_w4_gemm(layer, x)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, ref), i


def test_quantized_layer_end_to_end(fb):
    """Quantize, pack and multiply: the product with the values that the quantizer says its codes stand for."""
    import torch
    log("case quantize, pack, gemm")
    W = torch.from_numpy(weights(700, 1500, seed=8).astype(np.float16)).cuda()
    codes, scales, zeros, values = fb.fluxbin_w4_quantize(W, 128, values=True)
    layer = fb.fluxbin_w4_pack(codes, scales, zeros, 1500, 128)
    x = torch.randn(9, 1500, device="cuda").half()
    y = fb.fluxbin_w4_gemm(layer, x, out_fp32=True).double().cpu()
    ref = x.double().cpu() @ values.double().cpu().T
    # the values are rounded to fp16: 2^-11 of each term
    mag = x.double().cpu().abs() @ values.double().cpu().abs().T
    assert ((y - ref).abs() <= mag * (2.0 ** -11 + 300 * 2.0 ** -23)).all()
    assert (W.float() - values.float()).abs().max() <= 0.51 * scales.float().max()


@pytest.mark.parametrize("M,N", [(40, 300), (5, 3), (2, 1)])
def test_one_group_of_any_length(fb, M, N):
    """g far past the row is the same as g = N: codes, scales and products."""
    import torch
    log(f"case one group per row M={M} N={N}")
    W = torch.from_numpy(weights(M, N, seed=11).astype(np.float16)).cuda()
    x = torch.randn(3, N, device="cuda").half()
    ref = None
    for g in (N, 1 << 40, (1 << 63) - 1):
        codes, scales, zeros, values = fb.fluxbin_w4_quantize(W, g, values=True)
        got = [codes, scales, zeros, values, fb.fluxbin_w4_gemm(fb.fluxbin_w4_pack(codes, scales, zeros, N, g), x)]
        assert scales.shape == (M, 1)
        ref = ref or got
        assert all(torch.equal(a, b) for a, b in zip(ref, got))
