"""Every form of the 4-bit product that its plan can choose on 256 CUs (tests/test_w4_forms.py checks that these are all)
against 64-bit sums."""
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


# M, N, batches; each with groups of 32, 64 and 128, with and without zero points
FORMS = [
    (17, 300, (1, 5, 17)),                    # two wavefronts
    (20, 2100, (3, 16, 32)),                  # four
    (33, 2600, (4, 9, 24)),                   # eight
    (16, 5000, (2,)), (16, 28700, (1, 4)),    # sixteen, without and with parts of the columns
    (48, 14400, (8, 20)),                     # parts, up to 16 and 32 rows
    (8179, 300, (5, 17)),                     # two row tiles: two wavefronts,
    (8190, 2100, (16, 32)),                   # four,
    (8192, 2600, (5, 16, 17, 32)),            # eight, 32 of W's rows a workgroup
    (30, 130, (33,)), (40, 1100, (40,)),      # many rows, three tiles of 16: one part, several
    (5904, 260, (512,)), (24000, 130, (100,)), (8180, 1100, (49,)), (5120, 1100, (100,)),   # four
]


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("g", [32, 64, 128])
@pytest.mark.parametrize("M,N,batches", FORMS)
def test_form(fb, M, N, batches, g, asym):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(M + N + g)
    G = -(-N // g)
    codes = torch.randint(-2**31, 2**31, (M, -(-N // 8)), dtype=torch.int32, device="cuda", generator=gen)
    scales = (torch.randn((M, G), device="cuda", generator=gen) * 0.5 - 5).exp().half()
    zeros = torch.randint(0, 16, (M, G), dtype=torch.uint8, device="cuda", generator=gen) if asym else None
    layer = fb.fluxbin_w4_pack(codes, scales, zeros, N, g)
    n = torch.arange(N, device="cuda")
    q = (codes[:, n // 8] >> (4 * (n % 8))) & 15
    W = (q - (8 if zeros is None else zeros[:, n // g].int())).double() * scales[:, n // g].double()
    ws = fb.make_w4_workspace(layer, max(batches))
    for B in batches:
        log(f"case form M={M} N={N} g={g} asym={asym} B={B}")
        x = torch.randn((B, N), device="cuda", generator=gen).half()
        ws.fill_(0xFF)   # NaN wherever a call would read what it has not written
        y = fb.fluxbin_w4_gemm(layer, x, out_fp32=True, workspace=ws).double()
        wt = W.t().contiguous()
        bound = qo.w4_depth(N) * 2.0 ** -23 * (x.double().abs() @ wt.abs())
        assert ((y - x.double() @ wt).abs() <= bound).all()
