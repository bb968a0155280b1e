"""How close the attention over the 8-bit cache is to 64 bits before its final rounding, in every form: the norm of what is
left without that rounding, and the elementwise bound where it is narrow (few keys, small scores)."""
import numpy as np
import pytest

from oracle import quant_oracle as qo

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


# heads, group, head_dim, page, new rows, tokens: prompts whose rows fill 256 CUs, one beside few rows; single tokens, split
# over workgroups and not; prompts that do not fill the device, a few rows
FORMS = [(8, 8, 128, 64, [520], [700]), (8, 8, 64, 16, [520], [520]), (8, 8, 256, 32, [270], [400]),
         (32, 1, 128, 128, [1030], [1030]), (8, 8, 128, 64, [520, 3], [520, 900]), (2, 4, 128, 64, [1, 1], [700, 9000]),
         (2, 8, 64, 16, [1], [200]), (1, 8, 256, 64, [1], [3000]), (8, 8, 128, 64, [300], [300]),
         (2, 4, 128, 32, [8, 5], [600, 40])]


def run(s, new, G, q_scale, window):
    offsets = np.concatenate([[0], np.cumsum(new)])
    q = (s.rng.standard_normal((int(offsets[-1]), s.H * G, s.D)) * q_scale).astype(np.float16)
    got = s.fb.fluxbin_kv8_attention(s.cache, s.dev(q), *s.arrays(offsets, s.length), window=window).cpu().double().numpy()
    return got, s.plain.attention(q, offsets, s.length, s.table, s.D ** -0.5, True, window)


@pytest.mark.parametrize("H,G,D,P,new,ctx", FORMS)
def test_apart(fb, H, G, D, P, new, ctx):
    log(f"case precision H={H} G={G} D={D} P={P} new={new} ctx={ctx}")
    s = Setup(fb, len(new), H, D, P, max(ctx), seed=40)
    s.append(ctx)
    for q_scale in (0.1, 1.5):
        got, (ref, *_) = run(s, new, G, q_scale, 0)
        far = qo.attention_apart(got, ref) / qo.APART
        log(f"  {far:.3f} of the norm")
        assert far <= 1


@pytest.mark.parametrize("H,G,D,P,new,ctx", FORMS)
def test_few_keys(fb, H, G, D, P, new, ctx):
    log(f"case few keys H={H} G={G} D={D} P={P} new={new} ctx={ctx}")
    s = Setup(fb, len(new), H, D, P, max(ctx), seed=41)
    s.append(ctx)
    for window in (2, 4):
        got, (ref, mag, big, peak, _) = run(s, new, G, 0.03, window)
        sv = s.plain.scales[1][s.plain.scales[1] > 0]
        assert np.abs(np.log2(sv)).max() <= 8
        far = np.abs(got - ref) / qo.attention_bound(ref, mag, big, peak, window, log2_scale=8)
        log(f"  worst {far.max():.3f} of the bound")
        assert (far <= 1).all()
