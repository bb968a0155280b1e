"""What the checks of the attention's precision can see, on the CPU: fp32 arithmetic as the kernels do it passes them, the
same with softmax weights of one fp16 number, of bf16, or with scores held in fp16 does not."""
import numpy as np
import pytest

from oracle import quant_oracle as qo

F32 = np.float32


def data(n, D, q_scale, seed):
    """Keys with channels of different size and values, as codes and page scales; queries."""
    rng = np.random.default_rng(seed)
    P, rows = 64, 48
    kv = []
    for side in range(2):
        x = rng.standard_normal((n, D)) * (np.exp(rng.standard_normal(D) * 0.5) if side == 0 else 1.0)
        scale = np.array([np.abs(x[i:i + P]).max() / 127 for i in range(0, n, P)], F32).repeat(P)[:n]
        kv.append((np.rint(x / scale[:, None]), scale))
    return kv, (rng.standard_normal((rows, D)) * q_scale).astype(np.float16)


def reference(kv, q, first):
    k, v = (c * s.astype(np.float64)[:, None] for c, s in kv)
    s = q.astype(np.float64) @ k.T * q.shape[1] ** -0.5
    s[:, :first] = -np.inf
    e = np.exp(s - s.max(1, keepdims=True))
    e /= e.sum(1, keepdims=True)
    return e @ v


def split(p):
    hi = p.astype(np.float16)
    return hi.astype(np.float64) + (p - hi.astype(F32)).astype(np.float16).astype(np.float64)


def bf16(p):
    u = p.view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(F32).astype(np.float64)


FORMS = dict(two=(lambda s: s, split), one=(lambda s: s, lambda p: p.astype(np.float16).astype(np.float64)),
             bf16=(lambda s: s, bf16), scores=(lambda s: s.astype(np.float16).astype(F32), split))


def attention(kv, q, first, form):
    """p = 2^(s + log2 sv - top + 8) in fp32, fed as the form says; the sum is that of p / sv."""
    score, feed = FORMS[form]
    (kc, ks), (vc, vs) = kv
    dot = np.zeros((len(q), len(kc)), F32)
    for d in range(0, q.shape[1], 32):   # steps of the matrix instructions, rounded to fp32 in between
        dot = (dot + q[:, d:d + 32].astype(np.float64) @ kc[:, d:d + 32].T).astype(F32)
    s = score(dot * (ks * F32(q.shape[1] ** -0.5 * np.log2(np.e)))) + np.log2(vs)
    s[:, :first] = -np.inf
    p = np.exp2(s - s.max(1, keepdims=True) + F32(8)).astype(F32)
    o, total = np.zeros((len(q), vc.shape[1]), F32), np.zeros(len(q), F32)
    for j in range(0, len(kc), 32):
        o = (o + feed(p[:, j:j + 32]) @ vc[j:j + 32]).astype(F32)
        total = (total + (p[:, j:j + 32] / vs[j:j + 32]).astype(np.float64).sum(1)).astype(F32)
    return (o * (F32(1) / total)[:, None]).astype(np.float16)


@pytest.mark.parametrize("q_scale", [0.05, 1.5])
@pytest.mark.parametrize("n,D", [(5, 128), (64, 64), (700, 128), (4000, 256)])
def test_apart(n, D, q_scale):
    """The norm tells a weight's one fp16 number from two, whatever the number of keys."""
    kv, q = data(n, D, q_scale, seed=n + D)
    ref = reference(kv, q, 0)
    far = {form: qo.attention_apart(attention(kv, q, 0, form), ref) for form in FORMS}
    print({k: v / qo.APART for k, v in far.items()})
    assert far["two"] <= qo.APART
    assert far["one"] > qo.APART and far["bf16"] > qo.APART
    assert q_scale < 1 or far["scores"] > qo.APART


@pytest.mark.parametrize("form", list(FORMS))
def test_bound_of_few_keys(form):
    """Over a few keys and with small scores the elementwise bound tells them too (scores below 2^-4 do not show fp16)."""
    kv, q = data(640, 128, 0.05, seed=3)
    ref = reference(kv, q, 636)
    k, v = (np.abs(c) * s.astype(np.float64)[:, None] for c, s in kv)
    big = (np.abs(q.astype(np.float64)) @ k.T * 128 ** -0.5)[:, 636:].max(1)
    s = q.astype(np.float64) @ (kv[0][0] * kv[0][1].astype(np.float64)[:, None]).T * 128 ** -0.5
    e = np.exp(s[:, 636:] - s[:, 636:].max(1, keepdims=True))
    e /= e.sum(1, keepdims=True)
    bound = qo.attention_bound(ref, e @ v[636:], big, (e * 127 * kv[1][1][636:].astype(np.float64)).max(1), 4, log2_scale=8)
    far = (np.abs(attention(kv, q, 636, form).astype(np.float64) - ref) / bound).max()
    print(form, far)
    assert (far <= 1) == (form in ("two", "scores"))
