"""Operators next to the binary linears of a decoding step, as a program calls them: linears in 4 bits with group scales
and their quantizer, and a paged key/value cache in 8 bits with the attention that reads it.

A case is a dict of plain values. Four kinds of work ("op"):
  w4         y = What x for one packed 4-bit linear, one activation row or more, into a preallocated output with the
             workspace that a serving loop keeps.
  quantize   a weight matrix to 4-bit codes with group scales (and zero points), with the values that the codes stand for.
  append     new keys and values, quantized into the pages of a cache that holds earlier tokens, then the values of all
             cached tokens read back.
  attention  attention of each sequence's newest tokens over its cached ones.

Definitions. A group of g columns (the last one may be shorter) of a weight row has lo = min(w, 0), hi = max(w, 0);
s = fp16((hi - lo) * (1/15)), z = clamp(round(-lo / s), 0, 15), q = clamp(round(w / s) + z, 0, 15), or without zero points
s = fp16(max|w| * (1/7)), z = 8, q = clamp(round(w / s), -8, 7) + 8; a code stands for (q - z) s. A page and head of the
cache has one scale for its keys, one for its values: the larger of max|new| * (1/127) and, where the page holds earlier
tokens, its old scale; a code is round(v / s), an earlier code becomes round(code * (s_old / s)). Rounding is to nearest
even, and a quotient by s a product with 1 / s in 32 bits.
"""
import math

import torch

own = False   # True: the framework's operators instead of the plain forms


def _w4(name, M, N, B, g, asym=True, fp32=False):
    """g = 0: one group per row."""
    case = dict(op="w4", M=M, N=N, B=B, g=g, asym=asym, fp32=fp32)
    return dict(case, name=name) if name else case


def _quantize(name, M, N, g, asym=True, src="fp16"):
    case = dict(op="quantize", M=M, N=N, g=g, asym=asym, src=src)
    return dict(case, name=name) if name else case


def _cache(name, op, B, ctx, new, Hq, Hkv, D, P, window=0):
    """ctx, new: (least, most) cached tokens (the new ones among them) and new tokens of a sequence."""
    case = dict(op=op, B=B, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1], Hq=Hq, Hkv=Hkv, D=D, P=P,
                window=window)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest linear (a router, a small head), one row: launch latency and host path
        _w4("w4_tiny_b1", 512, 256, 1, 32, asym=False),
        # batch-1 decoding, the up projection of a 70B model's MLP, zero points per group of 128
        _w4("w4_mlp70b_b1", 28672, 8192, 1, 128),
        # sixteen sequences decoded together, the down projection of the same MLP
        _w4("w4_down70b_b16", 8192, 28672, 16, 128),
        # a prompt of 256 tokens through the up projection of a 7B model, fp32 output, finer groups
        _w4("w4_prefill7b_b256", 11008, 4096, 256, 64, fp32=True),
        # quantizing an MLP weight of a 7B model
        _quantize("quantize_mlp7b", 11008, 4096, 128),
        # an odd-sized fp32 weight, fine groups without zero points
        _quantize("quantize_odd", 1999, 3001, 32, asym=False, src="fp32"),
        # one new token of each of 32 short sequences into partly filled pages (grouped heads of a 70B model)
        _cache("append_decode_b32", "append", 32, (1, 128), (1, 1), 64, 8, 128, 64),
        # four prompts of different lengths written at once (40 heads of a 13B model)
        _cache("append_prompts", "append", 4, (301, 2048), (301, 2000), 40, 40, 128, 32),
        # one sequence with a short history, 32 heads of a 7B model: latency
        _cache("attention_short_b1", "attention", 1, (200, 200), (1, 1), 32, 32, 128, 16),
        # 32 sequences of 256 to 8192 tokens decoded together, grouped heads of a 70B model
        _cache("attention_decode_b32", "attention", 32, (256, 8192), (1, 1), 64, 8, 128, 64),
        # two long contexts
        _cache("attention_long_b2", "attention", 2, (50000, 65536), (1, 1), 64, 8, 128, 64),
        # chunks of two prompts over what is cached of them
        _cache("attention_chunk", "attention", 2, (1500, 4096), (700, 1024), 64, 8, 128, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_size(rng, lo, hi):
    n = _log(rng, lo, hi)   # half of the sizes whole chunks, as model dimensions are, the others odd
    return max(128, n // 128 * 128) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["w4"] * 4 + ["attention"] * 4 + ["quantize"] + ["append"] * 2)
    if op in ("w4", "quantize"):
        g, asym = rng.choice([32, 64, 128, 128, 256, 0]), rng.random() < 0.6
        while True:
            M, N = _draw_size(rng, 64, 28672), _draw_size(rng, 64, 28672)
            B = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 2, 16), _log(rng, 17, 64), _log(rng, 65, 512)])
            if M * N <= 28672 * 8192 and M * N * B <= 11008 * 4096 * 256:
                break
        if op == "w4":
            return _w4("", M, N, B, g, asym=asym, fp32=rng.random() < 0.3)
        while M * N > 11008 * 4096:
            M, N = max(64, M // 2), max(64, N * 3 // 4)
        return _quantize("", M, N, g, asym=asym, src=rng.choice(["fp16", "fp16", "fp32"]))
    Hkv, group = rng.choice([(1, 8), (2, 7), (4, 4), (8, 8), (8, 4), (8, 5), (8, 1), (32, 1), (40, 1), (8, 16), (4, 1)])
    D, P = rng.choice([64, 128, 128, 128, 256]), rng.choice([16, 32, 64, 64, 128])
    while True:
        B = _log(rng, 1, 64)
        kind = rng.choice(["one", "one", "few", "chunk"])
        hi = _log(rng, 16, 32768)
        lo = min(hi, _log(rng, 1, max(2, hi)))
        new = (1, 1) if kind == "one" else (1, rng.randint(2, 8)) if kind == "few" else (_log(rng, 1, 64), _log(rng, 64, 1024))
        new = (min(new[0], lo), min(new[1], hi))
        cached, pairs = B * hi * Hkv * D, B * hi * new[1] * Hkv * group
        if op == "append":
            if cached <= 4 * 2048 * 40 * 128 and B * new[1] * Hkv * D <= 4 * 2000 * 40 * 128:
                break
        elif cached <= 32 * 8192 * 8 * 128 and pairs <= 2 * 4096 * 1024 * 64 and pairs * D <= 2 * 4096 * 1024 * 64 * 128:
            break
    window = _log(rng, 16, 4096) if op == "attention" and rng.random() < 0.25 else 0
    return _cache("", op, B, (lo, hi), new, Hkv * group, Hkv, D, P, window)


# ---------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _spread(lo, hi, B):
    """B lengths from lo to hi, evenly spread over their logarithm, not in order of size."""
    step = next(k for k in (7, 5, 3, 1) if math.gcd(k, B) == 1)
    return [int(round(lo * (hi / lo) ** ((b * step % B) / max(1, B - 1)))) if B > 1 else hi for b in range(B)]


def _lengths(case):
    """(cached tokens, the new ones among them) of every sequence."""
    new, ctx = _spread(case["new_lo"], case["new_hi"], case["B"]), _spread(case["ctx_lo"], case["ctx_hi"], case["B"])
    return [max(c, n) for c, n in zip(ctx, new)], new


def _group(case):
    return case["g"] or case["N"]


def _w4_inputs(case, seed):
    """Codes as words of eight (column 8 w + t in bits 4 t of word w), fp16 scales, zero points or None, fp16 activations
    with 0.1% outlier channels."""
    gen, M, N, B = _gen(seed), case["M"], case["N"], case["B"]
    G = -(-N // _group(case))
    codes = torch.randint(-2**31, 2**31, (M, -(-N // 8)), dtype=torch.int32, device="cuda", generator=gen)
    scales = (torch.randn((M, G), device="cuda", generator=gen) * 0.3).exp().mul(0.004).half()
    zeros = torch.randint(5, 12, (M, G), dtype=torch.uint8, device="cuda", generator=gen) if case["asym"] else None
    x = torch.randn((B, N), device="cuda", generator=gen)
    x[:, torch.randperm(N, device="cuda", generator=gen)[:int(0.001 * N + 0.5)]] *= 20
    return codes, scales, zeros, x.half()


def _matrix(case, seed):
    """A weight matrix with 1% outlier columns."""
    gen, M, N = _gen(seed), case["M"], case["N"]
    W = torch.randn((M, N), device="cuda", generator=gen) * 0.02
    W[:, torch.randperm(N, device="cuda", generator=gen)[:int(0.01 * N + 0.5)]] *= 10
    return W.half() if case["src"] == "fp16" else W


def _keys_values(rows, case, gen):
    """Keys with channels of different size, a few far larger, as trained keys have, and values."""
    Hkv, D = case["Hkv"], case["D"]
    channel = (torch.randn((Hkv, D), device="cuda", generator=gen) * 0.4).exp()
    channel[:, torch.randperm(D, device="cuda", generator=gen)[:2]] *= 5
    k = torch.randn((rows, Hkv, D), dtype=torch.float16, device="cuda", generator=gen)
    k *= channel.half()
    return k, torch.randn((rows, Hkv, D), dtype=torch.float16, device="cuda", generator=gen)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    return _ints([0] + torch.tensor(lengths).cumsum(0).tolist())


def _cache_inputs(case, seed):
    """What a serving loop holds: earlier keys and values (all cached ones for attention), the new tokens' fused q | k | v
    rows, lengths, and a block table with the sequences' pages spread over the pool (-1 past a sequence's last page)."""
    gen = _gen(seed)
    ctx, new = _lengths(case)
    Hq, Hkv, D, P = case["Hq"], case["Hkv"], case["D"], case["P"]
    pages = [-(-c // P) for c in ctx]
    pool = sum(pages) + 8
    order = torch.randperm(pool, device="cuda", generator=gen).int()
    column, start = torch.arange(max(pages), device="cuda"), _offsets(pages)[:-1, None].long()
    table = torch.where(column < _ints(pages)[:, None], order[(start + column).clamp(max=pool - 1)], -1).int()
    earlier = ctx if case["op"] == "attention" else [c - n for c, n in zip(ctx, new)]
    k_old, v_old = _keys_values(sum(earlier), case, gen)
    T = sum(new)
    qkv = torch.randn((T, (Hq + 2 * Hkv) * D), dtype=torch.float16, device="cuda", generator=gen)
    if case["op"] == "append":
        k, v = _keys_values(T, case, gen)
        qkv[:, Hq * D:(Hq + Hkv) * D] = k.reshape(T, -1)
        qkv[:, (Hq + Hkv) * D:] = v.reshape(T, -1)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hkv * D, Hkv * D], dim=1))
    return dict(table=table, pool=pool, ctx=_ints(ctx), ctx_offsets=_offsets(ctx), earlier=_ints(earlier),
                earlier_offsets=_offsets(earlier), k_old=k_old, v_old=v_old, new_offsets=_offsets(new), q=q, k=k, v=v,
                rows=sum(ctx), T=T, most_new=max(new))


# ---------------------------------------------------------------------------------------------------- plain forms

def _unpack(codes, N):
    shifts = torch.arange(0, 32, 4, dtype=torch.int32, device="cuda")
    return ((codes[..., None] >> shifts) & 15).flatten(1)[:, :N].float()


def _wide(per_group, g, N):
    return per_group.float().repeat_interleave(g, dim=1)[:, :N]


def _plain_w4(s):
    N, g = s["x"].shape[1], s["g"]
    zero = 8.0 if s["zeros"] is None else _wide(s["zeros"], g, N)
    W = (_unpack(s["codes"], N) - zero) * _wide(s["scales"], g, N)
    return (s["x"].float() @ W.t()).to(s["y"].dtype)


def _plain_quantize(W, g, asym):
    M, N = W.shape
    G = -(-N // g)
    w = torch.nn.functional.pad(W.float(), (0, G * g - N)).unflatten(1, (G, g))
    if asym:
        lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
        scales = ((hi - lo) * (1.0 / 15)).half()
    else:
        scales = (w.abs().amax(-1) * (1.0 / 7)).half()
    s = scales.float()
    inv = torch.where(s > 0, torch.ones_like(s) / s, 0.0)
    if asym:
        z = (-lo * inv).round().clamp(0, 15)
        q = ((w * inv[..., None]).round() + z[..., None]).clamp(0, 15)
    else:
        z = torch.full_like(s, 8.0)
        q = (w * inv[..., None]).round().clamp(-8, 7) + 8
    values = ((q - z[..., None]) * s[..., None]).flatten(1)[:, :N].half()
    return dict(scales=scales, zeros=z.to(torch.uint8) if asym else None, values=values)


def _tokens(offsets, context, rows):
    """Sequence and position of every row: the rows of a sequence are its newest tokens."""
    i = torch.arange(rows, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(offsets, i, right=True) - 1
    return b, (context[b] - (offsets[b + 1] - i)).long()


def _plain_store(codes, scales, values, page, slot):
    """Writes values [T, H, D] to slots of pages in place. codes int8 [pool, P, H, D], scales fp32 [pool, H]."""
    pool, P, H, D = codes.shape
    x = values.float()
    amax = torch.zeros((pool, H), device="cuda").scatter_reduce_(
        0, page[:, None].expand(-1, H), x.abs().amax(-1), "amax")
    first = torch.full((pool,), P, device="cuda").scatter_reduce_(0, page, slot, "amin")   # P: no new token
    old = torch.where((first > 0)[:, None], scales, 0.0)
    new = torch.maximum(old, amax * (1.0 / 127))
    ratio = torch.where(new > 0, old / new, 0.0)
    touched = (first < P).nonzero().squeeze(1) if pool > 4 * page.numel() else slice(None)
    codes[touched] = (codes[touched].float() * ratio[touched][:, None, :, None]).round().to(torch.int8)
    scales.copy_(new)
    inv = torch.where(new > 0, torch.ones_like(new) / new, 0.0)
    codes[page, slot] = (x * inv[page][:, :, None]).round().clamp(-127, 127).to(torch.int8)


def _plain_append(s, offsets, context, k, v):
    b, at = _tokens(offsets, context, k.shape[0])
    P = s["k_codes"].shape[1]
    page, slot = s["table"][b, at // P].long(), at % P
    _plain_store(s["k_codes"], s["k_scales"], k, page, slot)
    _plain_store(s["v_codes"], s["v_scales"], v, page, slot)


def _plain_read(s):
    b, at = _tokens(s["ctx_offsets"], s["ctx"], s["rows"])
    P = s["k_codes"].shape[1]
    page, slot = s["table"][b, at // P].long(), at % P
    return dict(k=(s["k_codes"][page, slot].float() * s["k_scales"][page][:, :, None]).half(),
                v=(s["v_codes"][page, slot].float() * s["v_scales"][page][:, :, None]).half())


def _paged(codes, scales, table):
    """[B, H, tokens, D] in fp32."""
    t = table.clamp(min=0).long()
    x = codes[t].float() * scales[t][:, :, None, :, None]
    return x.flatten(1, 2).transpose(1, 2)


def _plain_attention(s):
    case, q = s["case"], s["q"]
    T, Hq, D = q.shape
    Hkv, B, n = case["Hkv"], case["B"], s["most_new"]
    K, V = _paged(s["k_codes"], s["k_scales"], s["table"]), _paged(s["v_codes"], s["v_scales"], s["table"])
    L = K.shape[2]
    seq, at = _tokens(s["new_offsets"], s["ctx"], T)
    row = torch.arange(T, device="cuda") - s["new_offsets"][seq]
    wide = torch.zeros((B, n, Hq, D), device="cuda")
    wide[seq, row] = q.float()
    where = torch.full((B, n), -1, dtype=torch.int64, device="cuda")
    where[seq, row] = at
    wide = wide.view(B, n, Hkv, -1, D).permute(0, 2, 1, 3, 4).flatten(2, 3)                  # [B, Hkv, n * group, D]
    scores = (wide @ K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    j = torch.arange(L, device="cuda")
    seen = j <= where[..., None]
    if case["window"]:
        seen &= j > where[..., None] - case["window"]
    seen = seen[:, None].repeat_interleave(Hq // Hkv, dim=2)
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    e = scores.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.where(total > 0, (e @ V) / total, 0.0)
    o = o.view(B, Hkv, n, -1, D).transpose(1, 2).flatten(2, 3)
    return o[seq, row].half()


# ---------------------------------------------------------------------------------------------------- the passes

def _library():
    from paper_2608_15602_amd import fluxbin
    return fluxbin


def _prepare_w4(case, seed):
    codes, scales, zeros, x = _w4_inputs(case, seed)
    y = torch.empty((case["B"], case["M"]), dtype=torch.float32 if case["fp32"] else torch.float16, device="cuda")
    s = dict(op="w4", x=x, y=y, g=_group(case))
    if own:
        fb = s["fb"] = _library()
        s["layer"] = fb.fluxbin_w4_pack(codes, scales, zeros, case["N"], _group(case))
        s["ws"] = fb.make_w4_workspace(s["layer"], case["B"])
        if case["B"] == 1:
            s["x"], s["y"] = x[0], y[0]
        s["fp32"], s["whole"] = case["fp32"], y
    else:
        s.update(codes=codes, scales=scales, zeros=zeros)
    return s


def _prepare_cache(case, seed):
    s = _cache_inputs(case, seed)
    Hkv, D, P = case["Hkv"], case["D"], case["P"]
    s.update(op=case["op"], case=case)
    k_old, v_old = s.pop("k_old"), s.pop("v_old")
    if own:
        fb = s["fb"] = _library()
        s["cache"] = fb.make_kv8_cache(s["pool"], P, Hkv, D)
        if k_old.shape[0]:
            fb.fluxbin_kv8_append(s["cache"], k_old, v_old, s["earlier_offsets"], s["earlier"], s["table"])
        s["ws"] = fb.make_kv8_workspace(s["cache"], s["T"], case["B"], case["Hq"])
        s["out"] = torch.empty((s["T"], case["Hq"], D), dtype=torch.float16, device="cuda")
    else:
        for side in "kv":
            s[side + "_codes"] = torch.zeros((s["pool"], P, Hkv, D), dtype=torch.int8, device="cuda")
            s[side + "_scales"] = torch.zeros((s["pool"], Hkv), device="cuda")
        if k_old.shape[0]:
            _plain_append(s, s["earlier_offsets"], s["earlier"], k_old, v_old)
    return s


def prepare(case, seed):
    if case["op"] == "w4":
        return _prepare_w4(case, seed)
    if case["op"] == "quantize":
        return dict(op="quantize", W=_matrix(case, seed), g=_group(case), asym=case["asym"], fb=_library() if own else None)
    return _prepare_cache(case, seed)


def _run_own(s):
    fb = s["fb"]
    if s["op"] == "w4":
        fb.fluxbin_w4_gemm(s["layer"], s["x"], y=s["y"], out_fp32=s["fp32"], workspace=s["ws"])
        return s["whole"]
    if s["op"] == "quantize":
        codes, scales, zeros, values = fb.fluxbin_w4_quantize(s["W"], s["g"], asymmetric=s["asym"], values=True)
        return dict(scales=scales, zeros=zeros, values=values)
    if s["op"] == "append":
        fb.fluxbin_kv8_append(s["cache"], s["k"], s["v"], s["new_offsets"], s["ctx"], s["table"])
        k, v = fb.fluxbin_kv8_read(s["cache"], s["ctx_offsets"], s["ctx"], s["table"], s["rows"])
        return dict(k=k, v=v)
    return fb.fluxbin_kv8_attention(s["cache"], s["q"], s["new_offsets"], s["ctx"], s["table"], out=s["out"],
                                    window=s["case"]["window"], workspace=s["ws"])


def run(state):
    if own:
        return _run_own(state)
    if state["op"] == "w4":
        return _plain_w4(state)
    if state["op"] == "quantize":
        return _plain_quantize(state["W"], state["g"], state["asym"])
    if state["op"] == "append":
        _plain_append(state, state["new_offsets"], state["ctx"], state["k"], state["v"])
        return _plain_read(state)
    return _plain_attention(state)


def work(case):
    if case["op"] in ("w4", "quantize"):
        M, N, G = case["M"], case["N"], -(-case["N"] // _group(case))
        weights = M * N / 2 + M * G * (2.5 if case["asym"] else 2)
        if case["op"] == "quantize":   # the matrix in, codes and scales and the values they stand for out
            return dict(bytes=M * N * (2 if case["src"] == "fp16" else 4) + weights + 2.0 * M * N, flops=6.0 * M * N)
        B = case["B"]
        return dict(bytes=weights + B * (2 * N + (4 if case["fp32"] else 2) * M), flops=2.0 * B * M * N)
    ctx, new = _lengths(case)
    Hq, Hkv, D, P, T = case["Hq"], case["Hkv"], case["D"], case["P"], sum(new)
    if case["op"] == "append":
        # the new tokens in and into the cache, then every cached token's codes in and its values out
        return dict(bytes=2.0 * Hkv * D * (3 * T + 3 * sum(ctx)) + 16.0 * Hkv * sum(-(-c // P) for c in ctx),
                    flops=6.0 * Hkv * D * (T + sum(ctx)))
    most = case["window"] or max(ctx)
    seen = [min(c, n + most - 1) for c, n in zip(ctx, new)]             # cached tokens that some new token sees
    pairs = sum(sum(min(c - n + i + 1, most) for i in range(n)) for c, n in zip(ctx, new))
    return dict(bytes=2.0 * Hkv * D * sum(seen) + 8.0 * Hkv * sum(-(-c // P) for c in seen) + 4.0 * T * Hq * D,
                flops=4.0 * D * Hq * pairs)


# ---------------------------------------------------------------------------------------------------- 64 bits

def _exact_w4(case, seed):
    codes, scales, zeros, x = _w4_inputs(case, seed)
    M, N, g = case["M"], case["N"], _group(case)
    xd = x.double().t().contiguous()
    y = torch.empty((case["B"], M), dtype=torch.float64, device="cuda")
    group_of = torch.arange(N, device="cuda") // g
    column = torch.arange(N, device="cuda")
    step = max(1, (1 << 25) // N)
    for i in range(0, M, step):
        rows = slice(i, min(M, i + step))
        q = (codes[rows].long()[:, column // 8] >> (4 * (column % 8))) & 15
        z = 8 if zeros is None else zeros[rows].long()[:, group_of]
        y[:, rows] = (((q - z).double() * scales[rows].double()[:, group_of]) @ xd).t()
    return y


def _exact_quantize(case, seed):
    W, g = _matrix(case, seed).double(), _group(case)
    M, N = W.shape
    out, scales = torch.empty_like(W), []
    for c in range(0, N, g):
        w = W[:, c:c + g]
        if case["asym"]:
            lo, hi = w.min(1, keepdim=True).values.clamp(max=0), w.max(1, keepdim=True).values.clamp(min=0)
            s = ((hi - lo) / 15).half().double()     # the scale is what the format stores: 16 bits
        else:
            lo, s = None, (w.abs().max(1, keepdim=True).values / 7).half().double()
        some = torch.where(s > 0, s, 1.0)
        if case["asym"]:
            z = torch.round(-lo / some).clamp(0, 15)
            q = (torch.round(w / some) + z).clamp(0, 15) - z
        else:
            q = torch.round(w / some).clamp(-8, 7)
        out[:, c:c + g] = q * s
        scales.append(s)
    return dict(scales=torch.cat(scales, 1), zeros=None, values=out)


def _exact_append(case, seed):
    s = _cache_inputs(case, seed)
    P, starts = case["P"], s["earlier_offsets"].tolist()
    fresh = s["new_offsets"].tolist()

    def side(old, new):
        parts = []
        for b in range(case["B"]):
            o, n = old[starts[b]:starts[b + 1]].double(), new[fresh[b]:fresh[b + 1]].double()
            whole = o.shape[0] // P * P
            seq = torch.cat([o, n])
            kept = torch.cat([torch.ones(o.shape[0]), torch.zeros(n.shape[0])]).cuda()
            pad = -seq.shape[0] % P
            x = torch.nn.functional.pad(seq, (0, 0, 0, 0, 0, pad)).unflatten(0, (-1, P))       # [pages, P, H, D]
            was = torch.nn.functional.pad(kept, (0, pad)).view(-1, P, 1, 1)
            first = (x * was).abs().amax((1, 3), keepdim=True) / 127
            full = torch.maximum(first, x.abs().amax((1, 3), keepdim=True) / 127)
            a, f = torch.where(first > 0, first, 1.0), torch.where(full > 0, full, 1.0)
            early = torch.round(torch.round(x / a) * (a / f)) * full
            parts.append(torch.where(was > 0, early, torch.round(x / f) * full).flatten(0, 1)[:seq.shape[0]])
        return torch.cat(parts)

    return dict(k=side(s["k_old"], s["k"]), v=side(s["v_old"], s["v"]))


def _exact_attention(case, seed):
    s = _cache_inputs(case, seed)
    P, D, Hq, Hkv = case["P"], case["D"], case["Hq"], case["Hkv"]
    at, rows = s["ctx_offsets"].tolist(), s["new_offsets"].tolist()

    def cached(x):
        """The values in the cache: the scale and the codes are what it stores, in 32 and 8 bits."""
        n = x.shape[0]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, -n % P)).unflatten(0, (-1, P))
        scale = x.abs().amax((1, 3), keepdim=True) * (1.0 / 127)
        codes = torch.round(x * torch.where(scale > 0, torch.ones_like(scale) / scale, 0.0))
        return (codes.double() * scale.double()).flatten(0, 1)[:n]

    out = torch.zeros((s["T"], Hq, D), dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        k, v = cached(s["k_old"][at[b]:at[b + 1]]), cached(s["v_old"][at[b]:at[b + 1]])
        q = s["q"][rows[b]:rows[b + 1]].double()
        n, c = q.shape[0], k.shape[0]
        pos, j = torch.arange(c - n, c, device="cuda")[:, None], torch.arange(c, device="cuda")
        seen = (j <= pos) & ((j > pos - case["window"]) if case["window"] else True)
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            a = (q[:, h] @ k[:, kv].t()) / math.sqrt(D)
            out[rows[b]:rows[b + 1], h] = torch.softmax(a.masked_fill(~seen, -math.inf), -1) @ v[:, kv]
    return out


def exact(case, seed):
    return dict(w4=_exact_w4, quantize=_exact_quantize, append=_exact_append,
                attention=_exact_attention)[case["op"]](case, seed)
