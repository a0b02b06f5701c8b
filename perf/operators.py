"""The attention side of the library as cases that can be timed and compared: norms and rotation of queries and keys, the
paged NVFP4 cache as it is written and read back, and attention over it in 4 bits.

`own` false: the operators in their plain form, elementary torch operations in 32 bits (64 where a rounding is decided, for
angles and for long sums).  `own` true: the calls of the library.  Both take what prepare() gives.
"""
import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
PLAIN, SEARCH = "plain", "search"


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # queries and keys of eight sequences that decode one token each, at far positions (a language model's step)
        {"name": "norm_rope_decode", "op": "norm_rope", "T": 8, "Hq": 32, "Hk": 8, "d": 128, "axes": 1, "pairs": 64, "interleaved": False, "far": 1000000},
        # a video transformer's training clip: 20 latent frames of 880 tokens, 24 heads, positions in time, height and width
        {"name": "norm_rope_video", "op": "norm_rope", "T": 17600, "Hq": 24, "Hk": 24, "d": 128, "axes": 3, "pairs": 64, "interleaved": True, "far": 64},
        # a short odd training batch, grouped keys, half of the head rotated
        {"name": "norm_rope_backward_short", "op": "norm_rope_backward", "T": 777, "Hq": 16, "Hk": 4, "d": 64, "axes": 2, "pairs": 16, "interleaved": False, "far": 4096},
        # the training clip's gradients
        {"name": "norm_rope_backward_video", "op": "norm_rope_backward", "T": 17600, "Hq": 24, "Hk": 24, "d": 128, "axes": 3, "pairs": 64, "interleaved": True, "far": 64},
        # 33 sequences append one token each and it is read back: latency
        {"name": "cache_write_decode", "op": "cache_write", "T": 33, "H": 8, "d": 128, "page": 16, "pages": 600, "rule": PLAIN, "smooth": False},
        # a chunk of four latent frames enters the cache: smoothed keys, scale search
        {"name": "cache_write_video", "op": "cache_write", "T": 3520, "H": 24, "d": 128, "page": 880, "pages": 21, "rule": SEARCH, "smooth": True},
        # a few scattered tokens of a small cache
        {"name": "cache_read_scattered", "op": "cache_read", "T": 217, "H": 3, "d": 80, "page": 32, "pages": 40, "smooth": False},
        # the whole window of 21 latent frames
        {"name": "cache_read_window", "op": "cache_read", "T": 18480, "H": 24, "d": 128, "page": 880, "pages": 21, "smooth": True},
        # five short sequences decode a token, one of them with an empty cache: latency
        {"name": "attention_decode_short", "op": "attention", "B": 5, "queries": 1, "lengths": 700, "ragged": True, "Hq": 24, "Hk": 24, "d": 64, "page": 16, "smooth": False,
         "causal": True, "window": 0, "sink": 0, "f32": False},
        # eight long sequences decode a token each, grouped heads
        {"name": "attention_decode_long", "op": "attention", "B": 8, "queries": 1, "lengths": 32768, "ragged": True, "Hq": 32, "Hk": 8, "d": 128, "page": 64, "smooth": True,
         "causal": True, "window": 0, "sink": 0, "f32": False},
        # ragged prompts behind caches of different lengths, causal with a sliding window and sink tokens
        {"name": "attention_prefill_ragged", "op": "attention", "B": 4, "queries": 1500, "lengths": 6000, "ragged": True, "Hq": 32, "Hk": 8, "d": 128, "page": 48, "smooth": False,
         "causal": True, "window": 2048, "sink": 16, "f32": True},
        # a chunk of four latent frames attends to the window of 21, itself among them
        {"name": "attention_video", "op": "attention", "B": 1, "queries": 3520, "lengths": 18480, "ragged": False, "Hq": 24, "Hk": 24, "d": 128, "page": 880, "smooth": True,
         "causal": False, "window": 0, "sink": 0, "f32": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_rope", "norm_rope_backward", "cache_write", "cache_read", "attention", "attention"])
    d = rng.choice([64, 80, 128, 128, 256])
    if op in ("norm_rope", "norm_rope_backward"):
        Hk = rng.randint(1, 24)
        Hq = Hk * rng.choice([1, 1, 2, 4]) if Hk <= 8 else Hk
        interleaved = rng.random() < 0.5
        pairs = rng.choice([d // 2, d // 2, d // 4]) if interleaved else 8 * rng.randint(1, d // 16)
        T = _log(rng, 1, max(1, min(17600, 17600 * 48 * 128 // ((Hq + Hk) * d))))
        return {"op": op, "T": T, "Hq": Hq, "Hk": Hk, "d": d, "axes": rng.randint(1, 3), "pairs": pairs, "interleaved": interleaved, "far": rng.choice([64, 4096, 1000000])}
    page = 16 * _log(rng, 1, 55)
    if op in ("cache_write", "cache_read"):
        H = rng.randint(1, 24)
        smooth = d != 80 and rng.random() < 0.5
        T = _log(rng, 1, max(1, min(18480, 18480 * 24 * 128 // (H * d))))
        pages = -(-T // page) + rng.randint(0, 5)
        case = {"op": op, "T": T, "H": H, "d": d, "page": page, "pages": pages, "smooth": smooth}
        return {**case, "rule": rng.choice([PLAIN, SEARCH])} if op == "cache_write" else case
    Hk = rng.randint(1, 16)
    Hq = Hk * rng.choice([1, 1, 2, 4, 7, 8])
    smooth = d != 80 and rng.random() < 0.5
    causal = rng.random() < 0.7
    B = _log(rng, 1, 48)
    queries = rng.choice([1, 1, 1, rng.randint(2, 17), _log(rng, 18, 2000), _log(rng, 18, 2000)])
    while B > 1 and B * queries * max(queries, 16) * Hq * d > 10 ** 11:
        B //= 2
    room = min(8 * 32768 * 8 * 128 // (B * Hk * d), 10 ** 11 // (B * queries * Hq * d), 131072)
    lengths = max(queries, _log(rng, 1, max(16, room)))
    window = rng.choice([0, 0, _log(rng, 16, 4096)])
    return {"op": "attention", "B": B, "queries": queries, "lengths": lengths, "ragged": rng.random() < 0.7, "Hq": Hq, "Hk": Hk, "d": d, "page": page, "smooth": smooth,
            "causal": causal, "window": window, "sink": rng.choice([0, 4, 100]) if window else 0, "f32": rng.random() < 0.3}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=F32)


def _axis_pairs(case):
    """Pairs of each axis: as even as they go, the first axis takes what is left over (22, 21, 21 of 64)."""
    n, P = case["axes"], case["pairs"]
    return [P - (n - 1) * (P // n)] + [P // n] * (n - 1)


def _norm_rope_inputs(case, g):
    T, Hq, Hk, d = case["T"], case["Hq"], case["Hk"], case["d"]
    split = _axis_pairs(case)
    # one row of the fused projection holds the token's queries, keys and values; per-channel gains as trained projections have
    gain = torch.exp(0.5 * _normal(g, (Hq + 2 * Hk) * d))
    x = (_normal(g, T, (Hq + 2 * Hk) * d) * gain).to(BF16)
    state = {"x": x, "q": x[:, : Hq * d].unflatten(1, (Hq, d)), "k": x[:, Hq * d : (Hq + Hk) * d].unflatten(1, (Hk, d)),
             "wq": (1 + 0.2 * _normal(g, d)).to(BF16), "wk": (1 + 0.2 * _normal(g, d)).to(BF16),
             "positions": torch.randint(0, case["far"], (T, case["axes"]), generator=g, device="cuda", dtype=torch.int32),
             "freqs": torch.cat([10000.0 ** (-torch.arange(n, dtype=F64) / max(n, 1)) for n in split]).to(F32).cuda()}
    if case["op"] == "norm_rope_backward":
        state["dq"], state["dk"] = (1e-3 * _normal(g, T, Hq, d)).to(BF16), (1e-3 * _normal(g, T, Hk, d)).to(BF16)
    return state


def _kv(g, T, H, d):
    """Keys with an offset of their own for each head and per-head magnitudes, values with per-head magnitudes."""
    scale = 0.5 + 3.5 * torch.rand((2, 1, H, 1), generator=g, device="cuda")
    k = (_normal(g, T, H, d) + _normal(g, 1, H, 1)) * scale[0]
    return k.to(BF16), (_normal(g, T, H, d) * scale[1]).to(BF16)


def _page_scales(g, pages, amax):
    """Tensor scales as calibration leaves them: the expected maximum over 2688, a little different from page to page."""
    return (amax / 2688.0 * (0.8 + 0.6 * torch.rand((2, pages), generator=g, device="cuda"))).to(F32)


def _filled_cache(case, g, pages, H, d):
    """A cache with every slot written (plain rule; what a slot holds does not matter to its readers)."""
    page = case["page"]
    n = pages * page
    cache = {"page": page, "k_codes": torch.empty((pages, page, H, d // 2), dtype=torch.uint8, device="cuda"),
             "k_scales": torch.empty((pages, page, H, d // 16), dtype=torch.uint8, device="cuda"),
             "v_codes": torch.empty((pages, page, H, d // 2), dtype=torch.uint8, device="cuda"),
             "v_scales": torch.empty((pages, page, H, d // 16), dtype=torch.uint8, device="cuda"),
             "k_mean": (_normal(g, pages, page, H) * 1.5).to(BF16) if case["smooth"] else None}
    cache["k_global"], cache["v_global"] = _page_scales(g, pages, 16.0)
    for kind in ("k", "v"):
        block = 0.5 + 3.5 * torch.rand((pages, 1, H, 1), generator=g, device="cuda")          # per-head magnitudes
        for at in range(0, pages, max(1, (1 << 24) // (page * H * d))):
            to = min(pages, at + max(1, (1 << 24) // (page * H * d)))
            x = (_normal(g, to - at, page, H, d) * block[at:to]).unflatten(3, (d // 16, 16))
            code, byte, _ = _encode(x, cache[kind + "_global"][at:to].view(-1, 1, 1, 1), 6.0)
            cache[kind + "_codes"][at:to] = _pack(code.flatten(3))
            cache[kind + "_scales"][at:to] = byte
    assert cache["k_codes"].numel() == n * H * d // 2
    return cache


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    if case["op"] in ("norm_rope", "norm_rope_backward"):
        return {**state, **_norm_rope_inputs(case, g)}
    if case["op"] == "cache_write":
        T, H, d, page, pages = (case[n] for n in ("T", "H", "d", "page", "pages"))
        k, v = _kv(g, T, H, d)
        amax = 24.0
        cache = {"page": page, "k_codes": torch.zeros((pages, page, H, d // 2), dtype=torch.uint8, device="cuda"),
                 "k_scales": torch.zeros((pages, page, H, d // 16), dtype=torch.uint8, device="cuda"),
                 "v_codes": torch.zeros((pages, page, H, d // 2), dtype=torch.uint8, device="cuda"),
                 "v_scales": torch.zeros((pages, page, H, d // 16), dtype=torch.uint8, device="cuda"),
                 "k_mean": torch.zeros((pages, page, H), dtype=BF16, device="cuda") if case["smooth"] else None}
        cache["k_global"], cache["v_global"] = _page_scales(g, pages, amax)
        if case["pages"] * page < 4 * T:      # a chunk: consecutive slots from some page on; else scattered ones
            slots = torch.arange(T, device="cuda") + (pages * page - T) // page * page
        else:
            slots = torch.randperm(pages * page, generator=g, device="cuda")[:T]
        return {**state, "cache": cache, "k": k, "v": v, "slots": slots.to(torch.int64)}
    if case["op"] == "cache_read":
        T, H, d, page, pages = (case[n] for n in ("T", "H", "d", "page", "pages"))
        cache = _filled_cache(case, g, pages, H, d)
        slots = torch.arange(T, device="cuda") if pages * page < 2 * T else torch.randperm(pages * page, generator=g, device="cuda")[:T]
        return {**state, "cache": cache, "slots": slots.to(torch.int64)}
    B, Hq, Hk, d, page = (case[n] for n in ("B", "Hq", "Hk", "d", "page"))
    n_q, n_kv = _ragged(case)
    per_seq = [-(-n // page) for n in n_kv]
    most = max(max(per_seq), 1)
    pages = max(sum(per_seq), 1)
    cache = _filled_cache(case, g, pages, Hk, d)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((B, most), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(per_seq):
        table[b, :n] = order[at : at + n]
        at += n
    starts = torch.tensor([sum(n_q[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    q = (2.0 * _normal(g, sum(n_q), Hq, d)).to(BF16)
    return {**state, "cache": cache, "q": q, "table": table.cuda(), "lens": torch.tensor(n_kv, dtype=torch.int32, device="cuda"), "starts": starts}


def _ragged(case):
    """Queries and cached tokens of each sequence, from the case alone.  Ragged: lengths from empty caches to the full one."""
    B = case["B"]
    if not case["ragged"]:
        return [case["queries"]] * B, [case["lengths"]] * B
    n_q = [max(1, case["queries"] * (B - b // 2) // B) for b in range(B)]
    n_kv = [case["lengths"] * ((7 * b) % B + 1) // B for b in range(B)]
    n_kv = [n_kv[b] if case["queries"] == 1 else max(n_kv[b], n_q[b]) for b in range(B)]
    if B >= 4 and case["queries"] == 1:
        n_kv[1] = 0
    return n_q, n_kv


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _round_e4m3(x):
    """Nearest E4M3 number to x >= 0 (64 bits), ties to even, at most 448; and its byte."""
    x = x.clamp(max=448.0)
    e = (torch.frexp(x).exponent - 1).clamp(min=-6)
    v = torch.ldexp(torch.round(torch.ldexp(x, 3 - e)), e - 3)
    e = (torch.frexp(v).exponent - 1).clamp(min=-6)
    m = torch.ldexp(v, 3 - e).to(torch.int32)                       # 8..15 for normal numbers, 0..7 for subnormal ones
    byte = torch.where(m >= 8, ((e + 7) << 3) + (m - 8), m)
    return v, byte.to(torch.uint8)


def _round_e2m1(y):
    """Nearest E2M1 magnitude to y >= 0, ties to the even code."""
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0).to(y.dtype)).to(y.dtype)
    return (torch.round(y / step) * step).clamp(max=6.0)


def _encode(x, sg, target):
    """Blocks [..., 16] -> signed values of the codes, scale bytes and block scales, in 64 bits; sg broadcasts over the blocks."""
    x, sg = x.to(F64), sg.to(F64)
    sb, byte = _round_e4m3(x.abs().amax(-1) / (target * sg))
    den = (sb * sg).unsqueeze(-1)
    y = torch.where(den > 0, x.abs() / den, 0.0)
    return torch.copysign(_round_e2m1(y), x), byte, sb


def _pack(values):
    """E2M1 values [..., n] -> bytes [..., n / 2], the even element in the low half."""
    m = values.abs()
    code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(values).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _decoded(codes, scales, dtype):
    """Codes [..., d/2] and scale bytes [..., d/16] -> code * block scale, [..., d]; both factors are short, the product is exact."""
    magnitudes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=dtype, device=codes.device)
    values = torch.cat([magnitudes, -magnitudes])
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(torch.int32)
    b = scales.to(torch.int32)
    sb = torch.where(b >= 8, torch.ldexp((8 + (b & 7)).to(dtype), (b >> 3) - 10), (b & 7).to(dtype) / 512)
    return (values[code].unflatten(-1, (-1, 16)) * sb.unsqueeze(-1)).flatten(-2)


def _rotation(state):
    """cos and sin [T, 1, P] of position times frequency, the angle in 64 bits."""
    axis = torch.repeat_interleave(torch.arange(state["case"]["axes"]), torch.tensor(_axis_pairs(state["case"]))).cuda()
    angle = state["positions"].to(F64)[:, axis] * state["freqs"].to(F64)
    return torch.cos(angle).to(F32).unsqueeze(1), torch.sin(angle).to(F32).unsqueeze(1)


def _rotate(y, cos, sin, interleaved):
    P = cos.shape[-1]
    if interleaved:
        a, b, rest = y[..., 0 : 2 * P : 2], y[..., 1 : 2 * P : 2], y[..., 2 * P :]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)
    a, b, rest = y[..., :P], y[..., P : 2 * P], y[..., 2 * P :]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)


EPS = 1e-6


def _norm_rope_plain(x, w, cos, sin, interleaved):
    x = x.to(F32)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return _rotate(x * r * w.to(F32), cos, sin, interleaved).to(BF16)


def _norm_rope_backward_plain(dy, x, w, cos, sin, interleaved):
    g = _rotate(dy.to(F32), cos, -sin, interleaved)
    x, w = x.to(F32), w.to(F32)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh, dxh = x * r, g * w
    dx = r * (dxh - xh * (dxh * xh).mean(-1, keepdim=True))
    return dx.to(BF16), (g * xh).sum((0, 1), dtype=F64).to(F32)


def _quantised_plain(x, sg, rule, mean):
    """Rows [T, H, d] with a tensor scale for each token -> the values that the cache holds for them, rounded to bf16."""
    x = x.to(F64)
    if mean:
        mu = x.mean(-1, keepdim=True).to(BF16).to(F64)
        x = (x - mu).to(BF16).to(F64)
    blocks, sg = x.unflatten(-1, (-1, 16)), sg.view(-1, 1, 1)
    code, _, sb = _encode(blocks, sg, 6.0)
    held = code * (sb * sg.to(F64)).unsqueeze(-1)
    if rule == SEARCH:
        code4, _, sb4 = _encode(blocks, sg, 4.0)
        held4 = code4 * (sb4 * sg.to(F64)).unsqueeze(-1)
        closer = (blocks - held4).square().sum(-1) < (blocks - held).square().sum(-1)
        held = torch.where(closer.unsqueeze(-1), held4, held)
    held = held.flatten(-2)
    return (held + mu if mean else held).to(BF16)


def _read_plain(cache, slots, dtype):
    """Values of the slots, [T, H, d] each, before any rounding to bf16."""
    page, at = slots // cache["page"], slots % cache["page"]
    k = _decoded(cache["k_codes"][page, at], cache["k_scales"][page, at], dtype) * cache["k_global"][page].to(dtype).view(-1, 1, 1)
    v = _decoded(cache["v_codes"][page, at], cache["v_scales"][page, at], dtype) * cache["v_global"][page].to(dtype).view(-1, 1, 1)
    return k if cache["k_mean"] is None else k + cache["k_mean"][page, at].to(dtype).unsqueeze(-1), v


def _attention_plain(state):
    case, cache = state["case"], state["cache"]
    B, Hq, Hk, d, page = (case[n] for n in ("B", "Hq", "Hk", "d", "page"))
    G, most_q = Hq // Hk, case["queries"]
    starts, lens = state["starts"].to(torch.int64), state["lens"].to(torch.int64)
    n_q, n_kv = starts[1:] - starts[:-1], state["table"].shape[1] * page
    # queries and keys padded to rectangles
    i, j = torch.arange(most_q, device="cuda"), torch.arange(n_kv, device="cuda")
    real = i < n_q.view(-1, 1)
    q = state["q"][torch.where(real, starts[:-1].view(-1, 1) + i, 0)].to(F32)                                   # [B, Q, Hq, d]
    q = q.unflatten(2, (Hk, G)).permute(0, 2, 3, 1, 4).reshape(B * Hk, G * most_q, d)
    slots = state["table"].to(torch.int64).clamp(min=0)[:, j // page] * page + j % page
    k, v = _read_plain(cache, slots.reshape(-1), F32)
    k = k.view(B, n_kv, Hk, d).permute(0, 2, 3, 1).reshape(B * Hk, d, n_kv)
    v = v.view(B, n_kv, Hk, d).permute(0, 2, 1, 3).reshape(B * Hk, n_kv, d)
    s = torch.matmul(q, k.contiguous()).mul_(1.0 / math.sqrt(d)).view(B, Hk, G, most_q, n_kv)
    last = (lens.view(-1, 1) - n_q.view(-1, 1) + i if case["causal"] else (lens.view(-1, 1) - 1).expand(B, most_q)).unsqueeze(-1)
    seen = (j <= last) & (j < lens.view(-1, 1, 1))
    if case["window"]:
        seen = seen & ((j > last - case["window"]) | (j < case["sink"]))
    s.masked_fill_(~seen.view(B, 1, 1, most_q, n_kv), -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    s.sub_(m).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B * Hk, G * most_q, n_kv), v.contiguous()).view(B, Hk, G, most_q, d) / total.clamp(min=1e-30)
    lse = m.squeeze(-1) + torch.log(total.squeeze(-1))
    o, lse = o.permute(0, 3, 1, 2, 4).reshape(B, most_q, Hq, d)[real], lse.permute(0, 3, 1, 2).reshape(B, most_q, Hq)[real]
    return {"out": o if case["f32"] else o.to(BF16), "lse": lse}


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] in ("norm_rope", "norm_rope_backward"):
        cos, sin = _rotation(state)
        if case["op"] == "norm_rope":
            return {"q": _norm_rope_plain(state["q"], state["wq"], cos, sin, case["interleaved"]),
                    "k": _norm_rope_plain(state["k"], state["wk"], cos, sin, case["interleaved"])}
        dq, dwq = _norm_rope_backward_plain(state["dq"], state["q"], state["wq"], cos, sin, case["interleaved"])
        dk, dwk = _norm_rope_backward_plain(state["dk"], state["k"], state["wk"], cos, sin, case["interleaved"])
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    if case["op"] == "cache_write":
        page = state["slots"] // state["cache"]["page"]
        return {"k": _quantised_plain(state["k"], state["cache"]["k_global"][page], case["rule"], case["smooth"]),
                "v": _quantised_plain(state["v"], state["cache"]["v_global"][page], case["rule"], False)}
    if case["op"] == "cache_read":
        k, v = _read_plain(state["cache"], state["slots"], F32)
        return {"k": k.to(BF16), "v": v.to(BF16)}
    return _attention_plain(state)


def _cache(nv, state):
    """The handle that a program keeps beside its cache's memory."""
    if "handle" not in state:
        c = state["cache"]
        state["handle"] = nv.NVFP4KvCache(c["k_codes"], c["k_scales"], c["k_global"], c["v_codes"], c["v_scales"], c["v_global"], k_mean=c["k_mean"])
    return state["handle"]


def _run_own(state):
    import paper_2605_18739_amd as nv

    case = state["case"]
    if case["op"] in ("norm_rope", "norm_rope_backward"):
        if "rope" not in state:
            state["rope"] = nv.NVFP4Rope(state["positions"], state["freqs"], _axis_pairs(case), interleaved=case["interleaved"])
        if case["op"] == "norm_rope":
            q, k = nv.nvfp4_qk_norm_rope(state["q"], state["k"], state["wq"], state["wk"], state["rope"], eps=EPS)
            return {"q": q, "k": k}
        dq, dk, dwq, dwk = nv.nvfp4_qk_norm_rope_backward(state["dq"], state["dk"], state["q"], state["k"], state["wq"], state["wk"], state["rope"], eps=EPS)
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    cache = _cache(nv, state)
    if case["op"] == "cache_write":
        nv.nvfp4_kv_cache_write(cache, state["k"], state["v"], state["slots"], scale_search=case["rule"] == SEARCH)
    if case["op"] in ("cache_write", "cache_read"):
        k, v = nv.nvfp4_kv_cache_read(cache, state["slots"])
        return {"k": k, "v": v}
    out, lse = nv.nvfp4_kv_attention(state["q"], cache, state["table"], state["lens"], state["starts"], case["queries"], causal=case["causal"], window=case["window"],
                                     sink=case["sink"], out_dtype=nv.OUT_F32 if case["f32"] else nv.OUT_BF16)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    op, d = case["op"], case["d"]
    if op in ("norm_rope", "norm_rope_backward"):
        n = case["T"] * (case["Hq"] + case["Hk"]) * d
        small = 4 * case["T"] * case["axes"] + 4 * case["pairs"] + 4 * d
        return {"bytes": 4 * n + small, "flops": 8 * n} if op == "norm_rope" else {"bytes": 6 * n + small + 8 * d, "flops": 18 * n}
    held = d / 2 + d / 16
    if op in ("cache_write", "cache_read"):
        rows, mean = case["T"] * case["H"], 2 if case["smooth"] else 0
        read = rows * (2 * held + mean + 4 * d)
        if op == "cache_read":
            return {"bytes": read + 8 * case["T"], "flops": 4 * rows * d}
        return {"bytes": 2 * read + 8 * case["T"], "flops": (16 if case["rule"] == PLAIN else 40) * rows * d}
    n_q, n_kv = _ragged(case)
    seen = touched = 0
    for a, n in zip(n_q, n_kv):
        W, S = case["window"], case["sink"]
        if case["causal"]:
            last = range(n - a, n)
            first = n - a
        else:
            last = [n - 1] * a
            first = n - 1
        seen += sum(_seen(p, W, S) for p in last)
        # cached tokens that some query sees
        touched += n if not W or first - W < 0 else min(n, min(S, max(first - W + 1, 0)) + n - max(first - W + 1, 0))
    rows = sum(n_q) * case["Hq"]
    cached = touched * case["Hk"] * (2 * held + (2 if case["smooth"] else 0))
    return {"bytes": cached + rows * (2 * d + (4 if case["f32"] else 2) * d + 4), "flops": 4 * d * case["Hq"] * seen}


def _seen(last, window, sink):
    """Tokens 0..last that a window (0: none) and sink tokens leave visible."""
    n = max(0, last + 1)
    return n if not window else min(n, window + min(sink, max(0, n - window)))


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_rotation(state, sign):
    """[T, d, d] rotations would be large: cos and sin of each element, the partner's index and the partner's sign instead."""
    case, d, P = state["case"], state["case"]["d"], state["case"]["pairs"]
    T = state["positions"].shape[0]
    cos, sin = torch.ones((T, d), dtype=F64, device="cuda"), torch.zeros((T, d), dtype=F64, device="cuda")
    partner = torch.arange(d, device="cuda")
    j = 0
    for axis, n in enumerate(_axis_pairs(case)):
        for _ in range(n):
            a, b = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + P)
            angle = sign * state["positions"][:, axis].double() * float(state["freqs"][j])
            cos[:, a] = cos[:, b] = torch.cos(angle)
            sin[:, a], sin[:, b] = -torch.sin(angle), torch.sin(angle)
            partner[a], partner[b] = b, a
            j += 1
    return cos, sin, partner


def _exact_norm_rope(state):
    case, answer = state["case"], {}
    for n in ("q", "k"):
        x, w = state[n].double(), state["w" + n].double()
        if case["op"] == "norm_rope":
            cos, sin, partner = _exact_rotation(state, 1.0)
            y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS) * w
            answer[n] = y * cos[:, None] + y[..., partner] * sin[:, None]
        else:
            cos, sin, partner = _exact_rotation(state, -1.0)
            dy = state["d" + n].double()
            g = dy * cos[:, None] + dy[..., partner] * sin[:, None]
            s = torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS)
            # y = w x / s: dx = w g / s - x sum(w g x) / (d s^3)
            answer["d" + n] = w * g / s - x * (w * g * x).sum(-1, keepdim=True) / (case["d"] * s ** 3)
            answer["dw" + n] = (g * x / s).sum(1).sum(0)
    return answer


def _exact_block_values(x, sg, target):
    """Nearest representable values by comparing with every midpoint (even code wins a tie); x [n, 16], sg [n]."""
    e4m3 = torch.tensor([m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1], dtype=F64, device="cuda")
    e2m1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64, device="cuda")

    def nearest(y, grid):
        mid = (grid[1:] + grid[:-1]) / 2
        low = torch.bucketize(y, mid)                       # midpoints below y
        up = torch.bucketize(y, mid, right=True)            # ... and those that y meets
        return grid[torch.where(low % 2 == 0, low, up)]

    sb = nearest(x.abs().amax(-1) / (target * sg), e4m3)
    den = (sb * sg).unsqueeze(-1)
    m = nearest(torch.where(den > 0, x.abs() / den.clamp(min=1e-300), torch.zeros_like(x)), e2m1)
    return torch.where(x < 0, -m, m) * den


def _exact_written(x, sg, rule, smooth):
    T, H, d = x.shape
    x = x.double()
    mu = (x.sum(-1, keepdim=True) / d).to(BF16).double() if smooth else torch.zeros((T, H, 1), dtype=F64, device="cuda")
    b = ((x - mu).to(BF16).double() if smooth else x).reshape(-1, 16)
    sg = sg.double().view(-1, 1, 1).expand(T, H, d // 16).reshape(-1)
    held = _exact_block_values(b, sg, 6.0)
    if rule == SEARCH:
        other = _exact_block_values(b, sg, 4.0)
        pick = ((b - other) ** 2).sum(-1) < ((b - held) ** 2).sum(-1)
        held[pick] = other[pick]
    return held.view(T, H, d) + mu


def _exact_slots(cache, slots, kind):
    """Values [T, H, d] in 64 bits, through a table of all 256 scale bytes."""
    page, at = torch.div(slots, cache["page"], rounding_mode="floor"), torch.remainder(slots, cache["page"])
    byte = torch.arange(128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    magnitude = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    value = torch.tensor([s * m for s in (1.0, -1.0) for m in magnitude], dtype=F64, device="cuda")
    c, s = cache[kind + "_codes"][page, at].long(), cache[kind + "_scales"][page, at].long()
    x = torch.empty((*c.shape[:-1], 2 * c.shape[-1]), dtype=F64, device="cuda")
    x[..., 0::2], x[..., 1::2] = value[c % 16], value[c // 16]
    x *= byte[s].repeat_interleave(16, -1) * cache[kind + "_global"].double()[page][:, None, None]
    if kind == "k" and cache["k_mean"] is not None:
        x += cache["k_mean"][page, at].double()[..., None]
    return x


def _exact_attention(state):
    case, cache = state["case"], state["cache"]
    Hq, G, page = case["Hq"], case["Hq"] // case["Hk"], case["page"]
    n_q, n_kv = _ragged(case)
    if sum(a * n for a, n in zip(n_q, n_kv)) * Hq * case["d"] > 3e11:
        return None
    outs, lses, at = [], [], 0
    for b in range(case["B"]):
        a, n = n_q[b], n_kv[b]
        out = torch.zeros((a, Hq, case["d"]), dtype=F64, device="cuda")
        lse = torch.full((a, Hq), -math.inf, dtype=F64, device="cuda")
        if n:
            j = torch.arange(n, device="cuda")
            slots = state["table"][b].long()[j // page] * page + j % page
            k, v = _exact_slots(cache, slots, "k"), _exact_slots(cache, slots, "v")
            pos = (n - a + torch.arange(a, device="cuda")) if case["causal"] else torch.full((a,), n - 1, device="cuda")
            hidden = j[None] > pos[:, None]
            if case["window"]:
                hidden |= (j[None] <= pos[:, None] - case["window"]) & (j[None] >= case["sink"])
            for h in range(Hq):
                s = state["q"][at : at + a, h].double() @ k[:, h // G].T.contiguous() / math.sqrt(case["d"])
                s = s.masked_fill(hidden, -math.inf)
                lse[:, h] = torch.logsumexp(s, -1)
                w = torch.exp(s - lse[:, h, None])
                out[:, h] = torch.where(torch.isfinite(lse[:, h, None]), w, torch.zeros_like(w)) @ v[:, h // G].contiguous()
        outs.append(out)
        lses.append(lse)
        at += a
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] in ("norm_rope", "norm_rope_backward"):
        return _exact_norm_rope(state)
    if case["op"] == "cache_write":
        page = torch.div(state["slots"], case["page"], rounding_mode="floor")
        return {"k": _exact_written(state["k"], state["cache"]["k_global"][page], case["rule"], case["smooth"]),
                "v": _exact_written(state["v"], state["cache"]["v_global"][page], case["rule"], False)}
    if case["op"] == "cache_read":
        return {"k": _exact_slots(state["cache"], state["slots"], "k"), "v": _exact_slots(state["cache"], state["slots"], "v")}
    return _exact_attention(state)
