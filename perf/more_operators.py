"""The feed-forward half of a block in 8 bits as cases that can be timed and compared: quantizers to E4M3 with a power-of-two
scale for each 128 elements, the matrix product of such operands, the gated projections with their activation, the norm of the
residual stream in front of them, and the backward passes.

`own` false: the operators in their plain form, elementary torch operations in 32 bits.  `own` true: the calls of the library.
Both take what prepare() gives.
"""
import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 128
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a chunk of hidden activations in front of the down projection
        {"name": "quantize_chunk", "op": "quantize", "R": 3520, "C": 14336, "axis": 0, "kind": "activation", "strided": False},
        # an up projection's weights after an optimizer step, for the forward pass and transposed for the backward pass
        {"name": "quantize_weights", "op": "quantize_2d", "R": 14336, "C": 4096, "kind": "weight", "strided": False},
        # eight sequences that decode a token each: norm in front of the feed-forward block (latency)
        {"name": "norm_decode", "op": "norm", "T": 8, "C": 4096, "residual": True, "bf16": False, "strided": False},
        # a training clip: the norm's output in 8 bits for the layer and in bf16 for its weights' gradient
        {"name": "norm_train", "op": "norm", "T": 17600, "C": 5120, "residual": True, "bf16": True, "strided": False},
        # its gradient, joined with that of the residual stream
        {"name": "norm_backward_train", "op": "norm_backward", "T": 17600, "C": 5120, "residual": True, "strided": False},
        # a down projection for five sequences that decode a token each: the weights' bytes
        {"name": "gemm_decode", "op": "gemm", "M": 5, "N": 4096, "K": 14336, "tiles": True, "f32": False, "fast": False},
        # odd sizes: a short prompt through a projection whose width is no multiple of a tile or of a block
        {"name": "gemm_odd", "op": "gemm", "M": 777, "N": 1111, "K": 2000, "tiles": True, "f32": False, "fast": False},
        # the down projection of a chunk, with the sums that the 8-bit matrix instruction makes
        {"name": "gemm_chunk", "op": "gemm", "M": 3520, "N": 4096, "K": 14336, "tiles": True, "f32": False, "fast": True},
        # a weights' gradient, contracted over the tokens of a training clip (both operands with scales along the tokens)
        {"name": "gemm_weight_gradient", "op": "gemm", "M": 4096, "N": 2048, "K": 17600, "tiles": False, "f32": True, "fast": False},
        # gate and up projection for eight sequences that decode a token each
        {"name": "gated_decode", "op": "gated", "M": 8, "F": 14336, "K": 4096, "act": "silu", "train": False},
        # gate and up projection of a training clip's chunk, with what the backward pass needs
        {"name": "gated_chunk", "op": "gated", "M": 3520, "F": 11008, "K": 4096, "act": "silu", "train": True},
        # the activation's gradient in 8 bits along both axes, and the activations again for the down projection's weights
        {"name": "gated_backward", "op": "gated_backward", "T": 7040, "F": 11008, "act": "silu", "strided": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "quantize", "quantize_2d", "norm", "norm_backward", "gemm", "gemm", "gemm", "gated", "gated", "gated_backward"])
    strided = rng.random() < 0.3
    if op == "quantize":
        C = 16 * _log(rng, 1, 896)
        return {"op": op, "R": _log(rng, 1, min(17600, 3520 * 14336 // C)), "C": C, "axis": rng.randint(0, 1), "kind": rng.choice(["activation", "gradient"]), "strided": strided}
    if op == "quantize_2d":
        C = 16 * _log(rng, 4, 512)
        return {"op": op, "R": 16 * _log(rng, 4, min(896, 14336 * 256 // C)), "C": C, "kind": "weight", "strided": strided}
    if op in ("norm", "norm_backward"):
        C = 16 * _log(rng, 4, 512)
        case = {"op": op, "T": _log(rng, 1, min(17600, 17600 * 5120 // C)), "C": C, "residual": rng.random() < 0.7, "strided": strided}
        return {**case, "bf16": rng.random() < 0.4} if op == "norm" else case
    if op == "gated_backward":
        F = 128 * _log(rng, 1, 112)
        return {"op": op, "T": _log(rng, 1, min(17600, 7040 * 11008 // F)), "F": F, "act": rng.choice(["silu", "gelu"]), "strided": strided}
    K = 16 * _log(rng, 8, 896)
    if op == "gated":
        F = 16 * _log(rng, 8, 896)
        room = min(4096, int(3.1e11 / (2 * F * K)))
        return {"op": op, "M": rng.choice([_log(rng, 1, 64), _log(rng, 1, room)]), "F": F, "K": K, "act": rng.choice(["silu", "silu", "gelu"]), "train": rng.random() < 0.4}
    N = rng.choice([16 * _log(rng, 4, 896), _log(rng, 50, 5000)])
    room = min(8192, int(2.0e11 / (N * K)))
    f32 = rng.random() < 0.3
    return {"op": op, "M": rng.choice([_log(rng, 1, 64), _log(rng, 1, room), _log(rng, 1, room)]), "N": N, "K": K, "tiles": rng.random() < 0.6, "f32": f32,
            "fast": not f32 and rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=F32)


def _matrix(g, R, C, kind, strided=False):
    """bf16 [R, C].  Activations: a few channels that are much larger; weights and gradients: small, with scales of their own for each row."""
    x = _normal(g, R, C + 24 if strided else C)
    if kind == "activation":
        x *= torch.exp(0.5 * _normal(g, x.shape[1])) * torch.where(torch.rand(x.shape[1], generator=g, device="cuda") < 0.01, 20.0, 1.0)
    else:
        x *= {"weight": 0.02, "gradient": 1e-3}[kind] * torch.exp(0.3 * _normal(g, R, 1))
    return x.to(BF16)[:, 8 : 8 + C] if strided else x.to(BF16)


def _held(x, tiles=False):
    """What a program holds of a matrix in 8 bits: codes and scales."""
    codes, scales = _quantized_tiles(x.to(F32)) if tiles else _quantized(x.to(F32))
    return {"codes": codes, "scales": scales}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state, op = {"case": case}, case["op"]
    if op in ("quantize", "quantize_2d"):
        return {**state, "x": _matrix(g, case["R"], case["C"], case["kind"], case["strided"])}
    if op in ("norm", "norm_backward"):
        T, C = case["T"], case["C"]
        state["weight"] = (1 + 0.2 * _normal(g, C)).to(BF16)
        state["x"] = _matrix(g, T, C, "activation", case["strided"])
        if op == "norm":
            state["residual"] = (8 * _normal(g, T, C)).to(BF16) if case["residual"] else None
        else:
            state["dy"] = _matrix(g, T, C, "gradient", case["strided"])
            state["dsum"] = (1e-3 * _normal(g, T, C)).to(BF16) if case["residual"] else None
        return state
    if op == "gated_backward":
        T, F = case["T"], case["F"]
        state["dh"] = _matrix(g, T, F, "gradient", case["strided"])
        state["gate_up"] = (1.3 * _normal(g, T, 2 * F)).to(BF16)
        return state
    if op == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        if case["tiles"]:
            return {**state, "a": _held(_matrix(g, M, K, "activation")), "w": _held(_matrix(g, N, K, "weight"), tiles=True)}
        return {**state, "a": _held(_matrix(g, M, K, "gradient")), "w": _held(_matrix(g, N, K, "activation"))}
    return {**state, "a": _held(_matrix(g, case["M"], case["K"], "activation")), "w": _held(_matrix(g, 2 * case["F"], case["K"], "weight"), tiles=True)}


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _ceil(n, to):
    return -(-n // to)


def _padded(x, rows, cols):
    R, C = x.shape
    return x if (R, C) == (rows, cols) else torch.nn.functional.pad(x, (0, cols - C, 0, rows - R))


def _exponent(amax):
    """The smallest e >= -127 with amax <= 448 * 2^e."""
    m, k = torch.frexp(amax)                                        # amax = m 2^k, 1/2 <= m < 1; 448 = 7/8 * 2^9
    return torch.where(amax > 0, torch.where(m <= 0.875, k - 9, k - 8), -127).clamp(min=-127)


def _power(e):
    """2^e in 32 bits, for the exponents of normal numbers."""
    return ((e.to(torch.int32) + 127) << 23).view(F32)


def _byte(e):
    return (e + 127).to(torch.uint8).view(E8M0)


def _quantized(x):
    """Matrix [R, C] in 32 bits -> E4M3 codes [R, C] and E8M0 scales [R, C / 128], a scale for 128 neighbours of a row."""
    R, C = x.shape
    b = _padded(x, R, BLOCK * _ceil(C, BLOCK)).view(R, -1, BLOCK)
    e = _exponent(b.abs().amax(-1))
    return (b * _power(-e).unsqueeze(-1)).to(E4M3).view(R, -1)[:, :C].contiguous(), _byte(e)


def _quantized_tiles(x):
    """... with a scale for 128 x 128 elements: [R / 128, C / 128]."""
    R, C = x.shape
    b = _padded(x, BLOCK * _ceil(R, BLOCK), BLOCK * _ceil(C, BLOCK)).unflatten(0, (-1, BLOCK)).unflatten(2, (-1, BLOCK))
    e = _exponent(b.abs().amax((1, 3)))
    codes = (b * _power(-e)[:, None, :, None]).to(E4M3)
    return codes.flatten(2, 3).flatten(0, 1)[:R, :C].contiguous(), _byte(e)


def _quantized_columns(x):
    """Matrix [T, C] -> its transpose [C, T], scales along T, T filled up with zeros to a multiple of 16."""
    return _quantized(_padded(x, 16 * _ceil(x.shape[0], 16), x.shape[1]).T.contiguous())


def _values(held, dtype=F32):
    """What codes and scales stand for."""
    rows, K = held["codes"].shape
    s = held["scales"].to(dtype)
    if s.shape[0] != rows:
        s = s.repeat_interleave(BLOCK, 0)[:rows]
    return held["codes"].to(dtype) * s.repeat_interleave(BLOCK, 1)[:, :K]


def _activation(act, g):
    """act(g) and its derivative."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _norm_plain(state):
    case, w = state["case"], state["weight"].to(F32)
    s = state["x"].to(F32)
    answer = {}
    if case["residual"]:
        answer["sum"] = (s + state["residual"].to(F32)).to(BF16)
        s = answer["sum"].to(F32)
    y = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + EPS) * w
    answer["codes"], answer["scales"] = _quantized(y)
    return {**answer, "y": y.to(BF16)} if case["bf16"] else answer


def _norm_backward_plain(state):
    w, x, dy = state["weight"].to(F32), state["x"].to(F32), state["dy"].to(F32)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh = x * r
    dx = r * (dy * w - xh * (dy * w * xh).mean(-1, keepdim=True))
    if state["dsum"] is not None:
        dx = dx + state["dsum"].to(F32)
    return {"dx": dx.to(BF16), "dweight": (dy * xh).sum(0, dtype=F64).to(F32)}


def _gated_plain(state):
    case = state["case"]
    gu = torch.matmul(_values(state["a"]), _values(state["w"]).T)
    g, u = gu[:, : case["F"]], gu[:, case["F"] :]
    h = _activation(case["act"], g)[0] * u
    codes, scales = _quantized(h)
    return {"codes": codes, "scales": scales, "gate_up": gu.to(BF16)} if case["train"] else {"codes": codes, "scales": scales}


def _gated_backward_plain(state):
    case = state["case"]
    g, u, dh = state["gate_up"][:, : case["F"]].to(F32), state["gate_up"][:, case["F"] :].to(F32), state["dh"].to(F32)
    a, slope = _activation(case["act"], g)
    d = torch.cat([dh * u * slope, dh * a], 1)
    answer = {}
    answer["codes"], answer["scales"] = _quantized(d)
    answer["codes_t"], answer["scales_t"] = _quantized_columns(d)
    answer["h_codes_t"], answer["h_scales_t"] = _quantized_columns(a * u)
    return answer


def run(state):
    if own:
        return _run_own(state)
    case, op = state["case"], state["case"]["op"]
    if op == "quantize":
        codes, scales = _quantized(state["x"].to(F32)) if case["axis"] == 0 else _quantized_columns(state["x"].to(F32))
        return {"codes": codes, "scales": scales}
    if op == "quantize_2d":
        codes, scales = _quantized_tiles(state["x"].to(F32))
        return {"codes": codes, "scales": scales, "codes_t": codes.view(torch.uint8).T.contiguous().view(E4M3), "scales_t": scales.view(torch.uint8).T.contiguous().view(E8M0)}
    if op == "gemm":
        y = torch.matmul(_values(state["a"]), _values(state["w"]).T)
        return {"y": y if case["f32"] else y.to(BF16)}
    return {"norm": _norm_plain, "norm_backward": _norm_backward_plain, "gated": _gated_plain, "gated_backward": _gated_backward_plain}[op](state)


def _run_own(state):
    import paper_2605_18739_amd as nv

    case, op = state["case"], state["case"]["op"]
    act = nv.ACT_SILU if case.get("act") == "silu" else nv.ACT_GELU_TANH
    if op == "quantize":
        q = nv.nvfp4_e4m3_quantize(state["x"], block_axis=case["axis"])
        return {"codes": q.codes, "scales": q.scales}
    if op == "quantize_2d":
        q, t = nv.nvfp4_e4m3_quantize_2d(state["x"])
        return {"codes": q.codes, "scales": q.scales, "codes_t": t.codes, "scales_t": t.scales}
    if op == "norm":
        q, y, s = nv.nvfp4_rms_norm(state["x"], state["weight"], state["residual"], eps=EPS, keep_bf16=case["bf16"])
        answer = {"codes": q.codes, "scales": q.scales}
        if case["residual"]:
            answer["sum"] = s
        return {**answer, "y": y} if case["bf16"] else answer
    if op == "norm_backward":
        dx, dweight = nv.nvfp4_rms_norm_backward(state["dy"], state["x"], state["weight"], state["dsum"], eps=EPS)
        return {"dx": dx, "dweight": dweight}
    if op == "gated_backward":
        d, d_t, h_t, _ = nv.nvfp4_gated_backward(state["dh"], state["gate_up"], act=act, recompute_h=True)
        return {"codes": d.codes, "scales": d.scales, "codes_t": d_t.codes, "scales_t": d_t.scales, "h_codes_t": h_t.codes, "h_scales_t": h_t.scales}
    if "handles" not in state:                                      # what a program keeps beside its operands' memory
        state["handles"] = [nv.E4M3Tensor(state[n]["codes"], state[n]["scales"]) for n in ("a", "w")]
    a, w = state["handles"]
    if op == "gemm":
        return {"y": nv.nvfp4_e4m3_gemm(a, w, out_dtype=nv.OUT_F32 if case["f32"] else nv.OUT_BF16, fast_sums=case["fast"])}
    q, _, gate_up = nv.nvfp4_e4m3_gemm_gated(a, w, act=act, keep_gate_up=case["train"])
    return {"codes": q.codes, "scales": q.scales, "gate_up": gate_up} if case["train"] else {"codes": q.codes, "scales": q.scales}


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def _held_bytes(rows, K, tiles=False):
    return rows * K + (_ceil(rows, BLOCK) if tiles else rows) * _ceil(K, BLOCK)


def work(case):
    op = case["op"]
    if op in ("quantize", "quantize_2d"):
        R, C = case["R"], case["C"]
        n = R * C
        if op == "quantize_2d":
            return {"bytes": 2 * n + 2 * _held_bytes(R, C, True), "flops": 2 * n}
        return {"bytes": 2 * n + (_held_bytes(R, C) if case["axis"] == 0 else _held_bytes(C, 16 * _ceil(R, 16))), "flops": 2 * n}
    if op == "norm":
        T, C = case["T"], case["C"]
        return {"bytes": T * C * (2 + (4 if case["residual"] else 0) + (2 if case["bf16"] else 0)) + _held_bytes(T, C) + 2 * C, "flops": 7 * T * C}
    if op == "norm_backward":
        T, C = case["T"], case["C"]
        return {"bytes": T * C * (6 + (2 if case["residual"] else 0)) + 6 * C, "flops": 12 * T * C}
    if op == "gated_backward":
        T, F = case["T"], case["F"]
        t = 16 * _ceil(T, 16)
        return {"bytes": 6 * T * F + _held_bytes(T, 2 * F) + _held_bytes(2 * F, t) + _held_bytes(F, t), "flops": 24 * T * F}
    M, K = case["M"], case["K"]
    if op == "gemm":
        N = case["N"]
        return {"bytes": _held_bytes(M, K) + _held_bytes(N, K, case["tiles"]) + M * N * (4 if case["f32"] else 2), "flops": 2 * M * N * K}
    F = case["F"]
    return {"bytes": _held_bytes(M, K) + _held_bytes(2 * F, K, True) + _held_bytes(M, F) + (4 * M * F if case["train"] else 0), "flops": 4 * M * F * K}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_grid():
    """The non-negative E4M3 numbers in order: code n is number n."""
    return torch.tensor([m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1], dtype=F64, device="cuda")


def _exact_nearest(y):
    """The nearest E4M3 number by comparing with every midpoint; the even code wins a tie."""
    grid = _exact_grid()
    mid, y = (grid[1:] + grid[:-1]) / 2, y.contiguous()
    low, up = torch.bucketize(y.abs(), mid), torch.bucketize(y.abs(), mid, right=True)          # midpoints below y, and those that y meets
    return torch.copysign(grid[torch.where(low % 2 == 0, low, up)], y)


def _exact_scale(amax):
    """The smallest power of two from 2^-127 on that amax is not above 448 times of, by comparing with all of them."""
    powers = torch.pow(torch.tensor(2.0, dtype=F64), torch.arange(-127, 121, dtype=F64)).cuda()
    return powers[torch.bucketize(amax.contiguous(), 448 * powers)]


def _exact_codes(x):
    """Rows in 64 bits -> the values of their codes and scales, block after block."""
    codes, scales = torch.empty_like(x), torch.empty((x.shape[0], _ceil(x.shape[1], BLOCK)), dtype=F64, device="cuda")
    for b in range(scales.shape[1]):
        v = x[:, b * BLOCK : (b + 1) * BLOCK]
        scales[:, b] = _exact_scale(v.abs().amax(1))
        codes[:, b * BLOCK : (b + 1) * BLOCK] = _exact_nearest(v / scales[:, b : b + 1])
    return codes, scales


def _exact_tile_codes(x):
    codes, scales = torch.empty_like(x), torch.empty((_ceil(x.shape[0], BLOCK), _ceil(x.shape[1], BLOCK)), dtype=F64, device="cuda")
    column = torch.arange(x.shape[1], device="cuda") // BLOCK
    for r in range(scales.shape[0]):
        band = x[r * BLOCK : (r + 1) * BLOCK]
        top = torch.zeros(scales.shape[1], dtype=F64, device="cuda").scatter_reduce_(0, column, band.abs().amax(0), "amax")
        scales[r] = _exact_scale(top)
        codes[r * BLOCK : (r + 1) * BLOCK] = _exact_nearest(band / scales[r][column])
    return codes, scales


def _exact_columns(x):
    T, C = x.shape
    wide = torch.zeros((C, 16 * _ceil(T, 16)), dtype=F64, device="cuda")
    wide[:, :T] = x.T
    return _exact_codes(wide)


def _exact_values(held):
    """Codes and scales by their bytes."""
    grid = _exact_grid()
    code = held["codes"].view(torch.uint8).long()
    v = grid[(code & 127).clamp(max=126)] * (1 - 2 * (code >> 7)).double()
    s = torch.pow(torch.tensor(2.0, dtype=F64, device="cuda"), held["scales"].view(torch.uint8).double() - 127)
    row = torch.arange(v.shape[0], device="cuda") // (1 if s.shape[0] == v.shape[0] else BLOCK)
    return v * s[row][:, torch.arange(v.shape[1], device="cuda") // BLOCK]


def _exact_activation(act, g):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    z = math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)                        # (1 + tanh(z / 2)) / 2 = sigmoid(z)
    s = torch.sigmoid(z)
    return g * s, s + g * s * torch.sigmoid(-z) * math.sqrt(8 / math.pi) * (1 + 0.134145 * g ** 2)


def exact(case, seed):
    state, op = prepare(case, seed), case["op"]
    if op == "quantize":
        codes, scales = _exact_codes(state["x"].double()) if case["axis"] == 0 else _exact_columns(state["x"].double())
        return {"codes": codes, "scales": scales}
    if op == "quantize_2d":
        codes, scales = _exact_tile_codes(state["x"].double())
        return {"codes": codes, "scales": scales, "codes_t": codes.T.contiguous(), "scales_t": scales.T.contiguous()}
    if op == "norm":
        s, answer = state["x"].double(), {}
        if case["residual"]:
            s = answer["sum"] = (s + state["residual"].double()).to(BF16).double()      # (rounded: the stream that later layers read)
        y = s / torch.sqrt((s * s).sum(1, keepdim=True) / case["C"] + EPS) * state["weight"].double()
        answer["codes"], answer["scales"] = _exact_codes(y)
        return {**answer, "y": y} if case["bf16"] else answer
    if op == "norm_backward":
        x, g = state["x"].double(), state["dy"].double() * state["weight"].double()
        norm = torch.sqrt((x * x).sum(1, keepdim=True) / case["C"] + EPS)
        # y = w x / norm: dx = w dy / norm - x sum(w dy x) / (C norm^3)
        dx = g / norm - x * (g * x).sum(1, keepdim=True) / (case["C"] * norm ** 3)
        dx = dx if state["dsum"] is None else dx + state["dsum"].double()
        return {"dx": dx, "dweight": (state["dy"].double() * x / norm).sum(0)}
    if op == "gated_backward":
        F = case["F"]
        gu, dh = state["gate_up"].double(), state["dh"].double()
        a, slope = _exact_activation(case["act"], gu[:, :F])
        d = torch.cat([dh * gu[:, F:] * slope, dh * a], 1)
        codes, scales = _exact_codes(d)
        codes_t, scales_t = _exact_columns(d)
        h_codes_t, h_scales_t = _exact_columns(a * gu[:, F:])
        return {"codes": codes, "scales": scales, "codes_t": codes_t, "scales_t": scales_t, "h_codes_t": h_codes_t, "h_scales_t": h_scales_t}
    y = _exact_values(state["a"]) @ _exact_values(state["w"]).T.contiguous()
    if op == "gemm":
        return {"y": y}
    F = case["F"]
    h = _exact_activation(case["act"], y[:, :F])[0] * y[:, F:]
    codes, scales = _exact_codes(h)
    return {"codes": codes, "scales": scales, "gate_up": y} if case["train"] else {"codes": codes, "scales": scales}
