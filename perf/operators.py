"""Cases of the block-scaled operators: rows and weights in 8 bits (e4m3) or 4 (e2m1), a power of two for every 32 elements of a row.

quant    rows of float32 / bfloat16 to e4m3 codes and scales
norm     residual addition, RMSNorm, e4m3 codes and scales
mx       products of e4m3 rows with e4m3 or e2m1 weights
swiglu   the gate/up product of such rows with silu(gate) * up in e4m3 codes and scales
w4       products of float32 / bfloat16 rows with e2m1 weights

Sizes are those of the LLaDA-8B-shaped model of the benchmark (d_model 4096, d_ff 12288), of its canvases (5 x 512 and 9 x 1280 tokens), of its
K/V-cached rounds (64 rows a canvas) and odd ones.  Codes are returned as float8_e4m3fn and scales as float8_e8m0fnu: the values they stand for.
"""
import math

import torch

own = False

E4M3, E2M1 = "e4m3", "e2m1"
TOP = {E4M3: 448.0, E2M1: 6.0}                      # largest value of a code
STEPS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)    # e2m1 by code; bit 3 is the sign
EPS = 1e-5


# ---------------------------------------------------------------- cases
def listed():
    return [
        # a single token between two layers: latency
        {"name": "norm_1x4096", "op": "norm", "M": 1, "K": 4096, "dtype": "bf16"},
        # nine canvases of 1280 tokens: the largest batch of a planned round
        {"name": "norm_11520x4096", "op": "norm", "M": 11520, "K": 4096, "dtype": "bf16"},
        # the attention's output of a cached round with four drafts, for the O projection
        {"name": "quant_320x4096", "op": "quant", "M": 320, "K": 4096, "dtype": "bf16"},
        # rows of no round width, float32
        {"name": "quant_2443x1411_f32", "op": "quant", "M": 2443, "K": 1411, "dtype": "f32"},
        # down projection of a cached round with four drafts, into the residual stream
        {"name": "mx_320x4096x12288", "op": "mx", "M": 320, "N": 4096, "K": 12288, "w": E4M3, "dtype": "bf16", "residual": True},
        # QKV of nine canvases of 1280 tokens: bound by the matrix rate
        {"name": "mx_11520x12288x4096", "op": "mx", "M": 11520, "N": 12288, "K": 4096, "w": E4M3, "dtype": "bf16", "residual": False},
        # a ragged canvas through a small float32 projection with 4-bit weights
        {"name": "mx_437x1003x1411_f32", "op": "mx", "M": 437, "N": 1003, "K": 1411, "w": E2M1, "dtype": "f32", "residual": True},
        # gate/up of one cached canvas with 4-bit weights: bound by the weights' bytes
        {"name": "swiglu_64x12288x4096", "op": "swiglu", "M": 64, "N": 12288, "K": 4096, "w": E2M1},
        # gate/up of five canvases of 512 tokens
        {"name": "swiglu_2560x12288x4096", "op": "swiglu", "M": 2560, "N": 12288, "K": 4096, "w": E4M3},
        # QKV of a single token: a matrix-vector product
        {"name": "w4_1x12288x4096", "op": "w4", "M": 1, "N": 12288, "K": 4096, "dtype": "bf16", "residual": False},
        # odd sizes, float32 rows
        {"name": "w4_33x4001x1411_f32", "op": "w4", "M": 33, "N": 4001, "K": 1411, "dtype": "f32", "residual": False},
        # O projection of a cached round with four drafts, rows as they are
        {"name": "w4_320x4096x4096", "op": "w4", "M": 320, "N": 4096, "K": 4096, "dtype": "bf16", "residual": True},
    ]


def _spread(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; half of them round ones where there is room."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n >= 256 and rng.random() < 0.5:
        n = n // 64 * 64
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(("norm", "quant", "mx", "mx", "swiglu", "w4", "w4"))
    case = {"op": op, "M": _spread(rng, 1, 1024 if op == "w4" else 11520), "K": _spread(rng, 32, 12288)}
    if op in ("norm", "quant"):
        case["M"] = min(case["M"], 11520 * 4096 // case["K"])
    else:
        case["N"] = _spread(rng, 16, 12288 if op == "swiglu" else 24576)
        most = 11520 * 12288 * 4096 // (2 if op == "swiglu" else 1)
        case["M"] = max(1, min(case["M"], most // (case["N"] * case["K"])))
    if op in ("mx", "swiglu"):
        case["w"] = rng.choice((E4M3, E2M1))
    if op != "swiglu":
        case["dtype"] = rng.choice(("bf16", "bf16", "f32"))
    if op in ("mx", "w4"):
        case["residual"] = rng.random() < 0.5
    return case


def _type(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _width(K):
    return (K + 127) // 128 * 128


# ---------------------------------------------------------------- inputs
def _rows(M, K, dtype, gen):
    """Activations: unit normal rows, with a few channels many times larger as the residual streams of trained models have them."""
    x = torch.randn(M, K, device="cuda", generator=gen)
    loud = torch.rand(K, device="cuda", generator=gen) < 0.004
    return (x * (1 + 19 * loud.float())).to(dtype)


def prepare(case, seed):
    """Codes, scales and rows in GPU memory, and the buffers that a decoding loop keeps for its results."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, M, K = case["op"], case["M"], case["K"]
    Kp, state = _width(K), dict(case)
    codes = lambda m, k: torch.empty(m, k, dtype=torch.float8_e4m3fn, device="cuda")  # noqa: E731
    scales = lambda m, k: torch.empty(k // 128, m, 4, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)  # noqa: E731
    if op in ("norm", "quant"):
        state["x"] = _rows(M, K, _type(case), gen)
        state["codes"], state["scales"] = codes(M, Kp), scales(M, Kp)
        if op == "norm":
            state["residual"] = _rows(M, K, _type(case), gen)
            state["gain"] = (1 + 0.2 * torch.randn(K, device="cuda", generator=gen)).to(_type(case))
            state["sum"] = torch.empty_like(state["x"])
        return state
    N = case["N"]
    w = torch.randn(2 * N if op == "swiglu" else N, K, device="cuda", generator=gen) * 0.02
    if op == "w4":
        state["x"] = _rows(M, K, _type(case), gen)
        state["W"], state["w_scale"] = _quantised(w, E2M1)
    else:
        state["A"], state["a_scale"] = _quantised(_rows(M, K, torch.float32, gen), E4M3)
        state["W"], state["w_scale"] = _quantised(w, case["w"])
    if op == "swiglu":
        state["codes"], state["scales"] = codes(M, _width(N)), scales(M, _width(N))
    else:
        state["res"] = torch.randn(M, N, device="cuda", generator=gen).to(_type(case)) if case["residual"] else None
        state["out"] = torch.empty(M, N, dtype=_type(case), device="cuda")
    return state


# ---------------------------------------------------------------- plain forms
def _two(e):
    """2^e in 64 bits, exactly, for whole e (torch's pow and exp2 may be a bit off)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantised(x, fmt):
    """Codes [M, Kp] (e2m1: two a byte, [M, Kp / 2]) and scales [Kp / 128, M, 4] of float32 rows."""
    M, K = x.shape
    Kp = _width(K)
    blocks = torch.nn.functional.pad(x, (0, Kp - K)).view(M, Kp // 32, 32)
    amax = blocks.abs().amax(2)
    mant, power = torch.frexp(amax)                            # amax = mant 2^power, mant in [0.5, 1)
    top = math.frexp(TOP[fmt])
    power = power - top[1] + (mant > top[0]).int()             # smallest power with amax <= top 2^power
    power = torch.where(amax > 0, power, -127).clamp(min=-127)
    y = (blocks.double() * _two(-power).unsqueeze(2)).float()
    scale = (power + 127).to(torch.uint8).view(M, Kp // 128, 4).transpose(0, 1).contiguous().view(torch.float8_e8m0fnu)
    y = y.view(M, Kp)
    if fmt == E4M3:
        return y.to(torch.float8_e4m3fn), scale
    a = y.abs()                                                # ties to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)) | (y.signbit().to(torch.uint8) << 3)
    return code[:, 0::2] | (code[:, 1::2] << 4), scale


def _values(codes, scale, fmt):
    """The float32 rows that codes and scales stand for."""
    if fmt == E2M1:
        table = torch.tensor(STEPS + tuple(-s for s in STEPS), device=codes.device)
        v = table[torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1).int()]
    else:
        v = codes.float()
    M, Kp = v.shape
    return (v.view(M, Kp // 32, 32) * scale.float().transpose(0, 1).reshape(M, Kp // 32, 1)).view(M, Kp)


def run(state):
    if own:
        return _own(state)
    op = state["op"]
    if op == "quant":
        codes, scale = _quantised(state["x"].float(), E4M3)
        return {"codes": codes, "scale": scale}
    if op == "norm":
        h = (state["x"].float() + state["residual"].float()).to(state["x"].dtype)
        inv = (1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + EPS)).float()      # 64 bits: codes next to a border
        codes, scale = _quantised(h.float() * inv * state["gain"].float(), E4M3)
        return {"sum": h, "codes": codes, "scale": scale}
    if op == "w4":
        a = torch.nn.functional.pad(state["x"].float(), (0, _width(state["K"]) - state["K"]))
        w = _values(state["W"], state["w_scale"], E2M1)
    else:
        a, w = _values(state["A"], state["a_scale"], E4M3), _values(state["W"], state["w_scale"], state["w"])
    c = a @ w.T
    if op == "swiglu":
        gate, up = c[:, :state["N"]], c[:, state["N"]:]
        codes, scale = _quantised(gate / (1 + torch.exp(-gate)) * up, E4M3)
        return {"codes": codes, "scale": scale}
    if state["res"] is not None:
        c = c + state["res"].float()
    return c.to(state["out"].dtype)


def _own(s):
    from paper_2601_12247_amd import binding as B
    op = s["op"]
    if op == "quant":
        codes, scale = B.quant_mx(s["x"], out=(s["codes"], s["scales"]))
        return {"codes": codes, "scale": scale}
    if op == "norm":
        h, codes, scale = B.add_rmsnorm_mx(s["x"], s["gain"], EPS, residual=s["residual"], sum_out=s["sum"], out=(s["codes"], s["scales"]))
        return {"sum": h, "codes": codes, "scale": scale}
    if op == "w4":
        return B.gemm_w4(s["x"], s["W"], s["w_scale"], residual=s["res"], out=s["out"])
    if op == "swiglu":
        codes, scale = B.gemm_mx_swiglu(s["A"], s["a_scale"], s["W"], s["w_scale"], out=(s["codes"], s["scales"]))
        return {"codes": codes, "scale": scale}
    return B.gemm_mx(s["A"], s["a_scale"], s["W"], s["w_scale"], residual=s["res"], out=s["out"])


# ---------------------------------------------------------------- work and exact results
def work(case):
    op, M, K = case["op"], case["M"], case["K"]
    size, Kp = (4 if case.get("dtype") == "f32" else 2), _width(K)
    rows = M * Kp * 33 / 32                                    # codes and scales
    if op == "quant":
        return {"bytes": M * K * size + rows, "flops": 2 * M * K}
    if op == "norm":
        return {"bytes": 3 * M * K * size + K * size + rows, "flops": 7 * M * K}
    N = case["N"]
    w = Kp * (17 / 32 if case.get("w", E2M1) == E2M1 else 33 / 32)
    if op == "swiglu":
        return {"bytes": rows + 2 * N * w + M * _width(N) * 33 / 32, "flops": 4 * M * N * K}
    return {"bytes": (M * K * size if op == "w4" else rows) + N * w + M * N * size * (2 if case["residual"] else 1), "flops": 2 * M * N * K}


def _grid64(y, K):
    """Codes and scales of float64 rows as float64 values, from the definition: the scale is the smallest power of two, from 2^-127 on, that
    brings the block's largest magnitude to 448 at most; the element is the nearest multiple of its binade's step, ties to even."""
    M = y.shape[0]
    Kp = _width(K)
    full = torch.zeros(M, Kp, dtype=torch.float64, device=y.device)
    full[:, :K] = y
    b = full.reshape(M, -1, 32)
    largest = b.abs().max(dim=2).values
    e = torch.ceil(torch.log2(torch.clamp(largest, min=2.0 ** -900) / 448))
    e = torch.where(largest > 448 * _two(e), e + 1, e)
    e = torch.where(largest <= 448 * _two(e - 1), e - 1, e)
    e = torch.clamp(e, min=-127)
    v = b / _two(e)[:, :, None]
    binade = torch.floor(torch.log2(torch.clamp(v.abs(), min=2.0 ** -900)))
    binade = torch.where(v.abs() < _two(binade), binade - 1, binade)
    binade = torch.where(v.abs() >= _two(binade + 1), binade + 1, binade)
    step = _two(torch.clamp(binade, min=-6) - 3)
    codes = torch.round(v / step) * step
    return codes.reshape(M, Kp), _two(e).reshape(M, -1, 4).permute(1, 0, 2).contiguous()


def _read64(codes, scale):
    """The float64 rows behind codes (float8 or pairs of 4 bits) and scales, by the bits' meaning."""
    s = _two(scale.view(torch.uint8).long() - 127).permute(1, 0, 2).reshape(scale.shape[1], -1)
    if codes.dtype == torch.uint8:
        both = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.int64, device=codes.device)
        both[:, 0::2], both[:, 1::2] = codes % 16, codes // 16
        e, m = both // 2 % 4, (both % 2).double()
        v = torch.where(e > 0, _two(e - 1) * (1 + m / 2), m / 2) * torch.where(both >= 8, -1.0, 1.0)
    else:
        bits = codes.view(torch.uint8).long()
        e, m = bits // 8 % 16, (bits % 8).double()
        v = torch.where(e > 0, _two(e - 7) * (1 + m / 8), m / 512) * torch.where(bits >= 128, -1.0, 1.0)
    return v * s.repeat_interleave(32, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    op, K = case["op"], case["K"]
    if op == "quant":
        codes, scale = _grid64(s["x"].double(), K)
        return {"codes": codes, "scale": scale}
    if op == "norm":
        total = s["x"].double() + s["residual"].double()
        h = total.to(s["x"].dtype).double()
        codes, scale = _grid64(h * torch.rsqrt((h * h).sum(1) / K + EPS)[:, None] * s["gain"].double(), K)
        return {"sum": total, "codes": codes, "scale": scale}
    w = _read64(s["W"], s["w_scale"])
    if op == "w4":
        c = torch.mm(s["x"].double(), w[:, :K].t())
    else:
        c = torch.mm(_read64(s["A"], s["a_scale"]), w.t())
    if op == "swiglu":
        gate, up = c.chunk(2, dim=1)
        codes, scale = _grid64(gate * torch.sigmoid(gate) * up, case["N"])
        return {"codes": codes, "scale": scale}
    return c if s["res"] is None else c + s["res"].double()
