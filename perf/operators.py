"""Cases that measure the 8-bit floating-point operators of the library on a GPU: the residual addition with RMS norm and
quantization (``xq_f8_norm_quant``), the block-scaled product (``xq_f8_gemm``, ``xq_f8_linear``) and the gated pair of
products (``xq_f8_gated``).

The 8-bit format: E4M3 elements with one E8M0 scale (a power of two, stored as its exponent + 127) for each group of 128
consecutive channels of a token row, and for each 128 x 128 block of a weight matrix.  A group's exponent is the smallest e
with max |v| <= 448 * 2^e; an element is the E4M3 value nearest to v / 2^e, ties to even.  Token rows are held as bytes
[M, Kq], Kq = K rounded up to 128 (padding: zero codes), and scale bytes [M, P], P = K / 128 rounded up to a multiple of
four (padding and groups of zeros: 127, a scale of one).

``run`` computes either the operators' plain form in torch (``own`` false), or calls the library (``own`` true).
"""
import math

import torch

own = False

EPS = 1e-5


# --- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # residual addition + RMS norm + quantization: one decoded token of an 8B-sized model, a decode batch of a 1B-sized one,
        # a ragged prefill of odd width that also wants the normalised rows in bf16 (for a layer that takes bf16 tokens), and
        # the first norm of a long prefill
        {"name": "norm_1x4096", "op": "norm", "M": 1, "K": 4096, "residual": True, "y": False},
        {"name": "norm_32x2048", "op": "norm", "M": 32, "K": 2048, "residual": True, "y": False},
        {"name": "norm_777x2876_y", "op": "norm", "M": 777, "K": 2876, "residual": False, "y": True},
        {"name": "norm_16384x8192", "op": "norm", "M": 16384, "K": 8192, "residual": True, "y": False},
        # product: the down projection of one token, the QKV projection of a decode batch from bf16 rows (quantization
        # included), a ragged middle size, the down projection of a prefill
        {"name": "gemm_1_14336_4096", "op": "gemm", "M": 1, "K": 14336, "N": 4096},
        {"name": "linear_16_4096_6144", "op": "linear", "M": 16, "K": 4096, "N": 6144},
        {"name": "gemm_333_2720_5005", "op": "gemm", "M": 333, "K": 2720, "N": 5005},
        {"name": "gemm_4096_14336_4096", "op": "gemm", "M": 4096, "K": 14336, "N": 4096},
        # gated pair: one token whose result goes on in bf16 (to an expanded W4A4 down projection), a decode batch and a ragged
        # prefill whose result goes on in 8 bits, a full prefill
        {"name": "gated_1_4096_14336_bf16", "op": "gated", "M": 1, "K": 4096, "N": 14336, "out8": False},
        {"name": "gated_24_2048_8192", "op": "gated", "M": 24, "K": 2048, "N": 8192, "out8": True},
        {"name": "gated_517_1800_5000", "op": "gated", "M": 517, "K": 1800, "N": 5000, "out8": True},
        {"name": "gated_4096_4096_14336", "op": "gated", "M": 4096, "K": 4096, "N": 14336, "out8": True},
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["norm", "gemm", "linear", "gated"])
    if op == "norm":
        return {"op": op, "M": size(1, 16384), "K": size(128, 8192), "residual": rng.random() < 0.7, "y": rng.random() < 0.3}
    while True:
        c = {"op": op, "M": size(1, 4096), "K": size(128, 14336), "N": size(128, 14336)}
        if rng.random() < 0.5:  # widths of models are mostly round
            c["K"], c["N"] = max(128, c["K"] // 128 * 128), max(128, c["N"] // 128 * 128)
        if op == "gated":
            c["out8"] = rng.random() < 0.6
        if c["M"] * c["K"] * c["N"] <= 4096 * 14336 * 4096:
            return c


# --- the format ----------------------------------------------------------------------------------------------------

def _up(v, a):
    return -(-v // a) * a


def _pad(v, cols):
    return v if v.shape[1] == cols else torch.cat([v, v.new_zeros(v.shape[0], cols - v.shape[1])], 1)


def _scale_bytes(amax):
    """Smallest e with amax <= 448 * 2^e, plus 127 (127 for zero): amax = m * 2^k with m in [0.5, 1), 448 = 0.875 * 2^9."""
    m, k = torch.frexp(amax)
    e = k - 9 + (m > 0.875).int()
    return torch.where(amax == 0, torch.zeros_like(e), e.clamp(-127, 127)) + 127


def _pow2(b):
    """2^(b - 127) as fp32, b a tensor of scale bytes in 1..254."""
    return (b.int() << 23).view(torch.float32)


def _quantize_rows(v, K):
    """fp32 rows [M, K] -> E4M3 [M, Kq], scale bytes [M, P]."""
    Kq, P = _up(K, 128), _up(K, 512) // 128
    g = _pad(v, Kq).view(v.shape[0], Kq // 128, 128)
    b = _scale_bytes(g.abs().amax(2))
    codes = (g * _pow2(254 - b).unsqueeze(2)).to(torch.float8_e4m3fn).view(v.shape[0], Kq)
    scales = torch.full((v.shape[0], P), 127, dtype=torch.uint8, device=v.device)
    scales[:, : Kq // 128] = b.to(torch.uint8)
    return codes, scales


def _quantize_blocks(W):
    """fp32 weights [N, K] -> codes uint8 [N, K], scale bytes [ceil(N / 128), ceil(K / 128)], one for each 128 x 128 block."""
    N, K = W.shape
    Nb, Kb = _up(N, 128) // 128, _up(K, 128) // 128
    p = torch.zeros(Nb * 128, Kb * 128, device=W.device)
    p[:N, :K] = W
    b = _scale_bytes(p.view(Nb, 128, Kb, 128).abs().amax((1, 3)))
    s = _pow2(254 - b).repeat_interleave(128, 0).repeat_interleave(128, 1)
    return (p * s).to(torch.float8_e4m3fn).view(torch.uint8)[:N, :K].contiguous(), b.to(torch.uint8)


def _rows(codes, scales, K):
    """The fp32 values that token codes and scales stand for, [M, K]."""
    M, Kq = codes.shape
    s = _pow2(scales[:, : Kq // 128])
    return (codes.view(torch.float8_e4m3fn).float().view(M, Kq // 128, 128) * s.unsqueeze(2)).view(M, Kq)[:, :K]


def _matrix(codes, scales):
    """The fp32 values that weight codes and block scales stand for, [N, K]."""
    N, K = codes.shape
    s = _pow2(scales).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    return codes.view(torch.float8_e4m3fn).float() * s


# --- inputs --------------------------------------------------------------------------------------------------------

def _activations(M, K, gen):
    """N(0, 1) rows with 1 % outlier channels and a heavy-tailed scale per token, bf16, row pitch a multiple of eight."""
    x = torch.zeros(M, _up(K, 8), dtype=torch.bfloat16, device="cuda")
    v = torch.randn(M, K, generator=gen, device="cuda")
    v *= torch.where(torch.rand(K, generator=gen, device="cuda") < 0.01, 30.0, 1.0)
    v *= torch.exp(0.5 * torch.randn(M, 1, generator=gen, device="cuda"))
    x[:, :K] = v
    return x[:, :K]


def _weights(N, K, gen):
    return _quantize_blocks(0.02 * torch.randn(N, K, generator=gen, device="cuda"))


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, M, K = case["op"], case["M"], case["K"]
    s = {}
    if op == "norm":
        s["x"] = _activations(M, K, gen)
        s["residual"] = _activations(M, K, gen) if case["residual"] else None
        s["gamma"] = (1.0 + 0.2 * torch.randn(K, generator=gen, device="cuda")).bfloat16()
        return s
    if op == "linear":
        s["x"] = _activations(M, K, gen)
    else:
        codes, s["scales"] = _quantize_rows(_activations(M, K, gen).float(), K)
        s["codes"] = codes.view(torch.uint8)
    s["w"] = [_weights(case["N"], K, gen) for _ in range(2 if op == "gated" else 1)]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op, M, K = case["op"], case["M"], case["K"]
    if not own:
        return s
    # what a program that uses the library keeps: weights objects, workspace, output buffers
    from paper_2503_17513_b200 import xq

    s["xq"] = xq

    def rows8(n):
        return (torch.empty(M, _up(n, 128), dtype=torch.uint8, device="cuda"), torch.empty(M, _up(n, 512) // 128, dtype=torch.uint8, device="cuda"))

    if op == "norm":
        s["out8"] = rows8(K)
        s["sum"] = torch.empty(M, _up(K, 8), dtype=torch.bfloat16, device="cuda")[:, :K] if case["residual"] else None
        s["y"] = torch.empty(M, _up(K, 8), dtype=torch.bfloat16, device="cuda")[:, :K] if case["y"] else None
        return s
    s["handle"] = [xq.xq_f8_weights_import(c, b) for c, b in s["w"]]
    s["ws"] = xq.new_f8_workspace(M, s["handle"][0])
    if op == "gated" and case["out8"]:
        s["out8"] = rows8(case["N"])
    else:
        s["out"] = torch.empty(M, case["N"], dtype=torch.bfloat16, device="cuda")
    return s


# --- one pass ------------------------------------------------------------------------------------------------------

def _eight(codes, scales):
    """8-bit rows as the values that codes and scale bytes stand for (views, nothing is computed)."""
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}


def _run_own(s):
    c, xq = s["case"], s["xq"]
    op, M = c["op"], c["M"]
    if op == "norm":
        xq.xq_f8_norm_quant(s["x"], s["gamma"], EPS, *s["out8"], residual=s["residual"], sum_out=s["sum"], y=s["y"])
        out = _eight(*s["out8"])
        if c["residual"]:
            out["sum"] = s["sum"]
        if c["y"]:
            out["y"] = s["y"]
        return out
    if op == "linear":
        xq.xq_f8_linear(s["x"], s["handle"][0], s["out"], s["ws"])
        return {"out": s["out"]}
    if op == "gemm":
        xq.xq_f8_gemm(s["codes"], s["scales"], M, s["handle"][0], s["out"], s["ws"])
        return {"out": s["out"]}
    if c["out8"]:
        xq.xq_f8_gated(s["codes"], s["scales"], M, *s["handle"], s["ws"], out_codes=s["out8"][0], out_scales=s["out8"][1])
        return _eight(*s["out8"])
    xq.xq_f8_gated(s["codes"], s["scales"], M, *s["handle"], s["ws"], out=s["out"])
    return {"out": s["out"]}


def _run_plain(s):
    c = s["case"]
    op, K = c["op"], c["K"]
    if op == "norm":
        t = s["x"].float()
        if c["residual"]:
            t = t + s["residual"].float()
        y = t * (1.0 / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)) * s["gamma"].float()
        out = _eight(*_quantize_rows(y, K))
        if c["residual"]:
            out["sum"] = t.bfloat16()
        if c["y"]:
            out["y"] = y.bfloat16()
        return out
    if op == "linear":
        x = _rows(*_quantize_rows(s["x"].float(), K), K)
    else:
        x = _rows(s["codes"], s["scales"], K)
    if op != "gated":
        return {"out": (x @ _matrix(*s["w"][0]).T).bfloat16()}
    g, u = x @ _matrix(*s["w"][0]).T, x @ _matrix(*s["w"][1]).T
    h = g / (1.0 + torch.exp(-g)) * u
    return _eight(*_quantize_rows(h, c["N"])) if c["out8"] else {"out": h.bfloat16()}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    M, K = case["M"], case["K"]
    G = _up(K, 128) // 128
    if case["op"] == "norm":
        per = 2 + 1 + (4 if case["residual"] else 0) + (2 if case["y"] else 0)  # x, codes; residual in and out; y
        return {"bytes": M * K * per + M * G + 2 * K, "flops": M * K * 6}
    N, mats = case["N"], 2 if case["op"] == "gated" else 1
    Nb = _up(N, 128) // 128
    tokens = M * K * 2 if case["op"] == "linear" else M * K + M * G
    result = M * N + M * Nb if case.get("out8") else 2 * M * N
    return {"bytes": tokens + mats * (N * K + Nb * G) + result, "flops": 2.0 * mats * M * N * K}


# --- the operators' definitions in 64 bits ---------------------------------------------------------------------------

def _e4m3_table(device):
    """Values of the 256 E4M3 bytes from the format's bit fields (sign, 4-bit exponent with bias 7, 3-bit mantissa)."""
    b = torch.arange(256, dtype=torch.float64, device=device)
    e, m, sign = torch.floor(b % 128 / 8), b % 8, 1 - 2 * torch.floor(b / 128)
    v = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * _two_to(e - 7))
    return sign * torch.where(b % 128 == 127, torch.nan, v)


def _two_to(e):
    """2^e in 64 bits for whole e, from the bits (the library's power function is an ulp off in places)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_scale(amax):
    """2^e with the smallest e such that amax <= 448 * 2^e (a logarithm names a candidate, comparisons settle it)."""
    e = torch.round(torch.log2(amax / 448.0))
    e = torch.where(amax == 0, torch.zeros_like(e), e)
    return _two_to(torch.where(amax > 448.0 * _two_to(e), e + 1, e))


def _exact_eight(v):
    """Scaled elements before their rounding to 8 bits, and the scales."""
    M, n = v.shape
    Kq, P = _up(n, 128), _up(n, 512) // 128
    g = torch.zeros(M, Kq, dtype=torch.float64, device=v.device)
    g[:, :n] = v
    g = g.view(M, Kq // 128, 128)
    s = _exact_scale(g.abs().max(2).values)
    scales = torch.ones(M, P, dtype=torch.float64, device=v.device)
    scales[:, : Kq // 128] = s
    return {"codes": (g / s.unsqueeze(2)).view(M, Kq), "scales": scales}


def _exact_rows(s, K):
    if "x" in s:  # bf16 tokens: their elements rounded to the nearest E4M3 value, which the product reads
        e = _exact_eight(s["x"].double())
        a = e["codes"].abs()
        step = _two_to(torch.frexp(a.clamp(min=2.0 ** -6))[1] - 4)
        q = torch.sign(e["codes"]) * torch.round(a / step) * step
        scale = e["scales"]
    else:
        q, scale = _e4m3_table("cuda")[s["codes"].long()], _two_to(s["scales"].long() - 127)
    return (q * scale.repeat_interleave(128, 1)[:, : q.shape[1]])[:, :K]


def _exact_matrix(codes, scales):
    N, K = codes.shape
    at = torch.arange(N, device="cuda") // 128, torch.arange(K, device="cuda") // 128
    return _e4m3_table("cuda")[codes.int()] * _two_to(scales.long() - 127)[at[0]][:, at[1]]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        t = s["x"].double()
        if case["residual"]:
            t = t + s["residual"].double()
        y = t * torch.rsqrt(t.square().sum(1, keepdim=True) / case["K"] + EPS) * s["gamma"].double()
        out = _exact_eight(y)
        if case["residual"]:
            out["sum"] = t
        if case["y"]:
            out["y"] = y
        return out
    x = _exact_rows(s, case["K"])
    p = [torch.matmul(x, _exact_matrix(*w).t()) for w in s["w"]]
    if case["op"] != "gated":
        return {"out": p[0]}
    h = p[0] * torch.sigmoid(p[0]) * p[1]
    return _exact_eight(h) if case["out8"] else {"out": h}
