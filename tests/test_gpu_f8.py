"""The 8-bit floating-point layer on the GPU against its definition in 64 bits (oracle/f8.py).

Bounds, with u = 2^-24 the unit roundoff of fp32:
 - quantization of bf16 rows: scaling by a power of two is exact, so codes and scales equal the definition's.
 - norm: t = x + r has one rounding, the sum of squares of up to 65536 terms is at most 64 additions deep in a thread and ten
   across threads (relative error of the sum <= 76 u, half of that in the root), division, root and two products add 5 u:
   y within DELTA = 2^-18 = 64 u, relative.  An 8-bit or bf16 output must be the rounding of some value in that interval, and
   a scale the scale of some maximum in it.
 - product: products of E4M3 values are exact in fp32; a tensor-core step adds 32 of them and may truncate the sum by two units of
   its last place, and the partial sums of at most 16 slices meet in fp32: |error| <= (K / 32 + 16) 2^-22 sum |x w|.  Then one rounding to bf16.
 - gated: the two products' errors through h = silu(G) U (|silu'| <= 1.1), plus 2^-19 |h| for exponential, division and
   products, plus 1e-36 |U| where exp(-G) leaves the fp32 range.
"""
import numpy as np
import pytest
import torch

from oracle import f8
from paper_2503_17513_b200 import synth

pytestmark = pytest.mark.gpu

DELTA = 2.0 ** -18
U = 2.0 ** -24


@pytest.fixture(scope="module")
def xq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2503_17513_b200 import xq as binding

    binding.lib()
    return binding


def bf16_rows(v: np.ndarray, ld=None, fill=0.0):
    """Device bf16 view [M, K] of row pitch ld (default: K rounded up to 8); its values in fp64."""
    M, K = v.shape
    ld = -(-K // 8) * 8 if ld is None else ld
    buf = torch.full((M, ld), fill, dtype=torch.bfloat16, device="cuda")
    buf[:, :K] = torch.from_numpy(np.ascontiguousarray(v)).to(torch.bfloat16).cuda()
    return buf[:, :K], buf[:, :K].double().cpu().numpy(), buf


def np64(t):
    return t.double().cpu().numpy()


def bf16_round(v):
    return torch.from_numpy(v.astype(np.float32)).to(torch.bfloat16).double().numpy()


def bf16_of(v64):
    """fp64 -> bf16 in one rounding (to odd in fp32 first, so that the second rounding cannot err)."""
    f = v64.astype(np.float32)
    bits = f.view(np.uint32).astype(np.int64)
    inexact = f.astype(np.float64) != v64
    low = np.where(inexact & (np.abs(f.astype(np.float64)) > np.abs(v64)), bits - 1, bits)  # truncate
    odd = np.where(inexact, low | 1, bits)
    return torch.from_numpy(odd.astype(np.uint32).view(np.float32)).to(torch.bfloat16).double().numpy()


def assert_between(got, lo, hi):
    ok = (got >= np.minimum(lo, hi)) & (got <= np.maximum(lo, hi))
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], lo[~ok][:5], hi[~ok][:5])


def assert_bf16_within(got, v, err):
    assert_between(got, bf16_of(v - err), bf16_of(v + err))


def assert_eight_within(codes, scales, v, err):
    """codes and scales are those of some rows within err of v (elementwise)."""
    M, K = v.shape
    Kq, G = f8.padded(K), f8.padded(K) // 128
    err = np.broadcast_to(err, v.shape)
    assert codes.shape == (M, Kq) and scales.shape == (M, f8.pitch(K))
    assert np.all(codes[:, K:] == 0) and np.all(scales[:, G:] == 127)
    lo = f8.scale_byte(f8.group_amax(np.maximum(np.abs(v) - err, 0)))
    hi = f8.scale_byte(f8.group_amax(np.abs(v) + err))
    b = scales[:, :G].astype(np.int64)
    zero_may = f8.group_amax(np.maximum(np.abs(v) - err, 0)) == 0  # the group may be all zero: scale one
    assert np.all(((b >= np.minimum(lo, hi)) & (b <= hi)) | (zero_may & ((b == 127) | (b <= hi))))
    s = np.repeat(f8.pow2(b), 128, axis=1)[:, :K]
    val = f8.e4m3_values()
    assert_between(val[codes[:, :K]], val[f8.encode((v - err) / s)], val[f8.encode((v + err) / s)])


def new_rows(xq, M, K):
    c, s = xq.new_f8_rows(M, K)
    c.fill_(0x55), s.fill_(0x55)
    return c, s


def rows_data(M, K, seed, zero_row=None):
    v = synth.bf16_bits_to_f32(synth.activations(M, K, seed=seed, tag=f"f8{M}x{K}", heavy_tail=M > 8)).astype(np.float64)
    if zero_row is not None and M > zero_row:
        v[zero_row] = 0
    return v


# ---- quantization and norm ------------------------------------------------------------------------

ROWS = [(1, 1), (1, 7), (2, 8), (3, 127), (5, 128), (4, 129), (2, 520), (17, 640), (33, 2048), (3, 2876), (1, 4096), (5, 8192), (2, 14336),
        (2, 20001), (1, 40000), (1, 65536), (1500, 320), (700, 4100)]


@pytest.mark.parametrize("M,K", ROWS)
def test_quant_is_the_definition(xq, M, K):
    X, x, _ = bf16_rows(rows_data(M, K, 3, zero_row=1))
    codes, scales = new_rows(xq, M, K)
    xq.xq_f8_quant(X, codes, scales)
    want = f8.quantize_rows(x)
    assert np.array_equal(scales.cpu().numpy(), want[1])
    got = codes.cpu().numpy()
    val = f8.e4m3_values()
    assert np.array_equal(val[got], val[want[0]])  # (a zero may carry either sign)


@pytest.mark.parametrize("M,K", ROWS)
@pytest.mark.parametrize("residual,y", [(True, False), (False, True), (True, True)])
def test_norm_quant(xq, M, K, residual, y):
    X, x, _ = bf16_rows(rows_data(M, K, 4, zero_row=1))
    R, r, _ = bf16_rows(rows_data(M, K, 5, zero_row=1))
    g = np.random.default_rng(6).standard_normal(K) * 0.3 + 1
    gamma = torch.from_numpy(g).to(torch.bfloat16).cuda()
    codes, scales = new_rows(xq, M, K)
    S = torch.empty_like(X.contiguous()) if K % 8 == 0 else bf16_rows(np.zeros((M, K)))[0]
    Y, _, _ = bf16_rows(np.zeros((M, K)))
    xq.xq_f8_norm_quant(X, gamma, 1e-5, codes, scales, residual=R if residual else None, sum_out=S, y=Y if y else None)
    t, want = f8.norm(x, r if residual else None, np64(gamma), float(np.float32(1e-5)))
    assert_bf16_within(np64(S), t, U * np.abs(t))
    err = DELTA * np.abs(want)
    assert_eight_within(codes.cpu().numpy(), scales.cpu().numpy(), want, err)
    if y:
        assert_bf16_within(np64(Y), want, err)


def test_norm_in_place_and_pitches(xq):
    """The residual stream updated in place, all pitches different, elements between K and the pitch untouched."""
    M, K = 37, 1003
    X, x, _ = bf16_rows(rows_data(M, K, 7), ld=1016)
    R, r, rbuf = bf16_rows(rows_data(M, K, 8), ld=1040, fill=7.0)
    Y, _, ybuf = bf16_rows(np.zeros((M, K)), ld=1008, fill=9.0)
    gamma = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    codes, scales = new_rows(xq, M, K)
    xq.xq_f8_norm_quant(X, gamma, 1e-6, codes, scales, residual=R, sum_out=R, y=Y)
    t, want = f8.norm(x, r, np.ones(K), float(np.float32(1e-6)))
    assert_bf16_within(np64(R), t, U * np.abs(t))
    assert_bf16_within(np64(Y), want, DELTA * np.abs(want))
    assert_eight_within(codes.cpu().numpy(), scales.cpu().numpy(), want, DELTA * np.abs(want))
    assert bool((rbuf[:, K:] == 7.0).all()) and bool((ybuf[:, K:] == 9.0).all())


def test_quant_special_values(xq):
    """Infinities, NaN, the smallest and largest magnitudes: each confined to its group."""
    K = 640
    v = np.ones((4, K)) * 3.0
    v[0, 5] = np.inf
    v[1, 130] = np.nan
    v[2, 256:384] = 1e-38
    v[2, 384:512] = 3e38
    v[3, 0:128] = np.nan
    X, x, _ = bf16_rows(v)
    codes, scales = new_rows(xq, 4, K)
    xq.xq_f8_quant(X, codes, scales)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    plain = f8.quantize_rows(np.full((1, 128), 3.0))
    assert s[0, 0] == 247 and c[0, 5] == 0x7E  # 448 * 2^120: beyond fp32, an infinity again
    assert np.isposinf(np.float32(448) * np.float32(2.0 ** 120))
    assert c[1, 130] & 0x7F == 0x7F and s[1, 1] == plain[1][0, 0] and np.all(np.delete(c[1], 130)[:K - 1] == plain[0][0, 0])
    assert np.all(c[3, :128] & 0x7F == 0x7F) and s[3, 0] == 127
    want = f8.quantize_rows(x[2:3])
    assert np.array_equal(c[2], want[0][0]) and np.array_equal(s[2], want[1][0])
    for row, group in [(0, 1), (1, 0), (2, 0), (3, 1)]:
        assert s[row, group] == plain[1][0, 0] and np.all(c[row, 128 * group : 128 * group + 128] == plain[0][0, 0])


def test_norm_special_rows(xq):
    """A row with an infinity or a NaN stays alone with it."""
    K = 256
    v = rows_data(4, K, 9)
    v[1, 3], v[2, 200] = np.inf, np.nan
    X, x, _ = bf16_rows(v)
    gamma = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    codes, scales = new_rows(xq, 4, K)
    Y, _, _ = bf16_rows(np.zeros((4, K)))
    xq.xq_f8_norm_quant(X, gamma, 1e-5, codes, scales, y=Y)
    y, c = np64(Y), codes.cpu().numpy()
    assert np.isnan(y[1, 3]) and np.all(np.delete(y[1], 3) == 0) and c[1, 3] & 0x7F == 0x7F
    assert np.isnan(y[2]).all() and np.all(c[2] & 0x7F == 0x7F)
    _, want = f8.norm(x[[0, 3]], None, np.ones(K), float(np.float32(1e-5)))
    assert_bf16_within(y[[0, 3]], want, DELTA * np.abs(want))


def test_norm_many_rows_past_32_bit_offsets(xq):
    """More than 2^31 elements: the last rows equal the same rows given alone."""
    K, M = 8192, (1 << 18) + 5
    X = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    tail, x, _ = bf16_rows(rows_data(9, K, 10))
    X[-9:] = tail
    gamma = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    codes, scales = new_rows(xq, M, K)
    S = torch.empty_like(X)
    xq.xq_f8_norm_quant(X, gamma, 1e-5, codes, scales, sum_out=S)
    c9, s9 = new_rows(xq, 9, K)
    xq.xq_f8_norm_quant(tail, gamma, 1e-5, c9, s9)
    assert torch.equal(codes[-9:], c9) and torch.equal(scales[-9:], s9) and torch.equal(S[-9:], tail)
    assert int(codes[:-9].max()) == 0 and bool((scales[:-9, :64] == 127).all())


# ---- weights --------------------------------------------------------------------------------------

@pytest.mark.parametrize("N,K", [(1, 1), (5, 130), (128, 128), (200, 300), (129, 2048), (300, 77)])
@pytest.mark.parametrize("where", ["cpu", "cuda"])
def test_prepare_import_export(xq, N, K, where):
    g = np.random.default_rng(11)
    W = torch.from_numpy(g.standard_normal((N, K)) * 0.02).to(torch.bfloat16)
    want = f8.quantize_blocks(W.double().numpy())
    codes, scales = xq.xq_f8_weights_export(xq.xq_f8_prepare_weights(W.to(where)))
    val = f8.e4m3_values()
    assert np.array_equal(val[codes], val[want[0]]) and np.array_equal(scales, want[1])
    rnd = g.integers(0, 256, (N, K)).astype(np.uint8), g.integers(0, 255, (-(-N // 128), -(-K // 128))).astype(np.uint8)
    w = xq.xq_f8_weights_import(torch.from_numpy(rnd[0]).to(where), torch.from_numpy(rnd[1]).to(where))
    assert (w.N, w.K) == (N, K)
    back = xq.xq_f8_weights_export(w)
    assert np.array_equal(back[0], rnd[0]) and np.array_equal(back[1], rnd[1])


# ---- products -------------------------------------------------------------------------------------

def eight_bit_tokens(M, K, seed):
    codes, scales = f8.quantize_rows(rows_data(M, K, seed, zero_row=2))
    return codes, scales, f8.dequantize_rows(codes, scales, K)


def eight_bit_weights(N, K, seed):
    W = np.random.default_rng(seed).standard_normal((N, K)) * 0.02
    W *= np.exp2(np.random.default_rng(seed + 1).integers(-2, 3, (-(-N // 128), 1))).repeat(128, axis=0)[:N]
    codes, scales = f8.quantize_blocks(W)
    return codes, scales, f8.dequantize_blocks(codes, scales)


def product(x, w):
    return x @ w.T, (x.shape[1] / 32 + 16) * 2.0 ** -22 * (np.abs(x) @ np.abs(w).T)


def cuda(a):
    return torch.from_numpy(a).cuda()


SIZES = [(1, 1, 1), (1, 16, 8), (1, 4096, 256), (2, 130, 129), (7, 300, 77), (8, 512, 640), (16, 2048, 384), (17, 640, 1000), (32, 1400, 256),
         (33, 128, 130), (48, 896, 520), (64, 2048, 136), (100, 1000, 1001), (128, 512, 512), (129, 384, 264), (200, 2176, 300), (256, 256, 1024),
         (300, 2720, 505), (520, 1152, 776), (1000, 640, 2000), (2100, 512, 1160)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_gemm(xq, M, K, N):
    xc, xs, x = eight_bit_tokens(M, K, 12)
    wc, wsc, w = eight_bit_weights(N, K, 13)
    h = xq.xq_f8_weights_import(wc, wsc)
    ws = xq.new_f8_workspace(M, h)
    out = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    xq.xq_f8_gemm(cuda(xc), cuda(xs), M, h, out, ws)
    assert xq.xq_poll_status(ws) == xq.OK
    want, err = product(x, w)
    assert_bf16_within(np64(out), want, err)


# sizes that run in tiles of 256, 192 and 128 columns, over several waves of tiles, with rows that do and do not start on 16 bytes
SLICED_SIZES = [(1, 14336, 256), (40, 9000, 130), (200, 14000, 256)]  # few tiles, K cut into eight slices
TILE_SIZES = [(3000, 640, 4000), (2500, 300, 6001), (2100, 1152, 4168), (2000, 900, 5003), (512, 4096, 4096), (600, 4096, 2001)]


@pytest.mark.parametrize("M,K,N", TILE_SIZES + SLICED_SIZES)
def test_gemm_tiles_and_slices(xq, M, K, N):
    test_gemm(xq, M, K, N)


def gated_want(x, g, u):
    G, eG = product(x, g)
    Uu, eU = product(x, u)
    s = f8.silu(G)
    h = s * Uu
    return h, 1.1 * eG * (np.abs(Uu) + eU) + np.abs(s) * eU + 2.0 ** -19 * np.abs(h) + 1e-36 * np.abs(Uu)


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("eight", [False, True])
def test_gated(xq, M, K, N, eight):
    xc, xs, x = eight_bit_tokens(M, K, 14)
    gc, gs, g = eight_bit_weights(N, K, 15)
    uc, us, u = eight_bit_weights(N, K, 17)
    hg, hu = xq.xq_f8_weights_import(gc, gs), xq.xq_f8_weights_import(uc, us)
    ws = xq.new_f8_workspace(M, hg)
    want, err = gated_want(x, g, u)
    if eight:
        oc, os_ = new_rows(xq, M, N)
        xq.xq_f8_gated(cuda(xc), cuda(xs), M, hg, hu, ws, out_codes=oc, out_scales=os_)
        assert xq.xq_poll_status(ws) == xq.OK
        assert_eight_within(oc.cpu().numpy(), os_.cpu().numpy(), want, err)
    else:
        out = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        xq.xq_f8_gated(cuda(xc), cuda(xs), M, hg, hu, ws, out=out)
        assert xq.xq_poll_status(ws) == xq.OK
        assert_bf16_within(np64(out), want, err)


@pytest.mark.parametrize("M,K,N", [(1500, 256, 4000), (700, 1100, 5003)] + SLICED_SIZES)
@pytest.mark.parametrize("eight", [False, True])
def test_gated_tiles_and_slices(xq, M, K, N, eight):
    test_gated(xq, M, K, N, eight)


def test_gated_large_gates(xq):
    """|G| in the hundreds: the exponential saturates, the result stays finite and right."""
    M, K, N = 20, 256, 256
    xc, xs, x = eight_bit_tokens(M, K, 18)
    g64 = np.random.default_rng(19).standard_normal((N, K)) * 4
    gc, gs = f8.quantize_blocks(g64)
    g = f8.dequantize_blocks(gc, gs)
    uc, us, u = eight_bit_weights(N, K, 20)
    hg, hu = xq.xq_f8_weights_import(gc, gs), xq.xq_f8_weights_import(uc, us)
    for M2 in (M, 150):
        xc2, xs2, x2 = (np.tile(a, (-(-M2 // M), 1))[:M2] for a in (xc, xs, x))
        ws = xq.new_f8_workspace(M2, hg)
        out = torch.empty((M2, N), dtype=torch.bfloat16, device="cuda")
        xq.xq_f8_gated(cuda(np.ascontiguousarray(xc2)), cuda(np.ascontiguousarray(xs2)), M2, hg, hu, ws, out=out)
        want, err = gated_want(x2, g, u)
        assert np.abs(x2 @ g.T).max() > 150 and np.isfinite(np64(out)).all()
        assert_bf16_within(np64(out), want, err)


@pytest.mark.parametrize("M", [5, 40, 300])
def test_nan_stays_in_its_row_and_channel(xq, M):
    K, N = 384, 300
    xc, xs, x = eight_bit_tokens(M, K, 21)
    wc, wsc, w = eight_bit_weights(N, K, 22)
    xc[3, 100] = 0x7F
    wc[7, 11] = 0xFF
    h = xq.xq_f8_weights_import(wc, wsc)
    ws = xq.new_f8_workspace(M, h)
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    xq.xq_f8_gemm(cuda(xc), cuda(xs), M, h, out, ws)
    got = np64(out)
    assert np.isnan(got[3]).all() and np.isnan(got[:, 7]).all()
    rows, cols = np.delete(np.arange(M), 3), np.delete(np.arange(N), 7)
    want, err = product(x[rows], w[cols])
    assert_bf16_within(got[np.ix_(rows, cols)], want, err)


@pytest.mark.parametrize("M", [4, 64, 260])
def test_scale_range(xq, M):
    """Scales of the groups far apart: each group enters with its own power of two."""
    K, N = 1280, 264
    g = np.random.default_rng(23)
    xc, wc = (g.integers(0, 127, s).astype(np.uint8) | (g.integers(0, 2, s).astype(np.uint8) << 7) for s in ((M, K), (N, K)))
    xs = np.full((M, f8.pitch(K)), 127, dtype=np.uint8)
    xs[:, : K // 128] = g.integers(110, 145, (M, K // 128))
    wsc = g.integers(110, 145, (-(-N // 128), K // 128)).astype(np.uint8)
    h = xq.xq_f8_weights_import(wc, wsc)
    ws = xq.new_f8_workspace(M, h)
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    xq.xq_f8_gemm(cuda(xc), cuda(xs), M, h, out, ws)
    want, err = product(f8.dequantize_rows(xc, xs, K), f8.dequantize_blocks(wc, wsc))
    assert_bf16_within(np64(out), want, err)


@pytest.mark.parametrize("M,K,N", [(1, 2048, 512), (16, 700, 300), (90, 520, 136), (400, 1000, 650)])
def test_linear_is_quant_then_gemm(xq, M, K, N):
    X, x, _ = bf16_rows(rows_data(M, K, 24), ld=-(-K // 8) * 8 + 16)
    wc, wsc, w = eight_bit_weights(N, K, 25)
    h = xq.xq_f8_weights_import(wc, wsc)
    ws = xq.new_f8_workspace(M, h)
    out, out2 = (torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xq.xq_f8_linear(X, h, out, ws)
    codes, scales = new_rows(xq, M, K)
    xq.xq_f8_quant(X, codes, scales)
    xq.xq_f8_gemm(codes, scales, M, h, out2, ws)
    assert torch.equal(out, out2)
    want, err = product(f8.dequantize_rows(*f8.quantize_rows(x), K), w)
    assert_bf16_within(np64(out), want, err)


def test_gemm_past_32_bit_offsets(xq):
    """More than 2^31 outputs: sampled rows equal the same rows given alone (their M differs, not their sums' order)."""
    M, K, N = (1 << 17) + 40, 128, 16512
    xc, xs, _ = eight_bit_tokens(1024, K, 26)
    wc, wsc, _ = eight_bit_weights(N, K, 27)
    h = xq.xq_f8_weights_import(wc, wsc)
    X, S = cuda(xc).repeat(M // 1024 + 1, 1)[:M].contiguous(), cuda(xs).repeat(M // 1024 + 1, 1)[:M].contiguous()
    ws = xq.new_f8_workspace(1024, h)
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    xq.xq_f8_gemm(X, S, M, h, out, ws)
    ref = torch.empty((1024, N), dtype=torch.bfloat16, device="cuda")
    xq.xq_f8_gemm(cuda(xc), cuda(xs), 1024, h, ref, ws)
    assert xq.xq_poll_status(ws) == xq.OK
    for lo in (0, M // 1024 // 2 * 1024, M // 1024 * 1024 - 1024):
        assert torch.equal(out[lo : lo + 1024], ref)
    assert torch.equal(out[M // 1024 * 1024 :], ref[: M % 1024])


@pytest.mark.parametrize("M", [1, 24, 90, 700])
def test_repeated_launches_and_a_chain(xq, M):
    """The feed-forward chain norm -> gated -> product, launched many times without waiting on another stream: the same bits
    each time, and those of the same calls made one at a time."""
    K, I = 1024, 1400
    X, _, _ = bf16_rows(rows_data(M, K, 28))
    gamma = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    hg, hu = (xq.xq_f8_weights_import(*eight_bit_weights(I, K, s)[:2]) for s in (29, 31))
    hd = xq.xq_f8_weights_import(*eight_bit_weights(K, I, 33)[:2])
    ws, wsd = xq.new_f8_workspace(M, hg), xq.new_f8_workspace(M, hd)

    def chain(wait):
        c, s = new_rows(xq, M, K)
        hc, hs = new_rows(xq, M, I)
        R = X.clone()
        out = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
        for call in (lambda: xq.xq_f8_norm_quant(X, gamma, 1e-5, c, s, residual=R, sum_out=R),
                     lambda: xq.xq_f8_gated(c, s, M, hg, hu, ws, out_codes=hc, out_scales=hs),
                     lambda: xq.xq_f8_gemm(hc, hs, M, hd, out, wsd)):
            call()
            if wait:
                torch.cuda.synchronize()
        return R, hc, hs, out

    ref = chain(True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [chain(False) for _ in range(40)]
    side.synchronize()
    assert xq.xq_poll_status(ws, side) == xq.OK and xq.xq_poll_status(wsd, side) == xq.OK
    for r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, ref))


@pytest.mark.parametrize("M,K,N,times", [(16, 4096, 6144, 300), (1, 14336, 2048, 200), (120, 2048, 4096, 200), (2048, 2048, 4096, 60), (768, 2048, 4000, 60)])
def test_products_repeat_bit_for_bit(xq, M, K, N, times):
    """Back-to-back launches under load: a stage handed over too early would change some of the outputs some of the time."""
    g = torch.Generator(device="cuda").manual_seed(5)
    codes = torch.randint(0, 127, (M, K), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(115, 130, (M, f8.pitch(K)), generator=g, device="cuda", dtype=torch.uint8)
    wc = torch.randint(0, 127, (N, K), generator=g, device="cuda", dtype=torch.uint8)
    wc |= torch.randint(0, 2, (N, K), generator=g, device="cuda", dtype=torch.uint8) << 7
    h = xq.xq_f8_weights_import(wc, torch.randint(115, 130, (-(-N // 128), -(-K // 128)), generator=g, device="cuda", dtype=torch.uint8))
    ws = xq.new_f8_workspace(M, h)
    ref, out = (torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xq.xq_f8_gemm(codes, scales, M, h, ref, ws)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(times // 4):
        for _ in range(3):
            xq.xq_f8_gemm(codes, scales, M, h, out, ws)
        out.fill_(float("nan"))
        xq.xq_f8_gemm(codes, scales, M, h, out, ws)
        differ += (out != ref).sum()
    assert int(differ) == 0 and xq.xq_poll_status(ws) == xq.OK


def test_layers_on_distinct_streams(xq):
    """Products of different layers on different streams with their own workspaces give what they give alone."""
    K, N = 2048, 1024
    jobs = []
    for i, M in enumerate((1, 16, 60, 500)):
        xc, xs, _ = eight_bit_tokens(M, K, 40 + i)
        h = xq.xq_f8_weights_import(*eight_bit_weights(N, K, 50 + 2 * i)[:2])
        out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        jobs.append((cuda(xc), cuda(xs), M, h, out, xq.new_f8_workspace(M, h)))
    ref = []
    for j in jobs:
        xq.xq_f8_gemm(*j)
        torch.cuda.synchronize()
        ref.append(j[4].clone())
        j[4].zero_()
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(10):
        for j, st in zip(jobs, streams):
            xq.xq_f8_gemm(*j, stream=st)
    torch.cuda.synchronize()
    for j, r in zip(jobs, ref):
        assert torch.equal(j[4], r)


def test_captured_in_a_graph(xq):
    M, K, N = 8, 1024, 512
    X, _, _ = bf16_rows(rows_data(M, K, 60))
    h = xq.xq_f8_weights_import(*eight_bit_weights(N, K, 61)[:2])
    ws = xq.new_f8_workspace(M, h)
    out, ref = (torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xq.xq_f8_linear(X, h, ref, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xq.xq_f8_linear(X, h, out, ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
    del graph


# ---- refusals -------------------------------------------------------------------------------------

def refused(xq, status, call, *a, **k):
    with pytest.raises(xq.XqError) as e:
        call(*a, **k)
    assert e.value.status == status


def test_refusals(xq):
    M, K, N = 4, 256, 128
    X, _, buf = bf16_rows(rows_data(M, K, 70), ld=264)
    codes, scales = new_rows(xq, M, K)
    gamma = torch.ones(K + 8, dtype=torch.bfloat16, device="cuda")
    bad = xq.ERR_INVALID_ARG
    odd = torch.empty(M * 300, dtype=torch.bfloat16, device="cuda")
    view = lambda off, ld: torch.as_strided(odd, (M, K), (ld, 1), off)
    refused(xq, bad, xq.xq_f8_quant, view(0, 257), codes, scales)   # pitch not a multiple of 8
    refused(xq, bad, xq.xq_f8_quant, view(0, 248), codes, scales)   # pitch below K
    refused(xq, bad, xq.xq_f8_quant, view(1, 264), codes, scales)   # rows not 16-byte aligned
    flat = torch.empty(M * K + 16, dtype=torch.uint8, device="cuda")
    refused(xq, bad, xq.xq_f8_quant, X, flat[8 : 8 + M * K], scales)
    refused(xq, bad, xq.xq_f8_quant, X, codes, flat[1 : 1 + 16])
    refused(xq, bad, xq.xq_f8_norm_quant, X, gamma[1 : K + 1], 1e-5, codes, scales)
    refused(xq, bad, xq.xq_f8_norm_quant, X, gamma[:K], -1.0, codes, scales)
    refused(xq, bad, xq.xq_f8_norm_quant, X, gamma[:K], float("nan"), codes, scales)
    refused(xq, bad, xq.xq_f8_norm_quant, X, gamma[:K], 1e-5, codes, scales, residual=view(1, 264))
    refused(xq, bad, xq.xq_f8_norm_quant, X, gamma[:K], 1e-5, codes, scales, y=view(0, 257))
    wc, wsc, _ = eight_bit_weights(N, K, 71)
    nan_scale = wsc.copy()
    nan_scale[0, 1] = 255
    refused(xq, bad, xq.xq_f8_weights_import, wc, nan_scale)
    refused(xq, bad, xq.xq_f8_weights_import, cuda(wc), cuda(nan_scale))
    h = xq.xq_f8_weights_import(wc, wsc)
    other = xq.xq_f8_weights_import(*eight_bit_weights(N + 1, K, 72)[:2])
    ws = xq.new_f8_workspace(M, h)
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    oflat = torch.empty(M * N + 8, dtype=torch.bfloat16, device="cuda")
    refused(xq, bad, xq.xq_f8_gemm, codes, scales, -1, h, out, ws)
    refused(xq, bad, xq.xq_f8_gemm, codes, scales, M, h, oflat[1 : 1 + M * N], ws)
    refused(xq, bad, xq.xq_f8_gemm, codes, scales, M, h, None, ws)
    refused(xq, xq.ERR_WORKSPACE, xq.xq_f8_gemm, codes, scales, M, h, out, ws[:128])
    refused(xq, xq.ERR_WORKSPACE, xq.xq_f8_linear, X, h, out, ws[:256])
    oc, os_ = new_rows(xq, M, N)
    refused(xq, bad, xq.xq_f8_gated, codes, scales, M, h, other, ws, out=out)
    refused(xq, bad, xq.xq_f8_gated, codes, scales, M, h, h, ws)
    refused(xq, bad, xq.xq_f8_gated, codes, scales, M, h, h, ws, out=out, out_codes=oc, out_scales=os_)
    refused(xq, bad, xq.xq_f8_gated, codes, scales, M, h, h, ws, out_codes=oc)
    # nothing to do is no error
    xq.xq_f8_gemm(codes, scales, 0, h, out, ws)
    xq.xq_f8_quant(X[:0], codes, scales)
    torch.cuda.synchronize()
