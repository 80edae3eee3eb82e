"""Block-scaled rows and their products (pvf_quant_mx, pvf_add_rmsnorm_mx, pvf_gemm_mx, pvf_gemm_mx_swiglu, pvf_gemm_w4) against
tests/mx_reference.py in float64.

Codes and scales are exact: they have to be the reference's.  Products are checked twice.  On whole numbers whose sums every order
of float32 additions keeps exactly (elements of at most 4, scales 2^-1 .. 2^1, so products are multiples of 2^-2 and sums below 2^20)
results have to be the rounded exact ones, bit for bit, whichever route computes them.  On random rows the tolerance is
  half a step of the result's type (2^-8 bf16, 2^-24 float32, relative to the result),
  + for the scaled matrix instruction, 7 * 2^-13 times the largest product of every 8 neighbouring k (seven products cut off 13 bits
    below it),
  + for float32 sums, 2^-24 times the magnitudes' sum for each of the additions of an element (K products at most, and a few waves' sums).
"""
import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import mx_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def rows(M, K, dtype, seed, spread=3.0):
    """Rows whose magnitudes differ from block to block."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g) * torch.exp2(spread * torch.randn(M, (K + 31) // 32, generator=g)).repeat_interleave(32, 1)[:, :K]
    return x.to(DT[dtype])


def shifted(x, by):
    """x on the device, beginning `by` elements behind an aligned address."""
    buf = torch.empty(x.numel() + by, dtype=x.dtype, device="cuda")
    return buf[by:].view(x.shape).copy_(x)


def guarded(shape, dtype, fill):
    """A tensor with `fill` bytes in front of it and behind it, and what tells whether they are left as they were."""
    n = torch.empty(shape, dtype=dtype).numel() * torch.empty(0, dtype=dtype).element_size()
    buf = torch.full((n + 512,), fill, dtype=torch.uint8, device="cuda")
    return buf[256:256 + n].view(dtype).view(shape), lambda: bool((buf[:256] == fill).all() and (buf[256 + n:] == fill).all())


def guarded_mx(M, K, fmt=R.E4M3):
    Kp = R.width(K)
    codes, c_ok = guarded((M, Kp) if fmt == R.E4M3 else (M, Kp // 2), torch.float8_e4m3fn if fmt == R.E4M3 else torch.uint8, 0xa5)
    scales, s_ok = guarded((Kp // 128, M, 4), torch.float8_e8m0fnu, 0xa5)
    return (codes, scales), lambda: c_ok() and s_ok()


# ---------------------------------------------------------------- quantiser
@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,shift", [(1, 1, 0), (1, 128, 0), (3, 31, 1), (2, 33, 3), (17, 127, 0), (64, 129, 5), (5, 511, 1), (16, 512, 0), (7, 513, 2),
                                       (33, 1411, 1), (320, 4096, 0), (1, 12288, 0), (129, 2056, 4)])
def test_quantised_rows_are_the_reference_s(fmt, dtype, M, K, shift):
    x = rows(M, K, dtype, seed=M * 31 + K)
    out, untouched = guarded_mx(M, K, fmt)
    B.quant_mx(shifted(x, shift), fmt, out=out)
    codes, byte = R.unpack(*out, fmt)
    want, want_byte = R.quantise(x.double(), fmt)
    assert torch.equal(byte, want_byte)
    assert torch.equal(codes, want)
    assert untouched()


@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
def test_quantised_extremes(fmt):
    """Ties, borders of the scale, denormals, the largest numbers, zeros of both signs, infinities and NaN, each in a block of its own."""
    x = torch.zeros(24, 160)
    top = R.TOP[fmt]
    table = R.e4m3_table() if fmt == R.E4M3 else R.E2M1_VALUES[:8].clone()
    ties = ((table[1:] + table[:-1]) / 2).float()
    for i in range(min(8, (len(ties) + 30) // 31)):
        t = ties[31 * i:31 * i + 31]
        x[i, :len(t)] = t * torch.where(torch.arange(len(t)) % 2 == 0, 1.0, -1.0)
        x[i, 31] = top
    x[8, :32] = torch.nextafter(torch.tensor(top), torch.tensor(1e9))          # just above a border: the next scale
    x[9, :32] = -top
    x[10, :32] = 2.0 ** -149 * torch.arange(32)                               # denormals: scale 2^-127
    x[11, :32] = top * 2.0 ** -127 * torch.linspace(-1, 1, 32)
    x[12, :32] = torch.finfo(torch.float32).max
    x[13, 32:64] = torch.randn(32, generator=torch.Generator().manual_seed(1)) * 1e38
    x[14, :32] = -0.0
    x[15, 5], x[15, 70], x[16, 33], x[17, 159] = float("inf"), float("-inf"), float("nan"), float("nan")
    x[15, :32] += 1.0
    x[18, 128:] = torch.arange(32.0)
    codes, byte = R.unpack(*B.quant_mx(x.cuda(), fmt), fmt)
    want, want_byte = R.quantise(x.double(), fmt)
    assert torch.equal(byte, want_byte)
    assert torch.equal(codes, want)


def test_quantised_rows_past_32_bits():
    """More than 2^32 bytes of rows: the last ones are quantised like the first."""
    M, K = 270000, 8192                                      # 4.4 GB of bf16
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    some = rows(4, K, "bf16", seed=5)
    x[:2].copy_(some[:2])
    x[-2:].copy_(some[2:])
    codes, scales = B.quant_mx(x)
    want, want_byte = R.quantise(some.double(), R.E4M3)
    for at, w in ((slice(0, 2), slice(0, 2)), (slice(M - 2, M), slice(2, 4))):
        c, b = R.unpack(codes[at], scales[:, at].contiguous(), R.E4M3)
        assert torch.equal(c, want[w]) and torch.equal(b, want_byte[w])
    assert not codes[M // 2].view(torch.uint8).any()


# ---------------------------------------------------------------- norm
def norm_reference(x, r, gain, eps):
    """h and the float32 rows that are quantised: float32 operations in the order include/pvf.h gives."""
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    inv = (1 / torch.sqrt(h.double().square().sum(1, keepdim=True) / h.shape[1] + torch.tensor(eps).double())).float()
    return h, (h.float() * inv) * gain.float()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,d,shift", [(1, 1, 0), (1, 4096, 0), (3, 33, 1), (5, 127, 0), (64, 128, 0), (2, 1411, 1), (7, 2048, 0), (3, 2049, 3), (320, 4096, 0),
                                       (4, 4100, 2), (2, 8192, 0), (2, 8193, 1), (3, 12288, 0), (1, 20001, 5)])
@pytest.mark.parametrize("residual", [False, True])
def test_normed_rows_are_the_reference_s(dtype, M, d, shift, residual):
    x, r = rows(M, d, dtype, d, 1.0), rows(M, d, dtype, d + 1, 1.0) if residual else None
    gain = (1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(2))).to(DT[dtype])
    h, y = norm_reference(x, r, gain, 1e-5)
    want, want_byte = R.quantise(y.double(), R.E4M3)
    out, untouched = guarded_mx(M, d)
    total, total_untouched = guarded((M, d), DT[dtype], 0xa5)
    got, *_ = B.add_rmsnorm_mx(shifted(x, shift), shifted(gain, shift), 1e-5, residual=shifted(r, shift) if residual else None, sum_out=total, out=out)
    codes, byte = R.unpack(*out, R.E4M3)
    assert torch.equal(got.cpu(), h)
    assert torch.equal(byte, want_byte)
    assert torch.equal(codes, want)
    assert untouched() and total_untouched()


@pytest.mark.parametrize("d", [4096, 9000])
def test_norm_in_place(d):
    """The sum may take the place of either addend, in rows that are held and in rows that are read twice."""
    x, r = rows(6, d, "bf16", 1, 1.0), rows(6, d, "bf16", 2, 1.0)
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    h, codes, scales = B.add_rmsnorm_mx(x.cuda(), gain, 1e-6, residual=r.cuda())
    for place in (0, 1):
        a, b = x.cuda(), r.cuda()
        h2, c2, s2 = B.add_rmsnorm_mx(a, gain, 1e-6, residual=b, sum_out=(a, b)[place])
        assert h2.data_ptr() == (a, b)[place].data_ptr()
        assert torch.equal(h, h2) and torch.equal(codes.view(torch.uint8), c2.view(torch.uint8)) and torch.equal(scales.view(torch.uint8), s2.view(torch.uint8))


def test_norm_of_rows_that_are_zero_or_not_finite():
    """A row of zeros: zeros (eps 1e-5), or NaN where eps is 0; a NaN or an infinity makes its row NaN and no other.  A float32 row whose squares
    are beyond float32 is normed: its sum is taken in float64."""
    x = rows(6, 256, "f32", 3)
    x[1] = 0
    x[2, 100] = float("nan")
    x[3, 7] = float("inf")
    x[4] *= 1e30
    gain = torch.ones(256, device="cuda")
    _, codes, scales = B.add_rmsnorm_mx(x.cuda(), gain, 1e-5)
    v = R.values(*R.unpack(codes, scales, R.E4M3), R.E4M3)
    _, y = norm_reference(x, None, gain.cpu(), 1e-5)
    assert (v[1] == 0).all() and torch.isnan(v[2]).all() and torch.isnan(v[3][:32]).all()
    for m in (0, 4, 5):
        want = R.values(*R.quantise(y[m:m + 1].double(), R.E4M3), R.E4M3)
        assert torch.equal(v[m:m + 1], want)
    _, codes, scales = B.add_rmsnorm_mx(x.cuda(), gain, 0.0)
    v = R.values(*R.unpack(codes, scales, R.E4M3), R.E4M3)
    assert torch.isnan(v[1]).all() and torch.isfinite(v[0]).all()


def test_norm_of_more_rows_than_a_launch_has_along_x():
    """2^24 rows are 2^32 threads.  The last rows are those of a call of their own, and nothing lies behind them."""
    M, d = (1 << 24) + 5, 32
    x = torch.zeros(M, d, dtype=torch.bfloat16, device="cuda")
    x[-300:] = rows(300, d, "bf16", 5).cuda()
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    out, untouched = guarded_mx(M, d)
    B.add_rmsnorm_mx(x, gain, 1e-5, out=out)
    _, codes, scales = B.add_rmsnorm_mx(x[-300:], gain, 1e-5)
    assert torch.equal(out[0][-300:].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(out[1][:, -300:].view(torch.uint8), scales.view(torch.uint8))
    assert not bool(out[0][:-300].view(torch.uint8).any()) and untouched()


def test_quantiser_of_more_rows_than_a_launch_has_along_x():
    M = 1 << 28
    x = torch.zeros(M, 1, dtype=torch.bfloat16, device="cuda")
    x[-300:] = rows(300, 1, "bf16", 6).cuda()
    out, untouched = guarded_mx(M, 1, R.E2M1)
    B.quant_mx(x, R.E2M1, out=out)
    codes, scales = B.quant_mx(x[-300:], R.E2M1)
    assert torch.equal(out[0][-300:], codes) and torch.equal(out[1][:, -300:].view(torch.uint8), scales.view(torch.uint8))
    assert untouched()


# ---------------------------------------------------------------- products
def whole(M, K, fmt, seed):
    """Codes of whole numbers up to 4 and scales of 2^-1 .. 2^1, and their values."""
    g = torch.Generator().manual_seed(seed)
    v = torch.zeros(M, R.width(K), dtype=torch.float64)
    v[:, :K] = torch.randint(-4, 5, (M, K), generator=g).double()
    byte = torch.randint(126, 129, (M, R.width(K) // 32), generator=g)
    table = R.e4m3_table() if fmt == R.E4M3 else R.E2M1_VALUES[:8].clone()
    codes = R.nearest(v.abs(), table) + (torch.signbit(v).long() << (7 if fmt == R.E4M3 else 3))
    return codes, byte, R.values(codes, byte, fmt)


def random_mx(M, K, fmt, seed, std=1.0):
    codes, byte = R.quantise(rows(M, K, "f32", seed, 1.0).double() * std, fmt)
    return codes, byte, R.values(codes, byte, fmt)


def cuda64(a, b):
    """a b^T in float64 on the device."""
    return (a.cuda() @ b.t().contiguous().cuda()).cpu()


def cut_off(a, w):
    """What the scaled instruction may lose of every result: 7 * 2^-13 times the largest of every 8 neighbouring products."""
    total = torch.zeros(a.shape[0], w.shape[0], dtype=torch.float64, device="cuda")
    a, w = a.cuda().abs(), w.cuda().abs()
    for k in range(0, a.shape[1], 8):
        total += (a[:, None, k:k + 8] * w[None, :, k:k + 8]).amax(2)
    return 7 * 2.0 ** -13 * total.cpu()


SHAPES = [(1, 1, 1), (1, 64, 128), (3, 17, 32), (16, 48, 300), (17, 33, 1411), (33, 100, 129), (64, 256, 4096), (65, 130, 640), (128, 128, 512), (130, 300, 260),
          (200, 515, 1024), (257, 384, 384), (320, 1024, 2048), (511, 769, 512), (640, 512, 1280)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
def test_products_of_whole_numbers(M, N, K, fmt, dtype, residual):
    a, a_b, av = whole(M, K, R.E4M3, M + K)
    w, w_b, wv = whole(N, K, fmt, N + K + 1)
    res = torch.randint(-50, 51, (M, N), generator=torch.Generator().manual_seed(3)).to(DT[dtype]) if residual else None
    want = cuda64(av, wv) + (res.double() if residual else 0)
    out, untouched = guarded((M, N), DT[dtype], 0xa5)
    B.gemm_mx(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), residual=res.cuda() if residual else None, out=out)
    assert torch.equal(out.cpu(), want.float().to(DT[dtype]))
    assert untouched()


LARGE = [(64, 4096, 300), (64, 12288, 256), (320, 4100, 385), (320, 12288, 256), (256, 24576, 128), (640, 4096, 300), (500, 12300, 200), (1280, 4096, 256), (1300, 4000, 130),
         (2560, 4096, 256), (2500, 4011, 100), (2560, 12288, 384), (2049, 9000, 513), (320, 4096, 512), (192, 4096, 1100), (256, 4096, 640), (2560, 12288, 512), (2049, 9000, 200),
         (2300, 12289, 250), (1024, 24576, 128)]


@pytest.mark.parametrize("M,N,K", LARGE)
@pytest.mark.parametrize("fmt,dtype", [(R.E4M3, "bf16"), (R.E2M1, "bf16"), (R.E4M3, "f32"), (R.E2M1, "f32")])
def test_products_of_whole_numbers_on_every_tile(M, N, K, fmt, dtype):
    """Sizes at which the tiles of many rows are taken, whole and ragged, one stage of k and several."""
    a, a_b, av = whole(M, K, R.E4M3, M + K)
    w, w_b, wv = whole(N, K, fmt, N + K + 1)
    out, untouched = guarded((M, N), DT[dtype], 0xa5)
    res = torch.randint(-50, 51, (M, N), generator=torch.Generator().manual_seed(3)).to(DT[dtype])
    B.gemm_mx(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), residual=res.cuda(), out=out)
    want = cuda64(av, wv) + res.double()
    assert torch.equal(out.cpu(), want.float().to(DT[dtype]))
    assert untouched()


@pytest.mark.parametrize("M,N,K", [(1, 40, 128), (5, 33, 65), (64, 96, 1411), (70, 200, 256), (300, 140, 4096)])
@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_of_random_rows(M, N, K, fmt, dtype):
    a, a_b, av = random_mx(M, K, R.E4M3, M + K)
    w, w_b, wv = random_mx(N, K, fmt, N + 1, 0.02)
    want, mag = cuda64(av, wv), cuda64(av.abs(), wv.abs())
    got = B.gemm_mx(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), dtype=DT[dtype]).cpu().double()
    tol = HALF_STEP[dtype] * want.abs() + 2.0 ** -24 * mag * (K + 16 if dtype == "f32" else K / 8 + 16) + (cut_off(av, wv) if dtype == "bf16" else 0)
    assert bool(((got - want).abs() <= tol).all()), ((got - want).abs() / tol).max()
    if dtype == "f32":                                       # rounding errors do not add up one way: far below the bound in the mean
        assert (got - want).norm() <= 1e-6 * want.norm()


@pytest.mark.parametrize("M,N,K", [(1, 1, 33), (1, 64, 128), (1, 12288, 4096), (2, 17, 31), (16, 48, 300), (17, 33, 1411), (33, 100, 129), (64, 257, 4096), (65, 130, 640),
                                   (130, 300, 264), (320, 1024, 2048), (511, 769, 520), (1024, 384, 1000), (4, 4096, 512), (3, 300, 1024), (16, 12288, 256), (33, 4001, 1411),
                                   (64, 4096, 256), (64, 12288, 520), (320, 4096, 512), (330, 12300, 264),
                                   (1, 12289, 1030), (4, 12288, 1024), (4, 12289, 1031), (2560, 4096, 200), (330, 12289, 515)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual,shift", [(False, 0), (True, 0), (False, 1)])
def test_4_bit_products_of_whole_numbers(M, N, K, dtype, residual, shift):
    """Rows of whole numbers: up to 2^7 for bf16, with 20 bits for float32 (three parts), whose sums stay below 2^24."""
    g = torch.Generator().manual_seed(M + N + K)
    x = torch.randint(-127, 128, (M, K), generator=g).float()
    w, w_b, wv = whole(N, K, R.E2M1, N + K + 1)
    if dtype == "f32":                                       # a few elements of 20 bits, one a row
        x = torch.randint(-4, 5, (M, K), generator=g).float()
        x[torch.arange(M), torch.arange(M) * 7 % K] = torch.randint(-2 ** 19, 2 ** 19, (M,), generator=g).float()
        w_b[:] = 127
        wv = R.values(w, w_b, R.E2M1)
    x = x.to(DT[dtype])
    res = torch.randint(-50, 51, (M, N), generator=g).to(DT[dtype]) if residual else None
    want = cuda64(x.double(), wv[:, :K]) + (res.double() if residual else 0)
    assert want.abs().max() < 2 ** 22
    out, untouched = guarded((M, N), DT[dtype], 0xa5)
    B.gemm_w4(shifted(x, shift), *R.pack(w, w_b, R.E2M1), residual=res.cuda() if residual else None, out=out)
    assert torch.equal(out.cpu(), want.float().to(DT[dtype]))
    assert untouched()


@pytest.mark.parametrize("M,N,K", [(1, 40, 128), (5, 33, 65), (64, 96, 1411), (70, 200, 256), (300, 140, 4096)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_4_bit_products_of_random_rows(M, N, K, dtype):
    x = rows(M, K, dtype, M + K, 1.0)
    w, w_b, wv = random_mx(N, K, R.E2M1, N + 1, 0.02)
    want, mag = cuda64(x.double(), wv[:, :K]), cuda64(x.double().abs(), wv[:, :K].abs())
    got = B.gemm_w4(x.cuda(), *R.pack(w, w_b, R.E2M1)).cpu().double()
    tol = HALF_STEP[dtype] * want.abs() + 2.0 ** -24 * mag * ((3 if dtype == "f32" else 1) * K + 16)
    assert bool(((got - want).abs() <= tol).all()), ((got - want).abs() / tol).max()
    if dtype == "f32":
        assert (got - want).norm() <= 1e-6 * want.norm()


def test_4_bit_products_of_more_tiles_than_a_launch_has_along_x():
    """Tiles of 16 rows and 512 threads: 2^27 rows are 2^32 threads."""
    M = (1 << 27) + 3
    x = (torch.arange(M, device="cuda", dtype=torch.int32) % 1021).float()[:, None]
    w, w_b = torch.zeros(1, 128, dtype=torch.int64), torch.full((1, 4), 127)
    w[0, 0] = 5                                              # 3.0
    out, untouched = guarded((M, 1), torch.float32, 0xa5)
    B.gemm_w4(x, *R.pack(w, w_b, R.E2M1), out=out)
    assert torch.equal(out, x * 3) and untouched()


@pytest.mark.parametrize("call", ["mx_e4m3", "mx_e2m1", "mx_f32", "w4_bf16", "w4_f32"])
def test_scales_over_their_whole_range(call):
    """Every scale byte from 0 to 254 stands for its power of two, 255 for NaN.  Rows with 2^(127 - b) against weights with 2^(b - 127), so that
    results are near 1 (bytes 8 to 240: the other side's powers are in float32's normal range)."""
    fmt = R.E4M3 if call in ("mx_e4m3", "mx_f32") else R.E2M1
    dtype = torch.float32 if call.endswith("f32") else torch.bfloat16
    b = torch.arange(8, 241)
    w = torch.full((len(b), 128), 2 if fmt == R.E2M1 else 0x38)         # ones
    w_b = b[:, None].repeat(1, 4)
    W = R.pack(w, w_b, fmt)
    if call.startswith("w4"):
        x = torch.pow(2.0, (127 - b).double()).float()[:, None].repeat(1, 128).to(dtype)
        got = B.gemm_w4(x.cuda(), *W).cpu()
    else:
        got = B.gemm_mx(*R.pack(torch.full((len(b), 128), 0x38), (254 - b)[:, None].repeat(1, 4), R.E4M3), *W, dtype=dtype).cpu()
    assert torch.equal(torch.diagonal(got).float(), torch.full((len(b),), 128.0))
    # zero scales beside ordinary rows add nothing that shows; NaN scales make NaN of the results that read them and of no others
    w_b = torch.full((3, 4), 127)
    w_b[1, 2], w_b[2, :] = 255, 0
    W = R.pack(torch.full((3, 128), 2 if fmt == R.E2M1 else 0x38), w_b, fmt)
    if call.startswith("w4"):
        got = B.gemm_w4(torch.ones(5, 128, dtype=dtype, device="cuda"), *W).cpu()
    else:
        got = B.gemm_mx(*R.pack(torch.full((5, 128), 0x38), torch.full((5, 4), 127), R.E4M3), *W, dtype=dtype).cpu()
    assert (got[:, 0] == 128).all() and torch.isnan(got[:, 1]).all() and (got[:, 2].abs() <= 128 * 2.0 ** -126).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_4_bit_products_of_rows_that_are_not_finite(dtype):
    """Infinities and NaN reach the results of their own row only; an infinity times weights of one sign stays one."""
    x = torch.ones(4, 300, dtype=DT[dtype])
    x[1, 200], x[2, 299] = float("inf"), float("nan")
    w, w_b = torch.full((20, R.width(300)), 2), torch.full((20, R.width(300) // 32), 127)
    w[:, 300:] = 0
    got = B.gemm_w4(x.cuda(), *R.pack(w, w_b, R.E2M1)).cpu()
    assert (got[0] == 300).all() and (got[3] == 300).all()
    assert (got[1] == float("inf")).all() and torch.isnan(got[2]).all()


@pytest.mark.parametrize("call,M,N", [("mx_e4m3", 4096, 4096), ("mx_e4m3", 70, 300), ("mx_e2m1", 1, 4096), ("mx_f32", 4096, 4096), ("mx_f32", 33, 500), ("w4_bf16", 1, 300),
                                      ("w4_f32", 1, 300), ("w4_f32", 40, 4096)])
def test_products_of_the_longest_rows(call, M, N):
    """2^22 elements a row, all zero but 2000 whole numbers, the last element among them: offsets within a tile of 256 rows reach 2^30 bytes."""
    K, g = 1 << 22, torch.Generator().manual_seed(M + N)
    fmt = R.E4M3 if call in ("mx_e4m3", "mx_f32") else R.E2M1
    at = torch.cat([torch.randperm(K // 2 - 1, generator=g)[:1999] * 2 + torch.randint(0, 2, (1999,), generator=g), torch.tensor([K - 1])]).unique().cuda()
    a = torch.randint(-4, 5, (M, len(at)), generator=g).float().cuda()
    w = torch.randint(-4, 5, (N, len(at)), generator=g).float().cuda()
    want = (a.double() @ w.double().t().contiguous()).float()
    ones = lambda rows: torch.full((K // 128, rows, 4), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)

    def e4m3(v):
        codes = torch.zeros(v.shape[0], K, dtype=torch.uint8, device="cuda")
        codes[:, at] = v.to(torch.float8_e4m3fn).view(torch.uint8)
        return codes.view(torch.float8_e4m3fn), ones(v.shape[0])

    if fmt == R.E4M3:
        W = e4m3(w)
    else:                                                    # no two of the 2000 share a byte
        codes = torch.zeros(N, K // 2, dtype=torch.uint8, device="cuda")
        four = torch.tensor([0, 2, 4, 5, 6], dtype=torch.uint8, device="cuda")[w.abs().long()] + (w < 0).to(torch.uint8) * 8
        codes[:, at // 2] = four << (at % 2 * 4).to(torch.uint8)
        W = codes, ones(N)
    dtype = torch.float32 if call.endswith("f32") else torch.bfloat16
    if call.startswith("w4"):
        x = torch.zeros(M, K, dtype=dtype, device="cuda")
        x[:, at] = a.to(dtype)
        got = B.gemm_w4(x, *W)
    else:
        got = B.gemm_mx(*e4m3(a), *W, dtype=dtype)
    assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("M,N,K", [(5, 33, 128), (70, 200, 256), (300, 4096, 512), (2560, 4096, 256), (2560, 12288, 256)])
@pytest.mark.parametrize("fmt,dtype", [(R.E4M3, "bf16"), (R.E2M1, "bf16"), (R.E4M3, "f32")])
def test_results_and_residuals_may_begin_at_any_element(M, N, K, fmt, dtype):
    a, a_b, av = whole(M, K, R.E4M3, M + K)
    w, w_b, wv = whole(N, K, fmt, N + K + 1)
    res = torch.randint(-50, 51, (M, N), generator=torch.Generator().manual_seed(3)).to(DT[dtype])
    want = (cuda64(av, wv) + res.double()).float().to(DT[dtype])
    for c, r in ((1, 3), (3, 0), (4, 1)):
        buf = torch.full((M * N + 16,), 77.0, dtype=DT[dtype], device="cuda")
        out = buf[c:c + M * N].view(M, N)
        B.gemm_mx(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), residual=shifted(res, r), out=out)
        assert torch.equal(out.cpu(), want)
        assert bool((buf[:c] == 77).all() and (buf[c + M * N:] == 77).all())


def test_norm_of_rows_that_begin_at_any_element():
    """x, residual, gain and sum each at another element."""
    x, r, gain = rows(37, 515, "bf16", 1), rows(37, 515, "bf16", 2), rows(1, 515, "bf16", 3)[0]
    h, codes, scales = B.add_rmsnorm_mx(x.cuda(), gain.cuda(), 1e-5, residual=r.cuda())
    out = shifted(torch.zeros_like(x), 5)
    _, c, s = B.add_rmsnorm_mx(shifted(x, 1), shifted(gain, 3), 1e-5, residual=shifted(r, 2), sum_out=out)
    assert torch.equal(out, h) and torch.equal(c.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(s.view(torch.uint8), scales.view(torch.uint8))


def test_product_into_its_residual():
    a, a_b, av = whole(70, 512, R.E4M3, 1)
    w, w_b, wv = whole(200, 512, R.E2M1, 2)
    h = torch.randint(-50, 51, (70, 200)).to(torch.bfloat16).cuda()
    want = (cuda64(av, wv) + h.cpu().double()).float().to(torch.bfloat16)
    got = B.gemm_mx(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, R.E2M1), residual=h, out=h)
    assert got.data_ptr() == h.data_ptr() and torch.equal(h.cpu(), want)
    x = torch.randint(-9, 10, (70, 512)).to(torch.bfloat16)
    want = (cuda64(x.double(), wv) + h.cpu().double()).float().to(torch.bfloat16)
    B.gemm_w4(x.cuda(), *R.pack(w, w_b, R.E2M1), residual=h, out=h)
    assert torch.equal(h.cpu(), want)


# ---------------------------------------------------------------- SwiGLU
def within_codes(got, want_values, slack):
    """Whether device codes and scales stand for values within half a step of `want_values` (float64), which may be off by `slack` themselves.
    The step of a code in a block with scale s is 2^(binade - 3) s, 2^-9 s at least; near a border the block's scale may be twice the
    reference's, and then so may the step."""
    codes, byte = R.unpack(*got, R.E4M3)
    v = R.values(codes, byte, R.E4M3)
    want = torch.zeros(v.shape, dtype=torch.float64)
    want[:, :want_values.shape[1]] = want_values
    err = torch.zeros_like(want)
    err[:, :want_values.shape[1]] = slack
    s = torch.pow(2.0, (byte - 127).double()).repeat_interleave(32, 1)
    binade = torch.floor(torch.log2((want.abs() + err).clamp(min=2.0 ** -300)))
    step = torch.maximum(torch.pow(2.0, binade - 3), s * 2.0 ** -9)
    amax = (want.abs() + err).view(want.shape[0], -1, 32).amax(2)
    tight = s.view(want.shape[0], -1, 32)[:, :, 0] <= torch.clamp(2 * amax / 448, min=2.0 ** -127) * (1 + 1e-9)   # the smallest scale that fits, or its double at a border
    return bool(((v - want).abs() <= step / 2 + err).all() and tight.all() and (codes[:, want_values.shape[1]:] == 0).all())


@pytest.mark.parametrize("M,ff,K", [(1, 1, 32), (1, 32, 128), (3, 17, 33), (16, 200, 300), (17, 129, 1411), (64, 256, 4096), (65, 130, 640), (130, 500, 260), (257, 384, 512),
                                    (320, 1024, 1024), (515, 257, 384), (64, 4100, 256), (1, 12288, 256), (320, 12288, 128), (1100, 3000, 264), (64, 12288, 1024), (50, 12300, 140), (300, 12288, 384), (2560, 2100, 700)])
@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
def test_swiglu(M, ff, K, fmt):
    """The slack of a product is that of test_products_of_random_rows without a rounding to bf16; silu(g) u moves by at most 1.1 |u| dg + |silu(g)| du
    (the slope of silu is below 1.1), and evaluates within 8 * 2^-23 in float32 (an exponential of up to 2^7 with 2^-23 of it, a
    reciprocal, two products) times 1 + |g|."""
    a, a_b, av = random_mx(M, K, R.E4M3, M + K)
    w, w_b, wv = random_mx(2 * ff, K, fmt, ff + 1, 0.05)
    p, mag = cuda64(av, wv), cuda64(av.abs(), wv.abs())
    err = 2.0 ** -24 * mag * (K / 8 + 16) + cut_off(av, wv)
    gate, up = p[:, :ff], p[:, ff:]
    silu = gate * torch.sigmoid(gate)
    slack = 1.1 * (up.abs() + err[:, ff:]) * err[:, :ff] + silu.abs() * err[:, ff:] + 8 * 2.0 ** -23 * (1 + gate.abs()) * (silu * up).abs()
    out, untouched = guarded_mx(M, ff)
    B.gemm_mx_swiglu(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), out=out)
    assert within_codes(out, silu * up, slack)
    assert untouched()


def test_swiglu_extremes():
    """Gates far from zero on either side: silu(g) is g or a zero, never NaN; a NaN row is NaN and no other."""
    K, ff = 128, 64
    a = torch.zeros(3, K)
    a[:, 0] = 1.0
    w = torch.zeros(2 * ff, K)
    w[:ff, 0] = torch.linspace(-400, 400, ff)
    w[ff:, 0] = 2.0
    A = B.quant_mx(a.cuda())
    A[1].view(torch.uint8)[0, 1, 0] = 255
    W = B.quant_mx(w.cuda())
    codes, scales = B.gemm_mx_swiglu(*A, *W)
    v = R.values(*R.unpack(codes, scales, R.E4M3), R.E4M3)
    wv = R.values(*R.unpack(*W, R.E4M3), R.E4M3)
    assert torch.isnan(v[1, :ff]).all() and torch.equal(v[0], v[2])
    want = wv[:ff, 0] * torch.sigmoid(wv[:ff, 0]) * 2
    assert bool(((v[0, :ff] - want).abs() <= 2.0 ** -4 * want.abs() + 800 * 2.0 ** -9 / 448 * 2).all())


# ---------------------------------------------------------------- together, streams, graphs
def layer(x, r, gain, W, h):
    """The projections of an FFN half and an output projection of single rows, as a decoding loop would chain them."""
    h, codes, scales = B.add_rmsnorm_mx(x, gain, 1e-5, residual=r, sum_out=h)
    act = B.gemm_mx_swiglu(codes, scales, *W["gate_up"])
    down = B.gemm_mx(*act, *W["down"], residual=h)
    back = B.gemm_mx(*B.quant_mx(down), *W["o"], dtype=x.dtype)
    return codes, scales, *act, down, back, B.gemm_w4(down, *W["head"])


def make_layer(M, d, ff, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    W = {"gate_up": B.quant_mx(n(2 * ff, d) * 0.05, B.MX_E2M1), "down": B.quant_mx(n(d, ff) * 0.05), "o": B.quant_mx(n(d, d) * 0.05, B.MX_E2M1),
         "head": B.quant_mx(n(300, d) * 0.05, B.MX_E2M1)}
    return n(M, d).to(DT[dtype]), n(M, d).to(DT[dtype]), (1 + 0.1 * n(d)).to(DT[dtype]), W


def raw(ts):
    return [t.clone().view(torch.uint8) if t.element_size() == 1 else t.clone() for t in ts]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,d,ff", [(1, 512, 1408), (37, 515, 999), (200, 512, 768)])
def test_a_layer_of_them(M, d, ff, dtype):
    """Each link against float64 from the codes that the link before it gave, then the whole chain again: the same bits."""
    x, r, gain, W = make_layer(M, d, ff, dtype, M)
    h = torch.empty_like(x)
    codes, scales, a_codes, a_scales, down, back, head = layer(x, r, gain, W, h)
    val = lambda c, s: R.values(*R.unpack(c, s, R.E4M3 if c.dtype == torch.float8_e4m3fn else R.E2M1), R.E4M3 if c.dtype == torch.float8_e4m3fn else R.E2M1)  # noqa: E731
    want_h, y = norm_reference(x.cpu(), r.cpu(), gain.cpu(), 1e-5)
    assert torch.equal(h.cpu(), want_h)
    assert torch.equal(R.unpack(codes, scales, R.E4M3)[0], R.quantise(y.double(), R.E4M3)[0])
    p = cuda64(val(codes, scales), val(*W["gate_up"]))
    act = p[:, :ff] * torch.sigmoid(p[:, :ff]) * p[:, ff:]
    av = val(a_codes, a_scales)[:, :ff]
    assert (av - act).norm() <= 2.0 ** -4 * act.norm()
    want = cuda64(val(a_codes, a_scales), val(*W["down"])) + h.cpu().double()
    step = HALF_STEP[dtype] * 1.01
    slack = 1e-6 if dtype == "f32" else 2.0 ** -10           # the cut-off of the scaled instruction relative to a row's largest result
    assert bool(((down.cpu().double() - want).abs() <= step * want.abs() + slack * want.abs().amax()).all())
    want = cuda64(down.cpu().double(), val(*W["head"])[:, :d])
    assert bool(((head.cpu().double() - want).abs() <= step * want.abs() + 2.0 ** -20 * want.abs().amax()).all())
    again = layer(x, r, gain, W, torch.empty_like(x))
    assert all(torch.equal(a, b) for a, b in zip(raw((codes, scales, a_codes, a_scales, down, back, head)), raw(again)))


def test_a_layer_in_a_graph_and_on_two_streams():
    """Captured and replayed with new rows between eager runs; two layers on two streams at once: the eager results each time."""
    x, r, gain, W = make_layer(64, 512, 768, "bf16", 1)
    x2, r2, _, _ = make_layer(64, 512, 768, "bf16", 2)
    xs, rs, hs = x.clone(), r.clone(), torch.empty_like(x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        layer(xs, rs, gain, W, hs)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer(xs, rs, gain, W, hs)
    for rep in range(4):
        xs.copy_((x, x2)[rep % 2])
        rs.copy_((r, r2)[rep % 2])
        graph.replay()
        want = raw(layer((x, x2)[rep % 2], (r, r2)[rep % 2], gain, W, torch.empty_like(x)))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(raw(captured), want)), rep
    wants = [raw(layer(a, b, gain, W, torch.empty_like(x))) for a, b in ((x, r), (x2, r2))]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for rep in range(3):
        for i, (a, b) in enumerate(((x, r), (x2, r2))):
            with torch.cuda.stream(streams[i]):
                got[i] = layer(a, b, gain, W, torch.empty_like(x))
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(raw(got[i]), wants[i]))


def test_nothing_to_do():
    """No rows, no columns."""
    codes, scales = B.quant_mx(torch.empty(0, 100, device="cuda"))
    assert codes.shape == (0, 128) and scales.shape == (1, 0, 4)
    _, c, s = B.add_rmsnorm_mx(torch.empty(0, 100, device="cuda"), torch.ones(100, device="cuda"), 1e-5)
    assert c.shape == (0, 128)
    W = B.quant_mx(torch.randn(64, 100, device="cuda"), B.MX_E2M1)
    assert B.gemm_mx(codes, scales, *W).shape == (0, 64)
    assert B.gemm_mx_swiglu(codes, scales, *W)[0].shape == (0, 128)
    assert B.gemm_w4(torch.empty(0, 100, device="cuda"), *W).shape == (0, 64)
    none = B.quant_mx(torch.empty(0, 100, device="cuda"), B.MX_E2M1)
    assert B.gemm_w4(torch.ones(3, 100, device="cuda"), *none).shape == (3, 0)
