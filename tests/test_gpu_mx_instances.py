"""Products of block-scaled rows on every kernel instance that the choice by sizes can take (tests/test_mx_instances.py sees that the shapes here reach them all).

Whole numbers as in tests/test_gpu_mx.py have to come out bit for bit; they say that every element meets its partner, but sums in fewer bits would pass them.
Random rows say how exactly sums are kept: each result is held to the bounds that tests/test_gpu_mx.py derives, and all of them together to a norm that single bounds, which
allow for errors that all add up one way, are far above:
  float32   1e-6 of the results' norm (the scaled instruction's cut-off would be 1.5e-5);
  bfloat16  a rounding is at most 2^(e - 8) for values from 2^e on and uniform below that, so its root mean square is 2^-8 / sqrt(3) = 2.26e-3 of them at most; 2.3e-3
            leaves 4e-4 (in squares) to the cut-off and the sums.
"""
import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import mx_reference as R
from tests.test_gpu_mx import HALF_STEP, cuda64, cut_off, guarded, random_mx, rows, shifted, whole
from tests.test_mx_instances import KINDS

# by kind and instance: (M, N, K) of one stage of 128 k (two where the instance takes pairs), and of 12 or 17
SHORT, LONG = {
    "mx_e4m3": [(1, 16, 72), (676, 82, 72), (34, 4163, 72), (1, 12469, 72), (51, 8292, 72), (49, 16412, 72), (66, 8690, 72), (83, 8518, 72), (133, 16414, 72), (197, 17275, 72),
                (3605, 1033, 72), (484, 17371, 72), (406, 17066, 130)],
    "mx_e2m1": [(1, 16, 72), (194, 310, 72), (33, 4117, 72), (1, 12296, 72), (57, 8227, 72), (51, 16385, 72), (66, 8234, 72), (81, 8605, 72), (130, 16901, 72), (201, 17552, 72),
                (3649, 1026, 72), (651, 13385, 72), (672, 16635, 200)],
    "mx_e4m3_f32": [(1, 16, 72), (146, 403, 72), (36, 8393, 72), (51, 8245, 72), (67, 8490, 72), (151, 16650, 72), (193, 13259, 72), (3531, 843, 130), (3614, 1092, 72)],
    "mx_e2m1_f32": [(1, 16, 72), (198, 306, 72), (34, 8309, 72), (50, 8431, 72), (69, 8232, 72), (155, 16465, 72), (193, 13494, 72), (386, 7275, 130), (266, 13907, 72)],
    "swiglu_e4m3": [(1, 16, 72), (1039, 16, 72), (3144, 147, 72), (2087, 129, 130), (261, 9734, 72), (3452, 257, 130)],
    "swiglu_e2m1": [(1, 16, 72), (1036, 16, 72), (3225, 131, 72), (2108, 142, 130), (264, 9885, 72), (3432, 259, 130)],
    "w4": [(1, 4125, 72), (1, 16, 72), (196, 305, 72), (5, 8320, 72), (908, 130, 72), (2726, 264, 72), (389, 641, 72), (49, 8211, 72), (2798, 330, 72), (163, 16542, 72)],
    "w4_shifted": [(1, 16, 72), (2, 16, 72), (5, 16, 72), (145, 1221, 72), (1236, 306, 72), (97, 12650, 72)],
    "w4_f32": [(1, 16, 72), (1, 4101, 72), (2, 16, 72), (2, 4255, 72), (305, 198, 72), (2066, 69, 72), (3104, 390, 72)],
    "w4_f32_shifted": [(1, 16, 72), (1, 8229, 72), (2, 16, 72), (5, 16, 72), (305, 197, 72), (2089, 74, 72), (2733, 67, 72), (3732, 258, 72), (3359, 129, 72)],
}, {
    "mx_e4m3": [(1, 16, 1411), (306, 194, 1411), (548, 452, 1411), (712, 673, 1411), (867, 849, 1411), (1443, 1041, 1411), (1258, 775, 1411), (966, 1220, 1411),
                (1885, 1637, 1411), (1453, 3236, 1411), (1611, 2453, 1411), (2130, 4640, 2056), (3334, 2379, 1411)],
    "mx_e2m1": [(1, 16, 1411), (198, 307, 1411), (612, 389, 1411), (613, 801, 1411), (1350, 518, 1411), (1180, 1295, 1411), (1221, 795, 1411), (894, 1354, 1411),
                (1731, 1770, 1411), (3121, 1548, 1411), (3626, 1032, 1411), (4018, 2439, 1411), (3863, 3127, 1411)],
    "mx_e4m3_f32": [(1, 16, 1411), (291, 209, 1411), (745, 675, 1411), (1217, 580, 1411), (1242, 774, 1411), (2459, 1602, 1411), (1924, 1575, 2056), (1161, 2566, 1411), (1409, 2838, 1411)],
    "mx_e2m1_f32": [(1, 16, 1411), (214, 289, 1411), (835, 590, 1411), (915, 800, 1411), (770, 1234, 1411), (1538, 2457, 1411), (2136, 1418, 2056), (1767, 1733, 1411), (2578, 1541, 1411)],
    "swiglu_e4m3": [(1, 16, 1411), (517, 132, 1411), (1249, 515, 2056), (817, 514, 1411), (1462, 2069, 2056), (1324, 899, 1411)],
    "swiglu_e2m1": [(1, 16, 1411), (514, 138, 1411), (868, 781, 2056), (677, 659, 1411), (1869, 1537, 2056), (1491, 784, 1411)],
    "w4": [(1, 4111, 1408), (1, 16, 1408), (305, 203, 1408), (387, 612, 1408), (296, 419, 1408), (1171, 777, 1408), (452, 570, 1408), (1237, 579, 1408), (1252, 774, 1408), (1952, 1557, 1408)],
    "w4_shifted": [(1, 16, 1411), (2, 16, 1411), (5, 16, 1411), (401, 472, 1411), (548, 708, 1411), (1103, 1374, 1411)],
    "w4_f32": [(1, 16, 1408), (1, 4107, 1408), (2, 16, 1408), (2, 4111, 1408), (209, 290, 1408), (518, 451, 1408), (1604, 912, 1408)],
    "w4_f32_shifted": [(1, 16, 1411), (1, 8209, 1411), (2, 16, 1411), (5, 16, 1411), (306, 194, 1411), (583, 400, 1411), (404, 615, 1411), (1201, 844, 1411), (843, 582, 1411)],
}
# eight waves that share k have several stages each from 1024 elements on; of few rows as many results as single roundings take to show
MORE = {"swiglu_e4m3": [(16, 8000, 1411)], "swiglu_e2m1": [(13, 8000, 1411)],
        "mx_e4m3_f32": [(1, 16, 4104)], "mx_e2m1_f32": [(3, 33, 4104)], "w4": [(1, 16, 4104), (16, 16, 4104), (1, 12290, 4104)], "w4_shifted": [(1, 16, 4101), (3, 17, 4101)],
        "w4_f32": [(1, 16, 4104), (1, 4107, 4104), (9, 16, 4104), (3, 4110, 4104)], "w4_f32_shifted": [(1, 16, 4101), (1, 8209, 4101), (3, 16, 4101), (9, 33, 4101)]}
PRODUCTS = [k for k in KINDS if not k.startswith("swiglu")]

pytestmark = pytest.mark.gpu


def cases(*tables, kinds=PRODUCTS):
    return [(k, *s) for t in tables for k in kinds for s in t.get(k, ())]


def product(kind, left, W, **kw):
    """The call of this kind: left are codes and scales, or rows."""
    call, _, dtype, aligned = KINDS[kind]
    if call == B.MX_W4:
        return B.gemm_w4(shifted(left, 0 if aligned else 1), *W, **kw)
    return B.gemm_mx(*R.pack(*left, R.E4M3), *W, dtype=dtype, **kw)


@pytest.mark.parametrize("kind,M,N,K", cases(SHORT, LONG, MORE))
def test_whole_numbers(kind, M, N, K):
    call, fmt, dtype, _ = KINDS[kind]
    g = torch.Generator().manual_seed(M + N + K)
    w, w_b, wv = whole(N, K, fmt, N + K + 1)
    if call == B.MX_W4:
        left = torch.randint(-127, 128, (M, K), generator=g).float()
        if dtype is torch.float32:                           # an element of 20 bits in each row, which has three parts
            left = torch.randint(-4, 5, (M, K), generator=g).float()
            left[torch.arange(M), torch.arange(M) * 7 % K] = torch.randint(-2 ** 19, 2 ** 19, (M,), generator=g).float()
            w_b[:] = 127
            wv = R.values(w, w_b, fmt)
        left = left.to(dtype)
        av = torch.zeros(M, wv.shape[1], dtype=torch.float64)
        av[:, :K] = left.double()
    else:
        *left, av = whole(M, K, R.E4M3, M + K)
    res = torch.randint(-50, 51, (M, N), generator=g).to(dtype)
    want = cuda64(av, wv) + res.double()
    assert want.abs().max() < 2 ** 22
    out, untouched = guarded((M, N), dtype, 0xa5)
    product(kind, left, R.pack(w, w_b, fmt), residual=res.cuda(), out=out)
    assert torch.equal(out.cpu(), want.float().to(dtype))
    assert untouched()


@pytest.mark.parametrize("kind,M,N,K", cases(LONG, MORE))
def test_random_rows(kind, M, N, K):
    call, fmt, dtype, _ = KINDS[kind]
    name = "f32" if dtype is torch.float32 else "bf16"
    w, w_b, wv = random_mx(N, K, fmt, N + 1, 0.02)
    if call == B.MX_W4:
        left = rows(M, K, name, M + K, 1.0)
        av = torch.zeros(M, wv.shape[1], dtype=torch.float64)
        av[:, :K] = left.double()
    else:
        *left, av = random_mx(M, K, R.E4M3, M + K)
    want, mag = cuda64(av, wv), cuda64(av.abs(), wv.abs())
    got = product(kind, left, R.pack(w, w_b, fmt)).cpu().double()
    scaled = call == B.MX_GEMM and name == "bf16"
    additions = (3 if call == B.MX_W4 and name == "f32" else 1) * (K / 8 if scaled else K) + 16
    tol = HALF_STEP[name] * want.abs() + 2.0 ** -24 * mag * additions + (cut_off(av, wv) if scaled else 0)
    assert bool(((got - want).abs() <= tol).all()), ((got - want).abs() / tol).max()
    assert (got - want).norm() <= (1e-6 if name == "f32" else 2.3e-3) * want.norm()


def test_4_bit_products_of_2_32_threads():
    """The largest number of threads along x is 2^32 - 1: tiles of 16 rows and 512 threads go on in y from 2^27 rows on."""
    M = (1 << 27) + 3
    assert B.gemm_mx_instance(B.MX_W4, M, 1, 4, B.MX_E2M1, torch.float32) == B.gemm_mx_instance(B.MX_W4, 16, 16, 4, B.MX_E2M1, torch.float32)     # 16 x 16, eight waves
    x = (torch.arange(M, device="cuda", dtype=torch.int32) % 1021).float()[:, None].repeat(1, 4)
    w, w_b = torch.zeros(1, 128, dtype=torch.int64), torch.full((1, 4), 127)
    w[0, :4] = torch.tensor([5, 2, 0, 10])                   # 3, 1, 0, -1
    out, untouched = guarded((M, 1), torch.float32, 0xa5)
    B.gemm_w4(x, *R.pack(w, w_b, R.E2M1), out=out)
    assert torch.equal(out, x[:, :1] * 3) and untouched()


@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_elements_at_the_ends_of_the_scales(fmt, dtype):
    """Every magnitude with the scales at either end, against 2^60 or 2^-60.  Bfloat16 results are the exact product rounded.  For float32 results elements become bfloat16: what lies
    below 2^-126 may be lost, and 2^128 and more is infinite."""
    n = 126 if fmt == R.E4M3 else 7
    codes = torch.zeros(n, 128, dtype=torch.int64)
    codes[:, 0] = torch.arange(1, n + 1)
    one = torch.zeros(1, 128, dtype=torch.int64)
    one[0, 0] = 0x38
    for byte in (0, 1, 2, 7, 8, 240, 246, 247, 248, 253, 254):
        by = 60 if byte < 127 else -60
        W = R.pack(codes, torch.full((n, 4), byte), fmt)
        v = R.values(codes, torch.full((n, 4), byte), fmt)[:, 0]
        got = B.gemm_mx(*R.pack(one, torch.full((1, 4), 127 + by), R.E4M3), *W, dtype=dtype).cpu().double()[0] * 2.0 ** -by
        if dtype is torch.bfloat16:
            assert torch.equal(got, v), byte                 # at most 4 bits each
        else:
            assert bool(((got - v).abs() <= 2.0 ** -126)[v < 2.0 ** 128].all()) and torch.equal(got[v >= 2.0 ** -120].isinf(), v[v >= 2.0 ** -120] >= 2.0 ** 128), byte


@pytest.mark.parametrize("exponent", [-126, -118, -110, -60])
def test_parts_of_small_float32_rows(exponent):
    """Rows of 24 bits go as three parts; what of them lies below 2^-126 may be lost, and no more."""
    x = torch.zeros(70, 128)
    x[:, 0] = (1 + torch.rand(70, generator=torch.Generator().manual_seed(1))) * 2.0 ** exponent
    w, w_b = torch.zeros(33, 128, dtype=torch.int64), torch.full((33, 4), 127 + 100)
    w[:, 0] = 2                                              # ones
    got = B.gemm_w4(x.cuda(), *R.pack(w, w_b, R.E2M1)).cpu().double() * 2.0 ** -100
    assert bool(((got - x[:, :1].double()).abs() <= 2.0 ** -126).all())
    assert exponent < -103 or torch.equal(got, x[:, :1].double().expand(70, 33))      # the last of 24 bits is above 2^-126


@pytest.mark.parametrize("kind,M,N,K", [c for c in cases(LONG, kinds=list(KINDS)) if c[1] > 32])
def test_blocks_that_are_not_finite(kind, M, N, K):
    """A NaN or an infinity in a block of a row, or of a row of weights, makes NaN of the results that read it (of SwiGLU, of the blocks that hold them) and of no others."""
    call, fmt, dtype, aligned = KINDS[kind]
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x = torch.randn(M, K, device="cuda", generator=g)
    w = torch.randn((2 if call == B.MX_SWIGLU else 1) * N, K, device="cuda", generator=g) * 0.05
    m, n = [0, M // 2, M - 1], [0, N // 3, N - 1]
    x[m, [K - 1, K // 2, 0]] = torch.tensor([float("nan"), float("inf"), float("nan")], device="cuda")
    w[n, [0, K - 1, K // 2]] = torch.tensor([float("inf"), float("nan"), float("-inf")], device="cuda")
    W = B.quant_mx(w, fmt)
    if call == B.MX_W4:
        bad = torch.isnan(product(kind, x.to(dtype), W))
        bad[m[1]] = True                                     # unquantised: an infinity may give one
    elif call == B.MX_GEMM:
        bad = torch.isnan(B.gemm_mx(*B.quant_mx(x), *W, dtype=dtype))
    else:
        codes, scales = B.gemm_mx_swiglu(*B.quant_mx(x), *W)
        bad = (scales.view(torch.uint8) == 255).transpose(0, 1).reshape(M, -1)[:, :(N + 31) // 32]
        n = [k // 32 for k in n]
    want = torch.zeros_like(bad)
    want[m] = True
    want[:, n] = True
    assert torch.equal(bad, want)
