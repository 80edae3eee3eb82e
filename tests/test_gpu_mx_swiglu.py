"""SwiGLU of block-scaled rows where single roundings show: gates far below zero, and the share of codes that are not the definition's."""
import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import mx_reference as R
from tests.test_gpu_mx import cuda64, guarded_mx, random_mx, within_codes
from tests.test_gpu_mx_instances import LONG, MORE, SHORT, cases
from tests.test_mx_instances import KINDS

pytestmark = pytest.mark.gpu


def as_terms(v, fmt):
    """Codes, bytes and values [n, 96] of rows whose elements 0, 32 and 64 add up to nearly v: each what the ones before it leave."""
    w = torch.zeros(len(v), 96, dtype=torch.float64)
    for k in (0, 32, 64):
        w[:, k] = v - w.sum(1)
        w = R.values(*R.quantise(w, fmt), fmt)[:, :96]
    return w


@pytest.mark.parametrize("ups", [2.0, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
@pytest.mark.parametrize("M", [3, 70])
def test_gates_far_below_zero(M, fmt, ups):
    """Blocks of 32 columns whose gates all lie near -78, -86, .. -254, and one with -400: silu leaves float32's normal range at -92 and its
    divisor float32 itself at -89, while a block's scale goes down to 2^-127 and a large factor brings the product back.  Products here are a few
    terms that float32 adds exactly, so what may be off is silu(g) u: an exponential (2^-23), three products and the correction of
    its argument (2^-24 each) are less than 2^-21 of it, and 2^-149 where it is below the normal range."""
    n = 24
    gate = -(78 + 8.0 * torch.arange(n)).repeat_interleave(32) - torch.arange(32).repeat(n) / 16
    gate[-32:] = -400
    ff, K = len(gate), 128
    w = torch.zeros(2 * ff, K, dtype=torch.float64)
    w[:ff, :96] = as_terms(gate.double(), fmt)
    w[ff:, 96] = ups * torch.where(torch.arange(ff) % 3 == 0, -1.5, 1.0)
    a = torch.zeros(M, K, dtype=torch.float64)
    a[:, 0::32] = 1 + torch.arange(M)[:, None] % 2 / 8.0
    (w, w_b), (a, a_b) = R.quantise(w, fmt), R.quantise(a, R.E4M3)
    p = cuda64(R.values(a, a_b, R.E4M3), R.values(w, w_b, fmt))
    want = p[:, :ff] * torch.exp(p[:, :ff]) / (1 + torch.exp(p[:, :ff])) * p[:, ff:]
    out, untouched = guarded_mx(M, ff)
    B.gemm_mx_swiglu(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), out=out)
    assert within_codes(out, want, 2.0 ** -21 * want.abs() + 2.0 ** -149)
    assert untouched()


def flips(got, want):
    """How many codes of blocks whose scale is the definition's stand for another value than the definition's, and how many scales differ."""
    codes, byte = R.unpack(*got, R.E4M3)
    c, b = R.quantise(want, R.E4M3)
    same = byte == b
    return int((R.values(codes, byte, R.E4M3) != R.values(c, b, R.E4M3))[same.repeat_interleave(32, 1)].sum()), int((~same).sum())


@pytest.mark.parametrize("kind,M,ff,K", cases(SHORT, LONG, MORE, kinds=["swiglu_e4m3", "swiglu_e2m1"]))
def test_swiglu_sums_in_float32(kind, M, ff, K):
    """SwiGLU decodes its operands and adds in float32.  A sum of K products of random signs is off by 0.4 2^-24 of its size at each of at most K / 8 + 16 additions (the root mean
    square of a rounding of 24 bits), which do not add up one way: 2.5 2^-24 sqrt(K / 8 + 16) of the products' root sum of squares is six times that.  silu(g) u is
    evaluated within 3 * 2^-23 (an exponential 2^-23; its correction, the reciprocal and two products 2^-24 each).  A code differs from the definition's where
    its value is nearer to a border of two codes than the error: with a sixth of the bound as the error's size and values that lie anywhere between
    the borders, in the sum of error / step of all codes.  The instruction with the cut-off would change 0.3 % of the codes, products rounded to bfloat16 some 2 %."""
    fmt = KINDS[kind][1]
    a, a_b, av = random_mx(M, K, R.E4M3, M + K)
    w, w_b, wv = random_mx(2 * ff, K, fmt, ff + 1, 0.05)
    p, size = cuda64(av, wv), cuda64(av * av, wv * wv).sqrt()
    err = 2.5 * 2.0 ** -24 * (K / 8 + 16) ** 0.5 * size
    gate, up = p[:, :ff], p[:, ff:]
    silu = gate * torch.sigmoid(gate)
    want = silu * up
    slack = 1.1 * (up.abs() + err[:, ff:]) * err[:, :ff] + silu.abs() * err[:, ff:] + 3 * 2.0 ** -23 * want.abs()
    out, untouched = guarded_mx(M, ff)
    B.gemm_mx_swiglu(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), out=out)
    assert within_codes(out, want, slack)
    s = torch.pow(2.0, (R.quantise(want, R.E4M3)[1] - 127).double()).repeat_interleave(32, 1)[:, :ff]
    step = torch.maximum(torch.pow(2.0, torch.floor(torch.log2(want.abs().clamp(min=2.0 ** -300))) - 3), s * 2.0 ** -9)
    expected = float((slack / 6 / step).clamp(max=1).sum())
    codes, scales = flips(out, want)
    assert codes <= expected + 6 * expected ** 0.5 + 3 and scales <= 1, (codes, expected, scales)
    assert untouched()


@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
@pytest.mark.parametrize("M", [1, 24, 100])
def test_silu_to_the_last_bits(M, fmt):
    """Products that float32 adds exactly, so that what may be off is silu(g) u: 3 * 2^-23 of it (above).  exp(-g) by a product that is rounded before
    the power is taken would be off by |g| 2^-24: 4 * 2^-23 from 8 on, ten times the bound at the far gates."""
    ff, K, g = 24576 if M == 1 else 6144, 128, torch.Generator().manual_seed(M)
    w = torch.zeros(2 * ff, K, dtype=torch.float64)
    centre = -torch.linspace(-12, 60, ff // 32, dtype=torch.float64).repeat_interleave(32)       # gates of a block lie together, so none is lost under the block's largest
    left = torch.round((centre + torch.rand(ff, generator=g, dtype=torch.float64)) * 256) / 256
    for k in (0, 32, 64):                                    # three codes add up to a gate, or nearly
        w[:ff, k] = left
        w[:ff, k] = R.values(*R.quantise(w[:ff], fmt), fmt)[:, k]
        left = left - w[:ff, k]
    w[ff:, 96] = torch.randint(0, 2, (ff,), generator=g).double() * 2 - 1
    a = torch.zeros(M, K, dtype=torch.float64)
    a[:, 0:96:32] = 1 + (torch.arange(M) % 8 / 8.0)[:, None]
    a[:, 96] = 1.0
    (w, w_b), (a, a_b) = R.quantise(w, fmt), R.quantise(a, R.E4M3)
    p = cuda64(R.values(a, a_b, R.E4M3), R.values(w, w_b, fmt))
    gate, up = p[:, :ff], p[:, ff:]
    assert torch.equal(p, p.float().double()) and gate.min() > -120
    want = gate / (1 + torch.exp(-gate)) * up
    out, untouched = guarded_mx(M, ff)
    B.gemm_mx_swiglu(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), out=out)
    assert within_codes(out, want, 3 * 2.0 ** -23 * want.abs())
    assert untouched()


@pytest.mark.parametrize("fmt", [R.E4M3, R.E2M1])
def test_far_gates_to_the_last_bits(fmt):
    """As above with gates of -80 to -240 and factors of some 2^100 (400 000 different codes): an argument of the exponential off by half a last place of 128 (2^-17) would move 1 code of 40 000
    beyond 3 * 2^-23 of the value (the argument is rounded to 2^-25, the exponential off by 2^-23, three products by 2^-24 each)."""
    M, ff, K, g = 64, 6144, 128, torch.Generator().manual_seed(5)
    w = torch.zeros(2 * ff, K, dtype=torch.float64)
    centre = -torch.linspace(81, 127, ff // 32, dtype=torch.float64).repeat_interleave(32)
    w[:ff, :96] = as_terms(torch.round((centre - torch.rand(ff, generator=g, dtype=torch.float64)) * 256) / 256, fmt)
    w[ff:, 96] = 2.0 ** 100 * (torch.randint(0, 2, (ff,), generator=g).double() * 2 - 1) * (1 + torch.randint(0, 2, (ff,), generator=g) / 2.0)
    a = torch.zeros(M, K, dtype=torch.float64)
    a[:, 0:96:32] = 1 + (torch.arange(M) % 8 / 8.0)[:, None]
    a[:, 96] = 1 + torch.arange(M) // 8 % 8 / 8.0
    (w, w_b), (a, a_b) = R.quantise(w, fmt), R.quantise(a, R.E4M3)
    p = cuda64(R.values(a, a_b, R.E4M3), R.values(w, w_b, fmt))
    gate, up = p[:, :ff], p[:, ff:]
    assert torch.equal(p, p.float().double()) and gate.max() <= -80 and gate.min() >= -256
    want = gate * torch.exp(gate) / (1 + torch.exp(gate)) * up
    out, untouched = guarded_mx(M, ff)
    B.gemm_mx_swiglu(*R.pack(a, a_b, R.E4M3), *R.pack(w, w_b, fmt), out=out)
    assert within_codes(out, want, 3 * 2.0 ** -23 * want.abs() + 2.0 ** -149)
    assert untouched()
