"""SwiGLU of block-scaled rows where single roundings show: gates far below zero, and the share of codes that are not the definition's."""
import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import mx_reference as R
from tests.test_gpu_mx import cuda64, guarded_mx, within_codes

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
