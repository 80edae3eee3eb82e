"""The float64 reference of block-scaled rows against torch's 8-bit types and hand-computed blocks, and the calls' refusals (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import mx_reference as R


def test_e4m3_codes_are_torch_s():
    g = torch.Generator().manual_seed(0)
    x = (torch.rand(64, 128, generator=g, dtype=torch.float64) * 2 - 1) * 448
    x[0, :127] = R.e4m3_table()
    x[1, :126] = (R.e4m3_table()[1:] + R.e4m3_table()[:-1]) / 2   # ties
    x[:, 0::32] = 448.0                                      # every block's scale is 1
    codes, byte = R.quantise(x, R.E4M3)
    assert (byte == 127).all()
    assert torch.equal(codes.to(torch.uint8), x.float().to(torch.float8_e4m3fn).view(torch.uint8))
    assert torch.equal(R.values(codes, byte, R.E4M3), x.float().to(torch.float8_e4m3fn).double())


def test_e2m1_codes_by_hand():
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :16] = torch.tensor([6, .25, .26, .75, 1.25, 1.75, 2.5, 3.5, 5, -5.01, -.24, -.75, 0, -2.5, 5.99, -6])
    codes, byte = R.quantise(x, R.E2M1)
    assert byte[0, 0] == 127
    assert codes[0, :16].tolist() == [7, 0, 1, 2, 2, 4, 4, 6, 6, 15, 8, 10, 0, 12, 7, 15]


@pytest.mark.parametrize("fmt,top", [(R.E4M3, 448.0), (R.E2M1, 6.0)])
def test_scales(fmt, top):
    for amax, want in ((top, 127), (top * 1.0001, 128), (top / 2, 126), (0.0, 0), (top * 2.0 ** -127, 0), (2.0 ** -149, 0), (float("inf"), 255),
                       (float("nan"), 255)):
        x = torch.zeros(1, 64, dtype=torch.float64)
        x[0, 40] = amax
        codes, byte = R.quantise(x, fmt)
        assert byte[0].tolist() == [0, want, 0, 0], amax
        assert (codes[0, :32] == 0).all() and (want < 255 or (codes == 0).all())


def test_pack_and_unpack():
    g = torch.Generator().manual_seed(1)
    for fmt in (R.E4M3, R.E2M1):
        codes, byte = R.quantise(torch.randn(5, 200, generator=g, dtype=torch.float64), fmt)
        c, s = R.pack(codes, byte, fmt, device="cpu")
        assert s.shape == (2, 5, 4) and c.shape == (5, 256 if fmt == R.E4M3 else 128)
        c2, b2 = R.unpack(c, s, fmt)
        assert torch.equal(c2, codes) and torch.equal(b2, byte)


# ---------------------------------------------------------------- refusals, before anything is launched
P = 4096          # an address that is never used: the calls below are refused, or empty
BAD = {"EINVAL": -1, "ESHAPE": -2}


def refused(rc, status, text):
    assert rc == BAD[status], rc
    assert text in B.lib().pvf_last_error(None).decode()


def test_quant_refuses():
    f = B.lib().pvf_quant_mx
    refused(f(None, 7, P, 0, P, P, 1, 32), "EINVAL", "dtype")
    refused(f(None, 0, P, 2, P, P, 1, 32), "EINVAL", "fmt")
    refused(f(None, 0, None, 0, P, P, 1, 32), "EINVAL", "x is NULL")
    refused(f(None, 0, P + 2, 0, P, P, 1, 32), "EINVAL", "between elements")
    refused(f(None, 1, P + 1, 0, P, P, 1, 32), "EINVAL", "between elements")
    refused(f(None, 0, P, 0, None, P, 1, 32), "EINVAL", "NULL")
    refused(f(None, 0, P, 0, P, None, 1, 32), "EINVAL", "NULL")
    refused(f(None, 0, P, 0, P + 8, P, 1, 32), "EINVAL", "16 bytes")
    refused(f(None, 0, P, 0, P, P + 2, 1, 32), "EINVAL", "scales of 4")
    refused(f(None, 0, P, 0, P, P, -1, 32), "EINVAL", "size")
    refused(f(None, 0, P, 0, P, P, 1, 0), "EINVAL", "size")
    refused(f(None, 0, P, 0, P, P, (1 << 28) + 1, 32), "ESHAPE", "beyond")
    refused(f(None, 0, P, 0, P, P, 1, (1 << 24) + 1), "ESHAPE", "beyond")
    assert f(None, 0, None, 0, None, None, 0, 32) == 0       # no rows: nothing to do


def test_norm_refuses():
    f = B.lib().pvf_add_rmsnorm_mx
    refused(f(None, 3, P, P, P, P, P, P, 1, 32, 1e-5), "EINVAL", "dtype")
    refused(f(None, 0, None, P, P, P, P, P, 1, 32, 1e-5), "EINVAL", "NULL")
    refused(f(None, 0, P, P, None, P, P, P, 1, 32, 1e-5), "EINVAL", "NULL")
    refused(f(None, 0, P, P + 1, P, P, P, P, 1, 32, 1e-5), "EINVAL", "between elements")
    refused(f(None, 0, P, P, P, P + 2, P, P, 1, 32, 1e-5), "EINVAL", "between elements")
    refused(f(None, 0, P, P, P, P, None, P, 1, 32, 1e-5), "EINVAL", "NULL")
    refused(f(None, 0, P, P, P, P, P, P, 1, 0, 1e-5), "EINVAL", "size")
    refused(f(None, 0, P, P, P, P, P, P, 1, 32, -1.0), "EINVAL", "eps")
    refused(f(None, 0, P, P, P, P, P, P, 1, 32, float("nan")), "EINVAL", "eps")
    assert f(None, 0, None, None, None, None, None, None, 0, 32, 1e-5) == 0


def test_products_refuse():
    f = B.lib().pvf_gemm_mx
    refused(f(None, 2, 0, P, P, P, P, P, None, 1, 1, 32), "EINVAL", "w_fmt")
    refused(f(None, 0, 9, P, P, P, P, P, None, 1, 1, 32), "EINVAL", "dtype")
    refused(f(None, 0, 0, None, P, P, P, P, None, 1, 1, 32), "EINVAL", "(A)")
    refused(f(None, 0, 0, P, P, P + 4, P, P, None, 1, 1, 32), "EINVAL", "(W)")
    refused(f(None, 0, 0, P, P, P, P + 1, P, None, 1, 1, 32), "EINVAL", "(W)")
    refused(f(None, 0, 0, P, P, P, P, None, None, 1, 1, 32), "EINVAL", "C is NULL")
    refused(f(None, 0, 1, P, P, P, P, P, P + 1, 1, 1, 32), "EINVAL", "between elements")
    refused(f(None, 0, 0, P, P, P, P, P, None, 1, -1, 32), "EINVAL", "size")
    refused(f(None, 0, 0, P, P, P, P, P, None, 1, 1, (1 << 24) + 1), "ESHAPE", "beyond")
    assert f(None, 0, 0, None, None, None, None, None, None, 0, 4, 32) == 0 and f(None, 0, 0, None, None, None, None, None, None, 4, 0, 32) == 0
    f = B.lib().pvf_gemm_mx_swiglu
    refused(f(None, 5, P, P, P, P, P, P, 1, 32, 32), "EINVAL", "w_fmt")
    refused(f(None, 0, P, P, P, P, P, None, 1, 32, 32), "EINVAL", "(act)")
    refused(f(None, 0, P, P, P, P, P + 8, P, 1, 32, 32), "EINVAL", "(act)")
    refused(f(None, 0, P, P, P, P, P, P, 1, (1 << 24) + 1, 32), "ESHAPE", "beyond")
    assert f(None, 0, None, None, None, None, None, None, 0, 32, 32) == 0
    f = B.lib().pvf_gemm_w4
    refused(f(None, 2, P, P, P, P, None, 1, 1, 32), "EINVAL", "dtype")
    refused(f(None, 0, P + 2, P, P, P, None, 1, 1, 32), "EINVAL", "between elements")
    refused(f(None, 0, P, None, P, P, None, 1, 1, 32), "EINVAL", "(W)")
    refused(f(None, 0, P, P, P, P + 2, None, 1, 1, 32), "EINVAL", "between elements")
    assert f(None, 0, None, None, None, None, None, 0, 1, 32) == 0


def test_rows_of_more_than_2_22_elements_are_refused():
    n = (1 << 22) + 1
    refused(B.lib().pvf_quant_mx(None, 0, P, 0, P, P, 1, n), "ESHAPE", "2^22")
    refused(B.lib().pvf_add_rmsnorm_mx(None, 0, P, P, P, P, P, P, 1, n, 1e-5), "ESHAPE", "2^22")
    refused(B.lib().pvf_gemm_mx(None, 0, 0, P, P, P, P, P, None, 1, 1, n), "ESHAPE", "2^22")
    refused(B.lib().pvf_gemm_mx_swiglu(None, 0, P, P, P, P, P, P, 1, n, 32), "ESHAPE", "2^22")
    refused(B.lib().pvf_gemm_mx_swiglu(None, 0, P, P, P, P, P, P, 1, 32, n), "ESHAPE", "2^22")
    refused(B.lib().pvf_gemm_w4(None, 0, P, P, P, P, None, 1, 1, n), "ESHAPE", "2^22")


def test_binding_refuses():
    """What the binding can tell from shapes and types alone, on CPU tensors."""
    x = torch.zeros(4, 200)
    codes, scales = B.mx_empty(4, 200, device="cpu")
    w4, w4s = B.mx_empty(8, 200, B.MX_E2M1, device="cpu")
    for call in (lambda: B.quant_mx(x),                                                       # not on a device
                 lambda: B.quant_mx(x, out=(codes[:2], scales)),
                 lambda: B.quant_mx(x, out=(codes, scales.view(torch.uint8))),
                 lambda: B.quant_mx(x, B.MX_E2M1, out=(codes, scales)),
                 lambda: B.add_rmsnorm_mx(x, torch.ones(199), 1e-5, out=(codes, scales)),
                 lambda: B.add_rmsnorm_mx(x, torch.ones(200), 1e-5, residual=x[:2], out=(codes, scales)),
                 lambda: B.gemm_mx(w4, w4s, codes, scales),                                   # 4-bit rows
                 lambda: B.gemm_mx(codes, scales, w4[:, :64], w4s),
                 lambda: B.gemm_mx(codes, scales, w4, w4s, residual=torch.zeros(4, 7)),
                 lambda: B.gemm_mx_swiglu(codes, scales, w4[:7], w4s[:, :7]),
                 lambda: B.gemm_w4(x, codes, scales),                                         # 8-bit weights
                 lambda: B.gemm_w4(x, w4, w4s, out=torch.zeros(4, 8, dtype=torch.bfloat16))):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(TypeError):
        B.quant_mx(x.double().cuda() if torch.cuda.is_available() else x.double())
    assert ctypes.sizeof(ctypes.c_void_p) == 8
