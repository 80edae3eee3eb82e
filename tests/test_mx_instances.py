"""Which kernel instance a product of block-scaled rows takes is decided on the host (pvf_gemm_mx_instance), so no GPU is needed to see that none is out of reach."""
import ctypes

import pytest
import torch

from paper_2601_12247_amd import binding as B

BF16, F32 = torch.bfloat16, torch.float32
# what has a list of instances of its own: call, weights, type, whether rows begin at 16 bytes
KINDS = {
    "mx_e4m3": (B.MX_GEMM, B.MX_E4M3, BF16, True), "mx_e2m1": (B.MX_GEMM, B.MX_E2M1, BF16, True),
    "mx_e4m3_f32": (B.MX_GEMM, B.MX_E4M3, F32, True), "mx_e2m1_f32": (B.MX_GEMM, B.MX_E2M1, F32, True),
    "swiglu_e4m3": (B.MX_SWIGLU, B.MX_E4M3, BF16, True), "swiglu_e2m1": (B.MX_SWIGLU, B.MX_E2M1, BF16, True),
    "w4": (B.MX_W4, B.MX_E2M1, BF16, True), "w4_shifted": (B.MX_W4, B.MX_E2M1, BF16, False),
    "w4_f32": (B.MX_W4, B.MX_E2M1, F32, True), "w4_f32_shifted": (B.MX_W4, B.MX_E2M1, F32, False),
}


def instance(kind, M, N, K):
    call, fmt, dtype, aligned = KINDS[kind]
    return B.gemm_mx_instance(call, M, N, K, fmt, dtype, aligned)


@pytest.mark.parametrize("kind", KINDS)
def test_every_instance_is_taken_by_some_product(kind):
    rows = (1, 2, 4, 5, 16, 17, 32, 33, 48, 64, 80, 96, 128, 160, 192, 224, 256, 320, 448, 512, 640, 832, 1024, 1280, 1792, 2560, 4100, 8300, 11520)
    columns = (16, 64, 130, 200, 256, 300, 400, 512, 640, 800, 1024, 1411, 2048, 2700, 4096, 4200, 6144, 8250, 12288, 16800, 22000)
    taken = {instance(kind, M, N, K) for M in rows for N in columns for K in (72, 520, 648)}
    assert len({count for _, count in taken}) == 1
    assert {index for index, _ in taken} == set(range(taken.pop()[1]))


def test_rows_that_do_not_begin_at_16_bytes_have_lists_of_their_own():
    """By their first address, or by their length: 1030 bfloat16 or 1411 float32 elements are no whole number of 16 bytes."""
    assert B.gemm_mx_instance(B.MX_W4, 5, 64, 1030) == B.gemm_mx_instance(B.MX_W4, 5, 64, 1030, aligned=False)
    assert B.gemm_mx_instance(B.MX_W4, 5, 64, 1411, dtype=F32) == B.gemm_mx_instance(B.MX_W4, 5, 64, 1411, dtype=F32, aligned=False)
    assert instance("w4", 5, 64, 1024)[1] != instance("w4_shifted", 5, 64, 1024)[1]


def test_instance_refuses():
    f, i = B.lib().pvf_gemm_mx_instance, ctypes.byref(ctypes.c_int32())
    for args in ((3, 0, 0, 1, 1, 1, 32), (0, 2, 0, 1, 1, 1, 32), (0, 0, 7, 1, 1, 1, 32), (1, 2, 0, 1, 1, 1, 32), (2, 0, 2, 1, 1, 1, 32), (0, 0, 0, 1, 0, 1, 32), (0, 0, 0, 1, 1, 0, 32),
                 (0, 0, 0, 1, 1, 1, 0), (0, 0, 0, 1, -1, 1, 32)):
        assert f(*args, i, i) == -1, args
    assert f(0, 0, 0, 1, 1, 1, (1 << 22) + 1, i, i) == -2
    assert f(0, 0, 0, 1, 1, 1, 32, None, i) == -1 and f(0, 0, 0, 1, 1, 1, 32, i, None) == -1
    assert f(1, 0, 7, 1, 1, 1, 32, i, i) == 0 and f(2, 7, 0, 0, 1, 1, 32, i, i) == 0        # what is not read


@pytest.mark.parametrize("kind", KINDS)
def test_gpu_tests_run_every_instance(kind):
    """With one stage of 128 k (or two, where stages go in pairs), and with twelve or more."""
    from tests.test_gpu_mx_instances import LONG, SHORT
    for shapes, stages in ((SHORT[kind], range(1, 3)), (LONG[kind], range(11, 100))):
        taken = [instance(kind, *s) for s in shapes]
        assert all((K + 127) // 128 in stages for _, _, K in shapes)
        assert [index for index, _ in taken] == list(range(taken[0][1]))
