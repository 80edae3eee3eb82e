"""Attention over pages of requests that are longer than their table: every row that sees a token is NaN, by the length as it was told, and rows that see none
are zeros.  Every other row against tests/page_reference.py, with the slack that it derives."""
import pytest
import torch

from tests import page_reference as R
from tests.test_gpu_pages import Pool

pytestmark = pytest.mark.gpu


def check(lens, n, told, H, Hkv, dh, dtype, width, causal):
    """`told`: the lengths in the call; `lens`: how many tokens of each request the table has pages for."""
    p = Pool(lens, H, Hkv, dh, 16, dtype, seed=len(lens) + dh, width=width, apart=16).rows(n)
    want, slack = R.attention(p.q, p.k, p.v, p.table, lens, p.cu, causal, dh ** -0.5)
    p.lens = told
    got = p.run(causal=causal, extra=2)
    for b in range(len(lens)):
        for i, r in enumerate(range(p.cu[b], p.cu[b + 1])):
            if told[b] <= width * 16:
                assert R.close(got[r], want[r], slack[r]), (b, i)
            elif causal and told[b] - n[b] + i + 1 <= 0:
                assert not got[r].any(), (b, i)
            else:
                assert bool(got[r].isnan().all()), (b, i)
    assert torch.equal(got.isnan(), p.run(causal=causal, extra=2).isnan())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("H,Hkv,dh", [(4, 4, 64), (8, 2, 128), (2, 1, 80), (2, 1, 256)])
@pytest.mark.parametrize("n", [3, 90])
def test_several_rows_of_a_request_longer_than_its_table(dtype, causal, H, Hkv, dh, n):
    """80 tokens in the table, 100 told, 90 rows: rows 0 .. see 11 .. tokens.  One token too many; rows that see less than the table holds; rows that see none."""
    check([80, 80, 70, 80, 80], [n, n, n, 2, n], [100, 81, 70, 2 ** 31 - 1, 85], H, Hkv, dh, dtype, 5, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [1, 40])
def test_a_table_without_columns(dtype, causal, n):
    check([0, 0, 0], [n, n, n], [5, 0, 100], 4, 2, 64, dtype, 0, causal)


@pytest.mark.parametrize("dtype,width,n", [
    ("bf16", 65, [1100]),                                  # many rows: keys of a tile divided, and joined
    ("f32", 26, [420]),
    ("bf16", 41, [1] * 30 + [700] + [1] * 30),             # few columns a tile, which go by the mean
])
def test_divided_and_joined(dtype, width, n):
    held = [width * 16 if x > 1 else 100 + 7 * b for b, x in enumerate(n)]
    told = [width * 16 + 40 if x > 1 else y for x, y in zip(n, held)]
    check(held, n, told, 1, 1, 64, dtype, width, True)
