"""Attention over pages where lengths and row offsets are not what a table or M has room for.  Requests longer than their table: every row that sees a token is
NaN, by the length as it was told, and rows that see none are zeros.  Every other row against tests/page_reference.py, with the slack that it derives."""
import pytest
import torch

from paper_2601_12247_amd import binding as B
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 70])
def test_row_offsets_at_the_ends_of_their_type(dtype, n):
    """Offsets of -2^31 and 2^31 - 1 behind sound ones: the requests that they end or begin have no rows, or those up to M, and nothing else is touched."""
    least, most = -2 ** 31, 2 ** 31 - 1
    p = Pool([100, 90, 80], 4, 2, 64, 16, dtype, seed=n).rows([n, n, n])
    want, slack = R.attention(p.q, p.k, p.v, p.table, p.lens, p.cu, False, 64 ** -0.5)
    q, k, v, table, lens = p.q.cuda(), p.k.cuda(), p.v.cuda(), p.table.cuda(), torch.tensor(p.lens, dtype=torch.int32, device="cuda")
    for cu, written in (([0, n, least, least + 1], 1), ([0, n, least + n, least], 1), ([least, n, 2 * n, most], 3), ([0, n, most, least], 2), ([most, least, -1, 0], 0)):
        buf = torch.full((3 * n + 8, 4, 64), 7.0, dtype=p.dtype, device="cuda")
        B.page_attention(q, k, v, table, lens, cu_rows=torch.tensor(cu, dtype=torch.int32, device="cuda"), out=buf[4: 4 + 3 * n])
        got, own = buf[4: 4 + 3 * n].cpu(), n if written == 2 else n * written      # with `most` behind n, request 1 has all rows from n on
        assert R.close(got[:own], want[:own], slack[:own])
        if written == 2:
            again, off = R.attention(p.q, p.k, p.v, p.table, p.lens, [0, n, 3 * n, 3 * n], False, 64 ** -0.5)
            assert R.close(got, again, off)
        else:
            assert bool((got[own:] == 7.0).all())
        assert bool((buf[:4] == 7.0).all() and (buf[4 + 3 * n:] == 7.0).all())
