"""The paged K/V cache at the borders between its ways of doing a call: more triples than workgroups, one launch and two, prompts that see their own tokens, one
beside many single rows, tables that the library refuses.  Against tests/page_reference.py, exactly or with the slack that it derives."""
import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import page_reference as R
from tests.test_gpu_pages import Pool, check_extend, i32, requests

pytestmark = pytest.mark.gpu


# Requests x key heads of 40 to 100 columns, one tile each, above the 2048 workgroups of a launch (1024 where d_head is above 128): a workgroup takes several
# triples, whole as the table has room for little (20 pages) or as they are dealt out (80).  Columns are heads, so that rows are few.
@pytest.mark.parametrize("width", [20, 80])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("nreq,Hkv,group,n,dh", [(300, 8, 20, 2, 64), (300, 8, 20, 2, 72), (270, 8, 45, 2, 128), (270, 8, 35, 3, 40), (140, 8, 11, 3, 256), (140, 8, 25, 3, 136)])
def test_more_triples_than_workgroups(nreq, Hkv, group, n, dh, causal, width):
    lens = [(37 * b) % 200 for b in range(nreq)]
    p = Pool(lens, Hkv * group, Hkv, dh, 16, "bf16", seed=nreq + dh, width=width, spread=2.0).rows([n - (b % 7 == 3) for b in range(nreq)])
    first = p.check(causal=causal, extra=1)
    assert torch.equal(first, p.run(causal=causal, extra=1))


@pytest.mark.parametrize("nreq,rows,W,P", [(64, [32] * 64, 20, 16), (64, [32] * 63 + [33], 20, 16), (1, [2048], 200, 16), (1, [2049], 200, 16),
                                           (65, [31] * 64 + [64], 20, 16), (65, [31] * 64 + [65], 20, 16), (2048, [1] * 2048, 4, 8), (2048, [1] * 2047 + [2], 4, 8),
                                           (2049, [1] * 2047 + [0, 1], 4, 8), (2047, [1] * 2046 + [2], 4, 8)])
@pytest.mark.parametrize("in_place", [False, True])
def test_extend_where_one_launch_becomes_two(nreq, rows, W, P, in_place):
    """2048 rows and 2049, 64 requests and 65, 2048 and 2049: with enough pages and without."""
    lens, _, table, free, n_free = requests(nreq, W * P // 3, 0, W, P, seed=nreq + rows[-1])
    M = sum(rows)
    assert M in (2048, 2049)
    check_extend(lens, rows, table, free, n_free, P, M, in_place=in_place)
    check_extend(lens, rows, table, free, max(1, M // (3 * P)), P, M, in_place=in_place)
    check_extend(lens, rows, table, free, n_free, P, M, start=[x // 2 for x in lens], in_place=in_place)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,dh,lens", [(4, 4, 128, [700]), (4, 1, 128, [513]), (2, 1, 64, [640, 1, 127, 0, 300]), (2, 2, 80, [500, 129]), (2, 1, 256, [333])])
def test_prompts_that_see_their_own_tokens(dtype, H, Hkv, dh, lens):
    """As many rows as tokens: row i sees i + 1."""
    for width in (None, 120):
        Pool(lens, H, Hkv, dh, 16, dtype, seed=dh, width=width).rows(lens).check(causal=True, extra=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nreq,H,Hkv,dh,prompt", [(80, 8, 2, 128, 300), (80, 8, 2, 64, 700), (20, 8, 2, 128, 512), (70, 2, 1, 256, 400)])
def test_a_prompt_beside_single_rows(dtype, nreq, H, Hkv, dh, prompt):
    """What a serving step looks like when a request enters: the instance goes by the mean number of rows, narrow for the most of these."""
    for at in (0, nreq // 2, nreq - 1):
        lens = [(61 * b) % 500 + 1 for b in range(nreq)]
        lens[at] = prompt
        Pool(lens, H, Hkv, dh, 16, dtype, seed=at, width=50).rows([prompt if b == at else 1 for b in range(nreq)]).check(causal=True, extra=2)


def test_tables_whose_rows_overlap_are_refused():
    """One row for all requests, and rows that share columns: an error, and nothing is written."""
    for table in (i32([3, 1, 0, 2, 4])[None].expand(3, 5), i32(list(range(9))).as_strided((3, 5), (2, 1))):
        before, free = table.clone(), i32([8, 9, 10, 11, 12, 13])
        lens, n_free, outs = i32([70, 70, 70]), i32([6]), [torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (3, 1, 4, 3, 4, 60, 60)]
        q, kv, out = (torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((3, 4, 64), (14, 2, 16, 64), (3, 4, 64)))
        with pytest.raises(B.PvfError, match="apart"):
            B.page_extend(lens, i32([20, 20, 20]), table, free, n_free, 16, out=tuple(outs))
        with pytest.raises(B.PvfError, match="apart"):
            B.page_trim(lens, i32([0, 0, 0]), table, free, n_free, 16, out=tuple(outs[:2] + [outs[2]]))
        with pytest.raises(B.PvfError, match="apart"):
            B.page_attention(q, kv, kv, table, lens, out=out)
        torch.cuda.synchronize()
        assert torch.equal(table, before) and free.tolist() == [8, 9, 10, 11, 12, 13] and all(bool((o == -77).all()) for o in outs) and bool((out == 7.0).all())
        one = B.page_attention(q, kv, kv, before, lens)                       # rows of its own for each
        assert bool((one == 7.0).all())
