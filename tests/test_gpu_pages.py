"""The paged K/V cache on the GPU against tests/page_reference.py: tables, slots and free lists exactly, rotated rows and attention in float64.

Tolerances: stored rows, half a step of their type and 8 roundings of float32 (angle 3.2 of them, sine and cosine 2, product and sum 2) of |a| + |b|;
attention, half a step of its type and the slack that page_reference.attention derives."""
import math

import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import page_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def guarded(n, fill=-77):
    """int32 [n] between sentinels, and what tells whether they are left as they were."""
    buf = torch.full((n + 64,), fill, dtype=torch.int32, device="cuda")
    return buf[32: 32 + n], lambda: bool((buf[:32] == fill).all() and (buf[32 + n:] == fill).all())


# ---------------------------------------------------------------- tables
def check_extend(seq_len, n_rows, table, free, n_free, P, M, start=None, in_place=False):
    B_, W = len(seq_len), len(table[0]) if table else 0
    want = R.extend(seq_len, n_rows, table, free, n_free, P, M, start)
    dev_table = torch.full((B_ + 2, W + 3), -77, dtype=torch.int32, device="cuda")     # rows lie apart
    dev_table[1: B_ + 1, :W] = i32(table).view(B_, W) if B_ else 0
    lens, count = i32(seq_len).view(-1), i32([n_free])
    sizes = (B_, 1, B_ + 1, B_, B_ + 1, M, M)
    outs = [guarded(n) for n in sizes]
    out = [o for o, _ in outs]
    if in_place:
        out[0], out[1] = lens, count
    B.page_extend(lens, i32(n_rows).view(-1), dev_table[1: B_ + 1, :W], i32(free).view(-1), count, P, start=None if start is None else i32(start).view(-1), out=tuple(out))
    for name, got in zip(("seq_len", "n_free", "cu_rows", "admitted", "place", "pos", "slot"), out):
        expect = want[name] if name != "n_free" else [want[name]]
        assert got.cpu().tolist() == expect, name
    assert dev_table[1: B_ + 1, :W].cpu().tolist() == want["table"]
    assert bool((dev_table[0] == -77).all() and (dev_table[-1] == -77).all() and (dev_table[:, W:] == -77).all())
    assert all(ok() for _, ok in outs)


def requests(nreq, most_len, most_rows, W, P, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda top, n: torch.randint(0, top + 1, (n,), generator=g).tolist()  # noqa: E731
    lens = [min(x, W * P) for x in r(most_len, nreq)]
    rows = r(most_rows, nreq)
    n_pages = nreq * W + 5
    pages = torch.randperm(n_pages, generator=g).tolist()
    table = [[pages.pop() if j < R.pages_of(lens[b], P) else -1 for j in range(W)] for b in range(nreq)]
    return lens, rows, table, pages + [-5] * 3, len(pages)


# (requests, longest, most rows, width, page size): one launch, and two (more than 2048 rows or 2048 requests)
SIZES = [(1, 0, 1, 1, 16), (1, 15, 1, 2, 16), (1, 16, 1, 2, 16), (5, 40, 3, 9, 8), (64, 500, 1, 40, 16), (63, 100, 200, 30, 16), (700, 30, 5, 9, 7), (2048, 9, 4, 20, 1),
         (9, 100, 3000, 200, 24), (2049, 20, 1, 9, 8), (1, 3, 20000, 400, 64), (3000, 64, 64, 20, 16), (1025, 10, 2, 4, 8)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("nreq,most_len,most_rows,W,P", SIZES)
def test_extend_is_the_reference_s(nreq, most_len, most_rows, W, P, in_place):
    lens, rows, table, free, n_free = requests(nreq, most_len, most_rows, W, P, seed=nreq + P)
    check_extend(lens, rows, table, free, n_free, P, sum(rows) + 3, in_place=in_place)


@pytest.mark.parametrize("nreq,most_len,most_rows,W,P", SIZES)
def test_extend_without_enough_of_anything(nreq, most_len, most_rows, W, P):
    """Too few pages, tables too narrow, more rows than there is room for, negative counts: exactly the requests that the rule names are turned away."""
    lens, rows, table, free, n_free = requests(nreq, most_len, most_rows, W, P, seed=7 * nreq + P)
    rows = [-3 if b % 11 == 5 else x for b, x in enumerate(rows)]
    total = sum(max(x, 0) for x in rows)
    check_extend(lens, rows, table, free, min(n_free, total // (3 * P) + 1), P, total, in_place=True)
    check_extend(lens, rows, table, free, 0, P, total * 2 // 3)
    check_extend(lens, rows, table, free, len(free) + 100, P, 0)
    narrow = max(1, W // 2)
    short = [min(x, narrow * P + 1) for x in lens]
    check_extend(short, rows, [t[:narrow] for t in table], free, n_free, P, total)


@pytest.mark.parametrize("nreq,W,P", [(9, 20, 64), (40, 30, 8), (2500, 6, 16)])
def test_extend_of_rows_that_are_written_again(nreq, W, P):
    """Windows inside a canvas: rows from `start` on, some behind the end, some starting outside."""
    lens, rows, table, free, n_free = requests(nreq, W * P * 2 // 3, P + 5, W, P, seed=W)
    g = torch.Generator().manual_seed(5)
    start = [int(torch.randint(-1, x + 2, (1,), generator=g)) for x in lens]
    for in_place in (False, True):
        check_extend(lens, rows, table, free, n_free, P, sum(rows), start=start, in_place=in_place)


def test_extend_of_nothing_and_of_odd_tables():
    check_extend([], [], [], [3, 4], 2, 16, 5)
    check_extend([], [], [], [3, 4], 2, 16, 9000)
    check_extend([0, 0], [0, 0], [[-1], [-1]], [1], 1, 16, 0)
    check_extend([-4, 5, 100], [2, 2, 2], [[-1, -1]] * 3, [1, 2], 2, 16, 6)          # lengths that cannot be
    check_extend([20, 3], [5, 5], [[7, -9], [1 << 30, -1]], [-2, 3], 2, 16, 10)         # entries that are no pages


def check_trim(lens, keep, table, free, n_free, P, in_place=False):
    nreq = len(lens)
    want = R.trim(lens, keep, table, free, n_free, P)
    dev, dev_free = i32(lens).view(-1), torch.full((len(free) + 64,), -77, dtype=torch.int32, device="cuda")
    dev_free[32: 32 + len(free)] = i32(free)
    count = i32([n_free])
    outs = [guarded(n) for n in (nreq, 1, nreq + 1)]
    out = [o for o, _ in outs]
    if in_place:
        out[0], out[1] = dev, count
    dev_table = i32(table)
    B.page_trim(dev, i32(keep).view(-1), dev_table, dev_free[32: 32 + len(free)], count, P, out=tuple(out))
    assert out[0].cpu().tolist() == want["seq_len"] and out[1].cpu().tolist() == [want["n_free"]] and out[2].cpu().tolist() == want["place"]
    assert dev_free[32: 32 + len(free)].cpu().tolist() == want["free"] and dev_table.cpu().tolist() == table
    assert bool((dev_free[:32] == -77).all() and (dev_free[32 + len(free):] == -77).all()) and all(ok() for _, ok in outs)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("nreq,most_len,W,P", [(1, 0, 1, 16), (1, 16, 1, 16), (5, 40, 9, 8), (64, 500, 40, 16), (700, 60, 9, 7), (2048, 20, 32, 1), (2049, 70, 9, 8),
                                               (100, 30000, 4000, 8), (3000, 640, 40, 16), (1, 70000, 70000, 1)])
def test_trim_is_the_reference_s(nreq, most_len, W, P, in_place):
    lens, _, table, free, n_free = requests(nreq, most_len, 0, W, P, seed=nreq + W)
    g = torch.Generator().manual_seed(nreq)
    keep = [x - int(torch.randint(0, max(x, 1) + 2, (1,), generator=g)) if b % 3 else x + b % 4 for b, x in enumerate(lens)]
    taken = sum(R.pages_of(x, P) for x in lens)
    check_trim(lens, keep, table, free[:n_free] + [-1] * taken, n_free, P, in_place)


def test_trim_of_more_pages_than_the_list_holds():
    table = [[1, 2, 3, 4], [5, 6, 7, 8]]
    check_trim([50, 64], [0, 0], table, [9, -1, -1, -1, -1], 1, 16)                   # room for 4 of 8
    check_trim([1000, -3], [-1, 5], table, [-1] * 9, -2, 16)                         # a length beyond the table, one below zero, a count below zero
    check_trim([50, 64], [50, 60], table, [9], 7, 16)                               # a count beyond the list
    check_trim([3000], [0], [list(range(3000))], [-1] * 2000, 0, 1)
    check_trim([70000], [0], [list(range(70000))], [-1] * 60000, 5, 1)


# ---------------------------------------------------------------- stores
def rows_apart(M, wide, apart, dtype, gen):
    buf = torch.randn(M, wide + apart, generator=gen).to(dtype).cuda()
    return buf[:, :wide]


def check_store(M, H, Hkv, dh, P, dtype, theta=1e4, apart=0, page_apart=0, in_place=False, top=5000, seed=0):
    g = torch.Generator().manual_seed(seed + M)
    t = DT[dtype]
    n_pages = R.pages_of(M, P) + 3
    qkv = rows_apart(M, (H + 2 * Hkv) * dh, apart, t, g)
    pos = torch.randint(0, top, (M,), generator=g, dtype=torch.int32)
    slot = torch.randperm(n_pages * P, generator=g)[:M].int()
    slot[M // 2: M // 2 + 2] = torch.tensor([-1, n_pages * P], dtype=torch.int32)[: max(0, min(2, M - M // 2 - 1))] if M > 3 else slot[M // 2: M // 2 + 2]
    page = Hkv * P * dh
    pool = torch.randn(n_pages, 2, page + page_apart, generator=g).to(t).cuda()
    k, v = (pool[:, i, :page].view(n_pages, Hkv, P, dh) for i in (0, 1))
    before, x = pool.clone(), qkv.cpu().double().view(M, H + 2 * Hkv, dh)
    q_out = qkv[:, : H * dh].view(M, H, dh) if in_place else torch.full((M, H, dh), 7.0, dtype=t, device="cuda")
    got = B.page_store(qkv, pos.cuda(), slot.cuda(), k, v, theta, q_out=q_out)
    kept = (slot >= 0) & (slot < n_pages * P)
    turned = R.rotate(x[:, : H + Hkv], pos, theta)
    half = dh // 2
    size = x[:, : H + Hkv, :half].abs() + x[:, : H + Hkv, half:].abs()
    slack = 8 * 2.0 ** -24 * torch.cat([size, size], 2)
    q = got.cpu()
    assert R.close(q[kept], turned[kept][:, :H], slack[kept][:, :H])
    left = x[~kept][:, :H] if in_place else torch.full_like(x[~kept][:, :H], 7.0)
    assert torch.equal(q[~kept].double(), left)
    at = slot[kept].long()
    for cache, rows, off in ((k, turned[:, H:], slack[:, H:]), (v, x[:, H + Hkv:], torch.zeros_like(x[:, H + Hkv:]))):
        assert R.close(cache.cpu()[at // P, :, at % P], rows[kept], off[kept])
    untouched = torch.ones(n_pages, P, dtype=torch.bool)
    untouched[at // P, at % P] = False
    for i, cache in ((0, k), (1, v)):
        was = before[:, i, :page].view(n_pages, Hkv, P, dh).transpose(1, 2).cpu()
        assert torch.equal(cache.transpose(1, 2).cpu()[untouched], was[untouched])
    assert torch.equal(pool[:, :, page:], before[:, :, page:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,H,Hkv,dh,P", [(1, 1, 1, 8, 8), (1, 32, 8, 128, 16), (2, 4, 4, 64, 16), (7, 12, 3, 80, 24), (33, 3, 3, 72, 8), (64, 32, 32, 128, 64), (513, 5, 1, 96, 40),
                                          (514, 2, 2, 256, 16), (1021, 7, 7, 24, 8), (600, 1, 2, 16, 8), (515, 0, 2, 64, 16),
                                          (1025, 3, 3, 64, 16), (1030, 4, 2, 128, 24), (1027, 2, 1, 80, 8), (1026, 5, 1, 32, 8), (1029, 1, 1, 8, 16)])
def test_stored_rows_are_the_reference_s(dtype, M, H, Hkv, dh, P):
    check_store(M, H, Hkv, dh, P, dtype)
    check_store(M, H, Hkv, dh, P, dtype, apart=16, page_apart=48, in_place=H > 0, theta=5e5, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_stored_rows_at_far_positions(dtype):
    """Angles of the last positions that 31 bits hold: float32 would be off by whole turns."""
    check_store(40, 4, 2, 128, 16, dtype, theta=1e4, top=2 ** 31 - 1)
    check_store(600, 2, 1, 64, 16, dtype, theta=1.5, top=2 ** 31 - 1)
    check_store(1400, 2, 1, 128, 16, dtype, theta=1e6, top=2 ** 31 - 1)


# ---------------------------------------------------------------- attention
class Pool:
    """Caches whose pages are filled with `junk` wherever no token lies, and requests with tables into them."""

    def __init__(self, lens, H, Hkv, dh, P, dtype, seed=0, junk=math.nan, width=None, spare=2, apart=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        t = DT[dtype]
        self.lens, self.H, self.Hkv, self.dh, self.P, self.dtype, self.gen = lens, H, Hkv, dh, P, t, g
        need = [R.pages_of(x, P) for x in lens]
        n_pages = sum(need) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        W = max(need + [1]) if width is None else width
        table = [[order.pop() if j < need[b] else -1 for j in range(W)] for b in range(len(lens))]
        self.table = torch.tensor(table, dtype=torch.int32).view(len(lens), W)
        pool = torch.full((n_pages, 2, Hkv * P * dh + apart), junk, dtype=t)
        self.k, self.v = (pool[:, i, : Hkv * P * dh].view(n_pages, Hkv, P, dh) for i in (0, 1))
        for b, length in enumerate(lens):
            for cache, scale in ((self.k, spread), (self.v, 1.0)):
                for j in range(need[b]):
                    n = min(P, length - j * P)
                    cache[table[b][j], :, :n] = (torch.randn(Hkv, n, dh, generator=g) * scale).to(t)
        self.pool = pool

    def rows(self, n):
        self.n = n
        self.cu = [0]
        for x in n:
            self.cu.append(self.cu[-1] + x)
        self.q = torch.randn(self.cu[-1], self.H, self.dh, generator=self.gen).to(self.dtype)
        return self

    def run(self, causal=False, scale=None, cu="given", extra=0, workspace=None):
        dev = self.pool.cuda()
        n_pages, page = dev.shape[0], self.Hkv * self.P * self.dh
        k, v = (dev[:, i, :page].view(n_pages, self.Hkv, self.P, self.dh) for i in (0, 1))
        M = self.cu[-1] + extra
        q = torch.cat([self.q, torch.full((extra, self.H, self.dh), math.nan, dtype=self.dtype)]).cuda()
        out = torch.full((M, self.H, self.dh), 7.0, dtype=self.dtype, device="cuda")
        B.page_attention(q, k, v, self.table.cuda(), i32(self.lens), cu_rows=i32(self.cu) if cu else None, causal=causal, scale=scale, out=out, workspace=workspace)
        assert bool((out[self.cu[-1]:] == 7.0).all()), "rows behind the last request"
        return out[: self.cu[-1]].cpu()

    def check(self, causal=False, scale=None, **kw):
        got = self.run(causal, scale, **kw)
        want, slack = R.attention(self.q, self.k, self.v, self.table, self.lens, self.cu, causal, self.dh ** -0.5 if scale is None else scale)
        assert R.close(got, want, slack), float(((got.double() - want).abs() - slack).nan_to_num().max())
        return got


LENGTHS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 255, 257, 300]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,dh,P", [(4, 4, 64, 16), (32, 8, 128, 16), (8, 1, 128, 64), (6, 2, 80, 24), (7, 1, 72, 8), (3, 3, 8, 8), (2, 1, 256, 16), (2, 2, 136, 40), (5, 5, 128, 512)])
@pytest.mark.parametrize("width", [None, 200])
def test_single_rows_at_every_border(dtype, H, Hkv, dh, P, width):
    """One row a request; tables as narrow as the requests are long (one launch where that is little) and wide ones (keys divided, two launches)."""
    Pool(LENGTHS, H, Hkv, dh, P, dtype, seed=H + dh, width=width).rows([1] * len(LENGTHS)).check()
    Pool(LENGTHS, H, Hkv, dh, P, dtype, seed=H + dh, width=width).rows([1] * len(LENGTHS)).check(causal=True, cu=None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,Hkv,dh,P,lens,n", [
    (4, 2, 64, 16, [40, 0, 5, 300, 129, 1], [3, 4, 9, 1, 0, 1]),           # rows without keys, requests without rows
    (8, 2, 128, 16, [500, 33, 17], [7, 8, 20]),                         # more rows than keys; 28 and 32 columns
    (28, 4, 128, 32, [1000, 129], [5, 2]),                              # 35 columns: a tile of 64
    (4, 4, 128, 64, [700, 64, 65, 63], [64, 64, 64, 64]),               # windows
    (2, 2, 80, 24, [333, 200], [130, 1]),                               # tiles of a long request, one row of a short one
    (4, 1, 256, 16, [260, 90], [40, 9]),
    (2, 1, 64, 8, [1025], [150]),
])
def test_several_rows(dtype, causal, H, Hkv, dh, P, lens, n):
    for width in (None, 300):
        Pool(lens, H, Hkv, dh, P, dtype, seed=dh, width=width, apart=16).rows(n).check(causal=causal, extra=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_and_ragged(dtype):
    """Requests that one worker takes many of and requests that many workers share, in one call."""
    lens = [9000, 1, 0, 4097, 128, 2000, 3, 700, 0, 12345]
    Pool(lens, 8, 2, 128, 16, dtype, seed=1).rows([1] * len(lens)).check()
    Pool(lens, 2, 2, 64, 64, dtype, seed=2, spread=4.0).rows([2, 1, 0, 3, 1, 1, 1, 5, 2, 1]).check(causal=True)
    Pool([20011], 4, 1, 80, 24, dtype, seed=3, spread=3.0).rows([1]).check()


def test_many_requests():
    """More requests than a wave has lanes, and than LDS has places for; items of one request spread over workers and of many in one."""
    lens = [(37 * b) % 301 for b in range(1300)]
    Pool(lens, 4, 2, 64, 16, "bf16", seed=4).rows([1] * 1300).check()
    n = [b % 3 for b in range(1300)]
    Pool(lens, 4, 2, 64, 16, "f32", seed=5, width=64).rows(n).check(causal=True)


# Requests x key heads of 128 rows (or 50, 64 columns): how triples are dealt to workers changes at 256 of them, at 7/8 of the workers and at all of them,
# with more than 64 requests, and where one request is much longer than the others.
@pytest.mark.parametrize("nreq,Hkv,n,dh,longest,causal", [
    (10, 30, 128, 128, 0, False), (10, 30, 128, 64, 0, True), (47, 10, 128, 64, 0, False), (75, 8, 128, 128, 0, True), (110, 10, 128, 64, 0, False), (70, 8, 50, 128, 0, True),
    (40, 7, 50, 64, 0, False), (130, 1, 128, 128, 0, True), (65, 4, 33, 72, 0, False), (9, 4, 128, 128, 9000, True), (70, 4, 128, 128, 9000, False), (66, 2, 64, 64, 5000, True),
    (1, 1, 128, 128, 30000, False), (1, 2, 50, 128, 20000, True), (3, 5, 300, 96, 3000, True), (40, 8, 100, 256, 0, False),
    (12, 8, 40, 256, 0, True), (6, 5, 128, 200, 4000, True), (3, 4, 33, 136, 5000, False), (300, 1, 20, 256, 0, True)])
def test_windows_dealt_to_workers(nreq, Hkv, n, dh, longest, causal):
    lens = [130 + (97 * b) % 331 for b in range(nreq)]
    rows = [n - (b % 5 == 3) * (b % 17) for b in range(nreq)]
    if longest:
        lens[nreq // 2] = longest
    pool = Pool(lens, Hkv, Hkv, dh, 16, "bf16", seed=nreq + n, width=max(80, -(-longest // 16)), spread=2.0).rows(rows)
    first = pool.check(causal=causal, extra=2)
    assert torch.equal(first, pool.run(causal=causal, extra=2))


@pytest.mark.parametrize("nreq,H,Hkv,n,dh", [(17, 12, 3, 5, 128), (3, 4, 1, 1, 80), (64, 8, 2, 2, 64), (65, 8, 2, 2, 64), (2, 6, 6, 40, 136), (5, 2, 2, 1, 256)])
def test_keys_divided_between_workers(nreq, H, Hkv, n, dh):
    """Lengths around what gives each worker one part, several, and parts that end inside another request."""
    for top in (700, 1411, 2600):
        lens = [top - (131 * b) % top for b in range(nreq)]
        Pool(lens, H, Hkv, dh, 24, "f32", seed=nreq + top, width=120).rows([n] * nreq).check(causal=top == 1411)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nreq,H,Hkv,n,dh", [(18, 8, 8, 1, 64), (40, 8, 8, 1, 64), (70, 8, 4, 1, 80), (130, 3, 3, 2, 64), (64, 8, 8, 1, 32), (30, 20, 10, 5, 128)])
def test_requests_of_like_lengths(dtype, nreq, H, Hkv, n, dh):
    """Whole triples, one a CU, and the others divided: 144 of them, 320, 280 of more than 64 requests, 390; 512, all divided; 300 of ten columns."""
    lens = [1100 - 7 * (b % 9) for b in range(nreq)]
    Pool(lens, H, Hkv, dh, 24, dtype, seed=nreq, width=100).rows([n] * nreq).check(causal=nreq % 4 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,n,width", [([300, 17, 90], 1, 20), ([5000, 17, 900], 1, 400), ([2000, 700, 5000], 40, 400)])
def test_results_in_place_of_the_queries(dtype, lens, n, width):
    pool = Pool(lens, 8, 2, 128, 16, dtype, seed=n, width=width).rows([n] * len(lens))
    want = pool.run()
    q, dev = pool.q.cuda(), pool.pool.cuda()
    k, v = (dev[:, i].view(dev.shape[0], 2, 16, 128) for i in (0, 1))
    B.page_attention(q, k, v, pool.table.cuda(), i32(lens), cu_rows=i32(pool.cu), out=q)
    assert torch.equal(q.cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales(dtype):
    for scale in (0.0, 0.7, -0.2, 3.0):
        Pool([300, 77], 4, 2, 64, 16, dtype, seed=6).rows([2, 1]).check(scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("odd", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dh", [64, 80, 128, 256])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_only(dtype, odd, dh):
    """A key's value is infinite or NaN: earlier rows of the same request are as if it were not there, later ones have it."""
    for at, length, n in ((290, 300, 16), (299, 300, 40), (260, 300, 41), (0, 20, 20), (31, 40, 25)):
        p = Pool([length, length], 4, 2, dh, 16, dtype, seed=7).rows([n, n])
        p.v[p.table[1, at // 16], 1, at % 16, dh // 2 + 1] = odd
        p.v[p.table[1, at // 16], 1, at % 16, 3] = odd
        got = p.check(causal=True)
        rows = got[n:, 2:, 3]
        sees = torch.arange(n) + length - n >= at
        assert bool((rows[sees].isfinite() == False).all()) and bool(rows[~sees].isfinite().all())  # noqa: E712


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("odd", [math.inf, -math.inf])
@pytest.mark.parametrize("n", [1, 12, 30])
def test_infinite_values_make_infinite_rows(dtype, odd, n):
    """Whatever the probability is: one (the key is the only one, or all keys are alike), or next to nothing."""
    for length in (1, 40, 300):
        p = Pool([length, length], 2, 1, 64, 16, dtype, seed=21).rows([n, n])
        if length == 40:
            p.k[:] = torch.where(p.k.isnan(), p.k, torch.ones_like(p.k))
        p.k[p.table[0, 0], 0, 0] = p.k[p.table[0, 0], 0, 0] * 4
        p.v[p.table[0, 0], 0, 0, 5] = odd
        assert bool((p.check()[:n, :, 5] == odd).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_that_are_not_finite(dtype):
    """NaN and infinite keys, seen and not seen: what softmax makes of them."""
    for odd in (math.nan, math.inf, -math.inf):
        p = Pool([100, 100], 2, 1, 64, 16, dtype, seed=8).rows([30, 30])
        p.k[p.table[1, 5], 0, 3, 7] = odd                                     # key 83, seen by rows 13 on
        p.q[:, :, 7] = p.q[:, :, 7].abs() + 0.5
        got = p.run(causal=True)
        keep = p.k.clone()
        p.k[p.table[1, 5], 0, 3, 7] = 0.25
        want, slack = R.attention(p.q, p.k, p.v, p.table, p.lens, p.cu, True, 64 ** -0.5)
        assert R.close(got[:43], want[:43], slack[:43])
        p.k = keep
        if odd == -math.inf:                                                  # the key has no part in any row
            assert bool(got[43:].isfinite().all())
        else:
            assert bool(got[43:].isnan().all())
    p = Pool([5], 2, 1, 64, 16, dtype, seed=9).rows([1])
    p.k[:] = torch.where(p.k.isnan(), p.k, torch.full_like(p.k, -math.inf))
    p.q.fill_(1.0)
    assert bool(p.run().isnan().all())                                        # keys, but none with a weight


def test_tables_that_name_no_page():
    """Entries outside the pool, and requests longer than their table: NaN in the rows that see such a token, no others."""
    for width in (20, 300):
        p = Pool([200, 200, 200, 200, 300], 4, 2, 64, 16, "bf16", seed=10, width=width).rows([1, 4, 4, 1, 1])
        p.table[0, 3] = -1
        p.table[1, 12] = 1 << 20                                              # tokens 192 ..: rows 0 .. see up to 197
        p.table[2, 13:] = -5                                                  # behind the last token
        p.lens[4] = 20 * 16 + 1 if width == 20 else 300 * 16 + 7
        got = p.check(causal=True)
        assert bool(got[0].isnan().all() and got[1:5].isnan().all()) and bool(got[5:10].isfinite().all()) and bool(got[10].isnan().all())


def test_rows_and_lengths_that_cannot_be():
    """Row offsets that run backwards or beyond M and negative lengths: nothing outside of out is touched, sound requests are right."""
    p = Pool([100, 100, 100], 4, 2, 64, 16, "bf16", seed=11).rows([2, 2, 2])
    q, k, v = p.q.cuda(), p.k.cuda(), p.v.cuda()
    buf = torch.full((10, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    want = p.run()
    B.page_attention(q, k, v, p.table.cuda(), i32([100, -5, 100]), cu_rows=i32([0, 2, 4, 900]), out=buf[2:8])
    got = buf.cpu()
    assert torch.equal(got[2:4], want[:2]) and torch.equal(got[6:8], want[4:]) and bool((got[4:6] == 0).all())
    B.page_attention(q, k, v, p.table.cuda(), i32([100, 100, 100]), cu_rows=i32([-7, 2, -3, 0]), out=buf[2:8])
    assert torch.equal(buf[:2].cpu(), got[:2]) and torch.equal(buf[4:].cpu(), got[4:]) and torch.equal(buf[2:4].cpu(), want[:2])


def test_strided_rows_and_unused_workspace():
    """q and out as parts of wider rows; a workspace of exactly the asked size between sentinels."""
    p = Pool([3000, 50], 8, 2, 128, 16, "bf16", seed=12).rows([2, 1])
    want = p.run()
    wide = torch.full((3, 16 * 128), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :1024] = p.q.cuda().view(3, 1024)
    out = wide[:, 1024:].view(3, 8, 128)
    k, v, table = p.k.cuda(), p.v.cuda(), p.table.cuda()
    need = B.page_attention_workspace(p.q.cuda(), k, table)
    assert need > 0
    ws = torch.full((need + 512,), 0xa5, dtype=torch.uint8, device="cuda")
    B.page_attention(wide[:, :1024].view(3, 8, 128), k, v, table, i32(p.lens), cu_rows=i32(p.cu), out=out, workspace=ws[256: 256 + need])
    assert torch.equal(out.cpu(), want) and bool((ws[:256] == 0xa5).all() and (ws[256 + need:] == 0xa5).all())
    assert torch.equal(wide[:, :1024].cpu().view(3, 8, 128), p.q)
    with pytest.raises(B.PvfError):
        B.page_attention(p.q.cuda(), k, v, table, i32(p.lens), cu_rows=i32(p.cu), workspace=ws[256: 256 + need - 16])


def test_caches_past_32_bits():
    """Pages more than 2^32 bytes and 2^31 elements apart: stores and reads of the last ones."""
    H, Hkv, dh, P = 4, 2, 64, 16
    apart = (1 << 30) + 64                                                    # elements
    pool = torch.zeros(3 * apart + 8192, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(pool, (4, Hkv, P, dh), (apart, P * dh, dh, 1))
    v = torch.as_strided(pool, (4, Hkv, P, dh), (apart, P * dh, dh, 1), 4096)
    g = torch.Generator().manual_seed(13)
    qkv = torch.randn(40, (H + 2 * Hkv) * dh, generator=g).to(torch.bfloat16).cuda()
    table = i32([[3, 0, 2]])
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    slot = table[0, (pos // P).long()] * P + pos % P
    q = B.page_store(qkv, pos, slot.int(), k, v, 1e4)
    x = R.rotate(qkv.cpu().double().view(40, 8, dh)[:, : H + Hkv], pos.cpu(), 1e4)
    assert R.close(k[3, :, 5].cpu(), x[5, H:], 8 * 2.0 ** -24 * 10 * torch.ones(Hkv, dh, dtype=torch.float64))
    got = B.page_attention(q, k, v, table, i32([40]), cu_rows=i32([0, 40]), causal=True)
    want, slack = R.attention(q.cpu(), k.cpu(), v.cpu(), table.cpu(), [40], [0, 40], True, dh ** -0.5)
    assert R.close(got, want, slack)
    last = B.page_attention(q[39:], k, v, table, i32([40]))
    assert R.close(last, want[39:], slack[39:])


def test_same_bits_every_time():
    p = Pool([5000, 300, 77], 8, 2, 128, 16, "bf16", seed=14).rows([1, 3, 2])
    first = p.run(causal=True)
    for fill in (0x00, 0xff):                                                # whatever the workspace held
        ws = torch.full((B.PAGE_WORKSPACE,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(p.run(causal=True, workspace=ws), first)


# ---------------------------------------------------------------- together
def rows_of(gen, n, wide, dtype):
    return torch.randn(n, wide, generator=gen).to(dtype).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_requests_served_together(dtype):
    """Prompts, single tokens, drafts that are taken back, a request that ends and a new one in its place: extend, store, attention and trim as a
    serving loop calls them; every step's pages against what each request has been given, and rows against attention over them."""
    H, Hkv, dh, P, W, n_pages, theta, nreq = 8, 2, 64, 16, 20, 60, 1e4, 5
    t = DT[dtype]
    g = torch.Generator().manual_seed(15)
    k, v = (torch.full((n_pages, Hkv, P, dh), math.nan, dtype=t, device="cuda") for _ in range(2))
    table = torch.full((nreq, W), -1, dtype=torch.int32, device="cuda")
    free, n_free, lens = torch.randperm(n_pages, generator=g).int().cuda(), i32([n_pages]), i32([0] * nreq)
    history = [torch.zeros(0, 2, 2 * Hkv, dh, dtype=torch.float64) for _ in range(nreq)]   # rotated k | v, and how far stored ones may be off
    steps = [[37, 5, 100, 1, 0], [1, 1, 1, 1, 1], [4, 4, 4, 0, 4], [1, 1, 1, 1, 1], [16, 0, 3, 200, 33], [1] * 5, [1] * 5]
    for step, n in enumerate(steps):
        M = sum(n) + 2                                                       # two padding rows
        lens, n_free, cu, admitted, place, pos, slot = B.page_extend(lens, i32(n), table, free, n_free, P, rows=M)
        assert admitted.cpu().tolist() == [1] * nreq
        qkv = rows_of(g, M, (H + 2 * Hkv) * dh, t)
        q = B.page_store(qkv, pos, slot, k, v, theta, q_out=torch.zeros(M, H, dh, dtype=t, device="cuda"))
        out = B.page_attention(q, k, v, table, lens, cu_rows=cu, causal=True)
        x = qkv.cpu().double().view(M, H + 2 * Hkv, dh)
        turned = R.rotate(x[:, : H + Hkv], pos.cpu(), theta)
        size = x[:, : H + Hkv].unflatten(2, (2, dh // 2)).abs().sum(2).repeat(1, 1, 2)
        at = cu.cpu().tolist()
        assert R.close(q[: at[-1]].cpu(), turned[: at[-1], :H], 8 * 2.0 ** -24 * size[: at[-1], :H]) and not q[at[-1]:].any()
        rows = torch.cat([turned[:, H:], x[:, H + Hkv:]], 1)
        off = torch.cat([8 * 2.0 ** -24 * size[:, H:], torch.zeros(M, Hkv, dh, dtype=torch.float64)], 1)
        kc, vc, tab = k.cpu(), v.cpu(), table.cpu()
        for b in range(nreq):                                                # what lies in the pages is what the request has been given, step after step
            history[b] = torch.cat([history[b], torch.stack([rows, off], 1)[at[b]: at[b + 1]]])
            page = tab[b, : R.pages_of(len(history[b]), P)].long()
            held = torch.cat([c[page].transpose(1, 2).reshape(-1, Hkv, dh) for c in (kc, vc)], 1)[: len(history[b])]
            assert R.close(held, history[b][:, 0], history[b][:, 1])
        assert lens.cpu().tolist() == [len(h) for h in history]
        want, slack = R.attention(q.cpu(), kc, vc, tab, lens.cpu(), at, True, dh ** -0.5)
        assert R.close(out[: at[-1]], want[: at[-1]], slack[: at[-1]])
        drop = [0, 0, 0, 0, 0] if step != 2 else [3, 4, 1, 0, 4]
        if step == 3:
            drop = [0, 10 ** 6, 0, 0, 0]                                      # request 1 ends
        keep = [max(0, len(h) - d) for h, d in zip(history, drop)]
        lens, n_free, place = B.page_trim(lens, i32(keep), table, free, n_free, P)
        history = [h[:x] for h, x in zip(history, keep)]
        used = sum(R.pages_of(x, P) for x in keep)
        assert n_free.item() == n_pages - used
        owned = [p for b in range(nreq) for p in table[b].cpu().tolist()[: R.pages_of(keep[b], P)]]
        assert sorted(owned + free.cpu().tolist()[: n_pages - used]) == list(range(n_pages))


def test_windows_over_shared_canvases():
    """Windows of a round of cached decoding: the backbone's canvas is in pages, drafts share them but for the pages of their window; all rows of a window
    see the whole canvas.  Against the attention of dense copies."""
    H, Hkv, dh, P, T, R_, K = 4, 4, 128, 64, 512, 64, 3
    g = torch.Generator().manual_seed(16)
    n_pages = 8 + K + 1
    k, v = (torch.zeros(n_pages, Hkv, P, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens, n_free, free = i32([0] * (1 + K)), i32([n_pages]), torch.arange(n_pages, dtype=torch.int32, device="cuda")
    table = torch.full((1 + K, 8), -1, dtype=torch.int32, device="cuda")
    lens, n_free, cu, _, _, pos, slot = B.page_extend(lens, i32([T] + [0] * K), table, free, n_free, P, rows=T)
    full = rows_of(g, T, 3 * H * dh, torch.bfloat16)
    B.page_store(full, pos, slot, k, v, 1e4)
    table[1:] = table[0]
    at = 5                                                                    # the window is page 5 of the canvas
    table[1:, at] = free[n_free.item() - K: n_free.item()]
    lens = i32([T] * (1 + K))
    M = (1 + K) * R_
    lens, n_free, cu, ok, _, pos, slot = B.page_extend(lens, i32([R_] * (1 + K)), table, free, n_free, P, start=i32([at * P] * (1 + K)), rows=M)
    assert ok.cpu().tolist() == [1] * (1 + K) and lens.cpu().tolist() == [T] * (1 + K)
    assert pos.cpu().tolist() == list(range(at * P, at * P + R_)) * (1 + K)
    win = rows_of(g, M, 3 * H * dh, torch.bfloat16)
    q = B.page_store(win, pos, slot, k, v, 1e4)
    got = B.page_attention(q, k, v, table, lens, cu_rows=cu)
    want, slack = R.attention(q.cpu(), k.cpu(), v.cpu(), table.cpu(), [T] * (1 + K), cu.cpu().tolist(), False, dh ** -0.5)
    assert R.close(got, want, slack)
    x = R.rotate(win.cpu().double().view(M, 3 * H, dh)[:, : 2 * H], pos.cpu(), 1e4)
    near = torch.full((H, R_, dh), 8 * 2.0 ** -24 * 12, dtype=torch.float64)
    for j in range(1 + K):
        assert R.close(k[table[j, at].long()].cpu(), x[j * R_: (j + 1) * R_, H:].transpose(0, 1), near)


# ---------------------------------------------------------------- streams, graphs, devices
def loop_state(nreq=3, seed=17):
    H, Hkv, dh, P, W = 4, 2, 64, 16, 300
    g = torch.Generator().manual_seed(seed)
    lens = [200, 31, 1000][:nreq]
    p = Pool(lens, H, Hkv, dh, P, "bf16", seed=seed, width=W, spare=40)
    used = set(p.table[p.table >= 0].tolist())
    rest = [x for x in range(p.k.shape[0]) if x not in used]
    dev = p.pool.cuda()
    k, v = (dev[:, i].view(-1, Hkv, P, dh) for i in (0, 1))
    return dict(k=k, v=v, table=p.table.cuda(), lens=i32(lens), n=i32([1] * nreq), free=i32(rest), n_free=i32([len(rest)]), qkv=rows_of(g, nreq, (H + 2 * Hkv) * dh, torch.bfloat16),
                outs=(i32([0] * (nreq + 1)), i32([0] * nreq), i32([0] * (nreq + 1)), i32([0] * nreq), i32([0] * nreq)), q=torch.zeros(nreq, H, dh, dtype=torch.bfloat16, device="cuda"),
                out=torch.zeros(nreq, H, dh, dtype=torch.bfloat16, device="cuda"), ws=torch.empty(B.PAGE_WORKSPACE, dtype=torch.uint8, device="cuda"))


def one_step(s):
    cu, admitted, place, pos, slot = s["outs"]
    B.page_extend(s["lens"], s["n"], s["table"], s["free"], s["n_free"], 16, out=(s["lens"], s["n_free"], cu, admitted, place, pos, slot))
    B.page_store(s["qkv"], pos, slot, s["k"], s["v"], 1e4, q_out=s["q"])
    B.page_attention(s["q"], s["k"], s["v"], s["table"], s["lens"], cu_rows=cu, causal=True, out=s["out"], workspace=s["ws"])


def test_steps_replayed_from_a_graph_are_eager_steps():
    """A whole step, lengths and free list updated in place, captured once and replayed: every replay has the eager step's bits.  Two graphs share
    the workspace."""
    eager, a, b = loop_state(), loop_state(), loop_state(seed=18)
    other = loop_state(seed=18)
    graphs = []
    for s in (a, b):
        s["ws"] = a["ws"]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            one_step(s)
        graphs.append(g)
    for step in range(20):
        for s in (eager, other):
            s["qkv"].copy_(torch.randn(s["qkv"].shape, generator=torch.Generator().manual_seed(step)).to(torch.bfloat16))
            one_step(s)
        for s, g, e in ((a, graphs[0], eager), (b, graphs[1], other)):
            s["qkv"].copy_(e["qkv"])
            g.replay()
        for s, e in ((a, eager), (b, other)):
            assert torch.equal(s["out"], e["out"]) and torch.equal(s["lens"], e["lens"]) and torch.equal(s["n_free"], e["n_free"])
            assert torch.equal(s["table"], e["table"])
        torch.cuda.synchronize()
    assert bool(eager["out"].isfinite().all()) and eager["lens"].cpu().tolist() == [220, 51, 1020]


def test_calls_on_two_streams_at_once():
    """Steps of two loops on streams of their own, enqueued in turn: each as alone."""
    alone, both = [loop_state(seed=s) for s in (19, 20)], [loop_state(seed=s) for s in (19, 20)]
    for s in alone:
        for _ in range(10):
            one_step(s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for s, st in zip(both, streams):
            with torch.cuda.stream(st):
                one_step(s)
    torch.cuda.synchronize()
    for x, y in zip(alone, both):
        assert torch.equal(x["out"], y["out"]) and torch.equal(x["lens"], y["lens"])
