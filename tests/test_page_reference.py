"""The references of tests/page_reference.py against counting, dense attention and complex rotations (CPU), and the refusals of the page calls."""
import ctypes
import math

import pytest
import torch

from paper_2601_12247_amd import binding as B
from tests import page_reference as R


def test_pages_given_and_taken_balance():
    """Extend and trim in turn: every page has one owner at any time, tables name the pages that lengths say."""
    g = torch.Generator().manual_seed(3)
    P, W, n_pages, nreq = 4, 6, 30, 7
    free, n_free = list(range(n_pages)), n_pages
    table, lens = [[-1] * W for _ in range(nreq)], [0] * nreq
    for step in range(60):
        n = torch.randint(0, 9, (nreq,), generator=g).tolist()
        r = R.extend(lens, n, table, free, n_free, P, M=200)
        for b in range(nreq):
            fits = lens[b] + n[b] <= W * P
            assert not r["admitted"][b] or fits
            assert r["seq_len"][b] == lens[b] + (n[b] if r["admitted"][b] else 0)
            rows = range(r["cu_rows"][b], r["cu_rows"][b + 1])
            assert len(rows) == n[b]
            for t, m in enumerate(rows):
                assert r["pos"][m] == lens[b] + t
                assert (r["slot"][m] >= 0) == bool(r["admitted"][b])
                if r["admitted"][b]:
                    assert r["slot"][m] == r["table"][b][r["pos"][m] // P] * P + r["pos"][m] % P
        table, lens, n_free = r["table"], r["seq_len"], r["n_free"]
        owned = [p for b in range(nreq) for p in table[b][: R.pages_of(lens[b], P)]]
        assert sorted(owned + free[:n_free]) == list(range(n_pages))
        keep = [max(0, x - int(torch.randint(0, 7, (1,), generator=g))) for x in lens]
        r = R.trim(lens, keep, table, free, n_free, P)
        lens, free, n_free = r["seq_len"], r["free"], r["n_free"]
        owned = [p for b in range(nreq) for p in table[b][: R.pages_of(lens[b], P)]]
        assert lens == keep and sorted(owned + free[:n_free]) == list(range(n_pages))


def test_attention_over_pages_is_dense_attention():
    g = torch.Generator().manual_seed(1)
    H, Hkv, dh, P, T = 6, 2, 16, 8, 37
    k, v = torch.randn(T, Hkv, dh, generator=g), torch.randn(T, Hkv, dh, generator=g)
    q = torch.randn(5, H, dh, generator=g)
    kc, vc = torch.full((7, Hkv, P, dh), math.nan), torch.full((7, Hkv, P, dh), math.nan)
    table = torch.tensor([[6, 1, 4, 0, 3]])
    for t in range(T):
        kc[table[0, t // P], :, t % P], vc[table[0, t // P], :, t % P] = k[t], v[t]
    for causal in (False, True):
        got, _ = R.attention(q, kc, vc, table, [T], [0, 5], causal, 0.3)
        kk, vv = (x.double().repeat_interleave(H // Hkv, 1).transpose(0, 1) for x in (k, v))
        s = q.double().transpose(0, 1) @ kk.transpose(1, 2) * 0.3
        if causal:
            s = s.masked_fill(torch.arange(T)[None, :] > torch.arange(T - 5, T)[:, None], -math.inf)
        want = (torch.softmax(s, -1) @ vv).transpose(0, 1)
        assert torch.allclose(got, want, rtol=1e-12, atol=1e-12)


def test_rotation_keeps_lengths_and_distances():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(1, 3, 16, generator=g, dtype=torch.float64)
    at = lambda p: R.rotate(x, torch.tensor([p]), 1e4)  # noqa: E731
    assert torch.allclose(at(12345).norm(dim=2), x.norm(dim=2))
    assert torch.allclose(at(0), x)
    assert torch.allclose((at(100)[0, 0] * at(107)[0, 1]).sum(), (at(1000)[0, 0] * at(1007)[0, 1]).sum())


# ---------------------------------------------------------------- refusals: nothing is launched
A = 4096   # stands for a tensor: these calls return before they read anything


def _extend(**kw):
    a = dict(stream=None, seq_len=A, start=None, n_rows=A, B=3, table=A, width=5, table_stride=5, page_size=16, free_pages=A, free_cap=9, n_free=A, M=7,
             seq_len_out=A, n_free_out=A, cu_rows=A, admitted=A, place=A, pos=A, slot=A)
    assert set(kw) <= set(a)
    return B.lib().pvf_page_extend(*{**a, **kw}.values())


def _trim(**kw):
    a = dict(stream=None, seq_len=A, keep=A, B=3, table=A, width=5, table_stride=5, page_size=16, free_pages=A, free_cap=9, n_free=A, seq_len_out=A,
             n_free_out=A, place=A)
    assert set(kw) <= set(a)
    return B.lib().pvf_page_trim(*{**a, **kw}.values())


def _store(**kw):
    a = dict(stream=None, dtype=1, qkv=A, qkv_stride=512, pos=A, slot=A, M=3, H=4, Hkv=2, d_head=64, rope_theta=1e4, q_out=A, q_stride=256, k_cache=A,
             v_cache=A, n_pages=4, page_size=16, k_page_stride=2048, v_page_stride=2048)
    assert set(kw) <= set(a)
    return B.lib().pvf_page_store(*{**a, **kw}.values())


def _attention(**kw):
    a = dict(stream=None, dtype=1, q=A, q_stride=256, k_cache=A, v_cache=A, n_pages=4, page_size=16, k_page_stride=2048, v_page_stride=2048, table=A, width=500,
             table_stride=500, seq_len=A, cu_rows=A, B=2, M=3, H=4, Hkv=2, d_head=64, causal=0, scale=1.0, out=A, out_stride=256, workspace=A,
             workspace_bytes=1 << 26)
    assert set(kw) <= set(a)
    return B.lib().pvf_page_attention(*{**a, **kw}.values())


EINVAL, ESHAPE, ENOTIMPL = -1, -2, -5


@pytest.mark.parametrize("status,kw", [
    *[(EINVAL, {name: None}) for name in ("seq_len", "n_rows", "table", "free_pages", "n_free", "seq_len_out", "n_free_out", "cu_rows", "admitted", "place", "pos", "slot")],
    (EINVAL, {"B": -1}), (EINVAL, {"width": -1}), (EINVAL, {"page_size": 0}), (EINVAL, {"table_stride": 4}), (EINVAL, {"M": -1}), (EINVAL, {"free_cap": -1}),
    (EINVAL, {"start": A + 2}), (EINVAL, {"slot": A + 1}),
    (ESHAPE, {"B": (1 << 20) + 1}), (ESHAPE, {"width": 1 << 27, "table_stride": 1 << 27}), (ESHAPE, {"M": (1 << 24) + 1}),
])
def test_extend_refuses(status, kw):
    assert _extend(**kw) == status and b"pvf_page_extend" in B.lib().pvf_last_error(None)


@pytest.mark.parametrize("status,kw", [
    *[(EINVAL, {name: None}) for name in ("seq_len", "keep", "table", "free_pages", "n_free", "seq_len_out", "n_free_out", "place")],
    (EINVAL, {"B": -1}), (EINVAL, {"page_size": -3}), (EINVAL, {"table_stride": 4}), (EINVAL, {"free_cap": -1}), (EINVAL, {"keep": A + 2}),
    (ESHAPE, {"B": (1 << 20) + 1}), (ESHAPE, {"page_size": 1 << 29}), (ESHAPE, {"width": (1 << 24) + 1, "table_stride": 1 << 25, "page_size": 1}),
])
def test_trim_refuses(status, kw):
    assert _trim(**kw) == status and b"pvf_page_trim" in B.lib().pvf_last_error(None)


@pytest.mark.parametrize("status,kw", [
    *[(EINVAL, {name: None}) for name in ("qkv", "pos", "slot", "q_out", "k_cache", "v_cache")],
    *[(EINVAL, {name: A + 8}) for name in ("qkv", "q_out", "k_cache", "v_cache")],
    (EINVAL, {"pos": A + 2}), (EINVAL, {"M": -1}), (EINVAL, {"H": -1}), (EINVAL, {"Hkv": 0}), (EINVAL, {"d_head": 0}), (EINVAL, {"n_pages": -1}),
    (EINVAL, {"dtype": 2}), (EINVAL, {"rope_theta": 0.0}), (EINVAL, {"rope_theta": math.inf}), (EINVAL, {"rope_theta": math.nan}),
    (EINVAL, {"qkv_stride": 504}), (EINVAL, {"qkv_stride": 516}), (EINVAL, {"q_stride": 252}), (EINVAL, {"k_page_stride": 2040}), (EINVAL, {"v_page_stride": 2050}),
    (ENOTIMPL, {"d_head": 60}), (ENOTIMPL, {"d_head": 264}), (ENOTIMPL, {"page_size": 12}), (ENOTIMPL, {"page_size": 65544}),
    (ESHAPE, {"M": (1 << 24) + 1}), (ESHAPE, {"H": 5000}), (ESHAPE, {"n_pages": 1 << 28}), (ESHAPE, {"M": 1 << 22, "H": 1 << 9}),
])
def test_store_refuses(status, kw):
    assert _store(**kw) == status and (b"pvf_page_store" in B.lib().pvf_last_error(None) or "dtype" in kw)


@pytest.mark.parametrize("status,kw", [
    *[(EINVAL, {name: None}) for name in ("q", "k_cache", "v_cache", "table", "seq_len", "out")],
    *[(EINVAL, {name: A + 8}) for name in ("q", "k_cache", "v_cache", "out")],
    (EINVAL, {"table": A + 2}), (EINVAL, {"seq_len": A + 1}), (EINVAL, {"cu_rows": A + 3}), (EINVAL, {"cu_rows": None}), (EINVAL, {"dtype": -1}),
    (EINVAL, {"H": 5}), (EINVAL, {"H": 0}), (EINVAL, {"Hkv": 0}), (EINVAL, {"causal": 2}), (EINVAL, {"scale": math.nan}), (EINVAL, {"scale": math.inf}),
    (EINVAL, {"n_pages": 0}), (EINVAL, {"q_stride": 248}), (EINVAL, {"out_stride": 260}), (EINVAL, {"k_page_stride": 2040}), (EINVAL, {"table_stride": 499}),
    (ENOTIMPL, {"d_head": 65}), (ENOTIMPL, {"d_head": 512}), (ENOTIMPL, {"page_size": 4}),
    (ESHAPE, {"workspace": None}), (ESHAPE, {"workspace": A + 8}), (ESHAPE, {"workspace_bytes": 1000}), (ESHAPE, {"width": 1 << 27, "table_stride": 1 << 27}),
    (ESHAPE, {"B": (1 << 20) + 1}), (ESHAPE, {"M": 1 << 25}),
])
def test_attention_refuses(status, kw):
    assert _attention(**kw) == status and (b"pvf_page_attention" in B.lib().pvf_last_error(None) or "dtype" in kw)


def test_workspace_is_bounded():
    """Every instance and a range of sizes: what a call wants is below PVF_PAGE_WORKSPACE; refused sizes give a negative status."""
    L = B.lib()
    for dtype in (0, 1):
        for dh in (8, 64, 72, 128, 136, 256):
            for H, Hkv in ((1, 1), (32, 8), (32, 1), (64, 64)):
                for nreq, rows in ((1, 1), (1, 100), (64, 1), (9, 128), (1000, 3)):
                    for width in (1, 33, 70000):
                        n = L.pvf_page_attention_workspace(dtype, nreq, nreq * rows, H, Hkv, dh, width, 64)
                        assert 0 <= n <= B.PAGE_WORKSPACE and n % 4 == 0
    assert L.pvf_page_attention_workspace(1, 1, 1, 32, 8, 128, 2, 16) == 0           # too short to be divided
    assert L.pvf_page_attention_workspace(1, 1, 1, 5, 2, 128, 2, 16) == EINVAL
    assert L.pvf_page_attention_workspace(1, 1, 1, 4, 2, 100, 2, 16) == ENOTIMPL


def test_binding_refuses_tensors_that_do_not_fit():
    """Shapes and types that the C call cannot see."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    kv = torch.zeros(4, 2, 16, 64)
    with pytest.raises(AssertionError):
        B.page_attention(torch.zeros(3, 4, 64), kv, kv, i32(3, 5), i32(3))                                  # not on a device
    for bad in (dict(q=torch.zeros(3, 4, 32)), dict(v=torch.zeros(4, 2, 8, 64)), dict(k=kv.transpose(1, 2)), dict(table=i32(2, 5)),
                dict(q=torch.zeros(3, 4, 128)[:, :, ::2]), dict(table=torch.zeros(3, 5, dtype=torch.int64)), dict(lens=torch.zeros(3))):
        a = dict(q=torch.zeros(3, 4, 64), k=kv, v=kv, table=i32(3, 5), lens=i32(3))
        a.update(bad)
        with pytest.raises((AssertionError, TypeError)):
            B.page_attention(*a.values())
    with pytest.raises(AssertionError):
        B.page_store(torch.zeros(3, 500), i32(3), i32(3), kv, kv, 1e4)                                      # not whole heads
    with pytest.raises(AssertionError):
        B.page_store(torch.zeros(3, 512), i32(2), i32(3), kv, kv, 1e4)
    with pytest.raises(AssertionError):
        B.page_extend(i32(3), i32(3), i32(3, 5), i32(9), i32(1), 16)                                        # neither rows nor out
    with pytest.raises(AssertionError):
        B.page_trim(i32(3), i32(4), i32(3, 5), i32(9), i32(1), 16)
    assert ctypes.sizeof(ctypes.c_int64) == 8
