"""Plain references of the paged K/V cache (pvf_page_extend, pvf_page_trim, pvf_page_store, pvf_page_attention), written from include/pvf.h: whole
numbers request by request, rows in float64, on the CPU.  tests/test_page_reference.py checks them against counting and dense attention."""
from __future__ import annotations

import math

import torch


def pages_of(tokens: int, P: int) -> int:
    return -(-tokens // P)


def extend(seq_len, n_rows, table, free, n_free, P, M, start=None):
    """Lists in, a dict of lists out; `table` is a list of lists that is not changed."""
    B, W = len(seq_len), len(table[0]) if table else 0
    table, top = [list(t) for t in table], min(max(n_free, 0), len(free))
    out = dict(seq_len=list(seq_len), cu_rows=[0], admitted=[], place=[top], pos=[], slot=[])
    rows = asked = 0
    left = top
    for b in range(B):
        n, length = n_rows[b], seq_len[b]
        first = length if start is None else start[b]
        rows += max(n, 0)
        sound = n >= 0 and 0 <= first <= length <= W * P and max(length, first + n) <= W * P and rows <= M
        need = 0
        if sound:
            need = pages_of(max(length, first + n), P) - pages_of(length, P)
            asked += need
        ok = sound and (need == 0 or asked <= top)
        if ok:
            for j in range(need):
                left -= 1
                table[b][pages_of(length, P) + j] = free[left]
            out["seq_len"][b] = max(length, first + n)
        out["admitted"].append(int(ok))
        out["place"].append(left)
        for p in range(first, first + max(n, 0)):
            if len(out["pos"]) < M:
                page = table[b][p // P] if ok else -1
                out["pos"].append(p)
                out["slot"].append(page * P + p % P if 0 <= page * P + p % P < 2 ** 31 and page >= 0 else -1)   # slots are 31 bits
        out["cu_rows"].append(min(rows, M))
    out["pos"] += [0] * (M - len(out["pos"]))
    out["slot"] += [-1] * (M - len(out["slot"]))
    out.update(table=table, n_free=left)
    return out


def trim(seq_len, keep, table, free, n_free, P):
    W, cap = len(table[0]) if table else 0, len(free)
    free, top = list(free), min(max(n_free, 0), len(free))
    out = dict(seq_len=[], place=[top])
    for b, (length, kept) in enumerate(zip(seq_len, keep)):
        length = min(max(length, 0), W * P)
        kept = min(max(kept, 0), length)
        for page in table[b][pages_of(kept, P): pages_of(length, P)]:
            if top < cap:
                free[top] = page
                top += 1
        out["seq_len"].append(kept)
        out["place"].append(top)
    out.update(free=free, n_free=top)
    return out


def rotate(x, pos, theta):
    """x [M, heads, dh] in float64, rotated to positions pos."""
    half = x.shape[2] // 2
    angle = pos.double()[:, None, None] * theta ** (-2.0 * torch.arange(half, dtype=torch.float64) / x.shape[2])
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)


def attention(q, k_cache, v_cache, table, seq_len, cu_rows, causal, scale):
    """(out, slack) in float64: the rows of q that belong to a request, NaN elsewhere; |error| of float32 arithmetic on float32 scores is at most slack
    (below).  All tensors on the CPU.

    slack: a score is a sum of d_head products in float32, off by at most d_head 2^-24 sum |q k| however it is ordered, times the scale; scaling, the
    subtraction of the maximum and the rounding of scale log2(e) add four roundings of at most the largest score; 2^x is good to 2^-22 of itself, and a
    probability in two bf16 parts to 2^-15.  That error of every p, in the sum over v and in the sum of p, and one rounding of each of at most
    len + 16 additions in both, counts against sum p |v|."""
    M, H, dh = q.shape
    Hkv, P = k_cache.shape[1], k_cache.shape[2]
    group, W = H // Hkv, table.shape[1]
    out = torch.full((M, H, dh), math.nan, dtype=torch.float64)
    slack = torch.zeros(M, H, dh, dtype=torch.float64)
    for b in range(len(seq_len)):
        length, r0, r1 = int(seq_len[b]), int(cu_rows[b]), int(cu_rows[b + 1])
        for r in range(r0, r1):
            sees = length - (r1 - r0) + (r - r0) + 1 if causal else length
            if sees <= 0:
                out[r] = 0
                continue
            page = table[b, : pages_of(sees, P)].long()
            if sees > W * P or bool((page < 0).any()) or bool((page >= k_cache.shape[0]).any()):
                continue                                                  # NaN
            k = k_cache[page].double().transpose(1, 2).reshape(-1, Hkv, dh)[:sees]
            v = v_cache[page].double().transpose(1, 2).reshape(-1, Hkv, dh)[:sees]
            qr = q[r].double().view(Hkv, group, dh)
            s = torch.einsum("hgd,khd->hgk", qr, k) * scale
            p = torch.softmax(s, 2)
            out[r] = torch.einsum("hgk,khd->hgd", p, v).reshape(H, dh)
            size = torch.einsum("hgd,khd->hgk", qr.abs(), k.abs()).amax(2, keepdim=True) * abs(scale)
            off = dh * 2.0 ** -24 * size + 4 * 2.0 ** -24 * s.abs().amax(2, keepdim=True) + 2.0 ** -22 + (2.0 ** -15 if q.dtype is torch.bfloat16 else 0)
            slack[r] = ((2 * off + 2 * (sees + 16) * 2.0 ** -24) * torch.einsum("hgk,khd->hgd", p, v.abs())).reshape(H, dh)
    return out, slack


HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def close(got, want, slack):
    """Whether got is want within slack and half a step of its own type, with NaN and infinities in the same places."""
    g, half = got.double().cpu(), HALF_STEP[got.dtype]
    same = (g == want) | (g.isnan() & want.isnan())
    near = (g - want).abs() <= half * want.abs() + (1 + half) * slack
    return bool((same | near).all())
