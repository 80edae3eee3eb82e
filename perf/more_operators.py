"""Cases of the paged K/V cache: keys and values of requests of different lengths in pages of one pool, page tables on the GPU.

extend     pages for the rows that requests are about to add: tables, positions and slots of the rows
trim       pages behind the tokens that requests keep, back to the free list
store      rotary embedding of fresh q and k, keys and values into their slots
attention  rows of each request against the keys and values in its pages

A cache is [pages, kv heads, tokens a page, d_head]; the slot of a token is page * tokens a page + place.  Sizes are those of the
LLaDA-8B-shaped model of the benchmark (32 heads of 128, canvases of 512 and 1280 tokens, windows of 64 and 128 rows), of the small
float32 model (4 heads of 64), of such models with grouped heads, and odd ones.
"""
import math

import torch

own = False

THETA = 500000.0
WORKSPACE = 1 << 26                                 # bytes that suffice for any attention call


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one row of the small float32 model over a canvas of 128 tokens: latency
        {"name": "attn_1x1x128_f32", "op": "attention", "B": 1, "rows": 1, "len": 128, "H": 4, "Hkv": 4, "dh": 64, "page": 16,
         "ragged": False, "causal": False, "dtype": "f32"},
        # a single request with a long history: all of the chip has to read one cache
        {"name": "attn_1x1x32768", "op": "attention", "B": 1, "rows": 1, "len": 32768, "H": 32, "Hkv": 8, "dh": 128, "page": 64,
         "ragged": False, "causal": True, "dtype": "bf16"},
        # 64 requests of 1 to 8192 tokens, one new token each: a serving step
        {"name": "attn_64x1x8192", "op": "attention", "B": 64, "rows": 1, "len": 8192, "H": 32, "Hkv": 8, "dh": 128, "page": 16,
         "ragged": True, "causal": True, "dtype": "bf16"},
        # windows of a planned round: nine canvases of 1280 tokens, 128 rows each, every row sees its whole canvas
        {"name": "attn_9x128x1280", "op": "attention", "B": 9, "rows": 128, "len": 1280, "H": 32, "Hkv": 32, "dh": 128, "page": 64,
         "ragged": False, "causal": False, "dtype": "bf16"},
        # a few rows at once of requests of any length, odd heads and pages, float32
        {"name": "attn_17x5x1411_f32", "op": "attention", "B": 17, "rows": 5, "len": 1411, "H": 12, "Hkv": 3, "dh": 80, "page": 24,
         "ragged": True, "causal": True, "dtype": "f32"},
        # one new token: latency
        {"name": "store_1", "op": "store", "M": 1, "H": 32, "Hkv": 8, "dh": 128, "page": 16, "dtype": "bf16"},
        # nine canvases of 1280 tokens enter the cache
        {"name": "store_11520", "op": "store", "M": 11520, "H": 32, "Hkv": 32, "dh": 128, "page": 64, "dtype": "bf16"},
        # odd heads and pages, float32
        {"name": "store_437_f32", "op": "store", "M": 437, "H": 12, "Hkv": 3, "dh": 80, "page": 24, "dtype": "f32"},
        # 64 requests go on by one token each
        {"name": "extend_64x1", "op": "extend", "B": 64, "rows": 1, "len": 8192, "page": 16},
        # 512 prompts of 1 to 1024 tokens enter the pool
        {"name": "extend_512x1024", "op": "extend", "B": 512, "rows": 1024, "len": 0, "page": 16},
        # 64 requests drop up to five rejected tokens
        {"name": "trim_64x5", "op": "trim", "B": 64, "drop": 5, "len": 8192, "page": 16},
        # 4096 requests of up to 8192 tokens give back up to all of them
        {"name": "trim_4096x8192", "op": "trim", "B": 4096, "drop": 8192, "len": 8192, "page": 16},
    ]


def _spread(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "store", "store", "extend", "trim"))
    page = rng.choice((8, 16, 16, 24, 32, 64, 128))
    case = {"op": op, "page": page}
    if op == "extend":
        case["B"] = _spread(rng, 1, 1024)
        case["rows"] = _spread(rng, 1, 1024 * 512 // max(case["B"], 512))
        case["len"] = rng.choice((0, _spread(rng, 1, 8192)))
        return case
    if op == "trim":
        case.update(B=_spread(rng, 1, 4096), len=_spread(rng, 16, 8192))
        case["drop"] = _spread(rng, 1, case["len"])
        return case
    Hkv = rng.choice((1, 2, 3, 4, 8, 8, 16, 32))
    case.update(Hkv=Hkv, H=Hkv * rng.choice([g for g in (1, 1, 2, 4, 7, 8) if g * Hkv <= 64]), dh=rng.choice((64, 128, 128, 128, 80, 96, 256)),
                dtype=rng.choice(("bf16", "bf16", "f32")))
    size = 4 if case["dtype"] == "f32" else 2
    if op == "store":
        most = 11520 * 96 * 128 * 2 // ((case["H"] + 2 * Hkv) * case["dh"] * size)
        case["M"] = _spread(rng, 1, min(most, 65536))
        return case
    rows = rng.choice((1, 1, 1, _spread(rng, 2, 16), _spread(rng, 17, 128)))
    wide = rows * case["H"] * case["dh"]
    case.update(B=_spread(rng, 1, max(1, min(256, 9 * 128 * 4096 // wide))), rows=rows, ragged=rng.random() < 0.7, causal=rng.random() < 0.6)
    most = min(500_000_000 // (case["B"] * Hkv * case["dh"] * size), 9 * 128 * 4096 * 1280 // (case["B"] * wide))
    case["len"] = max(rows, _spread(rng, 16, max(17, min(65536, most))))
    return case


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _sizes(n, most, least):
    """n whole numbers from least to most, evenly spread and in no order, the same ones every time."""
    return [least + int((0.381966 + 0.618034 * b) % 1.0 * (most - least + 1)) for b in range(n)]


def _lengths(case):
    """Tokens and rows of each request of an attention case."""
    B, most, rows = case["B"], case["len"], case["rows"]
    if not case["ragged"]:
        return [most] * B, [rows] * B
    n = _sizes(B, rows, 1)[::-1]
    return [max(length, r) for length, r in zip(_sizes(B, most, 1), n)], n


def _pages(tokens, page):
    return (tokens + page - 1) // page


# ---------------------------------------------------------------- inputs
def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _tables(lens, width, page, pool, gen):
    """Tables with the pages of `lens` tokens each, in no order, and what is left of a pool of that many pages."""
    order = torch.randperm(pool, device="cuda", generator=gen).int()
    n = torch.tensor([_pages(x, page) for x in lens], device="cuda")
    before = n.cumsum(0) - n
    j = torch.arange(width, device="cuda")
    taken = j[None, :] < n[:, None]
    table = torch.where(taken, order[torch.where(taken, before[:, None] + j, 0)], -1).int()
    return table, order[int(n.sum()):]


def prepare(case, seed):
    """Rows, pool, tables and free list in GPU memory, and the buffers that a serving loop keeps for its results."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, P, state = case["op"], case["page"], dict(case)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen, dtype=_type(case))  # noqa: E731
    if op in ("extend", "trim"):
        B = case["B"]
        lens = _sizes(B, case["len"], min(case["len"], 1))
        add = _sizes(B, case.get("rows", 0), min(case.get("rows", 0), 1))[::-1]
        width = _pages(max(a + b for a, b in zip(lens, add)), P)
        pool = sum(_pages(a + b, P) for a, b in zip(lens, add)) + 64
        table, left = _tables(lens, width, P, pool, gen)
        state.update(table=table, seq_len=_i32(lens), n_free=_i32([left.numel()]), new_len=_i32([0] * B), new_free=_i32([0]), place=_i32([0] * (B + 1)))
        state["free"] = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
        state["free"][: left.numel()] = left
        if op == "trim":
            drop = torch.randint(0, case["drop"] + 1, (B,), device="cuda", generator=gen)
            state["keep"] = (state["seq_len"] - drop).clamp(min=0).int()
            return state
        state.update(n_rows=_i32(add), M=sum(add), cu=_i32([0] * (B + 1)), admitted=_i32([0] * B))
        state.update(pos=_i32([0] * state["M"]), slot=_i32([0] * state["M"]))
        return state
    H, Hkv, dh = case["H"], case["Hkv"], case["dh"]
    if op == "store":
        M = case["M"]
        pool = _pages(M, P) + 1
        state.update(qkv=normal(M, (H + 2 * Hkv) * dh), k=normal(pool, Hkv, P, dh), v=normal(pool, Hkv, P, dh), q=normal(M, H, dh))
        state["slot"] = torch.randperm(pool * P, device="cuda", generator=gen)[:M].int()
        state["pos"] = torch.randint(0, 131072, (M,), device="cuda", generator=gen, dtype=torch.int32)
        return state
    lens, n = _lengths(case)
    pool = sum(_pages(x, P) for x in lens) + 1
    state["table"], _ = _tables(lens, _pages(max(lens), P), P, pool, gen)
    state.update(q=normal(sum(n), H, dh), k=normal(pool, Hkv, P, dh), v=normal(pool, Hkv, P, dh), out=normal(sum(n), H, dh), seq_len=_i32(lens),
                 most_rows=max(n), most_len=max(lens), cu=_i32([sum(n[:b]) for b in range(len(n) + 1)]))
    state["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return state


# ---------------------------------------------------------------- plain forms
def _extend(s):
    P, length, n, table, free = s["page"], s["seq_len"].long(), s["n_rows"].long(), s["table"], s["free"]
    B, W = table.shape
    end = length + n
    have = (length + P - 1) // P
    fits = (end <= W * P) & (n.cumsum(0) <= s["M"])
    need = torch.where(fits, (end + P - 1) // P - have, 0)
    total = need.cumsum(0)
    admitted = fits & ((need == 0) | (total <= s["n_free"]))
    given = torch.where(admitted, need, 0)
    place = s["n_free"] - torch.cat([given.new_zeros(1), given.cumsum(0)])
    j = torch.arange(W, device=table.device)[None, :] - have[:, None]
    new = (j >= 0) & (j < given[:, None])
    table.copy_(torch.where(new, free[(place[:-1, None] - 1 - j).clamp(0, free.numel() - 1)], table))
    cu = torch.cat([n.new_zeros(1), n.cumsum(0)])
    row = torch.arange(s["M"], device=table.device)
    r = torch.searchsorted(cu[1:], row, right=True)
    pos = length[r] + row - cu[r]
    slot = torch.where(admitted[r], table[r, (pos // P).clamp(max=W - 1)] * P + pos % P, -1)
    return {"table": table, "seq_len": torch.where(admitted, end, length).int(), "n_free": place[-1:].int(), "cu_rows": cu.int(), "admitted": admitted.int(),
            "place": place.int(), "pos": pos.int(), "slot": slot.int()}


def _trim(s):
    P, length, table, free = s["page"], s["seq_len"].long(), s["table"], s["free"]
    keep = torch.minimum(s["keep"].long().clamp(min=0), length)
    first, behind = (keep + P - 1) // P, (length + P - 1) // P
    place = s["n_free"] + torch.cat([first.new_zeros(1), (behind - first).cumsum(0)])
    j = torch.arange(table.shape[1], device=table.device)[None, :]
    out = (j >= first[:, None]) & (j < behind[:, None])
    free.index_copy_(0, (place[:-1, None] + j - first[:, None])[out], table[out])
    return {"free": free, "seq_len": keep.int(), "n_free": place[-1:].int(), "place": place.int()}


def _store(s):
    H, Hkv, dh, P = s["H"], s["Hkv"], s["dh"], s["page"]
    M, half = s["M"], dh // 2
    x = s["qkv"].float().view(M, H + 2 * Hkv, dh)
    angle = s["pos"].double()[:, None] * THETA ** (-torch.arange(half, device=x.device, dtype=torch.float64) * 2 / dh)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x[:, : H + Hkv, :half], x[:, : H + Hkv, half:]
    turned = torch.cat([a * cos - b * sin, b * cos + a * sin], 2).to(s["qkv"].dtype)
    page, at = s["slot"].long() // P, s["slot"].long() % P
    s["k"][page, :, at] = turned[:, H:]
    s["v"][page, :, at] = x[:, H + Hkv:].to(s["v"].dtype)
    return {"q": turned[:, :H], "k": s["k"], "v": s["v"]}


def _attention(s):
    H, Hkv, dh, P, B = s["H"], s["Hkv"], s["dh"], s["page"], s["B"]
    length, cu = s["seq_len"].long(), s["cu"].long()
    n = cu[1:] - cu[:-1]
    t = torch.arange(s["most_len"], device=cu.device)
    there = t[None, :] < length[:, None]                                    # [B, L]
    page = torch.where(there, s["table"][:, t // P].long(), 0)
    k = s["k"][page, :, (t % P).expand_as(page)].float().permute(0, 2, 3, 1).contiguous()      # [B, Hkv, dh, L]
    v = torch.where(there[:, :, None, None], s["v"][page, :, (t % P).expand_as(page)].float(), 0).permute(0, 2, 1, 3).contiguous()
    i = torch.arange(s["most_rows"], device=cu.device)
    row = (cu[:-1, None] + i).clamp(max=int(s["q"].shape[0]) - 1)             # [B, R]; rows behind a request's own are dropped at the end
    q = s["q"][row].float().view(B, -1, Hkv, H // Hkv, dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, dh)
    limit = length[:, None] - n[:, None] + i + 1 if s["causal"] else length[:, None].expand_as(row)
    seen = (t < limit[:, :, None])[:, None, :, None, :]                      # [B, 1, R, 1, L]
    score = (q @ k / math.sqrt(dh)).view(B, Hkv, i.numel(), H // Hkv, -1)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - torch.where(top == -math.inf, 0, top))
    total = e.sum(-1, keepdim=True)
    o = (e.view(B, Hkv, -1, t.numel()) @ v).view(B, Hkv, i.numel(), H // Hkv, dh) / torch.where(total == 0, 1, total)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, i.numel(), H, dh)
    return o[i[None, :] < n[:, None]].to(s["q"].dtype)


def run(state):
    if own:
        return _own(state)
    return {"extend": _extend, "trim": _trim, "store": _store, "attention": _attention}[state["op"]](state)


def _own(s):
    from paper_2601_12247_amd import binding as B
    op = s["op"]
    if op == "attention":
        return B.page_attention(s["q"], s["k"], s["v"], s["table"], s["seq_len"], cu_rows=s["cu"], causal=s["causal"], out=s["out"], workspace=s["workspace"])
    if op == "store":
        B.page_store(s["qkv"], s["pos"], s["slot"], s["k"], s["v"], THETA, q_out=s["q"])
        return {"q": s["q"], "k": s["k"], "v": s["v"]}
    if op == "extend":
        B.page_extend(s["seq_len"], s["n_rows"], s["table"], s["free"], s["n_free"], s["page"],
                      out=(s["new_len"], s["new_free"], s["cu"], s["admitted"], s["place"], s["pos"], s["slot"]))
        return {"table": s["table"], "seq_len": s["new_len"], "n_free": s["new_free"], "cu_rows": s["cu"], "admitted": s["admitted"], "place": s["place"],
                "pos": s["pos"], "slot": s["slot"]}
    B.page_trim(s["seq_len"], s["keep"], s["table"], s["free"], s["n_free"], s["page"], out=(s["new_len"], s["new_free"], s["place"]))
    return {"free": s["free"], "seq_len": s["new_len"], "n_free": s["new_free"], "place": s["place"]}


# ---------------------------------------------------------------- work and exact results
def work(case):
    op, P = case["op"], case["page"]
    if op in ("extend", "trim"):
        B = case["B"]
        lens = _sizes(B, case["len"], min(case["len"], 1))
        if op == "trim":                                                     # half of what may be dropped, on average
            moved = sum(_pages(x, P) - _pages(max(0, x - case["drop"] // 2), P) for x in lens)
            return {"bytes": B * 16 + moved * 8 + 8, "flops": 4 * B + moved}
        add = _sizes(B, case["rows"], min(case["rows"], 1))[::-1]
        moved = sum(_pages(a + b, P) - _pages(a, P) for a, b in zip(lens, add))
        return {"bytes": B * 24 + moved * 8 + sum(add) * 8 + 8, "flops": 6 * B + moved + 4 * sum(add)}
    size, H, Hkv, dh = (4 if case["dtype"] == "f32" else 2), case["H"], case["Hkv"], case["dh"]
    if op == "store":
        return {"bytes": case["M"] * (2 * (H + 2 * Hkv) * dh * size + 8), "flops": case["M"] * (H + Hkv) * dh * 3}
    lens, n = _lengths(case)
    seen = sum(r * x - (r * (r - 1) // 2 if case["causal"] else 0) for x, r in zip(lens, n))
    return {"bytes": sum(lens) * 2 * Hkv * dh * size + 2 * sum(n) * H * dh * size + sum(_pages(x, P) for x in lens) * 4, "flops": 4 * seen * H * dh}


def _exact_attention(s):
    """One request and one shared head at a time, in 64 bits."""
    lens, cu = s["seq_len"].tolist(), s["cu"].tolist()
    group, P = s["H"] // s["Hkv"], s["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    for b, length in enumerate(lens):
        rows = cu[b + 1] - cu[b]
        pages = s["table"][b, : _pages(length, P)].long()
        limit = length - rows + torch.arange(rows, device=out.device) + 1 if s["causal"] else torch.full((rows,), length, device=out.device)
        hidden = (torch.arange(length, device=out.device)[None, :] >= limit[:, None]).repeat_interleave(group, 0)
        for h in range(s["Hkv"]):
            k = s["k"][pages, h].reshape(-1, s["dh"])[:length].double()
            v = s["v"][pages, h].reshape(-1, s["dh"])[:length].double()
            q = s["q"][cu[b]: cu[b + 1], h * group: (h + 1) * group].reshape(-1, s["dh"]).double()
            p = torch.softmax((torch.mm(q, k.t()) * s["dh"] ** -0.5).masked_fill(hidden, -math.inf), 1)
            out[cu[b]: cu[b + 1], h * group: (h + 1) * group] = torch.mm(p, v).view(rows, group, -1)
    return out


def _exact_store(s):
    """Pairs as complex numbers, turned by exp(i angle); every slot from the row that goes there, or as it was."""
    H, Hkv, dh, M, P = s["H"], s["Hkv"], s["dh"], s["M"], s["page"]
    x = s["qkv"].double().view(M, H + 2 * Hkv, dh)
    z = torch.complex(x[..., : dh // 2], x[..., dh // 2:])
    power = torch.exp(torch.arange(0, dh, 2, device=x.device, dtype=torch.float64) * (-math.log(THETA) / dh))
    z = z[:, : H + Hkv] * torch.polar(torch.ones((), dtype=torch.float64, device=x.device), s["pos"].double()[:, None, None] * power)
    turned = torch.cat([z.real, z.imag], 2)

    def filled(cache, rows):
        flat = cache.double().permute(0, 2, 1, 3).reshape(-1, Hkv, dh)
        flat[s["slot"].long()] = rows
        return flat.view(-1, P, Hkv, dh).permute(0, 2, 1, 3).contiguous()

    return {"q": turned[:, :H], "k": filled(s["k"], turned[:, H:]), "v": filled(s["v"], x[:, H + Hkv:])}


def _exact_pages(s):
    """A free list popped and pushed request by request."""
    P, lens, free = s["page"], s["seq_len"].tolist(), s["free"].tolist()
    table, n_free = s["table"].tolist(), int(s["n_free"])
    B, W = len(lens), len(table[0])
    new_len, place, asked = list(lens), [n_free], 0
    if s["op"] == "trim":
        keep = s["keep"].tolist()
        for b in range(B):
            new_len[b] = min(max(keep[b], 0), lens[b])
            for page in table[b][_pages(new_len[b], P): _pages(lens[b], P)]:
                free[n_free] = page
                n_free += 1
            place.append(n_free)
        return {"free": _i32(free), "seq_len": _i32(new_len), "n_free": _i32([n_free]), "place": _i32(place)}
    add, cu, admitted, pos, slot, top = s["n_rows"].tolist(), [0], [0] * B, [], [], n_free
    for b in range(B):
        cu.append(cu[-1] + add[b])
        end, have = lens[b] + add[b], _pages(lens[b], P)
        if end <= W * P and cu[-1] <= s["M"]:
            need = _pages(end, P) - have
            asked += need
            admitted[b] = int(need == 0 or asked <= top)
        if admitted[b]:
            for j in range(need):
                n_free -= 1
                table[b][have + j] = free[n_free]
            new_len[b] = end
        place.append(n_free)
        pos += range(lens[b], end)
        slot += [table[b][t // P] * P + t % P if admitted[b] else -1 for t in range(lens[b], end)]
    return {"table": _i32(table), "seq_len": _i32(new_len), "n_free": _i32([n_free]), "cu_rows": _i32(cu), "admitted": _i32(admitted), "place": _i32(place),
            "pos": _i32(pos), "slot": _i32(slot)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "store": _exact_store, "extend": _exact_pages, "trim": _exact_pages}[case["op"]](s)
