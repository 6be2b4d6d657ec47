"""Operators of a key-value cache held in pages and in 4 bits, and the
alpha-entmax attention of single tokens that reads it: their plain forms and the
cases on which they are measured.

A page holds `page` tokens of every key head, as a uint8 tensor
[layers, pages, kv_heads, 2 (keys, values), page / 16, 17 d / 2]: tiles of 16
tokens, each 16 rows of d / 2 bytes (value 2 i of a token in the low half of byte
i, value 2 i + 1 in the high half) and then 16 rows of d / 32 scale bytes.  A value
is the number of its four bits (sign, and 0, 0.5, 1, 1.5, 2, 3, 4 or 6) times 2^(s - 127),
s being the scale byte of its 32 values; s = 255 stands for NaN.  The scale is the
smallest power of two from 2^-125 to 2^125 that leaves the largest of the 32 magnitudes at
most 7 (2^125 where none does; 6 and 7 are as far apart as half a step of the next numbers would be);
values are rounded to the nearest number, ties to the even code.  A table gives the
pages of each row (a request, or a beam).

ops
    append   cache_append of new tokens' keys and values, and cache_read of the
             rows that they have taken (the values that a later prefill sees)
    read     cache_read alone: the context of a chunk of a prompt
    update   cache_update: every row goes on from a row of the table (itself, a
             beam that was chosen, nothing) and grows by new tokens or loses its
             last; rows that share a page they are about to write get a copy
    compact  cache_compact: pages move to the lowest places of the pool
    decode   paged_decode: one query per request (or several, the last tokens of a
             draft) over the pages of its row

`own` chooses between the plain forms (elementary torch operations in 32 bits)
and the calls of the library.
"""
import math

import torch

own = False

NUMBERS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------- cases

def _append(name, requests, new, old, page, hk, d, dtype):
    return {"name": name, "op": "append", "requests": requests, "new": new, "old": old, "page": page, "hk": hk,
            "d": d, "dtype": dtype}


def _read(name, requests, length, page, hk, d, dtype):
    return {"name": name, "op": "read", "requests": requests, "length": length, "page": page, "hk": hk, "d": d,
            "dtype": dtype}


def _update(name, prompts, beams, length, width, spare, layers, page, hk, d, serve=False):
    return {"name": name, "op": "update", "prompts": prompts, "beams": beams, "length": length, "width": width,
            "spare": spare, "layers": layers, "page": page, "hk": hk, "d": d, "serve": serve}


def _compact(name, requests, length, pages, layers, page, hk, d):
    return {"name": name, "op": "compact", "requests": requests, "length": length, "pages": pages, "layers": layers,
            "page": page, "hk": hk, "d": d}


def _decode(name, requests, length, per, page, hq, hk, d, dtype, alpha, c):
    return {"name": name, "op": "decode", "requests": requests, "length": length, "per": per, "page": page, "hq": hq,
            "hk": hk, "d": d, "dtype": dtype, "alpha": alpha, "c": c}


def listed():
    return [
        # one decoding step of a batch: a token to each request, latency
        _append("append_step", 64, 1, 9216, 64, 8, 128, "bf16"),
        # a chunk of prompts, a ragged number of tokens each, some of them padding
        _append("append_prompts", 8, 4000, 1111, 32, 8, 128, "bf16"),
        # the context of two requests whose prompts go on, fp32, head dimension 64
        _read("read_context_f32", 2, 777, 16, 12, 64, "f32"),
        # the contexts of a batch of long prompts' next chunks
        _read("read_contexts", 8, 8192, 64, 8, 128, "bf16"),
        # a decoding step's pages: requests that grow, end, start from another's prompt, drop draft tokens
        _update("update_serve", 64, 1, 4096, 576, 300, 4, 16, 8, 128, serve=True),
        # one step of beam search over all layers: beams go on from those chosen, the last pages are copied
        _update("update_beams", 32, 8, 2000, 128, 400, 8, 32, 8, 128),
        # a small pool with holes
        _compact("compact_small", 6, 300, 160, 2, 16, 4, 64),
        # a pool half of whose pages were freed, to be given back or filled again
        _compact("compact_pool", 48, 2048, 4096, 6, 32, 8, 128),
        # one request: latency
        _decode("paged_one", 1, 4096, 1, 16, 16, 4, 128, "bf16", 1.5, 1.0),
        # a chat service's batch, lengths of every size
        _decode("paged_chat", 64, 9216, 1, 64, 32, 8, 128, "bf16", 1.5, 1.0),
        # long documents
        _decode("paged_long", 8, 65536, 1, 128, 32, 8, 128, "bf16", 1.5, 2.0),
        # a few short requests with drafts of three tokens, fp32, denser rows
        _decode("paged_drafts_f32", 5, 1000, 3, 32, 8, 2, 64, "f32", 1.25, 1.0),
    ]


def draw(rng):
    """Another case of the ranges of the listed ones."""
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    op = rng.choice(["append", "read", "update", "compact", "decode", "decode", "decode"])
    page, d = rng.choice([16, 32, 64, 128, 256]), rng.choice([64, 128])
    hq, hk = rng.choice([(32, 8), (16, 8), (16, 4), (16, 16), (12, 4), (12, 12), (8, 1), (14, 2), (4, 4), (40, 2)])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    case = {"op": op, "page": page, "hk": hk, "d": d}
    if op == "append":
        requests = logint(1, 128)
        new = logint(1, max(1, 32000 * 8 * 128 // (requests * hk * d) // (2 if dtype == "f32" else 1)))
        return dict(case, requests=requests, new=new, old=logint(1, 4096), dtype=dtype)
    if op == "read":
        requests = logint(1, 64)
        most = 8 * 8192 * 8 * 128 // (requests * hk * d) // (2 if dtype == "f32" else 1)
        return dict(case, requests=requests, length=logint(1, min(16384, most)), dtype=dtype)
    if op == "update":
        serve = rng.random() < 0.5
        prompts, beams = (logint(1, 256), 1) if serve else (logint(1, 32), rng.choice([2, 4, 5, 8]))
        layers, length = rng.choice([1, 2, 4, 8]), logint(1, 4096)
        # no more pages, and no more bytes in them, than the largest listed pool
        most = min(4096, 4096 * 6 * 32 * 8 * 128 // (layers * page * hk * d))
        while length > 1 and _update_pages(prompts, beams, length, page) > most:
            length = max(1, length // 2)
        width = -(-length // page) + rng.choice([1, 2, 16, 64])
        return dict(case, prompts=prompts, beams=beams, length=length, width=width,
                    spare=logint(1, 4 * prompts * beams), layers=layers, serve=serve)
    if op == "compact":
        layers = rng.choice([1, 2, 4, 6])
        most = min(4096, 4096 * 6 * 32 * 8 * 128 // (layers * page * hk * d))
        pages = logint(8, max(8, most))
        requests = logint(1, min(64, pages // 2))
        return dict(case, requests=requests, length=logint(1, max(1, pages // (2 * requests) * page)),
                    pages=pages, layers=layers)
    length, per = logint(1, 65536), rng.choice([1, 1, 1, 2, 4])
    # no more keys, and no more scores, than the listed cases have
    most = min(8 * 65536 * 8 * 128 // (length * hk * d), 8 * 65536 * 32 // (length * hq)) // (4 if dtype == "f32" else 1)
    return dict(case, requests=max(1, min(logint(1, 256), most // per)), length=length, per=per, hq=hq, dtype=dtype,
                alpha=rng.choice([1.5, 1.5, 1.25, 1.4, 2.0]), c=round(math.exp(rng.uniform(math.log(0.5), math.log(8.0))), 3))


def _spread(count, longest):
    """Lengths of `count` requests, spread over 1 .. longest."""
    return [longest - (longest - 1) * ((b * 5) % count) // count for b in range(count)]


def _row_bytes(case):
    """Bytes of one token of all key heads, keys and values."""
    return case["hk"] * 2 * (case["d"] // 2 + case["d"] // 32)


def _update_pages(prompts, beams, length, page):
    used = 0
    for n in _spread(prompts, length):
        used += -(-n // page) + (beams - 1) * (-(-n // page) - n // 2 // page)
    return used


def _counts(case):
    """Tokens that each row of an update gains, -2 for rows that drop a rejected draft."""
    rows = case["prompts"] * case["beams"]
    if not case["serve"]:
        return [1] * rows
    return [-2 if r % 7 == 3 else 40 if r % 11 == 5 else 1 for r in range(rows)]


def _parents(case):
    """The row that each row of an update goes on from, -1 for none."""
    beams, rows = case["beams"], case["prompts"] * case["beams"]
    if case["serve"]:  # some end, and some of their places go to requests that share another's tokens
        return [-1 if r % 16 == 9 else (r + 1) % rows if r % 16 == 13 else r for r in range(rows)]
    # half of the beams go on, twice each
    return [r // beams * beams + (r % beams * 3 // 2 * 2 + r // beams) % beams // 2 for r in range(rows)]


def _state(case, seed):
    """(table, lengths, pages of the pool) of an update or a compaction, as lists: which
    rows have which pages.  The pages' numbers are shuffled by the seed."""
    page, ids, table = case["page"], 0, []
    if case["op"] == "update":
        width, lengths = case["width"], []
        for n in _spread(case["prompts"], case["length"]):
            shared = n // 2 // page  # the prompt's whole pages
            first = list(range(ids, ids + shared))
            ids += shared
            for _ in range(case["beams"]):
                rest = -(-n // page) - shared
                table.append(first + list(range(ids, ids + rest)))
                ids += rest
                lengths.append(n)
        pool = ids + case["spare"]
    else:
        lengths, pool = _spread(case["requests"], case["length"]), case["pages"]
        width = -(-case["length"] // page) + 3
        for n in lengths:
            table.append(list(range(ids, ids + -(-n // page))))
            ids += -(-n // page)
    at = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).tolist()
    return [[at[p] for p in row] + [-1] * (width - len(row)) for row in table], lengths, pool


def work(case):
    e = 4 if case.get("dtype") == "f32" else 2
    token = _row_bytes(case)
    if case["op"] == "append":
        tokens = sum(_spread(case["requests"], case["new"]))
        # values in, codes out, codes in, values out
        return {"bytes": tokens * (4 * case["hk"] * case["d"] * e + 2 * token), "flops": tokens * case["hk"] * case["d"] * 12}
    if case["op"] == "read":
        tokens = sum(_spread(case["requests"], case["length"]))
        return {"bytes": tokens * (2 * case["hk"] * case["d"] * e + token), "flops": tokens * case["hk"] * case["d"] * 2}
    if case["op"] == "update":
        table, lengths, pool = _state(case, 0)
        new, _, _, moved = _update_by_hand(case, table, lengths, pool)
        entries = sum(sum(p >= 0 for p in row) for row in table + new)
        return {"bytes": 4 * entries + len(moved) * 2 * case["layers"] * case["page"] * token, "flops": 4 * entries}
    if case["op"] == "compact":
        table, lengths, pool = _state(case, 0)
        used = len({p for row in table for p in row if p >= 0})
        # of pages in random places those behind the first `used`
        moved = used * (pool - used) / pool
        return {"bytes": 8 * used + moved * 2 * case["layers"] * case["page"] * token, "flops": 4 * used + pool}
    keys = sum(_spread(case["requests"], case["length"]))
    queries = case["requests"] * case["per"]
    # queries of one draft read the same keys; the products as if no probability were zero
    return {"bytes": keys * token + queries * case["hq"] * case["d"] * e * 2,
            "flops": keys * case["per"] * case["hq"] * case["d"] * 4}


# ------------------------------------------------------------------ inputs

def _pack(x):
    """(codes [..., d / 2], scales [..., d / 32]) of values [..., d], bytes."""
    x = x.float().unflatten(-1, (-1, 32))
    bits = x.abs().amax(-1).view(torch.int32)  # (a NaN's are the largest)
    power = bits >> 23
    scale = (power - 2 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(2, 252)
    scale = torch.where(power == 255, 255, scale)
    y = x * ((254 - scale).clamp_min(0) << 23).view(torch.float32).unsqueeze(-1)
    m = y.abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    code = code + 8 * (x.view(torch.int32) < 0).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], scale.to(torch.uint8)


def _unpack(codes, scales):
    """Values in 32 bits."""
    numbers = torch.tensor(NUMBERS + tuple(-v for v in NUMBERS), device=codes.device)
    v = numbers[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    s = (scales.int() << 23).view(torch.float32)
    s = torch.where(scales == 255, math.nan, s)
    return (v.unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def _parts(cache, d):
    """(codes [.., pages, kv_heads, 2, tiles, 16, d / 2], scales [.., 16, d / 32]) of a cache, as views."""
    return (cache[..., :8 * d].unflatten(-1, (16, d // 2)), cache[..., 8 * d:].unflatten(-1, (16, d // 32)))


def _pool(shape, d, g):
    """A cache whose pages all hold keys and values: Gaussian, as a norm of heads leaves them."""
    cache = torch.empty(*shape[:-1], 17 * d // 2, dtype=torch.uint8, device="cuda")
    flat = cache.view(-1, 17 * d // 2)
    for at in range(0, flat.shape[0], 1 << 16):  # (2^27 values at a time)
        part = flat[at:at + (1 << 16)]
        codes, scales = _pack(torch.randn(part.shape[0], 16, d, generator=g, device="cuda"))
        part[:, :8 * d], part[:, 8 * d:] = codes.flatten(1), scales.flatten(1)
    return cache


def _table(lengths, page, spare, seed):
    """A table of rows of these lengths with pages of their own in a shuffled order, and the pool's pages."""
    each = [-(-n // page) for n in lengths]
    ids = torch.randperm(sum(each) + spare, generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    table = torch.full((len(each), max(each)), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(each):
        table[r, :n] = ids[at:at + n]
        at += n
    return table.cuda(), sum(each) + spare


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
    page, hk, d = case["page"], case["hk"], case["d"]
    st = {"case": case, "dtype": dt}
    if case["op"] in ("update", "compact"):
        table, lengths, pool = _state(case, seed)
        st["table"], st["lengths"] = _ints(table), _ints(lengths)
        # (any bytes are a page)
        st["cache"] = torch.randint(0, 256, (case["layers"], pool, hk, 2, page // 16, 17 * d // 2), generator=g,
                                    device="cuda", dtype=torch.uint8)
        if case["op"] == "update":
            st["parents"], st["counts"] = _ints(_parents(case)), _ints(_counts(case))
        return st
    B = case["requests"]
    if case["op"] == "append":
        new = _spread(B, case["new"])
        first = [0 if b % 4 == 1 else n for b, n in enumerate(_spread(B, case["old"]))]
        lengths = [a + n for a, n in zip(first, new)]
    else:
        lengths = _spread(B, case["length"])
    st["table"], pool = _table(lengths, page, 5, seed)
    shape = (pool, hk, 2, page // 16, 17 * d // 2)
    if case["op"] == "append":
        st["cache"] = torch.zeros(shape, dtype=torch.uint8, device="cuda")
        rows, positions = [], []
        for b, n in enumerate(new):
            rows += [b] * n
            positions += range(first[b], first[b] + n)
            if n > 100:  # padding behind a long chunk
                rows += [b] * (n % 3)
                positions += [-1] * (n % 3)
        st["rows"], st["positions"] = _ints(rows), _ints(positions)
        # parts of a fused projection's rows; magnitudes of different heads and channels differ
        x = torch.randn(len(rows), 3 * hk * d, generator=g, device="cuda")
        x *= torch.exp(torch.randn(3 * hk * d, generator=g, device="cuda"))
        x = x.to(dt)
        st["k"], st["v"] = x[:, hk * d:2 * hk * d].view(-1, hk, d), x[:, 2 * hk * d:].view(-1, hk, d)
        return st
    st["cache"] = _pool(shape, d, g)
    if case["op"] == "read":
        count = torch.tensor(lengths, device="cuda")
        st["rows"] = torch.repeat_interleave(torch.arange(B, device="cuda", dtype=torch.int32), count)
        starts = torch.repeat_interleave(count.cumsum(0) - count, count)
        st["positions"] = (torch.arange(sum(lengths), device="cuda") - starts).int()
        return st
    per = case["per"]
    st["q"] = torch.randn(B * per, case["hq"], d, generator=g, device="cuda").mul_(case["c"]).to(dt)
    st["lengths"] = _ints([max(0, n - per + 1 + i) for n in lengths for i in range(per)])
    st["rows"] = _ints([b for b in range(B) for _ in range(per)]) if per > 1 else None
    return st


def run(state):
    case = state["case"]
    if own:
        return _OWN[case["op"]](case, state)
    return _PLAIN[case["op"]](case, state)


# ------------------------------------------------------- the library's calls

def _own_append(case, s):
    import paper_2502_12082_amd as ea
    ea.cache_append(s["cache"], s["k"], s["v"], s["rows"], s["positions"], s["table"])
    return ea.cache_read(s["cache"], s["rows"], s["positions"], s["table"], dtype=s["dtype"])


def _own_read(case, s):
    import paper_2502_12082_amd as ea
    return ea.cache_read(s["cache"], s["rows"], s["positions"], s["table"], dtype=s["dtype"])


def _own_update(case, s):
    import paper_2502_12082_amd as ea
    return ea.cache_update(s["cache"], s["table"], s["lengths"], s["parents"], s["counts"]) + (s["cache"],)


def _own_compact(case, s):
    import paper_2502_12082_amd as ea
    return ea.cache_compact(s["cache"], s["table"], s["lengths"]) + (s["cache"],)


def _own_decode(case, s):
    import paper_2502_12082_amd as ea
    return ea.paged_decode(s["q"], s["cache"], s["table"], s["lengths"], rows=s["rows"], alpha=case["alpha"])


# -------------------------------------------------------------- plain forms

def _places(case, s):
    """(which tokens have a place, and its page, tile and row in the tile)."""
    page, positions = case["page"], s["positions"]
    held = positions >= 0
    positions = positions.clamp_min(0)
    return held, s["table"][s["rows"], positions // page].clamp_min(0), positions % page // 16, positions % 16


def _plain_read(case, s):
    held, page, tile, row = _places(case, s)
    codes, scales = _parts(s["cache"], case["d"])
    return tuple(torch.where(held[:, None, None], _unpack(codes[page, :, i, tile, row], scales[page, :, i, tile, row]),
                             0.0).to(s["dtype"]) for i in (0, 1))


def _plain_append(case, s):
    held, page, tile, row = _places(case, s)
    page, tile, row = page[held], tile[held], row[held]
    for into, k, v in zip(_parts(s["cache"], case["d"]), _pack(s["k"][held]), _pack(s["v"][held])):
        into[page, :, 0, tile, row], into[page, :, 1, tile, row] = k, v
    return _plain_read(case, s)


def _references(table, held, pool):
    """How often each page stands in the table's `held` entries."""
    ids = torch.where(held, table, pool).flatten().long()
    return torch.zeros(pool + 1, dtype=torch.int64, device=table.device).index_add_(0, ids, torch.ones_like(ids))[:pool]


def _plain_update(case, s):
    page, pool, dev = case["page"], s["cache"].shape[1], s["table"].device
    parents, rows, width = s["parents"].long(), s["parents"].shape[0], s["table"].shape[1]
    table, old = s["table"][parents.clamp_min(0)], s["lengths"][parents.clamp_min(0)] * (parents >= 0)
    wanted = (old + s["counts"]).clamp_min(0)
    fits = wanted <= width * page
    grows = (s["counts"] > 0) & fits
    at = torch.arange(width, device=dev)
    kept = (torch.where(fits, torch.minimum(old, wanted), old) + page - 1) // page
    refs = _references(table, at < kept[:, None], pool)
    # rows that are about to write to a page which others hold: a copy, but one of them may write where all would
    last = torch.gather(table, 1, (old // page).clamp_max(width - 1)[:, None].long())[:, 0].long()
    writes = grows & (old % page > 0)
    ids = torch.where(writes, last, pool)
    number = torch.arange(rows, device=dev)
    writers = torch.zeros(pool + 1, dtype=torch.int64, device=dev).index_add_(0, ids, torch.ones_like(ids))
    lowest = torch.full((pool + 1,), rows, device=dev).scatter_reduce_(0, ids, number, "amin")
    shared = refs[ids.clamp_max(pool - 1)]
    copies = writes & (shared > 1) & ((shared > writers[ids]) | (lowest[ids] != number))
    need = torch.where(grows, (wanted + page - 1) // page - kept, 0) + copies
    before = need.cumsum(0) - need
    order = torch.argsort((refs > 0).int(), stable=True).int()  # free pages, the lowest first
    done = (need == 0) | (before + need <= (refs == 0).sum())
    length = torch.where(fits & done, wanted, old)
    missing = torch.where(fits, torch.where(done, 0, need), -1)
    # the copy's page comes first, then those behind
    used = (length + page - 1) // page
    rank = before[:, None] + copies[:, None] + at - kept[:, None]
    new = order[rank.clamp(0, pool - 1)]
    copied = copies & done
    new = torch.where(at >= kept[:, None], new, table)
    new = torch.where(copied[:, None] & (at == (old // page)[:, None]), order[before.clamp_max(pool - 1)][:, None], new)
    new = torch.where(at < used[:, None], new, -1)
    s["cache"][:, order[before[copied]].long()] = s["cache"][:, last[copied]]
    return new, length, missing.int(), s["cache"]


def _plain_compact(case, s):
    pool, dev = s["cache"].shape[1], s["table"].device
    at = torch.arange(s["table"].shape[1], device=dev)
    held = at < ((s["lengths"] + case["page"] - 1) // case["page"])[:, None]
    used = _references(s["table"], held, pool) > 0
    count = used.sum()
    number = torch.arange(pool, device=dev)
    source, free = (used & (number >= count)).nonzero()[:, 0], (~used & (number < count)).nonzero()[:, 0]
    to = number.clone()
    to[source] = free
    s["cache"][:, free] = s["cache"][:, source]
    table = torch.where(held, to[s["table"].clamp_min(0).long()], -1).int()
    return table, count.int().view(1), s["cache"]


def _threshold(x, gamma, steps=30):
    """tau of every row of x (invalid entries -inf): Newton's steps on the
    convex sum [x - tau]^gamma - 1 from max x - 1, where it is not negative."""
    tau = x.amax(-1, keepdim=True) - 1.0
    for _ in range(steps):
        z = (x - tau).clamp_min(0.0)
        u = z if gamma == 2.0 else (z > 0).to(x.dtype) if gamma == 1.0 else z ** (gamma - 1.0)
        tau = tau + (((u * z).sum(-1, keepdim=True) - 1.0) / (gamma * u.sum(-1, keepdim=True))).clamp_min(0.0)
    return tau


def _plain_decode(case, s):
    hk, group, alpha, page = case["hk"], case["hq"] // case["hk"], case["alpha"], case["page"]
    gamma = 1.0 / (alpha - 1.0)
    table = s["table"] if s["rows"] is None else s["table"][s["rows"]]
    codes, scales = _parts(s["cache"], case["d"])
    ids = table.clamp_min(0).long()

    def rows_of(i):  # [queries, kv_heads, keys, d]
        x = _unpack(codes[ids, :, i], scales[ids, :, i])  # [queries, pages, kv_heads, tiles, 16, d]
        return x.transpose(1, 2).flatten(2, 4)

    q = s["q"].float().unflatten(1, (hk, group))
    x = ((alpha - 1.0) * case["d"] ** -0.5) * (q @ rows_of(0).transpose(-1, -2).contiguous())
    behind = torch.arange(x.shape[-1], device=x.device) >= s["lengths"][:, None]
    x.masked_fill_(behind[:, None, None], -math.inf)
    x = torch.where((s["lengths"] > 0)[:, None, None, None], x, 0.0)
    p = (x - _threshold(x, gamma)).clamp_min(0.0)
    p = p if gamma == 1.0 else p ** gamma
    p = torch.where(behind[:, None, None], 0.0, p)
    return (p @ rows_of(1)).flatten(1, 2).to(s["q"].dtype)


_PLAIN = {"append": _plain_append, "read": _plain_read, "update": _plain_update, "compact": _plain_compact,
          "decode": _plain_decode}
_OWN = {"append": _own_append, "read": _own_read, "update": _own_update, "compact": _own_compact,
        "decode": _own_decode}


# ----------------------------------------------- the definition, in 64 bits

def _values64(tiles, d):
    """[..., 16, d] in 64 bits of tiles [..., 17 d / 2]."""
    low, high = tiles[..., :8 * d] % 16, tiles[..., :8 * d] // 16
    code = torch.stack([low, high], -1).unflatten(-2, (16, d // 2)).flatten(-2).long()
    number = torch.tensor(NUMBERS, dtype=torch.float64, device=tiles.device)[code % 8] * (1 - 2 * (code // 8))
    s = tiles[..., 8 * d:].unflatten(-1, (16, d // 32)).double()
    scale = torch.where(s == 255, math.nan, torch.exp2(s - 127)).repeat_interleave(32, -1)
    return number * scale


def _rounded64(x):
    """What values stand for after they went to 4 bits and back."""
    x = x.double().unflatten(-1, (-1, 32))
    # scales one by one from the smallest up to where the largest magnitude fits
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.full_like(top, 2.0 ** -125)
    for _ in range(260):
        small = (top > 7.0 * scale) & (scale < 2.0 ** 125)
        if not small.any():
            break
        scale = torch.where(small, 2.0 * scale, scale)
    m = x.abs() / scale
    # the nearest multiple of the step of each magnitude (round goes to even ties, as the codes do)
    step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0))
    near = (torch.round(m / step) * step).clamp_max(6.0)
    return (torch.copysign(near, x) * scale).flatten(-2)


def _exact_append(case, s):
    held = (s["positions"] >= 0)[:, None, None]
    return tuple(torch.where(held, _rounded64(s[t]), 0.0) for t in ("k", "v"))


def _exact_read(case, s):
    out = [torch.empty(s["rows"].shape[0], case["hk"], case["d"], dtype=torch.float64, device="cuda") for _ in range(2)]
    at = 0
    for b, n in enumerate(_spread(case["requests"], case["length"])):
        ids = s["table"][b, :-(-n // case["page"])].long()
        x = _values64(s["cache"][ids], case["d"])  # [pages, heads, 2, tiles, 16, d]
        x = x.permute(2, 0, 3, 4, 1, 5).flatten(1, 3)[:, :n]
        out[0][at:at + n], out[1][at:at + n] = x[0], x[1]
        at += n
    return tuple(out)


def _update_by_hand(case, table, lengths, pool):
    """(table, lengths, missing, copies) of an update, row by row."""
    page, width = case["page"], case["width"]
    rows = []
    for parent, count in zip(_parents(case), _counts(case)):
        old = lengths[parent] if parent >= 0 else 0
        ids = table[parent][:-(-old // page)] if parent >= 0 else []
        new = max(0, old + count)
        fits = new <= width * page
        rows.append({"old": old, "new": new, "fits": fits, "grows": fits and count > 0,
                     "ids": list(ids[:-(-min(old, new) // page)] if fits else ids)})
    holders, writers = {}, {}
    for r, row in enumerate(rows):
        for p in row["ids"]:
            holders[p] = holders.get(p, 0) + 1
        if row["grows"] and row["old"] % page:
            writers.setdefault(row["ids"][-1], []).append(r)
    free = [p for p in range(pool) if p not in holders]
    taken, missing, copies = 0, [], []
    for r, row in enumerate(rows):
        last = row["ids"][-1] if row["ids"] else None
        sharers = writers.get(last, []) if row["grows"] and row["old"] % page else []
        copy = bool(sharers) and holders[last] > 1 and (holders[last] > len(sharers) or sharers[0] != r)
        need = (-(-row["new"] // page) - len(row["ids"]) if row["grows"] else 0) + copy
        mine, taken = free[taken:taken + need], taken + need
        missing.append(-1 if not row["fits"] else 0 if len(mine) == need else need)
        if missing[-1]:
            row["new"] = row["old"]
            continue
        if copy:
            copies.append((last, mine[0]))
            row["ids"][-1] = mine.pop(0)
        row["ids"] += mine
    return ([row["ids"] + [-1] * (width - len(row["ids"])) for row in rows], [row["new"] for row in rows], missing,
            copies)


def _exact_update(case, s):
    new, lengths, missing, copies = _update_by_hand(case, s["table"].tolist(), s["lengths"].tolist(),
                                                    s["cache"].shape[1])
    for source, to in copies:
        s["cache"][:, to] = s["cache"][:, source]
    return _ints(new), _ints(lengths), _ints(missing), s["cache"]


def _exact_compact(case, s):
    table, lengths = s["table"].tolist(), s["lengths"].tolist()
    rows = [row[:-(-n // case["page"])] for row, n in zip(table, lengths)]
    used = sorted({p for row in rows for p in row})
    holes = [p for p in range(len(used)) if p not in set(used)]
    to = {p: p for p in used}
    for source, hole in zip([p for p in used if p >= len(used)], holes):
        s["cache"][:, hole] = s["cache"][:, source]
        to[source] = hole
    return (_ints([[to[p] for p in row] + [-1] * (len(table[0]) - len(row)) for row in rows]), _ints([len(used)]),
            s["cache"])


def _exact_decode(case, s):
    group, d, alpha, page = case["hq"] // case["hk"], case["d"], case["alpha"], case["page"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    rows = range(o.shape[0]) if s["rows"] is None else s["rows"].tolist()
    for i, (r, n) in enumerate(zip(rows, s["lengths"].tolist())):
        if n == 0:
            continue
        x = _values64(s["cache"][s["table"][r, :-(-n // page)].long()], d)
        keys, values = x.permute(2, 1, 0, 3, 4, 5).flatten(2, 4)[:, :, :n]  # [heads, n, d] each
        q = s["q"][i].double().view(case["hk"], group, d)
        y = (alpha - 1.0) * d ** -0.5 * (q @ keys.transpose(1, 2).contiguous())
        hi = y.amax(-1, keepdim=True)
        lo = hi - 1.0
        for _ in range(56):  # bisection
            mid = 0.5 * (lo + hi)
            mass = torch.relu(y - mid).pow(1.0 / (alpha - 1.0)).sum(-1, keepdim=True)
            lo, hi = torch.where(mass >= 1.0, mid, lo), torch.where(mass >= 1.0, hi, mid)
        o[i] = (torch.relu(y - lo).pow(1.0 / (alpha - 1.0)) @ values).view(-1, d)
    return o


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "read": _exact_read, "update": _exact_update, "compact": _exact_compact,
            "decode": _exact_decode}[case["op"]](case, s)
