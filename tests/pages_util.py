"""Plain references, on the CPU, of the calls on a cache in pages and in 4 bits."""
import math

import torch

from tests.layer_util import entmax64

NUMBERS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def pack(x):
    """(codes [..., d], scales [..., d / 32]) of values [..., d] by their definition, in 64 bits."""
    x = x.double().unflatten(-1, (-1, 32))
    finite = torch.isfinite(x).all(-1)
    top = torch.where(finite, x.abs().amax(-1), 1.0)
    # the smallest e with top <= 7 * 2^e
    e = torch.full_like(top, -125.0)
    for power in range(-125, 125):
        e = torch.where(top > 7.0 * 2.0 ** power, power + 1.0, e)
    m = torch.where(finite[..., None], x.abs() / torch.exp2(e)[..., None], 0.0)
    far = (m[..., None] - NUMBERS).abs()
    best = far.amin(-1, keepdim=True)
    # the nearest number; of two as near, the one of the even code
    near = far == best
    code = torch.where(near & (torch.arange(8) % 2 == 0), torch.arange(8), 8).amin(-1)
    code = torch.where(code == 8, near.int().argmax(-1), code)
    code = code + 8 * torch.signbit(x).long()
    return code.flatten(-2), torch.where(finite, e + 127, 255.0).long()


def unpack(code, scale):
    v = NUMBERS[code % 8] * (1 - 2 * (code // 8))
    s = torch.where(scale == 255, math.nan, torch.exp2(scale.double() - 127))
    return v * s.repeat_interleave(32, -1)


def put(cache, page, at, head, which, code, scale):
    """Writes one row of codes [d] and scales [d / 32] into a layer's cache (on the CPU)."""
    d = code.shape[-1]
    tile = cache[page, head, which, at // 16]
    r = at % 16
    tile[r * (d // 2):(r + 1) * (d // 2)] = (code[0::2] + 16 * code[1::2]).to(torch.uint8)
    first = 8 * d + r * (d // 32)
    tile[first:first + d // 32] = scale.to(torch.uint8)


def values(cache):
    """All values of a layer's cache, in 64 bits: [pages, page_size, kv_heads, 2, d]."""
    cache = cache.cpu()
    d = cache.shape[-1] * 2 // 17
    codes = cache[..., :8 * d].unflatten(-1, (16, d // 2)).long()
    scales = cache[..., 8 * d:].unflatten(-1, (16, d // 32)).long()
    x = unpack(torch.stack([codes % 16, codes // 16], -1).flatten(-2), scales)  # [pages, heads, 2, tiles, 16, d]
    return x.permute(0, 3, 4, 1, 2, 5).flatten(1, 2)


def filled(cache, seed):
    """The cache with all pages holding random rows."""
    d = cache.shape[-1] * 2 // 17
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(cache.shape[:-1] + (16, d), generator=g)
    code, scale = pack(x)
    packed = torch.cat([(code[..., 0::2] + 16 * code[..., 1::2]).flatten(-2), scale.flatten(-2)], -1)
    return cache.copy_(packed.to(torch.uint8))


def shuffled_table(lengths, page, spare, seed, width=None):
    """(table, pages of the pool): rows of these lengths with pages of their own, in a shuffled order."""
    each = [-(-n // page) for n in lengths]
    ids = torch.randperm(sum(each) + spare, generator=torch.Generator().manual_seed(seed)).int()
    table = torch.full((len(each), width or max(max(each), 1)), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(each):
        table[r, :n] = ids[at:at + n]
        at += n
    return table, sum(each) + spare


def update_by_hand(table, lengths, parents, counts, page, pages):
    """(table, lengths, missing, copies) of an update, lists; one row after another."""
    width, rows = len(table[0]), []
    for parent, count in zip(parents, counts):
        old, ids = 0, []
        if 0 <= parent < len(table):
            old = min(max(lengths[parent], 0), width * page)
            ids = table[parent][:-(-old // page)]
        new = max(0, old + count)
        fits = new <= width * page
        new = new if fits else old
        rows.append([old, new, fits, list(ids[:-(-min(old, new) // page)])])
    real = lambda p: 0 <= p < pages
    holders, writers = {}, {}
    for r, (old, new, fits, ids) in enumerate(rows):
        for p in ids:
            if real(p):
                holders[p] = holders.get(p, 0) + 1
        if new > old and old % page and real(ids[-1]):
            writers.setdefault(ids[-1], []).append(r)
    free = [p for p in range(pages) if p not in holders]
    taken, missing, copies = 0, [], []
    for r, row in enumerate(rows):
        old, new, fits, ids = row
        copy = False
        if new > old and old % page and real(ids[-1]):
            sharers = writers[ids[-1]]
            copy = holders[ids[-1]] > 1 and (holders[ids[-1]] > len(sharers) or sharers[0] != r)
        need = (-(-new // page) - len(ids) if new > old else 0) + copy
        mine = free[taken:taken + need]
        taken += need
        missing.append(-1 if not fits else 0 if len(mine) == need else need)
        if missing[-1]:
            row[1] = old
            continue
        if copy:
            copies.append((ids[-1], mine[0]))
            ids[-1] = mine.pop(0)
        ids += mine
    return ([row[3] + [-1] * (width - len(row[3])) for row in rows], [row[1] for row in rows], missing, copies)


def compact_by_hand(table, lengths, page, pages):
    """(table, pages in use, moves)."""
    width = len(table[0])
    rows = [row[:-(-min(max(n, 0), width * page) // page)] for row, n in zip(table, lengths)]
    used = sorted({p for row in rows for p in row if 0 <= p < pages})
    held = set(used)
    holes = [p for p in range(len(used)) if p not in held]
    moves = list(zip([p for p in used if p >= len(used)], holes))
    to = dict(moves)
    return [[to.get(p, p) for p in row] + [-1] * (width - len(row)) for row in rows], len(used), moves


def keys_of(vals, table, row, n, page):
    """([n, heads, d] keys, values, which of them there are) of a row's first n tokens."""
    pages, width = vals.shape[0], table.shape[1]
    n = min(max(n, 0), width * page)
    ids = table[row].tolist() if 0 <= row < table.shape[0] else [-1] * width
    at = torch.arange(n)
    page_ids = torch.tensor([ids[p // page] for p in range(n)], dtype=torch.long)
    there = (page_ids >= 0) & (page_ids < pages)
    x = vals[page_ids.clamp(0, pages - 1), at % page]
    return x[:, :, 0], x[:, :, 1], there


def paged64(q, vals, table, lengths, rows, page, alpha, scale, tol=1e-6):
    """(o, how far a result may be off besides its last rounding).

    The second, for every query and head: scores are off by at most
      e = c (2^-19 (fp32: 2^-29) sum_b max |q_b| sum |k_b| + 16 T 2^-23 sum |q k|) + 2^-22 max |x|
    (the digits; the sums of T products of 128 values in 16 groups of 8, each
    addition within 2^-23 of the sum of magnitudes; the product with c), so tau by at
    most e and z by 2 e; p by gamma (z + 2 e)^(gamma - 1) 2 e; the solver
    leaves sum p off by up to tol; each p, and each step of the sum over n of them, is
    a rounding or two, and a general power 2^-18."""
    f32 = q.dtype == torch.float32
    alpha, scale = (float(torch.tensor(x, dtype=torch.float32)) for x in (alpha, scale))
    c, gamma = (alpha - 1.0) * scale, 1.0 / (alpha - 1.0)
    n, hq, d = q.shape
    hk = vals.shape[2]
    o, off = torch.zeros(n, hq, d, dtype=torch.float64), torch.zeros(n, hq, d, dtype=torch.float64)
    for i in range(n):
        r = i if rows is None else int(rows[i])
        keys, vs, there = keys_of(vals, table, r, int(lengths[i]), page)
        if keys.shape[0] == 0:
            continue
        for h in range(hq):
            k, v, qd = keys[:, h // (hq // hk)], vs[:, h // (hq // hk)], q[i, h].double().cpu()
            s = k @ qd
            s = torch.where(there & ~torch.isnan(s), s, -math.inf)
            some = s > -math.inf
            if not some.any():
                continue
            x = c * s
            p, u = entmax64(x[None], alpha)
            p = p[0]
            v = torch.where((p > 0)[:, None], v, 0.0)
            o[i, h] = p @ v
            ka = torch.where(some[:, None], k.abs(), 0.0)
            block = qd.abs().unflatten(0, (-1, 32)).amax(-1).repeat_interleave(32)
            e = c * (2.0 ** (-29 if f32 else -19) * (ka @ block).max() +
                     16 * (6 if f32 else 4) * 2.0 ** -23 * (ka @ qd.abs()).max()) + 2.0 ** -22 * x[some].abs().max()
            # z + 2 e of every key, where it is positive
            top = p.max() ** (1.0 / gamma)
            z = x - x.max() + top + 2 * e
            slope = torch.where(z > 0, gamma * z.clamp_min(1e-300) ** (gamma - 1.0), 0.0) * 2 * e
            va = torch.where((z > 0)[:, None], torch.where(torch.isnan(vs[:, h // (hq // hk)]), 0.0, vs[:, h // (hq // hk)].abs()), 0.0)
            roundings = (int((p > 0).sum()) + 16) * 2.0 ** -24 + (2.0 ** -18 if gamma not in (1.0, 2.0, 4.0) else 0.0)
            off[i, h] = slope @ va + (p @ v.abs()) * (roundings + tol) + tol * v.abs().amax(0)
    return o, off
