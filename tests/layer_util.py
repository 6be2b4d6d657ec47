"""Plain 64-bit references, on the CPU, of the calls on [tokens, heads, d]
tensors, and the tolerances that their roundings give."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # of a rounding, relative


def entmax64(x, alpha):
    """(p, u) of the rows of x = (alpha - 1) scores (-inf: no key): p = [x - tau]^gamma
    with sum 1, u = [x - tau]^(gamma - 1) where p > 0.  Rows without keys are 0."""
    gamma = 1.0 / (alpha - 1.0)
    top = x.amax(-1, keepdim=True)
    some = top > -math.inf
    y = torch.where(some, x - torch.where(some, top, 0.0), -math.inf)
    lo, hi = torch.full_like(top, -1.0), torch.zeros_like(top)
    for _ in range(60):
        mid = 0.5 * (lo + hi)
        over = ((y - mid).clamp_min(0.0) ** gamma).sum(-1, keepdim=True) >= 1.0
        lo, hi = torch.where(over, mid, lo), torch.where(over, hi, mid)
    z = (y - lo).clamp_min(0.0)
    return z ** gamma, torch.where(z > 0, z.clamp_min(1e-300) ** (gamma - 1.0), 0.0)


def attention64(q, k, v, alpha, scale, causal, dout=None):
    """One sequence: q [n, Hq, d], k, v [n, Hk, d].  Returns o and, with dout,
    dq, dk, dv and the sums of |operands| that a rounding of p multiplies in dv."""
    alpha, scale = (float(torch.tensor(x, dtype=torch.float32)) for x in (alpha, scale))
    n, hq, _ = q.shape
    group = hq // k.shape[1]
    q, k, v = (t.double().cpu() for t in (q, k, v))
    o, dq, dk, dv, dv_abs = (torch.zeros_like(t) for t in (q, q, k, v, v))
    hidden = torch.ones(n, n, dtype=torch.bool).triu(1)
    for h in range(hq):
        g = h // group
        x = (alpha - 1.0) * scale * (q[:, h] @ k[:, g].t())
        if causal:
            x = x.masked_fill(hidden, -math.inf)
        p, u = entmax64(x, alpha)
        o[:, h] = p @ v[:, g]
        if dout is None:
            continue
        do = dout[:, h].double().cpu()
        dp = do @ v[:, g].t()
        ds = u * (dp - (u * dp).sum(-1, keepdim=True) / u.sum(-1, keepdim=True))
        dq[:, h] = scale * (ds @ k[:, g])
        dk[:, g] += scale * (ds.t() @ q[:, h])
        dv[:, g] += p.t() @ do
        dv_abs[:, g] += p.t() @ do.abs()
    return (o,) if dout is None else (o, dq, dk, dv, dv_abs)


def packed64(q, k, v, cu, alpha, scale, causal, dout=None):
    """attention64 of every sequence; rows of no sequence are 0."""
    outs = None
    for a, b in zip(cu[:-1], cu[1:]):
        if b <= a:
            continue
        r = attention64(q[a:b], k[a:b], v[a:b], alpha, scale, causal, None if dout is None else dout[a:b])
        if outs is None:
            like = (q,) if dout is None else (q, q, k, v, v)
            outs = [torch.zeros(t.shape, dtype=torch.float64) for t in like]
        for x, y in zip(outs, r):
            x[a:b] = y
    return outs


def decode64(q, k_cache, v_cache, lengths, k_prefix, v_prefix, alpha, scale):
    alpha, scale = (float(torch.tensor(x, dtype=torch.float32)) for x in (alpha, scale))
    B, hq, d = q.shape
    hk = k_cache.shape[2]
    o = torch.zeros(B, hq, d, dtype=torch.float64)
    cpu = lambda t: t.double().cpu()
    for b in range(B):
        n = min(max(int(lengths[b]), 0), k_cache.shape[1])
        keys, values = cpu(k_cache[b, :n]), cpu(v_cache[b, :n])
        if k_prefix is not None:
            keys, values = torch.cat([cpu(k_prefix), keys]), torch.cat([cpu(v_prefix), values])
        if keys.shape[0] == 0:
            continue
        for h in range(hq):
            g = h // (hq // hk)
            x = (alpha - 1.0) * scale * (keys[:, g] @ cpu(q[b, h]))
            p, _ = entmax64(x[None], alpha)
            o[b, h] = (p @ values[:, g])[0]
    return o


def rotary64(x, weight, positions, freqs, sections, eps, interleaved, dout=None):
    """(y,) or (y, dx, dw) of one of norm_rotary's tensors."""
    x = x.double().cpu()
    n, _, d = x.shape
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double().cpu()
    f, rot = freqs.double().cpu(), 2 * freqs.shape[0]
    pos = positions.cpu().double().view(-1, n)
    axis = [a for a, s in enumerate(sections) for _ in range(s)]
    phi = torch.stack([pos[a] * f[i] for i, a in enumerate(axis)], 1) if rot else torch.zeros(n, 0, dtype=torch.float64)
    co, si = phi.cos()[:, None], phi.sin()[:, None]
    i = torch.arange(rot // 2)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)

    def turn(t, sign):
        t = t.clone()
        a, b = t[..., first].clone(), t[..., second].clone()
        t[..., first], t[..., second] = a * co - sign * b * si, sign * a * si + b * co
        return t

    # (the eps that the library is given, a 32-bit number)
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32)))
    xh = x * r
    y = turn(xh * w, 1.0)
    if dout is None:
        return (y,)
    dy = turn(dout.double().cpu(), -1.0)
    g = dy * w
    return y, r * (g - xh * (g * xh).mean(-1, keepdim=True)), (dy * xh).sum((0, 1))


def check(name, got, want, atol, extra=None):
    """|got - want| <= half a step of got's type + extra + atol, elementwise."""
    got_d = got.double().cpu()
    tol = HALF_STEP[got.dtype] * want.abs() + atol
    if extra is not None:
        tol = tol + extra
    bad = (got_d - want).abs() - tol
    worst = float(bad.max()) if bad.numel() else 0.0
    err = float((got_d - want).abs().max()) if bad.numel() else 0.0
    print("%s: error %.3g, %.3g %s its tolerance" % (name, err, abs(worst), "past" if worst > 0 else "inside"), flush=True)
    assert not torch.isnan(got_d).any(), name
    assert worst <= 0.0, (name, err, worst)
