"""Operators around alpha-entmax attention in a transformer: their plain forms
and the cases on which they are measured.

ops
    rotary  norm_rotary: RMS norm of every query and key head and the rotation
            by the token's position (one position, or time, height and width),
            read from the fused projection's rows; `train` adds its backward
    packed  packed_forward: alpha-entmax attention of sequences of different
            lengths packed into one row of tokens, with grouped heads; `train`
            adds packed_backward
    prefix  prefix_decode: one new token per request against a prefix that all
            requests share and each request's own cache

`own` chooses between the plain forms (elementary torch operations in 32 bits)
and the calls of the library.  Queries and keys are Gaussian, as the norm of a
head leaves them, queries times a temperature c: the larger c, the sparser the
probabilities.  Training cases take alpha 1.5 or 1.25: at alpha = 2 the
gradient jumps where a probability reaches zero, so that two correct results
differ by whole terms wherever a score rounds across the threshold.
"""
import math

import torch

own = False


# ------------------------------------------------------------------- cases

def _rotary(name, tokens, hq, hk, d, dtype, train, axes=1, rot=None, interleaved=False):
    return {"name": name, "op": "rotary", "tokens": tokens, "hq": hq, "hk": hk, "d": d,
            "dtype": dtype, "train": train, "axes": axes, "rot": rot or d, "interleaved": interleaved}


def _packed(name, lens, hq, hk, d, dtype, train, alpha, c, causal=True):
    return {"name": name, "op": "packed", "lens": lens, "hq": hq, "hk": hk, "d": d, "dtype": dtype,
            "train": train, "alpha": alpha, "c": c, "causal": causal}


def _prefix(name, requests, prefix, cap, hq, hk, d, dtype, alpha, c):
    return {"name": name, "op": "prefix", "requests": requests, "prefix": prefix, "cap": cap,
            "hq": hq, "hk": hk, "d": d, "dtype": dtype, "alpha": alpha, "c": c}


def listed():
    return [
        # one decoding step of a small batch: latency
        _rotary("rotary_decode", 16, 32, 8, 128, "bf16", False),
        # a long prompt with images: positions of time, height and width
        _rotary("rotary_prompt_3axes", 16384, 32, 8, 128, "bf16", False, axes=3),
        # a training step's tokens, a ragged number of them, fp32, interleaved pairs
        _rotary("rotary_step_ragged_f32", 8191, 12, 12, 64, "f32", True, interleaved=True),
        # a training step in bf16, half of the dimensions rotated
        _rotary("rotary_step", 32768, 16, 8, 128, "bf16", True, rot=64),
        # a handful of short requests' prompts: launches
        _packed("packed_short_prompts", "17,1,64,130,5", 12, 4, 64, "bf16", False, 1.5, 1.0),
        # prompts of very different lengths, grouped heads
        _packed("packed_prompts", "4096,2048,1111,777,4000,130,2500,1700", 32, 8, 128, "bf16", False, 1.5, 1.0),
        # fine-tuning on packed documents
        _packed("packed_step", "3000,1200,2048,1500,444", 16, 4, 128, "bf16", True, 1.5, 1.0),
        # the same with one long document, head dimension 64, sparser rows
        _packed("packed_step_long", "8192", 16, 16, 64, "bf16", True, 1.5, 4.0),
        # a gradient check's size: fp32, alpha 1.25, both directions of attention
        _packed("packed_step_f32", "400,63,257", 8, 2, 64, "f32", True, 1.25, 1.0, causal=False),
        # one request without a shared prefix: latency
        _prefix("decode_one", 1, 0, 4096, 16, 4, 128, "bf16", 1.5, 1.0),
        # a chat service's system prompt and its users' turns
        _prefix("decode_shared", 64, 8192, 1024, 32, 8, 128, "bf16", 1.5, 1.0),
        # many questions about one long document
        _prefix("decode_long_prefix", 32, 65536, 300, 32, 8, 128, "bf16", 1.5, 2.0),
    ]


def draw(rng):
    """Another case of the ranges of the listed ones."""
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotary", "packed", "packed", "prefix"])
    f32 = rng.random() < 0.2
    dtype = "f32" if f32 else "bf16"
    hq, hk = rng.choice([(32, 8), (16, 8), (16, 4), (16, 16), (12, 4), (12, 12), (8, 1), (14, 2), (4, 4)])
    d = rng.choice([64, 128])
    c = round(math.exp(rng.uniform(math.log(0.5), math.log(8.0))), 3)
    if op == "rotary":
        tokens = min(logint(1, 32768), 32768 * 24 * 128 // ((hq + hk) * d) // (2 if f32 else 1))
        axes = rng.choice([1, 1, 3])
        return {"op": op, "tokens": tokens, "hq": hq, "hk": hk, "d": d, "dtype": dtype,
                "train": rng.random() < 0.5, "axes": axes, "rot": rng.choice([d, d, d // 2]),
                "interleaved": rng.random() < 0.3}
    if op == "packed":
        train = rng.random() < 0.5
        # at most the largest listed case's products, at fp32's sixteenth of the rate
        budget = 16 * 8192 * 4096 * 64 * 3 / (3 if train else 1) / (16 if f32 else 1)
        longest = int(math.sqrt(2 * budget / (hq * d)))
        lens, left = [], budget
        for _ in range(logint(1, 40)):
            n = logint(1, min(8192, longest))
            cost = hq * d * n * n
            if cost <= left:
                lens.append(n)
                left -= cost
        if not lens:
            lens = [longest // 2]
        return {"op": op, "lens": ",".join(map(str, lens)), "hq": hq, "hk": hk, "d": d, "dtype": dtype,
                "train": train, "alpha": rng.choice([1.5, 1.5, 1.25] + ([] if train else [2.0])), "c": c,
                "causal": rng.random() < 0.8}
    prefix = 0 if rng.random() < 0.2 else logint(64, 65536)
    cap = logint(1, 8192)
    # no more than the longest listed prefix's score rows, or the largest cache
    most = min(32 * 32 * 65836 // (hq * (prefix + cap)), 64 * 8 * 1024 * 128 * 4 // (hk * d * cap))
    return {"op": op, "requests": max(1, min(logint(1, 256), most // (4 if f32 else 1))), "prefix": prefix,
            "cap": cap, "hq": hq, "hk": hk, "d": d, "dtype": dtype,
            "alpha": rng.choice([1.5, 1.5, 1.25, 2.0]), "c": c}


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _own_lengths(case):
    """Rows in each request's own cache: spread over 1 .. cap, all different where they can be."""
    B, cap = case["requests"], case["cap"]
    return [cap - (cap - 1) * ((b * 5) % B) // B for b in range(B)]


def _sections(case):
    """Rotated pairs of each axis."""
    pairs = case["rot"] // 2
    if case["axes"] == 1:
        return (pairs,)
    side = pairs * 3 // 8
    return (pairs - 2 * side, side, side)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    d, hq, hk = case["d"], case["hq"], case["hk"]
    if case["op"] == "rotary":
        values = case["tokens"] * (hq + hk) * d
        # in and out; the backward reads both again and writes the gradient
        return {"bytes": values * e * (4 if case["train"] else 2), "flops": values * (24 if case["train"] else 9)}
    if case["op"] == "packed":
        lens = _lens(case)
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lens)
        rows = sum(lens) * d * e
        # q and o (do, dq), k and v (dk, dv); the products as if no probability were zero
        return {"bytes": rows * (2 * hq + 2 * hk + ((2 * hq + 2 * hk) if case["train"] else 0)),
                "flops": pairs * hq * d * (14 if case["train"] else 4)}
    keys = case["prefix"] + sum(_own_lengths(case))
    pairs = case["requests"] * case["prefix"] + sum(_own_lengths(case))
    return {"bytes": keys * hk * d * e * 2 + case["requests"] * hq * d * e * 2, "flops": pairs * hq * d * 4}


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    d, hq, hk = case["d"], case["hq"], case["hk"]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale).to(dt)

    st = {"case": case}
    if case["op"] == "rotary":
        n = case["tokens"]
        # the rows of a fused projection: queries, keys, values side by side
        x = normal(n, (hq + 2 * hk) * d, scale=1.7)
        st["q"] = x[:, :hq * d].view(n, hq, d)
        st["k"] = x[:, hq * d:(hq + hk) * d].view(n, hk, d)
        st["q_weight"] = torch.rand(d, generator=g, device="cuda").add_(0.5).to(dt)
        st["k_weight"] = torch.rand(d, generator=g, device="cuda").add_(0.5).to(dt)
        # rotations per position, from 1 radian down to base^-1 of one
        pairs = case["rot"] // 2
        st["freqs"] = (500000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)).float()
        first = torch.randint(0, 100000, (1,), generator=g, device="cuda", dtype=torch.int32)
        at = torch.arange(n, device="cuda", dtype=torch.int32)
        if case["axes"] == 1:
            st["positions"] = at + first
        else:  # frames of 24 x 32 patches
            st["positions"] = torch.stack([at // 768 + first, at // 32 % 24 + first, at % 32 + first])
        st["sections"] = _sections(case)
        if case["train"]:
            st["dq"], st["dk"] = normal(n, hq, d), normal(n, hk, d)
        return st
    if case["op"] == "packed":
        lens = _lens(case)
        n = sum(lens)
        st["q"], st["k"], st["v"] = normal(n, hq, d, scale=case["c"]), normal(n, hk, d), normal(n, hk, d)
        if case["train"]:
            st["do"] = normal(n, hq, d)
        ends = [0]
        for m in lens:
            ends.append(ends[-1] + m)
        st["cu"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
        if own:  # laid out once for all layers of a step
            import paper_2502_12082_amd as ea
            st["plan"] = ea.packed_plan(st["cu"], n, max_seqlen=max(lens), causal=case["causal"])
        return st
    B, P, cap = case["requests"], case["prefix"], case["cap"]
    st["q"] = normal(B, hq, d, scale=case["c"])
    st["k_cache"], st["v_cache"] = normal(B, cap, hk, d), normal(B, cap, hk, d)
    st["k_prefix"], st["v_prefix"] = (normal(P, hk, d), normal(P, hk, d)) if P else (None, None)
    st["lengths"] = torch.tensor(_own_lengths(case), dtype=torch.int32, device="cuda")
    return st


def run(state):
    case = state["case"]
    if own:
        return _OWN[case["op"]](case, state)
    return _PLAIN[case["op"]](case, state)


# ------------------------------------------------------- the library's calls

def _own_rotary(case, s):
    import paper_2502_12082_amd as ea
    args = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], sections=s["sections"],
                interleaved=case["interleaved"])
    out = ea.norm_rotary(s["q"], s["k"], s["positions"], s["freqs"], **args)
    if case["train"]:
        out += ea.norm_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["freqs"], **args)
    return out


def _own_packed(case, s):
    import paper_2502_12082_amd as ea
    o, res = ea.packed_forward(s["q"], s["k"], s["v"], s["plan"], alpha=case["alpha"], need_bwd=case["train"])
    if case["train"]:
        return (o,) + ea.packed_backward(s["q"], s["k"], s["v"], s["do"], res)
    return o


def _own_prefix(case, s):
    import paper_2502_12082_amd as ea
    return ea.prefix_decode(s["q"], s["k_cache"], s["v_cache"], s["lengths"], k_prefix=s["k_prefix"],
                            v_prefix=s["v_prefix"], alpha=case["alpha"])


# -------------------------------------------------------------- plain forms

def _pairs(x, rot, interleaved):
    """The two halves of every rotated pair of x [..., d], and the dimensions that stay."""
    r, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        return r[..., 0::2], r[..., 1::2], rest
    return r[..., :rot // 2], r[..., rot // 2:], rest


def _unpairs(a, b, rest, interleaved):
    r = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([r, rest], -1)


def _cos_sin(s, dtype):
    """[tokens, 1, pairs] each; far positions need their angles in 64 bits."""
    pos = s["positions"].view(-1, s["q"].shape[0]).double()
    axis = torch.repeat_interleave(torch.arange(len(s["sections"])), torch.tensor(s["sections"])).to(pos.device)
    phi = pos[axis].t() * s["freqs"].double()
    return torch.cos(phi).to(dtype)[:, None], torch.sin(phi).to(dtype)[:, None]


def _plain_rotary(case, s):
    cos, sin = _cos_sin(s, torch.float32)
    rot, inter = case["rot"], case["interleaved"]
    out, grads, dweights = [], [], []
    for x0, w0, dz0 in ((s["q"], s["q_weight"], s.get("dq")), (s["k"], s["k_weight"], s.get("dk"))):
        x, w = x0.float(), w0.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        xh = x * r
        a, b, rest = _pairs(xh * w, rot, inter)
        out.append(_unpairs(a * cos - b * sin, a * sin + b * cos, rest, inter).to(x0.dtype))
        if case["train"]:
            a, b, rest = _pairs(dz0.float(), rot, inter)
            dy = _unpairs(a * cos + b * sin, b * cos - a * sin, rest, inter)
            gw = dy * w
            grads.append((r * (gw - xh * (gw * xh).mean(-1, keepdim=True))).to(x0.dtype))
            dweights.append((dy * xh).sum((0, 1), dtype=torch.float64).float())
    return tuple(out + grads + dweights)


def _threshold(x, gamma, steps=30):
    """tau of every row of x (invalid entries -inf): Newton's steps on the
    convex sum [x - tau]^gamma - 1 from max x - 1, where it is not negative."""
    top = x.amax(-1, keepdim=True)
    tau = top - 1.0
    for _ in range(steps):
        z = (x - tau).clamp_min(0.0)
        u = z if gamma == 2.0 else (z > 0).to(x.dtype) if gamma == 1.0 else z ** (gamma - 1.0)
        tau = tau + (((u * z).sum(-1, keepdim=True) - 1.0) / (gamma * u.sum(-1, keepdim=True))).clamp_min(0.0)
    return tau


def _plain_packed(case, s):
    q, k, v = s["q"], s["k"], s["v"]
    d, group, alpha = case["d"], case["hq"] // case["hk"], case["alpha"]
    scale, gamma = d ** -0.5, 1.0 / (alpha - 1.0)
    o = torch.empty_like(q)
    grads = [torch.empty_like(t) for t in (q, k, v)] if case["train"] else []
    at = 0
    for n in _lens(case):
        rows = slice(at, at + n)
        at += n
        hidden = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1) if case["causal"] else None
        # as many heads at a time as keep a score matrix under a gigabyte
        step = max(1, min(case["hk"], (1 << 28) // (group * n * n)))
        for h0 in range(0, case["hk"], step):
            kh = slice(h0, min(h0 + step, case["hk"]))
            heads = slice(kh.start * group, kh.stop * group)
            qf = q[rows, heads].float().transpose(0, 1).unflatten(0, (-1, group))
            kf, vf = (t[rows, kh].float().transpose(0, 1).unsqueeze(1) for t in (k, v))
            x = ((alpha - 1.0) * scale) * (qf @ kf.transpose(-1, -2).contiguous())
            if hidden is not None:
                x.masked_fill_(hidden, -math.inf)
            z = (x - _threshold(x, gamma)).clamp_min(0.0)
            p = z if gamma == 1.0 else z ** gamma
            o[rows, heads] = (p @ vf).flatten(0, 1).transpose(0, 1).to(o.dtype)
            if not case["train"]:
                continue
            u = z ** (gamma - 1.0)
            dof = s["do"][rows, heads].float().transpose(0, 1).unflatten(0, (-1, group))
            dp = dof @ vf.transpose(-1, -2).contiguous()
            ds = u * (dp - (u * dp).sum(-1, keepdim=True) / u.sum(-1, keepdim=True)) * scale
            grads[0][rows, heads] = (ds @ kf).flatten(0, 1).transpose(0, 1).to(q.dtype)
            grads[1][rows, kh] = (ds.transpose(-1, -2).contiguous() @ qf).sum(1).transpose(0, 1).to(q.dtype)
            grads[2][rows, kh] = (p.transpose(-1, -2).contiguous() @ dof).sum(1).transpose(0, 1).to(q.dtype)
    return (o, *grads) if case["train"] else o


def _plain_prefix(case, s):
    d, hk, group, alpha = case["d"], case["hk"], case["hq"] // case["hk"], case["alpha"]
    B, P, cap = case["requests"], case["prefix"], case["cap"]
    c, gamma = (alpha - 1.0) * d ** -0.5, 1.0 / (alpha - 1.0)
    q = s["q"].float().view(B, hk, group, d)
    own_k, own_v = (s[t].float().transpose(1, 2) for t in ("k_cache", "v_cache"))
    x = c * (q @ own_k.transpose(-1, -2).contiguous())
    behind = torch.arange(cap, device=q.device) >= s["lengths"][:, None]
    x.masked_fill_(behind[:, None, None], -math.inf)
    if P:
        rows = q.transpose(0, 1).reshape(hk, B * group, d)
        pre_k, pre_v = (s[t].float().transpose(0, 1) for t in ("k_prefix", "v_prefix"))
        shared = c * (rows @ pre_k.transpose(-1, -2).contiguous())
        x = torch.cat([shared.view(hk, B, group, P).transpose(0, 1), x], -1)
    p = (x - _threshold(x, gamma)).clamp_min(0.0)
    p = p if gamma == 1.0 else p ** gamma
    o = p[..., P:] @ own_v
    if P:
        shared = p[..., :P].transpose(0, 1).reshape(hk, B * group, P) @ pre_v
        o = o + shared.view(hk, B, group, d).transpose(0, 1)
    return o.reshape(B, case["hq"], d).to(s["q"].dtype)


_PLAIN = {"rotary": _plain_rotary, "packed": _plain_packed, "prefix": _plain_prefix}
_OWN = {"rotary": _own_rotary, "packed": _own_packed, "prefix": _own_prefix}


# ----------------------------------------------- the definition, in 64 bits

def _entmax64(x, alpha):
    """(p, u) of the rows of x, the scores before the factor alpha - 1, by
    bisection of the threshold: u = p^(2 - alpha) where p > 0."""
    y = x * (alpha - 1.0)
    hi = y.amax(-1, keepdim=True)
    lo = hi - 1.0
    power = 1.0 / (alpha - 1.0)
    for _ in range(56):
        mid = 0.5 * (lo + hi)
        z = torch.relu(y - mid)
        mass = (z if power == 1.0 else z * z if power == 2.0 else z.pow(power)).sum(-1, keepdim=True)
        lo, hi = torch.where(mass >= 1.0, mid, lo), torch.where(mass >= 1.0, hi, mid)
    p = torch.relu(y - lo).pow(power)
    return p, torch.where(p > 0, p.pow(2.0 - alpha), 0.0)


def _exact_rotary(case, s):
    n, pairs, inter = case["tokens"], case["rot"] // 2, case["interleaved"]
    pos = s["positions"].reshape(case["axes"], n).double()
    turn = torch.empty(n, pairs, dtype=torch.complex128, device=pos.device)
    at = 0
    for axis, count in enumerate(_sections(case)):
        phi = torch.outer(pos[axis], s["freqs"].double()[at:at + count])
        turn[:, at:at + count] = torch.polar(torch.ones_like(phi), phi)
        at += count
    first = 2 * torch.arange(pairs) if inter else torch.arange(pairs)
    second = first + (1 if inter else pairs)
    outs, grads, dweights = [], [], []
    for name in ("q", "k"):
        x, w = s[name].double(), s[name + "_weight"].double()
        xh = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        y = xh * w
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        outs.append(y)
        if case["train"]:
            dy = s["d" + name].double().clone()
            z = torch.complex(dy[..., first], dy[..., second]) * turn.conj()[:, None]
            dy[..., first], dy[..., second] = z.real, z.imag
            dweights.append((dy * xh).sum((0, 1)))
            dy = dy * w
            dy = dy - xh * (dy * xh).mean(-1, keepdim=True)
            grads.append(dy / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6))
    return tuple(outs + grads + dweights)


def _exact_packed(case, s):
    q, k, v = (s[t].double() for t in ("q", "k", "v"))
    group, scale = case["hq"] // case["hk"], case["d"] ** -0.5
    o, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    start = 0
    for n in _lens(case):
        end = start + n
        for h in range(case["hq"]):
            qh, kh, vh = q[start:end, h], k[start:end, h // group], v[start:end, h // group]
            x = scale * (qh @ kh.t())
            if case["causal"]:
                x = x.masked_fill(torch.arange(n, device=x.device) > torch.arange(n, device=x.device)[:, None],
                                  -math.inf)
            p, u = _entmax64(x, case["alpha"])
            o[start:end, h] = p @ vh
            if case["train"]:
                do = s["do"][start:end, h].double()
                dp = do @ vh.t()
                ds = u * dp - u * ((u * dp).sum(-1) / u.sum(-1))[:, None]
                dq[start:end, h] = scale * (ds @ kh)
                dk[start:end, h // group] += scale * (ds.t() @ qh)
                dv[start:end, h // group] += p.t() @ do
        start = end
    return (o, dq, dk, dv) if case["train"] else o


def _exact_prefix(case, s):
    group, scale, P = case["hq"] // case["hk"], case["d"] ** -0.5, case["prefix"]
    o = torch.zeros(case["requests"], case["hq"], case["d"], dtype=torch.float64, device=s["q"].device)
    for b, m in enumerate(_own_lengths(case)):
        for h in range(case["hk"]):
            keys, values = s["k_cache"][b, :m, h].double(), s["v_cache"][b, :m, h].double()
            if P:
                keys = torch.cat([s["k_prefix"][:, h].double(), keys])
                values = torch.cat([s["v_prefix"][:, h].double(), values])
            mine = slice(h * group, (h + 1) * group)
            p, _ = _entmax64(scale * (s["q"][b, mine].double() @ keys.t()), case["alpha"])
            o[b, mine] = p @ values
    return o


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "packed": _exact_packed, "prefix": _exact_prefix}[case["op"]](case, s)
