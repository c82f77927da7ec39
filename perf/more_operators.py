"""Training through coreset attention, and serving drafted and image tokens from
the 4-bit cache: the operators, measured.

Five kinds of calls:

  grad     the gradients of coreset attention with respect to queries, keys,
           values and the coreset's log-weights (probabilities formed anew),
  axes     query and key rows turned by positions with several axes (time,
           height, width), or turned back (the gradient of that),
  tree     a tree of drafted tokens: from every token's parent the set of
           drafts that it attends to, and its position,
  attend   attention of the tree's tokens over the cached rows before the
           drafts and over their own ancestors among the drafts,
  keep     the accepted path's rows moved to the end of the cache's rows (read
           back here as the values they stand for, with the key bounds).

``run`` computes them in plain torch, or with ``own`` set through the library.

Cached rows.  A row of d channels is d/32 groups of 32 channels; a group holds
32 codes of 4 bits (sign, 2 exponent bits, 1 mantissa bit: 0, .5, 1, 1.5, 2, 3,
4, 6 and their negatives; channel 2i in the low half of byte i) and one scale
byte s, which stands for 2^(s-127).  Blocks are 64 rows; bounds[b, h, k] holds
the least and the largest cached key value of every channel over block k's rows.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 64


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _grad(name, B, H, n_q, n, n_out, d, dtype, out, weighted):
    """n_out of n key rows are the coreset; out: the type of the attention's
    output and of its gradient; weighted: with log-weights."""
    return dict(name=name, op="grad", B=B, H=H, n_q=n_q, n=n, n_out=n_out, d=d, dtype=dtype,
                out=out, weighted=weighted)


def _axes(name, B, Hq, Hk, T, d, rot, axes, order, dtype, layout, inverse):
    """order: the axes take runs of pairs ("runs"), or pairs in turn ("turns")."""
    return dict(name=name, op="axes", B=B, Hq=Hq, Hk=Hk, T=T, d=d, rot=rot, axes=axes,
                order=order, dtype=dtype, layout=layout, inverse=inverse)


def _tree(name, B, T, width):
    """T drafted tokens per sequence, `width` of them per level."""
    return dict(name=name, op="tree", B=B, T=T, width=width)


def _attend(name, B, Hq, Hk, T, width, n, d, dtype, ragged):
    """T drafted tokens behind a cache of n - T rows (the longest sequence's;
    ragged: others are shorter, and some of their T tokens are padding)."""
    return dict(name=name, op="attend", B=B, Hq=Hq, Hk=Hk, T=T, width=width, n=n, d=d,
                dtype=dtype, ragged=ragged)


def _keep(name, B, Hk, T, P, n, d):
    """Up to P of T drafted rows are kept, of caches with n rows."""
    return dict(name=name, op="keep", B=B, Hk=Hk, T=T, P=P, n=n, d=d)


def listed():
    return [
        # one layer's step on a small float32 model: latency
        _grad("grad_small", 1, 1, 1024, 1024, 32, 64, "fp32", "fp32", False),
        # a long context, 128 coreset rows between 32 sinks and a window of 32
        _grad("grad_long", 4, 16, 16384, 16384, 192, 128, "bf16", "bf16", True),
        # a wide coreset, odd sizes everywhere, the output kept in float32
        _grad("grad_wide", 3, 5, 2047, 4095, 333, 128, "bf16", "fp32", True),
        # a prompt of images and video: three axes, runs of pairs
        _axes("axes_prompt", 1, 32, 8, 16384, 128, 128, 3, "runs", "bf16", "half", False),
        # the gradient: float32 rows, two axes in turn, half of the head turned, odd length
        _axes("axes_grad", 3, 12, 12, 2047, 64, 32, 2, "turns", "fp32", "interleaved", True),
        # the drafts of one step
        _tree("tree_step", 8, 64, 8),
        # many sequences, large trees
        _tree("tree_large", 64, 1024, 16),
        # a few drafts of a small float32 model over a short cache: launches and latency
        _attend("attend_short", 2, 16, 4, 9, 3, 1000, 64, "fp32", True),
        # 64 drafts for each of 8 sequences of different lengths, 4 queries per key head
        _attend("attend_step", 8, 32, 8, 64, 8, 65536, 128, "bf16", True),
        # one large tree over a long prompt
        _attend("attend_large", 1, 32, 8, 1021, 16, 16384, 128, "bf16", False),
        # up to 7 of 64 drafts accepted, 8 sequences
        _keep("keep_step", 8, 8, 64, 7, 8192, 128),
        # hundreds of rows for each of 64 sequences
        _keep("keep_many", 64, 8, 1024, 500, 4096, 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("grad", "grad", "grad", "grad", "axes", "tree", "attend", "attend", "attend",
                     "keep"))
    d = rng.choice((32, 64, 128, 128))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    Hk = rng.choice((1, 2, 3, 4, 8, 8))
    G = rng.choice((1, 2, 3, 4, 4, 6, 8, 16))
    if op == "grad":
        B, H = _log(rng, 1, 8), rng.choice((1, 2, 3, 8, 12, 16))
        n_out = _log(rng, 1, 1024)
        # at most a fifth of the largest listed case's products
        most = min(16384, max(1, 4 * 16 * 16384 * 192 * 128 // (5 * B * H * n_out * d)))
        n_q = _log(rng, 1, most)
        n = max(n_out, _log(rng, n_out, 16384))
        return dict(op=op, B=B, H=H, n_q=n_q, n=n, n_out=n_out, d=d, dtype=dtype,
                    out=dtype if rng.random() < 0.6 else rng.choice(("bf16", "fp32")),
                    weighted=rng.random() < 0.5)
    if op == "axes":
        rot = d if rng.random() < 0.6 else rng.choice([r for r in (16, 32, 64) if r <= d])
        B = _log(rng, 1, 32)
        T = _log(rng, 1, max(1, 16384 * 40 // (B * Hk * (G + 1)))) if rng.random() < 0.7 else 1
        return dict(op=op, B=B, Hq=Hk * G, Hk=Hk, T=min(T, 16384), d=d, rot=rot,
                    axes=rng.choice((1, 2, 3, 3, 4)), order=rng.choice(("runs", "turns")),
                    dtype=dtype, layout=rng.choice(("half", "interleaved")),
                    inverse=rng.random() < 0.4)
    T = _log(rng, 1, 1024)
    width = min(T, _log(rng, 1, 32))
    if op == "tree":
        return dict(op=op, B=_log(rng, 1, 64), T=T, width=width)
    if op == "attend":
        G = min(G, 16 if T <= 64 else 4)
        n = _log(rng, max(T, 64), 65536 if T <= 64 else 16384)
        B = _log(rng, 1, min(64, max(1, 4 * 65536 // n)) if T <= 64 else 2)
        return dict(op=op, B=B, Hq=Hk * G, Hk=Hk, T=T, width=width, n=n, d=d, dtype=dtype,
                    ragged=rng.random() < 0.5)
    T = max(T, 2)
    return dict(op=op, B=_log(rng, 1, 64), Hk=Hk, T=T, P=_log(rng, 1, T // 2),
                n=_log(rng, T, 4096), d=d)


def _places(case):
    """(rows before the drafts, number of drafts) of every sequence, as lists."""
    B, T, n = case["B"], case["T"], case["n"]
    at, count = [], []
    for b in range(B):
        rows = n - T
        if case.get("ragged", True) and b:
            rows = rows * ((37 * b) % 61 + 3) // 64
        at.append(rows)
        count.append(T - (b % 3) * T // 5 if case.get("ragged", False) else T)
    return at, count


def _kept(case):
    """How many drafts of every sequence are accepted."""
    P = case["P"]
    return [P - (b * 5) % P if b else P for b in range(case["B"])]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=gen.device, dtype=torch.float32)


def _ints(values, device):
    return torch.tensor(values, dtype=torch.int32, device=device)


def _key_rows(gen, B, H, n, d):
    """Key rows: N(0,1), a few channels three times as large, and an offset of
    their own for every 64 rows, so that blocks differ."""
    x = _randn(gen, B, H, n, d)
    x *= torch.where(_randn(gen, H, 1, d) > 1.8, 3.0, 1.0)
    drift = 0.7 * _randn(gen, B, H, (n + BLOCK - 1) // BLOCK, d)
    return x + drift.repeat_interleave(BLOCK, 2)[:, :, :n]


def _fill_cache(gen, case):
    """A cache that holds n rows of every sequence."""
    B, H, n, d = case["B"], case["Hk"], case["n"], case["d"]
    nb = (n + BLOCK - 1) // BLOCK
    u8 = dict(dtype=torch.uint8, device=gen.device)
    c = dict(k_codes=torch.empty(B, H, n, d // 2, **u8),
             k_scales=torch.empty(B, H, n, d // 32, **u8),
             v_codes=torch.empty(B, H, n, d // 2, **u8),
             v_scales=torch.empty(B, H, n, d // 32, **u8),
             bounds=torch.empty(B, H, nb, 2, d, dtype=torch.bfloat16, device=gen.device))
    for b in range(B):
        k = _key_rows(gen, 1, H, n, d)
        c["k_codes"][b:b + 1], c["k_scales"][b:b + 1] = _encode(k)
        k = _decode(c["k_codes"][b], c["k_scales"][b])
        k = torch.nn.functional.pad(k, (0, 0, 0, nb * BLOCK - n), mode="replicate") \
            .view(H, nb, BLOCK, d)  # copies of the last row change no bound
        c["bounds"][b, :, :, 0], c["bounds"][b, :, :, 1] = k.amin(2), k.amax(2)
        del k
        c["v_codes"][b:b + 1], c["v_scales"][b:b + 1] = _encode(_randn(gen, 1, H, n, d))
    return c


def _parents(gen, B, T, width):
    """Level by level, every token's parent one of the level before it."""
    t = torch.arange(T, device=gen.device)
    level = torch.div(t, width, rounding_mode="floor")
    pick = torch.randint(0, width, (B, T), generator=gen, device=gen.device)
    return torch.where(level > 0, (level - 1) * width + pick, -1).to(torch.int32)


def _axis_positions(gen, case):
    """Images and video: frames of a grid, each token's frame, row and column
    (and, with four axes, the clip), behind a text of random length."""
    B, T = case["B"], case["T"]
    t = torch.arange(T, device=gen.device)
    wide = max(1, int(math.sqrt(T) / 2))
    high = max(1, wide - 1)

    def part(step, size):
        return torch.div(t, step, rounding_mode="floor") % size
    axes = [part(wide * high, 1 << 20), part(wide, high), part(1, wide), part(4096, 1 << 20)]
    first = torch.randint(0, 100000, (B, 1, 1), generator=gen, device=gen.device)
    return (first + torch.stack(axes, -1)[:, :case["axes"]]).to(torch.int32)


def prepare(case, seed):
    device = torch.device("cuda" if torch.cuda.is_available() else "cpu")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    s = {"case": case}
    B = case["B"]
    if case["op"] == "grad":
        H, n_q, n, m, d = (case[x] for x in ("H", "n_q", "n", "n_out", "d"))
        dt = DTYPES[case["dtype"]]
        s["Q"] = _randn(gen, B, H, n_q, d).to(dt)
        k = _randn(gen, B, H, n, d)
        # one key row in twenty is four times as long
        k *= torch.where(torch.rand(B, H, n, 1, generator=gen, device=device) < 0.05, 4.0, 1.0)
        s["K"] = k.to(dt)
        s["V"] = _randn(gen, B, H, n, d).to(dt)
        pick = torch.rand(B, H, n, generator=gen, device=device).argsort(-1)[..., :m]
        s["idx"] = pick.sort(-1)[0].to(torch.int32).contiguous()
        s["dO"] = _randn(gen, B, H, n_q, d).to(DTYPES[case["out"]])
        s["logw"] = None
        if case["weighted"]:
            # a third of the rows, at both ends, stand for themselves, the others for n / n_out
            j = torch.arange(m, device=device)
            middle = (j >= m // 6) & (j < m - m // 6)
            s["logw"] = torch.where(middle, math.log(n / m), 0.0).float().expand(B, H, m) \
                .contiguous()
        return s
    if case["op"] == "axes":
        T, d, rot, dt = case["T"], case["d"], case["rot"], DTYPES[case["dtype"]]
        s["X"] = _randn(gen, B, case["Hq"], T, d).to(dt)
        s["Y"] = _randn(gen, B, case["Hk"], T, d).to(dt)
        s["pos"] = _axis_positions(gen, case)
        i = torch.arange(rot // 2, device=device)
        axis = i * case["axes"] * 2 // rot if case["order"] == "runs" else i % case["axes"]
        s["axis"] = axis.to(torch.int32)
        f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        s["turns"] = (f / (2 * math.pi)).to(device)
        return s
    if case["op"] == "tree":
        s["parents"] = _parents(gen, B, case["T"], case["width"])
        s["at"] = torch.randint(0, 100000, (B,), generator=gen, device=device).to(torch.int32)
        return s
    at, count = _places(case)
    s["at"] = _ints(at, device)
    s["cache"] = _fill_cache(gen, case)
    if case["op"] == "attend":
        T = case["T"]
        s["count"] = _ints(count, device) if case["ragged"] else None
        s["seen"] = _ancestors(_parents(gen, B, T, case["width"]))[0]
        s["Q"] = _randn(gen, B, case["Hq"], T, case["d"]).to(DTYPES[case["dtype"]])
        return s
    # accepted paths: the first draft, then ones behind the kept rows' places (so that a pass
    # over the same state moves the same rows again), -1 behind
    T, P = case["T"], case["P"]
    rest = torch.rand(B, T - P, generator=gen, device=device).argsort(-1)[:, :P - 1].sort(-1)[0] + P
    path = torch.cat((torch.zeros(B, 1, dtype=rest.dtype, device=device), rest), 1)
    there = torch.arange(P, device=device) < _ints(_kept(case), device).unsqueeze(1)
    s["path"] = torch.where(there, path, -1).to(torch.int32)
    return s


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _encode(x):
    """Codes [.., d/2] and scale bytes [.., d/32] of finite float32 rows [.., d]."""
    g = x.unflatten(-1, (-1, 32))
    m, p = torch.frexp(g.abs().amax(-1))
    e = (p - torch.where(m <= 0.875, 3, 2)).clamp(-125, 125)
    e = torch.where(m == 0, torch.full_like(e, -125), e)
    y = torch.ldexp(g.abs(), -e.unsqueeze(-1))
    c = (y > 0.25).to(torch.uint8)
    c += y >= 0.75
    c += y > 1.25
    c += y >= 1.75
    c += y > 2.5
    c += y >= 3.5
    c += y > 5.0
    c |= (g < 0).to(torch.uint8) << 3
    c = c.flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    """float32 rows [.., d] that codes and scale bytes stand for."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    m = (c & 7).float()
    # 0, .5, 1, 1.5 then 2, 3, 4, 6
    v = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2.0, m * 2.0 - 8.0))
    v = torch.where(c >= 8, -v, v).unflatten(-1, (-1, 32))
    return torch.ldexp(v, (scales.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)


def _plain_grad(s):
    case = s["case"]
    B, H, n, m, d = (case[x] for x in ("B", "H", "n", "n_out", "d"))
    at = s["idx"].long().unsqueeze(-1).expand(B, H, m, d)
    q, k, v = s["Q"].float(), s["K"].gather(2, at).float(), s["V"].gather(2, at).float()
    do = s["dO"].float()
    c = 1.0 / math.sqrt(d)
    p = (q @ k.transpose(-1, -2)).mul_(c)
    if s["logw"] is not None:
        p += s["logw"].unsqueeze(2)
    p = torch.exp_(p.sub_(p.amax(-1, keepdim=True)))
    p /= p.sum(-1, keepdim=True)
    dv = p.transpose(-1, -2) @ do
    ds = do @ v.transpose(-1, -2)
    ds = (ds - (p * ds).sum(-1, keepdim=True)) * p
    dq = (ds @ k) * c
    dk = (ds.transpose(-1, -2) @ q) * c
    dt = DTYPES[case["dtype"]]
    full = [torch.zeros(B, H, n, d, dtype=dt, device=q.device).scatter_(2, at, g.to(dt))
            for g in (dk, dv)]
    out = dict(dQ=dq.to(dt), dK=full[0], dV=full[1])
    if s["logw"] is not None:
        out["dlogw"] = ds.sum(2, dtype=torch.float64).float()
    return out


def _plain_axes(s):
    case = s["case"]
    rot, inter = case["rot"], case["layout"] == "interleaved"
    pos = s["pos"][..., s["axis"].long()].double().unsqueeze(1)  # [B, 1, T, rot / 2]
    angle = pos * s["turns"] * (2 * math.pi)
    cos, sin = angle.cos().float(), angle.sin().float()
    if case["inverse"]:
        sin = -sin

    def turn(x):
        a = x.float()
        r = a[..., :rot]
        lo, hi = (r[..., 0::2], r[..., 1::2]) if inter else r.chunk(2, -1)
        lo, hi = lo * cos - hi * sin, hi * cos + lo * sin
        r = torch.stack((lo, hi), -1).flatten(-2) if inter else torch.cat((lo, hi), -1)
        return torch.cat((r, a[..., rot:]), -1).to(x.dtype)

    return turn(s["X"]), turn(s["Y"])


def _ancestors(parents):
    """Which drafts each draft attends to (itself and its ancestors: bit j % 64
    of word j / 64 is draft j), and its depth."""
    B, T = parents.shape
    j = torch.arange(T, device=parents.device)
    see = ((parents.unsqueeze(-1) == j) | (j.unsqueeze(-1) == j)).float()  # [B, T, T]
    for _ in range(max(1, (T - 1).bit_length())):
        see = ((see @ see) > 0).float()  # ancestors up to twice as far
    depth = see.sum(-1).to(torch.int32) - 1
    words = (T + 63) // 64
    bits = torch.nn.functional.pad(see.to(torch.int64), (0, words * 64 - T)).view(B, T, words, 64)
    return (bits << torch.arange(64, device=parents.device)).sum(-1), depth


def _plain_tree(s):
    seen, depth = _ancestors(s["parents"])
    return seen, s["at"].unsqueeze(1) + depth


def _plain_attend(s):
    case, c = s["case"], s["cache"]
    B, Hq, H, T, d, n = (case[x] for x in ("B", "Hq", "Hk", "T", "d", "n"))
    dev = s["Q"].device
    q = s["Q"].float().view(B, H, Hq // H * T, d)
    # a cached row is seen if it lies before the drafts, or is a draft whose bit is set
    bits = (s["seen"].unsqueeze(-1) >> torch.arange(64, device=dev)) & 1
    bits = bits.flatten(2)[..., :T] > 0
    t = torch.arange(T, device=dev)
    there = t < s["count"].unsqueeze(1) if s["count"] is not None else (t >= 0).expand(B, T)
    bits = bits & there.unsqueeze(1)
    row = torch.arange(n, device=dev) - s["at"].unsqueeze(1)  # [B, n]: the draft it holds
    inside = (row >= 0) & (row < T)
    seen = bits.gather(2, row.clamp(0, T - 1).unsqueeze(1).expand(B, T, n)) & inside.unsqueeze(1)
    seen = (seen | (row < 0).unsqueeze(1)).view(B, 1, 1, T, n)
    seen = seen.expand(B, 1, Hq // H, T, n).reshape(B, 1, Hq // H * T, n)
    k = _decode(c["k_codes"], c["k_scales"])
    v = _decode(c["v_codes"], c["v_scales"])
    p = q @ k.transpose(-1, -2)
    p *= 1.0 / math.sqrt(d)
    p = p.masked_fill_(~seen, -torch.inf)
    p = torch.exp_(p.sub_(p.amax(-1, keepdim=True).clamp(min=-3e38)))
    o = (p @ v) / p.sum(-1, keepdim=True).clamp(min=1e-37)
    o = o.view(B, Hq, T, d) * there.view(B, 1, T, 1)
    return o.to(DTYPES[case["dtype"]])


def _plain_keep(s):
    case, c = s["case"], s["cache"]
    B, H, P, d, n = (case[x] for x in ("B", "Hk", "P", "d", "n"))
    dev = s["at"].device
    at, path = s["at"].long().unsqueeze(1), s["path"].long()
    i = torch.arange(B, device=dev).unsqueeze(1)
    p = torch.arange(P, device=dev)
    moved = path >= 0
    to = at + p
    source = torch.where(moved, at + path, to)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        c[name][i, :, to] = c[name][i, :, source]
    end = at + moved.sum(1, keepdim=True)  # [B, 1]
    # the blocks from the last row before the drafts to the last kept row, over the rows up to it
    touched = (P + BLOCK - 2) // BLOCK + 2
    first = torch.div((at - 1).clamp(min=0), BLOCK, rounding_mode="floor")
    k = first + torch.arange(touched, device=dev)
    rows = k.unsqueeze(-1) * BLOCK + torch.arange(BLOCK, device=dev)
    there = (rows < end.unsqueeze(-1)).view(B, 1, touched, BLOCK, 1)
    at_rows = rows.clamp(max=n - 1).flatten(1)
    x = _decode(c["k_codes"][i, :, at_rows].transpose(1, 2),
                c["k_scales"][i, :, at_rows].transpose(1, 2)).view(B, H, touched, BLOCK, d)
    lo = torch.where(there, x, torch.inf).amin(3)
    hi = torch.where(there, x, -torch.inf).amax(3)
    bounds = torch.stack((lo, hi), 3).to(torch.bfloat16)
    # a block behind the last row stands for the first one again
    full = k * BLOCK < end
    k = torch.where(full, k, k[:, :1])
    bounds = torch.where(full.view(B, 1, touched, 1, 1), bounds, bounds[:, :, :1])
    c["bounds"][i, :, k] = bounds.transpose(1, 2)
    out = [_decode(c[x + "_codes"][i, :, to].transpose(1, 2),
                   c[x + "_scales"][i, :, to].transpose(1, 2)).to(torch.bfloat16) for x in "kv"]
    return end.squeeze(1).to(torch.int32), out[0], out[1], c["bounds"]


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if not own:
        return {"grad": _plain_grad, "axes": _plain_axes, "tree": _plain_tree,
                "attend": _plain_attend, "keep": _plain_keep}[op](state)
    return _own(state, op)


def _own(s, op):
    from paper_2606_10944_amd import (Q4Cache, thin_attention_backward, thin_q4_keep, thin_q4_load,
                                      thin_q4_tree, thin_q4_tree_attention, thin_rotary_axes)
    case = s["case"]
    if op == "grad":
        g = thin_attention_backward(s["Q"], s["K"], s["V"], s["idx"], s["dO"], logw=s["logw"],
                                    need_logw=s["logw"] is not None)
        return dict(zip(("dQ", "dK", "dV", "dlogw"), g))
    if op == "axes":
        return thin_rotary_axes(s["X"], s["pos"], s["turns"], s["axis"], Y=s["Y"],
                                layout=case["layout"], inverse=case["inverse"])
    if op == "tree":
        return thin_q4_tree(s["parents"], s["at"])
    if "handle" not in s:
        s["handle"] = Q4Cache.over(**s["cache"])
    cache = s["handle"]
    if op == "attend":
        return thin_q4_tree_attention(s["Q"], cache, s["at"], s["seen"], count=s["count"])
    end = thin_q4_keep(cache, s["at"], s["path"])
    k, v = thin_q4_load(cache, s["at"], case["P"], dtype=torch.bfloat16)
    return end, k, v, cache.bounds


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    B = case["B"]
    if case["op"] == "grad":
        H, n_q, n, m, d = (case[x] for x in ("H", "n_q", "n", "n_out", "d"))
        size, out = (2 if case[x] == "bf16" else 4 for x in ("dtype", "out"))
        S = B * H
        # queries, the output's gradient and the coreset read; every gradient written whole;
        # five products
        return {"bytes": S * (n_q * d * (2 * size + out) + m * (2 * d * size + 4) + 2 * n * d * size
                              + (8 * m if case["weighted"] else 0)),
                "flops": 10 * S * n_q * m * d}
    if case["op"] == "axes":
        rows = B * (case["Hq"] + case["Hk"]) * case["T"]
        # each channel read and written once; two products and a sum for each
        return {"bytes": 2 * rows * case["d"] * (2 if case["dtype"] == "bf16" else 4)
                + B * case["T"] * case["axes"] * 4, "flops": 3 * rows * case["rot"]}
    T = case["T"]
    words = (T + 63) // 64
    if case["op"] == "tree":
        return {"bytes": B * T * (4 + 8 * words + 4) + 4 * B, "flops": B * T * words}
    at, count = _places(case)
    H, d = case["Hk"], case["d"]
    row = d // 2 + d // 32  # one cached row, keys or values
    if case["op"] == "attend":
        size, Hq, width = 2 if case["dtype"] == "bf16" else 4, case["Hq"], case["width"]
        keys = sum(a + c for a, c in zip(at, count))
        # a draft sees one draft of every level up to its own
        pairs = sum(c * a + sum(t // width + 1 for t in range(c)) for a, c in zip(at, count))
        return {"bytes": H * keys * 2 * row + 2 * Hq * sum(count) * d * size
                + sum(count) * words * 8, "flops": 4 * Hq * pairs * d}
    kept = sum(_kept(case))
    # kept rows read and written, then P rows read back and written as values; the bounds of
    # the blocks that hold kept rows, whose other keys are read
    blocks = sum((a + k - 1) // BLOCK - max(a - 1, 0) // BLOCK + 1
                 for a, k in zip(at, _kept(case)))
    return {"bytes": H * (kept * 4 * row + B * case["P"] * 2 * (row + 2 * d)
                          + blocks * (4 * d + BLOCK // 2 * row)), "flops": 2 * H * kept * d}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_values(codes, scales):
    """What codes and scale bytes stand for, by table, in 64 bits."""
    table = torch.tensor(GRID + [-v for v in GRID], dtype=torch.float64, device=codes.device)
    v = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64,
                    device=codes.device)
    v[..., 0::2] = table[(codes % 16).int()]
    v[..., 1::2] = table[torch.div(codes, 16, rounding_mode="floor").int()]
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _exact_grad(s, case):
    B, H, n_q, n, m, d = (case[x] for x in ("B", "H", "n_q", "n", "n_out", "d"))
    f64 = dict(dtype=torch.float64, device=s["Q"].device)
    out = dict(dQ=torch.empty(B, H, n_q, d, **f64), dK=torch.zeros(B, H, n, d, **f64),
               dV=torch.zeros(B, H, n, d, **f64), dlogw=torch.empty(B, H, m, **f64))
    for b in range(B):
        for h in range(H):
            i = s["idx"][b, h].long()
            q, do = s["Q"][b, h].double(), s["dO"][b, h].double()
            k, v = s["K"][b, h, i].double(), s["V"][b, h, i].double()
            z = q @ k.T / math.sqrt(d)
            if s["logw"] is not None:
                z = z + s["logw"][b, h].double()
            p = torch.softmax(z, -1)
            # the derivative of a softmax row: diag(p) - p p^T
            g = do @ v.T
            dz = p * g - p * (p * g).sum(-1, keepdim=True)
            out["dQ"][b, h] = dz @ k / math.sqrt(d)
            out["dK"][b, h, i] = dz.T @ q / math.sqrt(d)
            out["dV"][b, h, i] = p.T @ do
            out["dlogw"][b, h] = dz.sum(0)
    if s["logw"] is None:
        del out["dlogw"]
    return out


def _exact_axes(s, case):
    B, T, rot = case["B"], case["T"], case["rot"]
    pair = torch.arange(rot // 2, device=s["X"].device)
    i, j = pair, pair + rot // 2
    if case["layout"] == "interleaved":
        i, j = 2 * pair, 2 * pair + 1
    turn = torch.empty(B, 1, T, rot // 2, dtype=torch.float64, device=s["X"].device)
    for p in range(rot // 2):
        at = s["pos"][:, :, int(s["axis"][p])].double()
        turn[:, 0, :, p] = (at * s["turns"][p]) % 1.0
    z = torch.polar(torch.ones_like(turn), turn * (-2 * math.pi if case["inverse"] else
                                                   2 * math.pi))
    out = []
    for x in (s["X"], s["Y"]):
        y = x.double()
        w = torch.complex(y[..., i], y[..., j]) * z
        y[..., i], y[..., j] = w.real, w.imag
        out.append(y)
    return tuple(out)


def _exact_attend(s, case):
    B, Hq, H, T, d, n = (case[x] for x in ("B", "Hq", "Hk", "T", "d", "n"))
    at, count = _places(case)
    c = s["cache"]
    G = Hq // H
    out = torch.zeros(B, Hq, T, d, dtype=torch.float64, device=s["Q"].device)
    for b in range(B):
        a, m = at[b], count[b]
        see = torch.ones(m, a + m, dtype=torch.bool, device=out.device)
        for j in range(m):
            see[:, a + j] = torch.div(s["seen"][b, :m, j // 64], 2 ** (j % 64),
                                      rounding_mode="floor") % 2 == 1 if j % 64 < 63 \
                else s["seen"][b, :m, j // 64] < 0
        for h in range(H):
            k = _exact_values(c["k_codes"][b, h, :a + m], c["k_scales"][b, h, :a + m])
            v = _exact_values(c["v_codes"][b, h, :a + m], c["v_scales"][b, h, :a + m])
            for g in range(h * G, (h + 1) * G):
                z = s["Q"][b, g, :m].double() @ k.T / math.sqrt(d)
                out[b, g, :m] = torch.softmax(torch.where(see, z, -torch.inf), -1) @ v
    return out


def _exact_keep(s, case):
    B, P = case["B"], case["P"]
    at, _ = _places(case)
    c = s["cache"]
    bounds = c["bounds"].double()
    rows = []
    for x in "kv":
        new = []
        for b in range(B):
            a, m = at[b], _kept(case)[b]
            v = _exact_values(c[x + "_codes"][b, :, :a + case["T"]],
                              c[x + "_scales"][b, :, :a + case["T"]])
            w = v.clone()
            for i in range(m):
                w[:, a + i] = v[:, a + int(s["path"][b, i])]
            new.append(w[:, a:a + P])
            if x == "k":
                for j in range(max(a - 1, 0) // BLOCK, -(-(a + m) // BLOCK)):
                    part = w[:, j * BLOCK:min((j + 1) * BLOCK, a + m)]
                    bounds[b, :, j, 0], bounds[b, :, j, 1] = part.amin(1), part.amax(1)
        rows.append(torch.stack(new))
    return None, rows[0], rows[1], bounds


def exact(case, seed):
    if case["op"] == "tree":
        return None  # whole numbers only
    s = prepare(case, seed)
    return {"grad": _exact_grad, "axes": _exact_axes, "attend": _exact_attend,
            "keep": _exact_keep}[case["op"]](s, case)
