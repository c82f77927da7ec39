"""The gradient of coreset attention in float64 from its formulas (torch on the CPU), and how
far float32 sums and the types' roundings may take the kernels from it."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def coreset(K, V, idx, logw):
    """Rows of K and V that idx lists (zeros for keys that are not there) and which are."""
    n = K.shape[-2]
    there = (idx >= 0) & (idx < n)
    if logw is not None:
        there = there & (logw != -math.inf)
    at = idx.clamp(0, n - 1).long().unsqueeze(-1).expand(*idx.shape, K.shape[-1])
    z = there.unsqueeze(-1)
    zero = torch.zeros((), dtype=torch.float64)
    return (torch.where(z, K.double().gather(-2, at), zero),
            torch.where(z, V.double().gather(-2, at), zero), there)


def scatter(n, idx, there, rows):
    """[.., n, d]: rows added at the places that idx lists."""
    out = torch.zeros(*idx.shape[:-1], n, rows.shape[-1], dtype=torch.float64)
    at = torch.where(there, idx, 0).long().unsqueeze(-1).expand_as(rows)
    return out.scatter_add_(-2, at, torch.where(there.unsqueeze(-1), rows, 0.0))


def forward(q, k, v, bias):
    """softmax(q k^T / sqrt d + bias) v; rows that see nothing are zeros."""
    z = q @ k.transpose(-1, -2) / math.sqrt(q.shape[-1]) + bias.unsqueeze(-2)
    m = z.amax(-1, keepdim=True)
    p = torch.where(m > -math.inf, torch.exp(z - torch.where(m > -math.inf, m, 0.0)), 0.0)
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / torch.where(total > 0, total, 1.0), 0.0)
    return p @ v, p, z


def gradient(Q, K, V, idx, logw, dO):
    """{name: (gradient, bound)}.

    S = sum |q_c k_c| / sqrt d.  A score is a float32 sum of d products (off by 2^-19 S with the
    scale and the log-weight's addition), so a weight is off by r = 2^-18 S + 2^-20 of itself,
    the maximum's error being in both (and 2^-22 |logw|).  g is such a sum as well, off by 2^-19 G,
    G = sum |do_c v_c|; of bf16 rows with a float32 dO, whose two bf16 parts hold 17 bits, by
    2^-17 G more.  sum p g is off by 2 r sum p |g| + sum p dg, and ds = p (g - sum p g) by r |ds| + p
    (dg + that).  ds and p round to bf16 beside bf16 rows (dO too, if it is float32, in dV).  A sum
    of N terms in float32 adds N 2^-24 of their magnitudes, and the gradient rounds.  Below the
    least normal number float32 holds nothing: a weight or a product p (g - ..) smaller than 2^-126
    may become 0, so that a weight is off by `least` = 2^-125 more, and ds by least (G + |D| + 1).
    (Seen: a weight of e^-91 in a dK of 1e-36.)"""
    u = HALF[Q.dtype]
    low = Q.dtype == torch.bfloat16
    n, d = K.shape[-2:]
    q, do = Q.double(), dO.double()
    k, v, there = coreset(K, V, idx, logw)
    lw = torch.zeros(idx.shape, dtype=torch.float64) if logw is None else logw.double()
    bias = torch.where(there, lw, -math.inf)
    _, p, _ = forward(q, k, v, bias)
    rd = 1.0 / math.sqrt(d)
    kt, vt = k.transpose(-1, -2), v.transpose(-1, -2)
    g = do @ vt
    G = do.abs() @ vt.abs()
    S = (q.abs() @ kt.abs() * rd).amax(-1, keepdim=True)
    big = torch.where(there, lw.abs(), 0.0).amax(-1, keepdim=True).unsqueeze(-1)
    D = (p * g).sum(-1, keepdim=True)
    ds = p * (g - D)
    r = 2.0 ** -18 * S + 2.0 ** -20 + 2.0 ** -22 * big
    dg = (2.0 ** -19 + (2.0 ** -17 if low and dO.dtype == torch.float32 else 0.0)) * G
    dD = 2 * r * (p * g.abs()).sum(-1, keepdim=True) + (p * dg).sum(-1, keepdim=True)
    least = 2.0 ** -125
    eds = r * ds.abs() + p * (1 + r) * (dg + dD) + least * (G + D.abs() + 1) * there.unsqueeze(-2)
    edr = eds + (u * (ds.abs() + eds) if low else 0.0)
    n_q, m = q.shape[-2], k.shape[-2]
    eq, ek = (m + 64) * 2.0 ** -24, (n_q + 64) * 2.0 ** -24
    T = lambda x: x.transpose(-1, -2)  # noqa: E731
    out = {}

    def put(name, value, bound, where=None):
        if where is not None:
            value, bound = scatter(n, idx, there, value), scatter(n, idx, there, bound)
        out[name] = (value, bound + (u if name != "dlogw" else 2.0 ** -24) * (value.abs() + bound)
                     + 1e-37)
    put("dQ", ds @ k * rd, (edr + eq * (ds.abs() + edr)) @ k.abs() * rd)
    put("dK", T(ds) @ q * rd, T(edr + ek * (ds.abs() + edr)) @ q.abs() * rd, True)
    ep = p * (r + (u if low else 0.0) + (u if low and dO.dtype == torch.float32 else 0.0)) * 1.01 \
        + least * there.unsqueeze(-2)
    put("dV", T(p) @ do, T(ep + ek * (p + ep)) @ do.abs(), True)
    put("dlogw", ds.sum(-2), (eds + ek * (ds.abs() + eds)).sum(-2))
    return out
