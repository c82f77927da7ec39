"""The 4-bit cache's operators and rotary positions in float64, from their
definitions (torch on the CPU)."""
import math

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
BLOCK = 64


def encode(x):
    """(codes [.., d], scale bytes [.., d/32]) of rows x: the nearest of the eight
    magnitudes (ties: the even code) under 2^e, e the least with amax <= 7 2^e."""
    g = x.double()
    g = torch.where(g.isnan(), torch.zeros_like(g), g).unflatten(-1, (-1, 32))
    amax = g.abs().amax(-1)
    e = torch.full(amax.shape, -125, dtype=torch.int64)
    for k in range(-125, 125):
        e = torch.where(amax > 7.0 * 2.0 ** k, torch.full_like(e, k + 1), e)
    y = g.abs() / torch.exp2(e.double()).unsqueeze(-1)
    y = y.clamp(max=6.0)
    off = (y.unsqueeze(-1) - GRID).abs()
    least = off.amin(-1, keepdim=True)
    near = off == least
    # of two equally near codes the even one
    code = torch.where(near, torch.arange(8).expand_as(off) + 8 * (torch.arange(8) % 2),
                       torch.full_like(off, 99).long()).amin(-1) % 8
    code = code + 8 * (g < 0).long()
    return code.flatten(-2), (e + 127)


def values(codes, scales):
    v = GRID[codes % 8] * torch.where(codes >= 8, -1.0, 1.0).double()
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def unpack(packed):
    """4-bit codes [.., d] of packed bytes [.., d/2]."""
    p = packed.long()
    return torch.stack((p % 16, p // 16), -1).flatten(-2)


def cached(codes, scales):
    """Values of a cache's packed codes and scale bytes (moved to the CPU)."""
    return values(unpack(codes.cpu()), scales.cpu().long())


def bounds(k, n):
    """[.., nb, 2, d] of the first n rows of values k [.., n_max, d]."""
    out = []
    for b in range(0, n, BLOCK):
        part = k[..., b:min(b + BLOCK, n), :]
        out.append(torch.stack((part.amin(-2), part.amax(-2)), -2))
    return torch.stack(out, -3)


def rotary(x, pos, turns, layout, amp, inverse):
    """x [B,H,T,d], pos [B,T] (ints), turns [rot/2]."""
    y = x.double().clone()
    r = turns.numel()
    i, j = (torch.arange(r), torch.arange(r) + r)
    if layout == "interleaved":
        i, j = 2 * i, 2 * i + 1
    a = (pos.double().unsqueeze(-1) * turns.double()) % 1.0 * 2 * math.pi
    a = (-a if inverse else a).unsqueeze(1)
    c, s = amp * a.cos(), amp * a.sin()
    y[..., i], y[..., j] = (x.double()[..., i] * c - x.double()[..., j] * s,
                            x.double()[..., j] * c + x.double()[..., i] * s)
    return y


def block_scores(q, bnd):
    """[nb] of a group's queries q [G, d] against bounds bnd [nb, 2, d]."""
    p = q.double().unsqueeze(1).unsqueeze(2) * bnd.double().unsqueeze(0)  # [G, nb, 2, d]
    return p.amax(2).sum(-1).sum(0)


def select(scores, last, n_sel, n_sinks, n_window):
    """The chosen blocks (ascending list) of one token whose own row is `last`."""
    if last < 0:
        return []
    n = last // BLOCK + 1
    forced = sorted(set(range(min(n_sinks, n))) | set(range(max(0, n - n_window), n)))
    if n <= n_sel:
        return list(range(n))
    rest = [k for k in range(n) if k not in set(forced)]
    key = lambda k: -scores[k] if not math.isnan(scores[k]) else math.inf  # noqa: E731
    rest.sort(key=lambda k: (key(k), k))
    return sorted(forced + rest[:n_sel - len(forced)])


def attention(q, k, v, weight):
    """(o, A, S) of queries q [R, d] over rows k, v [n, d] that count weight [R, n]
    times: the output, sum p |v| / sum p, and the largest sum |q_c k_c| / sqrt d."""
    q, d = q.double(), q.shape[-1]
    s = q @ k.T / math.sqrt(d)
    s = torch.where(weight > 0, s, torch.full_like(s, -math.inf))
    m = s.amax(-1, keepdim=True)
    p = torch.where(weight > 0, weight * torch.exp(s - m), torch.zeros_like(s))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    big = (q.abs() @ k.abs().T / math.sqrt(d)) * (weight > 0)
    return p @ v, p @ v.abs(), big.amax(-1, keepdim=True)
