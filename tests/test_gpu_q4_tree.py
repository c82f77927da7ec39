"""Drafted trees over the 4-bit cache and positions with several axes, on the GPU
against their definitions in float64."""
import pytest
import torch

import q4_reference as ref
from paper_2606_10944_amd import (Q4Cache, thin_q4_attention, thin_q4_keep, thin_q4_select,
                                  thin_q4_store, thin_q4_tree, thin_q4_tree_attention, thin_rotary,
                                  thin_rotary_axes, thin_rotary_turns)
from test_gpu_q4 import (DEV, attention_bound, filled, gen, i32, randn, rotary_bound,
                         same_contents, strided)

pytestmark = pytest.mark.gpu
BUFFERS = ("k_codes", "k_scales", "v_codes", "v_scales", "bounds")


# ---------------------------------------------------------------------------
# Positions with axes
# ---------------------------------------------------------------------------
def rotary_axes(x, pos, turns, axis, layout, amp, inverse):
    """Channel pair by channel pair: the turn by the position of the pair's axis."""
    y = x.double().clone()
    r = turns.numel()
    for p in range(r):
        i, j = (2 * p, 2 * p + 1) if layout == "interleaved" else (p, p + r)
        a = int(axis[p])
        where = pos[:, :, a] if 0 <= a < pos.shape[2] else torch.zeros_like(pos[:, :, 0])
        pair = x[..., [i, j]].repeat(1, 1, 1, 1)
        both = ref.rotary(pair, where, turns[p:p + 1], "half", amp, inverse)
        y[..., i], y[..., j] = both[..., 0], both[..., 1]
    return y


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot,B,H,T,axes", [
    (128, 128, 2, 3, 5, 3), (128, 32, 1, 1, 1, 1), (64, 64, 3, 2, 17, 2), (64, 48, 2, 1, 41, 4),
    (32, 32, 1, 5, 70, 3), (32, 16, 33, 2, 1, 4)])
def test_rotary_axes(dtype, layout, d, rot, B, H, T, axes):
    g = gen(101)
    turns, amp = thin_rotary_turns(rot, scaling="bands", factor=4.0, length=8192.0)
    x, y = randn(g, B, H, T, d, dtype=dtype), randn(g, B, 2 * H, T, d, dtype=dtype)
    pos = torch.randint(-100, 2_000_000, (B, T, axes), generator=g, dtype=torch.int32)
    orders = [torch.arange(rot // 2) * axes // (rot // 2), torch.arange(rot // 2) % axes,
              torch.randint(-1, axes + 2, (rot // 2,), generator=g)]  # (some are no axis)
    for axis in orders:
        for inverse in (False, True):
            a, b = thin_rotary_axes(x.to(DEV), pos.to(DEV), turns.to(DEV),
                                    axis.to(torch.int32).to(DEV), Y=strided(y), layout=layout,
                                    amp=amp, inverse=inverse)
            for got, v in ((a, x), (b, y)):
                want = rotary_axes(v, pos, turns, axis, layout, amp, inverse)
                err = (got.cpu().double() - want).abs()
                assert (err <= rotary_bound(v, want, turns, layout, amp, dtype)).all()


def test_one_axis_is_the_plain_turn_and_in_place():
    g = gen(102)
    turns, _ = thin_rotary_turns(64)
    x = randn(g, 2, 3, 9, 128, dtype="bf16").to(DEV)
    pos = torch.randint(0, 100000, (2, 9), generator=g, dtype=torch.int32).to(DEV)
    axis = torch.zeros(32, dtype=torch.int32, device=DEV)
    want = thin_rotary(x, pos, turns.to(DEV))
    assert torch.equal(thin_rotary_axes(x, pos.unsqueeze(2), turns.to(DEV), axis), want)
    s = strided(x.cpu())
    assert thin_rotary_axes(s, pos.unsqueeze(2), turns.to(DEV), axis, out=s) is s
    assert torch.equal(s, want)


def test_rotary_axes_gradient():
    """The inverse turn is the gradient: <turn(x), w> = <x, back(w)>, and the formula's by
    autograd in float64."""
    g = gen(103)
    turns, _ = thin_rotary_turns(32)
    x, w = randn(g, 2, 2, 7, 64), randn(g, 2, 2, 7, 64)
    pos = torch.randint(0, 50000, (2, 7, 3), generator=g, dtype=torch.int32)
    axis = torch.arange(16) % 3
    a = (pos.to(DEV), turns.to(DEV), axis.to(torch.int32).to(DEV))
    got = thin_rotary_axes(w.to(DEV), *a, inverse=True).cpu().double()
    xg = x.double().requires_grad_()
    y = torch.stack([ref.rotary(xg[..., [p, p + 16]], pos[:, :, p % 3], turns[p:p + 1], "half",
                                1.0, False) for p in range(16)])  # [16, B, H, T, 2]
    rest = (xg[..., 32:] * w[..., 32:].double()).sum()
    sides = torch.stack([w[..., [p, p + 16]].double() for p in range(16)])
    ((y * sides).sum() + rest).backward()
    assert ((got - xg.grad).abs() <= rotary_bound(w, xg.grad, turns, "half", 1.0, "fp32")).all()


# ---------------------------------------------------------------------------
# Trees
# ---------------------------------------------------------------------------
def tree_of(parents):
    """(sees [T, T] bool, depth [T]) by walking up from every draft."""
    T = len(parents)
    see, depth = torch.zeros(T, T, dtype=torch.bool), []
    for t in range(T):
        a, n = t, 0
        while True:
            see[t, a] = True
            p = parents[a]
            if p < 0 or p >= a:
                break
            a, n = p, n + 1
        depth.append(n)
    return see, torch.tensor(depth, dtype=torch.int32)


def unpacked(seen, T):
    """[.., T] bool of mask words [.., words]."""
    s = seen.cpu()
    return torch.stack([(s[..., j // 64] >> (j % 64)) & 1 for j in range(T)], -1).bool()


def packed(see):
    """Mask words of [.., T] bool."""
    T = see.shape[-1]
    words = [torch.zeros(see.shape[:-1], dtype=torch.int64) for _ in range((T + 63) // 64)]
    for j in range(T):
        words[j // 64] |= see[..., j].long() << (j % 64)
    return torch.stack(words, -1)


def some_parents(g, B, T, kind):
    t = torch.arange(T)
    if kind == "chain":
        p = (t - 1).expand(B, T)
    elif kind == "star":
        p = torch.where(t > 0, 0, -1).expand(B, T)
    elif kind == "roots":
        p = torch.full((B, T), -1)
    elif kind == "far":  # one parent per word of 64, one hop each
        p = torch.where(t >= 64, t - 64, -1).expand(B, T)
    elif kind == "wild":  # entries that are no earlier draft, too
        p = torch.randint(-3, T + 3, (B, T), generator=g)
    else:
        p = (torch.rand(B, T, generator=g) * (t + 1)).long() - 1
    return p.to(torch.int32).contiguous()


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 200, 257, 1024])
@pytest.mark.parametrize("kind", ["random", "chain", "star", "roots", "far", "wild"])
def test_tree(T, kind):
    g = gen(104)
    B = 3
    parents = some_parents(g, B, T, kind)
    at = [0, 5, 100000]
    seen, pos = thin_q4_tree(parents.to(DEV), i32(at))
    assert seen.shape == (B, T, (T + 63) // 64)
    for b in range(B):
        see, depth = tree_of(parents[b].tolist())
        assert torch.equal(seen[b].cpu(), packed(see))
        assert torch.equal(pos[b].cpu(), at[b] + depth)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
def check_tree(c, q, at, count, see, got, dtype):
    """Against the definition, a key head at a time; see [B, T, T] bool."""
    B, Hq, T, d = q.shape
    G = Hq // c.H
    got = got.cpu().double()
    for b in range(B):
        m = T if count is None else max(0, min(T, count[b]))
        n = max(0, min(c.n_max, at[b] + m))
        row = torch.arange(n)
        w = (row < at[b]).expand(T, n).clone()
        for j in range(m):
            if 0 <= at[b] + j < n:
                w[:, at[b] + j] = see[b, :, j]
        w[m:] = False
        w = w.double().repeat(G, 1)
        for h in range(c.H):
            o = got[b, h * G:(h + 1) * G].reshape(G * T, d)
            if n == 0:
                assert (o == 0).all()
                continue
            want, A, S = ref.attention(q[b, h * G:(h + 1) * G].reshape(G * T, d),
                                       ref.cached(c.k_codes[b, h, :n], c.k_scales[b, h, :n]),
                                       ref.cached(c.v_codes[b, h, :n], c.v_scales[b, h, :n]), w)
            assert (o[(w == 0).all(1)] == 0).all()
            ok = (o - want).abs() <= attention_bound(want, A, S, dtype)
            assert ok.all(), (b, h, (~ok).nonzero()[:3].tolist())


TREES = [
    # d, B, H, G, T, n_max, at, count: one workgroup per tile, keys shared out by lengths, many
    # query rows with and without shared keys; drafts across words, blocks, the cache's end
    (128, 1, 1, 1, 1, 1, [0], None),
    (64, 2, 2, 3, 9, 300, [250, 31], [9, 4]),
    (32, 3, 1, 8, 5, 100, [0, 97, -2], None),
    (128, 3, 2, 4, 33, 700, [660, 0, 700], [33, 0, 20]),
    (64, 2, 3, 2, 70, 400, [330, 11], [70, 65]),
    (128, 2, 2, 4, 8, 9000, [8990, 100], [8, 7]),
    (32, 9, 1, 5, 30, 5000, [4970, 0, 17, 300, 64, 2000, 5, 4999, 1], [30] * 8 + [12]),
    (128, 4, 16, 4, 130, 700, [0, 300, 570, 650], None),
    (64, 16, 8, 2, 130, 300, list(range(0, 160, 10)), [130] * 15 + [77]),
    (128, 1, 8, 4, 129, 5000, [4870], None),
    (64, 2, 2, 1, 1024, 4500, [3476, 0], [1024, 1000]),
    (32, 7, 4, 4, 40, 5000, [4960, 0, -50, 700, 5000, 63, 64], [40, 40, 40, 39, 40, 0, 1]),
    (64, 20, 2, 8, 33, 4500, [4467, *range(0, 1900, 100)], [33] * 18 + [-1, 50]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,G,T,n_max,at,count", TREES)
def test_tree_attention(dtype, d, B, H, G, T, n_max, at, count):
    g = gen(105)
    c = filled(g, B, H, n_max, d, [max(0, min(n_max, a + T)) for a in at])
    q = randn(g, B, H * G, T, d, dtype=dtype)
    cnt = None if count is None else i32(count)
    parents = some_parents(g, B, T, "random")
    seen, _ = thin_q4_tree(parents.to(DEV), i32(at))
    see = torch.stack([tree_of(parents[b].tolist())[0] for b in range(B)])
    o = strided(torch.zeros_like(q))
    got = thin_q4_tree_attention(strided(q), c, i32(at), seen, count=cnt, O=o)
    assert got is o
    check_tree(c, q, at, count, see, got, dtype)
    assert torch.equal(thin_q4_tree_attention(q.to(DEV), c, i32(at), seen, count=cnt), got)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,n_max,H,B", [(5, 200, 1, 2), (70, 300, 2, 2), (150, 400, 16, 8),
                                         (66, 6000, 2, 2)])
def test_any_mask_is_legal(dtype, T, n_max, H, B):
    """Masks that are no tree: later drafts, not oneself, nothing; bits behind the drafts."""
    g = gen(106)
    G, d = 4, 64
    at = [0, n_max - T] * (B // 2)
    count = [T, T - 2] * (B // 2)
    c = filled(g, B, H, n_max, d, [a + T for a in at])
    q = randn(g, B, H * G, T, d, dtype=dtype)
    see = torch.rand(B, T, T, generator=g) < 0.4
    see[:, 1] = False  # (sees nothing where no row lies before the drafts)
    see[:, 3] = True
    seen = packed(see)
    if T % 64:
        seen[..., -1] |= -1 << (T % 64)  # bits of no draft
    got = thin_q4_tree_attention(q.to(DEV), c, i32(at), seen.to(DEV), count=i32(count))
    check_tree(c, q, at, count, see, got, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,n_max,at", [(40, 900, [860, 3]), (40, 9000, [8960, 3]),
                                        (130, 5000, [4870, 1000])])
def test_a_chain_is_causal_attention(dtype, T, n_max, at):
    """Every draft the child of the one before: the bits of thin_q4_attention."""
    g = gen(107)
    c = filled(g, 2, 8, n_max, 128, [a + T for a in at])
    q = randn(g, 2, 16, T, 128, dtype=dtype).to(DEV)
    seen, pos = thin_q4_tree(some_parents(g, 2, T, "chain").to(DEV), i32(at))
    assert pos.cpu().tolist() == [[a + t for t in range(T)] for a in at]
    got = thin_q4_tree_attention(q, c, i32(at), seen)
    want = thin_q4_attention(q, c, i32(at))
    # the workgroups' shares of the keys differ, and with them the order of the sums
    err = (got.double() - want.double()).abs().cpu()
    for b in range(2):
        for h in range(8):
            n = at[b] + T
            k = ref.cached(c.k_codes[b, h, :n], c.k_scales[b, h, :n])
            v = ref.cached(c.v_codes[b, h, :n], c.v_scales[b, h, :n])
            for i in (2 * h, 2 * h + 1):
                w = (torch.arange(n) <= at[b] + torch.arange(T).unsqueeze(1)).double()
                o, A, S = ref.attention(q[b, i].cpu(), k, v, w)
                assert (err[b, i] <= 2 * attention_bound(o, A, S, dtype)).all()


# ---------------------------------------------------------------------------
# Keep
# ---------------------------------------------------------------------------
def kept_rows(path, at, n_max):
    """How many entries of a path count."""
    for i, p in enumerate(path):
        if p < 0 or at < 0 or at + p >= n_max or at + i >= n_max:
            return i
    return len(path)


KEEPS = [
    # d, B, H, n_max, at, paths
    (128, 2, 2, 300, [100, 62], [[0, 3, 9, -1], [2, 5, 7, 11]]),
    (64, 3, 1, 130, [64, 0, 127], [[1, 2, 3], [63, 64, 100], [0, 1, 2]]),
    (32, 4, 3, 100, [10, 99, -3, 100], [[4, -1, 8], [0, 0, 0], [5, 6, 7], [0, 1, 2]]),
    (64, 2, 2, 500, [3, 128], [[9, 9, 0, 2, 1], [5, 4, 3, 2, 1]]),  # any order, twice
    (128, 1, 2, 2000, [63], [list(range(1, 1000, 3))]),
    (64, 2, 1, 1500, [447, 20], [list(range(0, 1024))] * 2),
    (32, 2, 2, 64, [64, 0], [[0], [-1]]),
    (128, 2, 1, 200, [70, 64], [[-1, 3], [-5, 2]]),  # nothing accepted
    (32, 1, 1, 70, [5], [[2**31 - 1, 1]]),
]


@pytest.mark.parametrize("d,B,H,n_max,at,paths", KEEPS)
def test_keep(d, B, H, n_max, at, paths):
    g = gen(108)
    c = filled(g, B, H, n_max, d, [n_max] * B)
    before = {k: getattr(c, k).cpu().clone() for k in BUFFERS}
    end = c.keep(i32(at), i32(paths))
    after = {k: getattr(c, k).cpu() for k in BUFFERS}
    for b in range(B):
        m = kept_rows(paths[b], at[b], n_max)
        assert int(end[b]) == at[b] + m
        for k in BUFFERS[:4]:
            want = before[k][b].clone()
            for i in range(m):
                want[:, at[b] + i] = before[k][b][:, at[b] + paths[b][i]]
            assert torch.equal(after[k][b], want)
        want = before["bounds"][b].double()
        last = at[b] + m - 1
        if 0 <= last < n_max:
            rows = ref.cached(after["k_codes"][b], after["k_scales"][b])
            for j in range(max(at[b] - 1, 0) // 64, last // 64 + 1):
                part = rows[:, j * 64:min(j * 64 + 64, last + 1)]
                want[:, j, 0], want[:, j, 1] = part.amin(1), part.amax(1)
        assert torch.equal(after["bounds"][b].double(), want)


def test_kept_rows_are_those_of_a_store():
    """Rows stored as drafts and kept leave the cache that storing the accepted rows alone
    leaves, bounds too, and the next selection is the same."""
    g = gen(109)
    B, H, n_max, d, T = 2, 2, 400, 64, 100
    at, paths = [130, 61], [[0, 2, 5, 40, 41, 77], [1, 9, 10, 66, 98, 99]]
    c = filled(g, B, H, n_max, d, at)
    other = Q4Cache.over(*[getattr(c, k).clone() for k in BUFFERS])
    k, v = randn(g, B, H, T, d, dtype="bf16").to(DEV), randn(g, B, H, T, d, dtype="bf16").to(DEV)
    thin_q4_store(k, v, c, i32(at))
    end = c.keep(i32(at), i32(paths))
    pick = torch.tensor(paths, device=DEV).view(B, 1, 6, 1).expand(B, H, 6, d)
    thin_q4_store(k.gather(2, pick), v.gather(2, pick), other, i32(at))
    for b in range(B):
        n = int(end[b])
        assert n == at[b] + 6
        for name in BUFFERS[:4]:
            assert torch.equal(getattr(c, name)[b, :, :n], getattr(other, name)[b, :, :n])
        blocks = (n + 63) // 64
        assert torch.equal(c.bounds[b, :, :blocks], other.bounds[b, :, :blocks])
    q = randn(g, B, 2 * H, 1, d, dtype="bf16").to(DEV)
    last = end - 1
    assert torch.equal(thin_q4_select(q, c, last, 2, n_window=1),
                       thin_q4_select(q, other, last, 2, n_window=1))


# ---------------------------------------------------------------------------
# Together, streams, graphs, refusals
# ---------------------------------------------------------------------------
def test_drafts_as_they_are_used():
    """A prompt, then rounds of drafts and accepted paths: the rows left are those of the
    accepted tokens at their positions, and outputs follow the definition."""
    g = gen(110)
    B, H, G, d, n_max = 2, 2, 2, 64, 400
    turns, _ = thin_rotary_turns(64)
    t = turns.to(DEV)
    c = Q4Cache(B, H, n_max, d, device=DEV)
    n = 150
    k, v, q = (randn(g, B, x, n, d, dtype="bf16").to(DEV) for x in (H, H, H * G))
    at = i32([0, 0])
    c.step(q, k, v, at, count=i32([150, 90]), turns=t)
    at = i32([150, 90])
    rows = [[(k[b, :, i], i) for i in range(m)] for b, m in enumerate((150, 90))]
    for T in (1, 12, 70):
        parents = some_parents(g, B, T, "random")
        q, k, v = (randn(g, B, x, T, d, dtype="bf16").to(DEV) for x in (H * G, H, H))
        o = c.draft(q, k, v, at, parents.to(DEV), turns=t)
        lens = at.tolist()
        sees, paths = [], []
        for b in range(B):
            see, depth = tree_of(parents[b].tolist())
            sees.append(see)
            leaf = int(depth.argmax())
            paths.append(see[leaf].nonzero().flatten().tolist()[:5])
        qr, _ = thin_rotary(q, torch.stack([lens[b] + tree_of(parents[b].tolist())[1]
                                            for b in range(B)]).to(DEV), t, Y=k)
        check_tree(c, qr.cpu(), lens, None, torch.stack(sees), o, "bf16")
        for b in range(B):
            rows[b] += [(k[b, :, p], lens[b] + i) for i, p in enumerate(paths[b])]
        P = max(len(p) for p in paths)
        at = c.keep(at, i32([p + [-1] * (P - len(p)) for p in paths]))
        assert at.tolist() == [len(r) for r in rows]
    for b in range(B):
        m = len(rows[b])
        kept = torch.stack([r for r, _ in rows[b]], 1).unsqueeze(0)
        pos = torch.tensor([[p for _, p in rows[b]]], dtype=torch.int32, device=DEV)
        codes, scales = ref.encode(thin_rotary(kept, pos, t)[0].cpu())
        assert torch.equal(ref.cached(c.k_codes[b, :, :m], c.k_scales[b, :, :m]),
                           ref.values(codes, scales))


def test_draft_with_axes_and_a_shared_tree():
    g = gen(111)
    B, H, d, T, n_max = 2, 2, 64, 7, 100
    turns = thin_rotary_turns(32)[0].to(DEV)
    axis = i32([p % 3 for p in range(16)])
    pos = torch.randint(0, 999, (B, T, 3), generator=g, dtype=torch.int32).to(DEV)
    q, k, v = (randn(g, B, x, T, d, dtype="bf16").to(DEV) for x in (4, H, H))
    at = i32([50, 20])
    caches = [filled(gen(112), B, H, n_max, d, [50, 20]) for _ in range(2)]
    tree = thin_q4_tree(some_parents(g, B, T, "random").to(DEV), at)
    o = caches[0].draft(q, k, v, at, tree=tree, turns=turns, pos=pos, axis=axis)
    qr, kr = thin_rotary_axes(q, pos, turns, axis, Y=k)
    thin_q4_store(kr, v, caches[1], at)
    assert torch.equal(o, thin_q4_tree_attention(qr, caches[1], at, tree[0]))
    assert same_contents(*caches)


@pytest.mark.parametrize("T,n_max", [(8, 300), (20, 9000), (200, 5000)])
def test_replayed_drafts_follow_their_inputs(T, n_max):
    """A captured step (tree, turn, store, attention, keep) on another stream, replayed with
    new rows, parents, paths and positions, eager work between; two graphs alive."""
    g = gen(113)
    B, H, G, d = 2, 2, 2, 128
    turns = thin_rotary_turns(d)[0].to(DEV)
    caches = [filled(gen(114), B, H, n_max, d, [n_max, n_max]) for _ in range(3)]
    q, k, v = (torch.zeros(B, x, T, d, dtype=torch.bfloat16, device=DEV) for x in (H * G, H, H))
    at, parents, path = i32([0, 0]), i32([[-1] * T] * B), i32([[0, 1, 2]] * B)

    def step(c):
        o = c.draft(q, k, v, at, parents, turns=turns)
        return o, c.keep(at, path)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in caches:
            step(c)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for c in caches[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(c))
        graphs.append(graph)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(randn(g, *x.shape, dtype="bf16"))
        at.copy_(i32([n_max - T - 3 * i, 70 + i]))
        parents.copy_(some_parents(g, B, T, ("random", "chain")[i % 2]))
        path.copy_(i32([[i, i + 2, i + 3], [1, -1, 2]]))
        for graph in graphs:
            graph.replay()
        want = step(caches[2])
        torch.cuda.synchronize()
        for got in outs:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert same_contents(caches[0], caches[2]) and same_contents(caches[1], caches[2])


def test_calls_on_a_stream_of_their_own():
    g = gen(115)
    c = filled(g, 2, 2, 6000, 64, [6000, 6000])
    other = Q4Cache.over(*[getattr(c, k).clone() for k in BUFFERS])
    q = randn(g, 2, 4, 5, 64, dtype="bf16").to(DEV)
    at, parents, path = i32([5990, 17]), i32([[-1, 0, 0, 1, 3]] * 2), i32([[0, 1, 3, 4]] * 2)
    x, pos, axis = q[:, :2].contiguous(), i32([[[1, 2]] * 5] * 2), i32([0, 1] * 16)
    turns = thin_rotary_turns(64)[0].to(DEV)

    def calls(c, stream=None):
        seen, p = thin_q4_tree(parents, at, stream=stream)
        o = thin_q4_tree_attention(q, c, at, seen, stream=stream)
        return seen, p, o, thin_q4_keep(c, at, path, stream=stream), \
            thin_rotary_axes(x, pos, turns, axis, stream=stream)

    want = calls(c)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = calls(other, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert same_contents(c, other)


def test_binding_refuses_what_does_not_fit():
    from paper_2606_10944_amd._lib import THIN_EDTYPE, THIN_EINVAL, THIN_EWORKSPACE, ThinError
    g = gen(116)
    B, H, T, d = 2, 2, 6, 64
    c = filled(g, B, H, 5000, d, [5000, 5000])
    was = Q4Cache.over(*[getattr(c, k).clone() for k in BUFFERS])
    q = randn(g, B, 4, T, d, dtype="bf16").to(DEV)
    kv = randn(g, B, H, T, d, dtype="bf16").to(DEV)
    at, parents = i32([10, 20]), i32([[-1] * T] * B)
    seen, pos = thin_q4_tree(parents, at)
    turns, axis = thin_rotary_turns(d)[0].to(DEV), i32([0] * 32)

    def refused(status, f, *a, **kw):
        with pytest.raises(ThinError) as e:
            f(*a, **kw)
        assert e.value.status == status

    for bad in (parents[0], parents.long(), parents.cpu(), parents[:1], parents[:, ::2]):
        refused(THIN_EINVAL, thin_q4_tree, bad, at)
    refused(THIN_EINVAL, thin_q4_tree, i32([[-1] * 1025] * B), at)
    refused(THIN_EINVAL, thin_q4_tree, parents, at, seen=seen[:, :3])
    refused(THIN_EINVAL, thin_q4_tree, parents, at, pos=pos.long())
    for bad in (seen.to(torch.int32), seen.cpu(), seen[:1], seen[:, :5], torch.cat([seen, seen], 2)):
        refused(THIN_EINVAL, thin_q4_tree_attention, q, c, at, bad)
        refused(THIN_EINVAL, c.draft, q, kv, kv, at, tree=(bad, pos))
    for bad in (q[:, :3], q[:1], q.cpu()):
        refused(THIN_EINVAL, thin_q4_tree_attention, bad, c, at, seen)
    refused(THIN_EDTYPE, thin_q4_tree_attention, q.half(), c, at, seen)
    refused(THIN_EINVAL, thin_q4_tree_attention, q, c, at, seen, O=q.float())
    small = torch.empty(16, dtype=torch.uint8, device=DEV)
    refused(THIN_EWORKSPACE, thin_q4_tree_attention, q, c, at, seen, workspace=small)
    for bad in (at.long(), at[:1], at.cpu()):
        refused(THIN_EINVAL, thin_q4_keep, c, bad, parents)
    for bad in (parents[0], parents[:1], parents[:, ::2], i32([[0] * 1025] * B),
                torch.empty(B, 0, dtype=torch.int32, device=DEV)):
        refused(THIN_EINVAL, thin_q4_keep, c, at, bad)
    refused(THIN_EINVAL, thin_q4_keep, c, at, parents, end=at)
    refused(THIN_EINVAL, c.draft, q, kv, kv, at)
    refused(THIN_EINVAL, c.draft, q, kv, kv, at, parents[:, :3])
    refused(THIN_EINVAL, c.draft, q, kv, kv, at, parents, pos=pos)
    refused(THIN_EINVAL, c.draft, q, kv, kv, at, parents, turns=turns, pos=pos[:, :3])
    refused(THIN_EINVAL, c.draft, q, kv[:, :1], kv, at, parents)
    refused(THIN_EINVAL, c.draft, q, kv[:, :, :3], kv[:, :, :3], at, parents)
    refused(THIN_EINVAL, thin_q4_tree, parents, at, pos=parents)
    refused(THIN_EINVAL, c.draft, q, kv, kv, at, parents, O=q[:, :2])
    p3 = i32([[[0, 0, 0]] * T] * B)
    for bad in (pos, p3[:, :2], p3.long(), torch.cat([p3, p3], 2)):
        refused(THIN_EINVAL, thin_rotary_axes, q, bad, turns, axis)
    for bad in (axis[:31], axis.long(), axis.cpu(), axis[None]):
        refused(THIN_EINVAL, thin_rotary_axes, q, p3, turns, bad)
    torch.cuda.synchronize()
    assert same_contents(c, was)
