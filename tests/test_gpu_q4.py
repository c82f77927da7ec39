"""Rotary positions and the 4-bit key/value cache on the GPU against their
definitions in float64."""
import math

import pytest
import torch

import q4_reference as ref
from paper_2606_10944_amd import (Q4Cache, thin_q4_attention, thin_q4_load, thin_q4_select,
                                  thin_q4_store, thin_rotary, thin_rotary_turns)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype="fp32"):
    return torch.randn(*shape, generator=g).to(DT[dtype])


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def strided(x):
    """The same rows as a [B, T, heads, d] tensor's view (rows between heads) with
    spare channels behind each row."""
    B, H, T, d = x.shape
    wide = torch.full((B, T, H, 2 * d), 7.0, dtype=x.dtype)
    wide[..., :d] = x.transpose(1, 2)
    return wide.to(DEV)[..., :d].transpose(1, 2)


def half_step(dtype):
    return torch.finfo(DT[dtype]).eps / 2


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------
# A turned value is x c - y s with c, s = amp cos, amp sin.  2 x the fraction of a
# turn rounds to float32 (2^-25, an angle of pi 2^-25), sincospi adds at most two
# units of 2^-24 x 2, the factor amp, two products and the difference one 2^-24
# each: in all below 3 * 2^-22 of amp (|x| + |y|), then the output's rounding.
def rotary_bound(x, want, turns, layout, amp, dtype):
    r = turns.numel()
    i = torch.arange(r)
    i, j = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + r)
    b = want.abs() * half_step(dtype)
    both = (x.double()[..., i].abs() + x.double()[..., j].abs()) * abs(amp) * 3 * 2.0 ** -22
    b[..., i] += both
    b[..., j] += both
    b[..., 2 * r:] = 0
    return b


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot,B,H,T,scaling", [
    (128, 128, 2, 3, 5, "none"), (128, 32, 1, 1, 1, "linear"), (128, 96, 1, 2, 33, "bands"),
    (64, 64, 3, 2, 17, "base"), (64, 16, 2, 1, 40, "none"), (32, 32, 1, 5, 70, "bands"),
    (32, 16, 33, 2, 1, "none")])
def test_rotary(dtype, layout, d, rot, B, H, T, scaling):
    g = gen(1)
    turns, amp = thin_rotary_turns(rot, scaling=scaling, factor=4.0, length=8192.0)
    x, y = randn(g, B, H, T, d, dtype=dtype), randn(g, B, 2 * H, T, d, dtype=dtype)
    pos = torch.randint(-100, 2_000_000, (B, T), generator=g, dtype=torch.int32)
    first = pos[:, 0].contiguous()
    run = first.unsqueeze(1) + torch.arange(T, dtype=torch.int32)
    t = turns.to(DEV)
    for p, where in ((pos, pos), (first, run)):
        for inverse in (False, True):
            a, b = thin_rotary(x.to(DEV), p.to(DEV), t, Y=strided(y), layout=layout, amp=amp,
                               inverse=inverse)
            for got, v in ((a, x), (b, y)):
                want = ref.rotary(v, where, turns, layout, amp, inverse)
                err = (got.cpu().double() - want).abs()
                assert (err <= rotary_bound(v, want, turns, layout, amp, dtype)).all()


def test_rotary_in_place_strided_and_alone():
    g = gen(2)
    turns, _ = thin_rotary_turns(64)
    x = randn(g, 2, 3, 9, 128, dtype="bf16")
    t, p = turns.to(DEV), i32([5, 1000])
    want = thin_rotary(x.to(DEV), p, t)
    s = strided(x)
    assert thin_rotary(s, p, t, out=s) is s
    assert torch.equal(s, want)
    out = torch.zeros(2, 9, 3, 128, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    thin_rotary(x.to(DEV), p, t, out=out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient(layout):
    """The inverse turn of a gradient is the gradient of the turn: against the
    formula's by autograd in float64, and <turn(x), w> = <x, back(w)>."""
    g = gen(3)
    turns, amp = thin_rotary_turns(32, scaling="bands", factor=4.0, length=4096.0)
    x, w = randn(g, 2, 2, 7, 64), randn(g, 2, 2, 7, 64)
    pos = torch.randint(0, 50000, (2, 7), generator=g, dtype=torch.int32)
    got = thin_rotary(w.to(DEV), pos.to(DEV), turns.to(DEV), layout=layout, amp=amp, inverse=True)
    got = got.cpu().double()
    xg = x.double().requires_grad_()
    (ref.rotary(xg, pos, turns, layout, amp, False) * w.double()).sum().backward()
    assert ((got - xg.grad).abs() <= rotary_bound(w, xg.grad, turns, layout, amp, "fp32")).all()
    # the turn is linear, so differences are exact up to rounding
    y = thin_rotary(x.to(DEV), pos.to(DEV), turns.to(DEV), layout=layout, amp=amp).cpu().double()
    lhs, rhs = float((y * w.double()).sum()), float((x.double() * got).sum())
    # each side sums 1792 products whose factors are off by at most rotary_bound
    bound = float((rotary_bound(x, y, turns, layout, amp, "fp32") * w.double().abs()).sum()
                  + (rotary_bound(w, got, turns, layout, amp, "fp32") * x.double().abs()).sum())
    assert abs(lhs - rhs) <= bound


# ---------------------------------------------------------------------------
# Store and load
# ---------------------------------------------------------------------------
def fresh(B, H, n_max, d, fill=0x55):
    c = Q4Cache(B, H, n_max, d, device=DEV)
    for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
        t.fill_(fill)
    c.bounds.fill_(123.0)
    return c


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("B,H,n_max,T,at,count", [
    (1, 1, 1, 1, [0], None), (2, 3, 200, 1, [63, 64], None), (3, 2, 130, 70, [0, 1, 60], None),
    (3, 1, 200, 65, [100, 0, 135], [65, 0, 30]), (2, 2, 100, 64, [-10, 80], None),
    (2, 1, 64, 3, [64, 70], None), (2, 1, 300, 129, [127, 1], [129, 200]),
    (3, 2, 100, 2, [70, 105, 98], [0, 2, -3])])
def test_store(dtype, d, B, H, n_max, T, at, count):
    g = gen(4)
    k = randn(g, B, H, T, d, dtype=dtype) * torch.exp2(
        torch.randint(-20, 20, (B, H, T, 1), generator=g).float()).to(DT[dtype])
    v = randn(g, B, H, T, d, dtype=dtype)
    c = fresh(B, H, n_max, d)
    # older rows, in one call
    old = randn(g, B, H, n_max, d)
    if max(at) > 0:
        thin_q4_store(old.to(DEV), old.to(DEV), c, i32([0] * B),
                      count=i32([max(0, a) for a in at]))
    before = [t.cpu().clone() for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.bounds)]
    thin_q4_store(strided(k), v.to(DEV), c, i32(at), count=None if count is None else i32(count))
    after = [t.cpu() for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.bounds)]
    for b in range(B):
        new = range(max(0, -at[b]), min(T if count is None else min(T, count[b]), n_max - at[b]))
        rows = [at[b] + t for t in new]
        for x, i in ((k, 0), (v, 2)):
            codes, scales = ref.encode(x[b, :, new.start:max(new.start, new.stop)])
            got = ref.unpack(after[i][b][:, rows])
            assert torch.equal(got % 8, codes % 8)
            assert torch.equal((got >= 8) & (got % 8 > 0), (codes >= 8) & (codes % 8 > 0))
            assert torch.equal(after[i + 1][b][:, rows].long(), scales)
            rest = [r for r in range(n_max) if r not in set(rows)]
            assert torch.equal(after[i][b][:, rest], before[i][b][:, rest])
            assert torch.equal(after[i + 1][b][:, rest], before[i + 1][b][:, rest])
        touched = sorted({r // 64 for r in rows})
        untouched = [j for j in range(c.bounds.shape[2]) if j not in set(touched)]
        assert torch.equal(after[4][b][:, untouched], before[4][b][:, untouched])
        if rows:
            want = ref.bounds(ref.cached(after[0][b], after[1][b]), rows[-1] + 1)
            assert torch.equal(after[4][b][:, touched].double(), want[:, touched])


def test_store_special_values():
    """Ties, the largest values, infinities, NaN, zeros and subnormal numbers."""
    big = torch.finfo(torch.float32).max
    rows = torch.zeros(8, 32)
    rows[0, :9] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0])
    rows[1, :9] = -rows[0, :9] * 2.0 ** -40
    rows[2, :3] = torch.tensor([big, 1.0, -big])
    rows[3, :3] = torch.tensor([math.inf, 1e30, -math.inf])
    rows[4, :3] = torch.tensor([math.nan, 1.0, 3.0])
    rows[5, :] = math.nan
    rows[6, :3] = torch.tensor([1e-40, -1e-45, 2.0 ** -126])
    rows[7, :2] = torch.tensor([7.0000005, 3.5000002])
    x = rows.view(1, 1, 8, 32)
    c = fresh(1, 1, 8, 32)
    thin_q4_store(x.to(DEV), x.to(DEV), c, i32([0]))
    codes, scales = ref.encode(x)
    assert torch.equal(c.k_scales.cpu().long(), scales)
    k, v = thin_q4_load(c, i32([0]), 8, dtype=torch.float32)
    assert torch.equal(k.cpu().double(), ref.values(codes, scales)) and torch.equal(k, v)
    assert k.isfinite().all()


@pytest.mark.parametrize("d", [32, 64, 128])
def test_load(d):
    g = gen(5)
    c = fresh(2, 3, 90, d)
    x, y = randn(g, 2, 3, 90, d), randn(g, 2, 3, 90, d)
    thin_q4_store(x.to(DEV), y.to(DEV), c, i32([0, 0]))
    for dtype in (torch.float32, torch.bfloat16):
        k, v = thin_q4_load(c, i32([-3, 70]), 30, dtype=dtype)
        for got, codes, scales in ((k, c.k_codes, c.k_scales), (v, c.v_codes, c.v_scales)):
            want = torch.zeros(2, 3, 30, d, dtype=torch.float64)
            all_ = ref.cached(codes, scales)
            want[0, :, 3:] = all_[0, :, :27]
            want[1, :, :20] = all_[1, :, 70:]
            assert torch.equal(got.cpu().double(), want)


def test_calls_without_new_rows_leave_the_bounds():
    """No token (count 0), or tokens behind the cache: nothing changes, though rows of the
    position's block stand before it."""
    g = gen(23)
    c = fresh(3, 1, 100, 64)
    x = randn(g, 3, 1, 100, 64).to(DEV)
    thin_q4_store(x, x, c, i32([0, 0, 0]))
    before = [t.clone() for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.bounds)]
    thin_q4_store(x[:, :, :4] * 9, x[:, :, :4], c, i32([70, 101, 2000000000]),
                  count=i32([0, 4, 4]))
    for t, was in zip((c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.bounds), before):
        assert torch.equal(t, was)


def test_rewound_rows_leave_the_bounds():
    g = gen(6)
    c = fresh(1, 1, 200, 64)
    x = randn(g, 1, 1, 150, 64)
    x[:, :, 100:] *= 50
    thin_q4_store(x.to(DEV), x.to(DEV), c, i32([0]))
    thin_q4_store(x[:, :, :1].to(DEV), x[:, :, :1].to(DEV), c, i32([100]))
    want = ref.bounds(ref.cached(c.k_codes, c.k_scales), 101)
    assert torch.equal(c.bounds.cpu().double()[:, :, :2], want)


# ---------------------------------------------------------------------------
# Selection
# ---------------------------------------------------------------------------
def filled(g, B, H, n_max, d, rows):
    """A cache whose sequence b holds rows[b] rows; the rest is not stored."""
    c = fresh(B, H, n_max, d, fill=0xff)
    x = randn(g, B, H, n_max, d) * 2
    x += randn(g, B, H, (n_max + 63) // 64, d).repeat_interleave(64, 2)[:, :, :n_max]
    thin_q4_store(x.to(DEV), randn(g, B, H, n_max, d).to(DEV), c, i32([0] * B), count=i32(rows))
    return c


def check_select(c, q, at, count, n_sel, n_sinks, n_window, got):
    B, Hq, T, d = q.shape
    G = Hq // c.H
    bnd = c.bounds.cpu().double()
    got = got.cpu()
    for b in range(B):
        for h in range(c.H):
            for t in range(T):
                last = min(at[b] + t, c.n_max - 1)
                if count is not None and t >= count[b]:
                    last = -1
                sc = ref.block_scores(q[b, h * G:(h + 1) * G, t], bnd[b, h]).tolist()
                want = ref.select(sc, last, n_sel, n_sinks, n_window)
                assert got[b, h, t].tolist() == want + [-1] * (n_sel - len(want)), (b, h, t)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,G,T,n_max,at,count,sel", [
    (128, 2, 2, 4, 1, 3000, [2999, 700], None, (7, 1, 2)),
    (64, 1, 1, 1, 5, 1, [0], None, (1, 0, 1)),
    (64, 3, 1, 3, 1, 700, [-1, 640, 900], None, (4, 1, 1)),
    (32, 2, 3, 17, 9, 1000, [600, 0], [9, 4], (5, 2, 3)),
    (128, 1, 1, 2, 3, 9000, [8990], None, (60, 0, 1)),
    (64, 1, 2, 1, 2, 40000, [39998], None, (33, 3, 5)),
    (32, 1, 1, 2, 2, 140000, [139000], None, (100, 1, 2))])
def test_select(dtype, d, B, H, G, T, n_max, at, count, sel):
    g = gen(7)
    rows = [max(0, min(n_max, a + T)) for a in at]
    c = filled(g, B, H, n_max, d, rows)
    q = randn(g, B, H * G, T, d, dtype=dtype)
    got = thin_q4_select(strided(q), c, i32(at), sel[0], n_sinks=sel[1], n_window=sel[2],
                         count=None if count is None else i32(count))
    check_select(c, q, at, count, *sel, got)


def test_select_ties_and_nan():
    """Equal scores at the border take the lowest blocks; a NaN score is the least."""
    g = gen(8)
    c = fresh(1, 1, 64 * 300, 64)
    c.bounds.zero_()
    c.bounds[:, :, 200:210] = 1.0
    q = randn(g, 1, 1, 1, 64)
    got = thin_q4_select(q.to(DEV), c, i32([64 * 300 - 1]), 20, n_sinks=1, n_window=1)
    check_select(c, q, [64 * 300 - 1], None, 20, 1, 1, got)
    c.bounds[:, :, 3:290] = math.nan
    got = thin_q4_select(q.to(DEV), c, i32([64 * 300 - 1]), 20, n_sinks=1, n_window=1)
    check_select(c, q, [64 * 300 - 1], None, 20, 1, 1, got)
    q[:] = math.nan
    got = thin_q4_select(q.to(DEV), c, i32([64 * 300 - 1]), 20, n_sinks=0, n_window=1)
    assert got.flatten().tolist() == list(range(19)) + [299]


# Enough tokens for the launch that scores 16 of them at a time (64 workgroups).
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,G,T,n_max,at,count,sel", [
    (128, 4, 4, 4, 67, 9000, [0, 8900, 4000, 700], [67, 67, 30, 0], (9, 1, 2)),
    (64, 1, 32, 3, 33, 2000, [1990], None, (5, 0, 1)),
    (32, 2, 40, 1, 9, 30000, [-4, 29000], None, (40, 2, 3)),
    (128, 1, 33, 17, 20, 300, [200], None, (1, 0, 1))])
def test_select_of_prompts(dtype, d, B, H, G, T, n_max, at, count, sel):
    g = gen(21)
    rows = [max(0, min(n_max, a + T)) for a in at]
    c = filled(g, B, H, n_max, d, rows)
    q = randn(g, B, H * G, T, d, dtype=dtype)
    got = thin_q4_select(strided(q), c, i32(at), sel[0], n_sinks=sel[1], n_window=sel[2],
                         count=None if count is None else i32(count))
    check_select(c, q, at, count, *sel, got)


@pytest.mark.parametrize("kind", ["equal", "near", "nan", "inf", "zero", "tiny", "nan query"])
@pytest.mark.parametrize("nb,n_sel", [(100, 20), (600, 70), (1500, 9)])
def test_select_of_prompts_at_borders(kind, nb, n_sel):
    """Scores that float32 sums cannot tell apart, and values that are none."""
    g = gen(22)
    H, T, d = 64, 3, 64
    c = fresh(1, H, 64 * nb, d)
    x = torch.randn(1, 1, 1, 2, d, generator=g).bfloat16().expand(1, H, nb, 2, d).clone()
    if kind == "near":
        # differences of 2^-20 of a channel and less, both ways
        step = torch.randint(-3, 4, (1, H, nb, 2), generator=g).float() * 2.0 ** -20
        x[..., 5] = step.bfloat16()
    if kind == "nan":
        x[:, :, nb // 3:nb // 2] = math.nan
    if kind == "inf":
        x[:, ::2, nb // 3:nb // 2, 1, 4] = math.inf
    if kind == "zero":
        x.zero_()
    if kind == "tiny":
        x = (torch.randn(1, H, nb, 2, d, generator=g) * 2.0 ** -124).bfloat16()
    # (least, then largest)
    c.bounds.copy_(torch.stack((torch.minimum(x[..., 0, :], x[..., 1, :]),
                                torch.maximum(x[..., 0, :], x[..., 1, :])), -2))
    q = randn(g, 1, 2 * H, T, d, dtype="bf16")
    if kind == "tiny":
        q = (q.float() * 2.0 ** -20).bfloat16()
    if kind == "nan query":
        q[:, ::3, 1] = math.nan
    at = 64 * nb - T
    got = thin_q4_select(q.to(DEV), c, i32([at]), n_sel, n_sinks=1, n_window=2).cpu()
    for h in range(0, H, 7):
        check_select_head(c, q, at, n_sel, 1, 2, got, h)


def check_select_head(c, q, at, n_sel, n_sinks, n_window, got, h):
    G = q.shape[1] // c.H
    for t in range(q.shape[2]):
        sc = ref.block_scores(q[0, h * G:(h + 1) * G, t], c.bounds[0, h].cpu()).tolist()
        want = ref.select(sc, at + t, n_sel, n_sinks, n_window)
        assert got[0, h, t].tolist() == want, (h, t)


def test_select_of_small_queries_beside_large_bounds():
    """Sums of queries whose second bf16 part lies below the normal numbers, scores of
    ordinary size that differ by 2^-10 and less."""
    g = gen(25)
    H, T, d, nb = 64, 3, 64, 300
    c = fresh(1, H, 64 * nb, d)
    x = torch.randn(1, 1, 1, 2, d, generator=g).expand(1, H, nb, 2, d).clone()
    x[..., 5] += torch.randn(1, H, nb, 2, generator=g) * 2.0 ** -7
    x = (x * 2.0 ** 110).bfloat16()
    c.bounds.copy_(torch.stack((torch.minimum(x[..., 0, :], x[..., 1, :]),
                                torch.maximum(x[..., 0, :], x[..., 1, :])), -2))
    q = (torch.randn(1, 2 * H, T, d, generator=g) * 2.0 ** -121).bfloat16()
    at = 64 * nb - T
    got = thin_q4_select(q.to(DEV), c, i32([at]), 40, n_sinks=1, n_window=2).cpu()
    for h in range(0, H, 7):
        check_select_head(c, q, at, 40, 1, 2, got, h)


@pytest.mark.parametrize("d,n_max", [(32, 2000), (128, 2000), (64, 12000)])
def test_select_of_long_prompts(d, n_max):
    """More than 1024 times 16 tokens."""
    g = gen(27)
    H, T = 64, 290
    c = filled(g, 1, H, n_max, d, [n_max])
    q = randn(g, 1, 2 * H, T, d, dtype="bf16")
    at = n_max - T
    got = thin_q4_select(q.to(DEV), c, i32([at]), 9, n_sinks=1, n_window=2).cpu()
    for h in (0, 31, 63):
        check_select_head(c, q, at, 9, 1, 2, got, h)


@pytest.mark.parametrize("count", [None, [40, 17, 0]])
def test_select_of_prompts_in_large_caches(count):
    """Tokens that see more blocks than the launch of 16 tokens holds beside others."""
    g = gen(26)
    B, H, T, d, n = 3, 12, 40, 32, 140000
    at = [131072 - 20, 139950, 700]
    c = fresh(B, H, n, d)
    x = torch.randn(B, H, (n + 63) // 64, 2, d, generator=g)
    c.bounds.copy_(x.sort(-2)[0].bfloat16())
    q = randn(g, B, 2 * H, T, d, dtype="bf16")
    got = thin_q4_select(q.to(DEV), c, i32(at), 9,
                         count=None if count is None else i32(count)).cpu()
    bnd = c.bounds.cpu()
    for b in range(B):
        for h in (0, 7, 11):
            for t in range(T):
                last = at[b] + t if count is None or t < count[b] else -1
                sc = ref.block_scores(q[b, 2 * h:2 * h + 2, t], bnd[b, h]).tolist()
                want = ref.select(sc, min(last, n - 1), 9, 1, 2)
                assert got[b, h, t].tolist() == want + [-1] * (9 - len(want)), (b, h, t)


def test_select_in_pieces():
    """More tokens than the scores held at a time: 8 slices x 2049 blocks."""
    g = gen(9)
    n = 131073
    c = filled(g, 1, 8, n, 32, [n])
    q = randn(g, 1, 8, 600, 32, dtype="bf16").to(DEV)
    got = thin_q4_select(q, c, i32([n - 600]), 9)
    for t in (0, 510, 511, 512, 599):
        one = thin_q4_select(q[:, :, t:t + 1], c, i32([n - 600 + t]), 9)
        assert torch.equal(got[:, :, t:t + 1], one)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
# float32 queries: the matrix instructions add a row's d products in float32 (2^-24 of the
# sum of magnitudes for each of at most d additions, far fewer in sequence: 16 for d = 128
# with the parts of the queries), the scale and the exponential another few 2^-24 of the
# score: at most 2^-19 S, S = the largest sum |q_c k_c| / sqrt d.  A weight's relative error
# is that, twice (its own and the maximum's), and the sums of weights and of products
# 2^-20; the output rounds by half a step.  All of it is taken twice.  bf16 queries: a
# weight rounds by half a step of bf16 as well; the second half-step that the factor of two
# leaves covers what the scaled instruction cuts (1e-6 S for normal values, 6e-5 S seen at
# most: below 2^-8 up to S = 32).
def attention_bound(want, A, S, dtype):
    rel = 2 * 2.0 ** -19 * S + 2.0 ** -20 + (half_step("bf16") if dtype == "bf16" else 0.0)
    return rel * A * 2 + half_step(dtype) * want.abs() + 1e-30


def check_attention(c, q, at, count, blocks, got, dtype, tokens=None):
    B, Hq, T, d = q.shape
    G = Hq // c.H
    got = got.cpu().double()
    nb = (c.n_max + 63) // 64
    for b in range(B):
        for h in range(c.H):
            k = ref.cached(c.k_codes[b, h], c.k_scales[b, h])
            v = ref.cached(c.v_codes[b, h], c.v_scales[b, h])
            for t in (range(T) if tokens is None else tokens):
                last = min(at[b] + t, c.n_max - 1)
                if count is not None and t >= count[b]:
                    last = -1
                n = max(0, last + 1)
                w = torch.ones(n, dtype=torch.float64)
                if blocks is not None:
                    w[:] = 0
                    for j in blocks[b, h, t].tolist():
                        if 0 <= j < nb:
                            w[j * 64:(j + 1) * 64] += 1
                rows = slice(h * G, (h + 1) * G)
                o = got[b, rows, t]
                if n <= 0 or not (w > 0).any():
                    assert (o == 0).all()
                    continue
                want, A, S = ref.attention(q[b, rows, t], k[:n], v[:n], w.expand(G, n))
                assert ((o - want).abs() <= attention_bound(want, A, S, dtype)).all(), (b, h, t)


def check_dense(c, q, at, count, got, dtype):
    """check_attention without lists, a slice at a time."""
    B, Hq, T, d = q.shape
    G = Hq // c.H
    got = got.cpu().double()
    for b in range(B):
        last = torch.arange(T) + at[b]
        last = torch.where(torch.arange(T) < (T if count is None else count[b]),
                           last.clamp(max=c.n_max - 1), -1)
        n = max(0, int(last.max()) + 1)
        w = (torch.arange(n) <= last.unsqueeze(1)).double().repeat(G, 1)  # [G * T, n]
        for h in range(c.H):
            o = got[b, h * G:(h + 1) * G].reshape(G * T, d)
            if n == 0:
                assert (o == 0).all()
                continue
            want, A, S = ref.attention(q[b, h * G:(h + 1) * G].reshape(G * T, d),
                                       ref.cached(c.k_codes[b, h, :n], c.k_scales[b, h, :n]),
                                       ref.cached(c.v_codes[b, h, :n], c.v_scales[b, h, :n]), w)
            ok = (o - want).abs() <= attention_bound(want, A, S, dtype)
            assert ok.all(), (b, h, (~ok).nonzero()[:3].tolist())


# Enough query rows for the kernel that shares decoded rows, the last workgroup of a slice
# partly filled; the last three with workgroups that share a tile's keys, too.
PROMPT = [
    (128, 4, 16, 4, 130, 700, [0, 300, 570, 650], None),
    (64, 8, 8, 1, 513, 600, [0, 5, 87, -20, 60, 300, 1, 80], [513, 500, 0, 400, 1, 300, 129, 64]),
    (32, 16, 16, 16, 9, 300, list(range(0, 288, 18)), None),
    (128, 2, 50, 3, 171, 171, [0, 0], [171, 100]),
    (64, 43, 2, 7, 55, 200, [3 * b for b in range(43)], None),
    (128, 1, 8, 4, 67, 5000, [4900], None),
    (64, 4, 4, 2, 70, 3000, [2930, 0, -30, 1500], [70, 70, 60, 0]),
    (32, 2, 3, 9, 60, 9000, [8940, 1000], None),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,G,T,n_max,at,count", PROMPT)
def test_attention_of_prompts(dtype, d, B, H, G, T, n_max, at, count):
    g = gen(20)
    rows = [max(0, min(n_max, a + T)) for a in at]
    c = filled(g, B, H, n_max, d, rows)
    q = randn(g, B, H * G, T, d, dtype=dtype)
    o = strided(torch.zeros_like(q))
    got = thin_q4_attention(strided(q), c, i32(at), count=None if count is None else i32(count),
                            O=o)
    check_dense(c, q, at, count, got, dtype)
    again = thin_q4_attention(q.to(DEV), c, i32(at), count=None if count is None else i32(count))
    assert torch.equal(again, got)


ATT = [
    # d, B, H, G, T, n_max, at, count
    (128, 1, 1, 1, 1, 1, [0], None),
    (128, 2, 2, 4, 1, 700, [699, 31], None),
    (64, 3, 2, 3, 1, 260, [-1, 0, 300], None),
    (32, 2, 1, 8, 1, 5000, [4999, 128], None),
    (64, 1, 3, 1, 5, 100, [95], None),
    (128, 2, 1, 5, 7, 300, [200, 0], [7, 3]),
    (64, 1, 2, 16, 3, 500, [400], None),
    (128, 1, 1, 20, 2, 200, [100], None),
    (32, 2, 2, 2, 33, 90, [-5, 60], [33, 0]),
    (128, 1, 2, 2, 130, 400, [270], None),
    (64, 1, 1, 4, 300, 300, [0], None),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,G,T,n_max,at,count", ATT)
def test_attention(dtype, d, B, H, G, T, n_max, at, count):
    g = gen(10)
    rows = [max(0, min(n_max, a + T)) for a in at]
    c = filled(g, B, H, n_max, d, rows)
    q = randn(g, B, H * G, T, d, dtype=dtype)
    o = strided(torch.zeros_like(q))
    got = thin_q4_attention(strided(q), c, i32(at), count=None if count is None else i32(count),
                            O=o)
    assert got is o
    check_attention(c, q, at, count, None, got, dtype)
    again = thin_q4_attention(q.to(DEV), c, i32(at), count=None if count is None else i32(count))
    assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,G,T,n_max,at,count,n_sel", [
    (128, 2, 2, 4, 1, 3000, [2999, 700], None, 6), (64, 1, 2, 1, 3, 1000, [900], None, 5),
    (32, 2, 1, 18, 2, 500, [400, -1], [2, 1], 3), (128, 1, 1, 2, 40, 2000, [1900], None, 9),
    (64, 1, 1, 6, 1, 20000, [19999], None, 200)])
def test_attention_over_blocks(dtype, d, B, H, G, T, n_max, at, count, n_sel):
    g = gen(11)
    rows = [max(0, min(n_max, a + T)) for a in at]
    c = filled(g, B, H, n_max, d, rows)
    q = randn(g, B, H * G, T, d, dtype=dtype)
    nb = (n_max + 63) // 64
    # any order, blocks behind the token, twice the same, -1 and places outside
    blocks = torch.randint(0, nb, (B, H, T, n_sel), generator=g, dtype=torch.int32)
    blocks[..., 0] = -1
    if n_sel > 4:
        blocks[..., 1] = blocks[..., 2]
        blocks[..., 3] = nb
        blocks[0, 0, 0] = -1  # nothing listed
    got = thin_q4_attention(q.to(DEV), c, i32(at), blocks=blocks.to(DEV),
                            count=None if count is None else i32(count))
    check_attention(c, q, at, count, blocks, got, dtype)
    chosen = thin_q4_select(q.to(DEV), c, i32(at), n_sel, n_sinks=1, n_window=1,
                            count=None if count is None else i32(count))
    got = thin_q4_attention(q.to(DEV), c, i32(at), blocks=chosen,
                            count=None if count is None else i32(count))
    check_attention(c, q, at, count, chosen.cpu(), got, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lengths", [[4200] * 20, [4200, 1, 0, 4199, 77] * 5, [0] * 19 + [4200]])
def test_attention_shares_of_many_sequences(dtype, lengths):
    """Sequences of one length, of many and almost none: every one's keys are shared out."""
    g = gen(15)
    B = len(lengths)
    c = filled(g, B, 2, 4200, 32, lengths)
    q = randn(g, B, 6, 1, 32, dtype=dtype)
    at = [n - 1 for n in lengths]
    check_attention(c, q, at, None, None, thin_q4_attention(q.to(DEV), c, i32(at)), dtype)


def test_attention_large_scores():
    """Scores in the thousands: the running maximum moves, weights underflow."""
    g = gen(12)
    c = fresh(1, 1, 900, 64)
    k = randn(g, 1, 1, 900, 64) * torch.linspace(0.1, 60, 900).view(1, 1, 900, 1)
    thin_q4_store(k.to(DEV), randn(g, 1, 1, 900, 64).to(DEV), c, i32([0]))
    for dtype in ("fp32", "bf16"):
        q = randn(g, 1, 4, 3, 64, dtype=dtype) * 5
        check_attention(c, q, [897], None, None, thin_q4_attention(q.to(DEV), c, i32([897])), dtype)


def test_attention_nan_query_stays_in_its_row():
    g = gen(13)
    c = filled(g, 1, 1, 300, 64, [300])
    for dtype in ("fp32", "bf16"):
        q = randn(g, 1, 4, 3, 64, dtype=dtype)
        want = thin_q4_attention(q.to(DEV), c, i32([297]))
        q[0, 1, 2, 5] = math.nan
        got = thin_q4_attention(q.to(DEV), c, i32([297]))
        assert got[0, 1, 2].isnan().all()
        keep = torch.ones(4, 3, dtype=torch.bool)
        keep[1, 2] = False
        assert torch.equal(got[0][keep], want[0][keep])


@pytest.mark.parametrize("T", [3, 700])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attention_infinite_query_has_no_softmax(dtype, T):
    """Scores of +-infinity and 0 times infinity: the row is not a number, others keep theirs."""
    g = gen(14)
    c = filled(g, 8, 4, 1024, 64, [1024] * 8)
    q = randn(g, 8, 8, T, 64, dtype=dtype).to(DEV)
    at = i32([1024 - T] * 8)
    want = thin_q4_attention(q, c, at)
    q[3, 1, 2, 5] = math.inf
    q[5, 6, T - 1, 63] = -math.inf
    got = thin_q4_attention(q, c, at)
    odd = torch.zeros(8, 8, T, dtype=torch.bool, device=DEV)
    odd[3, 1, 2] = odd[5, 6, T - 1] = True
    assert got[odd].isnan().all()
    assert torch.equal(got[~odd], want[~odd])


def test_long_cache_offsets():
    """Rows whose byte offsets pass 32 bits: 2^21 rows x 40 heads x 64 bytes."""
    n, H = 1 << 21, 40
    c = Q4Cache(1, H, n, 128, device=DEV)
    for t in (c.k_codes, c.v_codes):
        t.zero_()
    for t in (c.k_scales, c.v_scales):
        t.fill_(127)
    c.bounds.zero_()
    assert c.k_codes.numel() > 2 ** 32
    g = gen(14)
    x = randn(g, 1, H, 70, 128)
    at = n - 70
    thin_q4_store(x.to(DEV), x.to(DEV), c, i32([at]))
    k, v = thin_q4_load(c, i32([at]), 70)
    codes, scales = ref.encode(x)
    assert torch.equal(k.cpu().double(), ref.values(codes, scales))
    q = randn(g, 1, H, 1, 128, dtype="bf16") * 4
    blocks = thin_q4_select(q.to(DEV), c, i32([n - 1]), 3, n_sinks=0, n_window=1)
    # every block but the last two holds zeros: their scores are 0
    got = thin_q4_attention(q.to(DEV), c, i32([n - 1]), blocks=blocks)
    for h in (0, H - 1):
        last = c.bounds[0, h, -2:].cpu()
        s = float(ref.block_scores(q[0, h:h + 1, 0], last)[0])
        want = [n // 64 - 2, n // 64 - 1] if s > 0 else [1, n // 64 - 1]
        assert blocks[0, h, 0].tolist() == [0] + want
        rows = torch.cat([torch.arange(j * 64, j * 64 + 64) for j in blocks[0, h, 0].tolist()])
        kk = ref.cached(c.k_codes[0, h, rows.to(DEV)], c.k_scales[0, h, rows.to(DEV)])
        vv = ref.cached(c.v_codes[0, h, rows.to(DEV)], c.v_scales[0, h, rows.to(DEV)])
        o, A, S = ref.attention(q[0, h:h + 1, 0], kk, vv, torch.ones(1, 192, dtype=torch.float64))
        err = (got[0, h:h + 1, 0].cpu().double() - o).abs()
        assert (err <= attention_bound(o, A, S, "bf16")).all()


# ---------------------------------------------------------------------------
# Together, streams, graphs
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("n_sel", [0, 4])
def test_steps_together(n_sel):
    """A padded prompt, then steps: every output against the whole definition."""
    g = gen(15)
    B, H, G, d, n_max = 2, 2, 3, 64, 900
    turns, amp = thin_rotary_turns(32, scaling="bands", factor=2.0, length=512.0)
    t = turns.to(DEV)
    c = Q4Cache(B, H, n_max, d, device=DEV)
    lens = [0, 0]
    for T, count in ((600, [600, 411]), (1, None), (3, [2, 3]), (1, None)):
        q, k, v = (randn(g, B, n, T, d, dtype="bf16") for n in (H * G, H, H))
        cnt = [T, T] if count is None else count
        got = c.step(q.to(DEV), k.to(DEV), v.to(DEV), i32(lens), turns=t, amp=amp,
                     count=None if count is None else i32(count), n_sel=n_sel, n_window=1)
        # the rows of the cache are those of the turned keys: to half a bf16 step
        # of the turn they may round to a neighbouring code, so the reference takes
        # the library's turned rows and is exact from there
        qr, kr = thin_rotary(q.to(DEV), i32(lens), t, Y=k.to(DEV), amp=amp)
        for b in range(B):
            codes, scales = ref.encode(kr[b, :, :cnt[b]].cpu())
            rows = slice(lens[b], lens[b] + cnt[b])
            assert torch.equal(ref.cached(c.k_codes[b][:, rows], c.k_scales[b][:, rows]),
                               ref.values(codes, scales))
        blocks = None
        if n_sel:
            blocks = thin_q4_select(qr, c, i32(lens), n_sel, n_window=1,
                                    count=None if count is None else i32(count))
            if T < 10:
                check_select(c, qr.cpu(), lens, count, n_sel, 1, 1, blocks)
            blocks = blocks.cpu()
        check_attention(c, qr.cpu(), lens, count, blocks, got, "bf16",
                        tokens=None if T < 10 else [0, 1, 255, 410, 411, 599])
        lens = [a + x for a, x in zip(lens, cnt)]


def same_contents(a, b):
    return all(torch.equal(getattr(a, name), getattr(b, name))
               for name in ("k_codes", "k_scales", "v_codes", "v_scales", "bounds"))


def test_replayed_step_follows_its_positions():
    """A captured step on another stream, replayed with new rows and positions."""
    g = gen(16)
    B, H, G, d, n_max = 2, 2, 4, 128, 2000
    turns, _ = thin_rotary_turns(128)
    t = turns.to(DEV)
    caches = [filled(gen(17), B, H, n_max, d, [1500, 70]) for _ in range(2)]
    q, k, v = (torch.zeros(B, n, 1, d, dtype=torch.bfloat16, device=DEV) for n in (H * G, H, H))
    at = i32([1500, 70])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        caches[0].step(q, k, v, at, turns=t, n_sel=6)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = caches[0].step(q, k, v, at, turns=t, n_sel=6)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(randn(g, *x.shape, dtype="bf16"))
        at.copy_(i32([1500 + i, 70 + i]))
        graph.replay()
        want = caches[1].step(q, k, v, at.clone(), turns=t, n_sel=6)
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        assert same_contents(*caches)


@pytest.mark.parametrize("T,n_max,d,n_sel", [(33, 60000, 32, 5), (70, 5000, 128, 0)])
def test_replayed_prompt_follows_its_positions(T, n_max, d, n_sel):
    """A captured chunk (choice with over 64 KiB of LDS; shared tiles and their join),
    replayed with new rows, positions and counts, eager work between."""
    g = gen(24)
    B, H, G = 2, 32 if n_sel else 2, 2
    caches = [filled(gen(25), B, H, n_max, d, [n_max, n_max]) for _ in range(2)]
    q, k, v = (torch.zeros(B, n, T, d, dtype=torch.bfloat16, device=DEV) for n in (H * G, H, H))
    at, count = i32([n_max - T, 100]), i32([T, T])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in caches:
            c.step(q, k, v, at, count=count, n_sel=n_sel)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = caches[0].step(q, k, v, at, count=count, n_sel=n_sel)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(randn(g, *x.shape, dtype="bf16"))
        at.copy_(i32([n_max - T - 7 * i, 100 + 900 * i]))
        count.copy_(i32([T - i, T if i % 2 else 1]))
        graph.replay()
        want = caches[1].step(q, k, v, at.clone(), count=count.clone(), n_sel=n_sel)
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        assert same_contents(*caches)


def test_binding_refuses_what_does_not_fit():
    from paper_2606_10944_amd._lib import THIN_EDTYPE, THIN_EINVAL, THIN_EWORKSPACE, ThinError
    g = gen(26)
    c = filled(g, 2, 2, 5000, 64, [5000, 5000])
    q = randn(g, 2, 4, 1, 64, dtype="bf16").to(DEV)
    at = i32([10, 20])
    turns = thin_rotary_turns(64)[0].to(DEV)
    kv = randn(g, 2, 2, 1, 64).to(DEV)
    wide = torch.zeros(2, 4, 1, 128, dtype=torch.bfloat16, device=DEV)

    def refused(status, f, *a, **kw):
        with pytest.raises(ThinError) as e:
            f(*a, **kw)
        assert e.value.status == status

    for bad in (q.cpu(), q[:1], q[..., :32], q[:, :3], q[0], wide[..., ::2]):
        refused(THIN_EINVAL, thin_q4_attention, bad, c, at)
        refused(THIN_EINVAL, thin_q4_select, bad, c, at, 4)
    refused(THIN_EINVAL, thin_q4_attention, wide[..., 4:68], c, at)  # not 16-byte aligned
    refused(THIN_EDTYPE, thin_q4_attention, q.half(), c, at)
    for bad in (at.long(), at[:1], at.cpu(), torch.stack((at, at), 1)[:, 0]):
        refused(THIN_EINVAL, thin_q4_attention, q, c, bad)
        refused(THIN_EINVAL, thin_q4_attention, q, c, at, count=bad)
        refused(THIN_EINVAL, thin_q4_store, kv, kv, c, bad)
        refused(THIN_EINVAL, thin_rotary, q, bad, turns)
    refused(THIN_EINVAL, thin_q4_attention, q, c, at, O=q.float())
    refused(THIN_EINVAL, thin_q4_attention, q, c, at, O=torch.zeros_like(q[:1]).expand(2, 4, 1, 64))
    refused(THIN_EINVAL, thin_q4_attention, q, c, at, blocks=i32([[1]]))
    refused(THIN_EINVAL, thin_q4_attention, q, c, at,
            blocks=torch.zeros(2, 2, 1, 4, dtype=torch.int64, device=DEV))
    refused(THIN_EWORKSPACE, thin_q4_attention, q, c, at,
            workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))
    refused(THIN_EINVAL, thin_q4_select, q, c, at, 4, n_sinks=3)
    refused(THIN_EINVAL, thin_q4_select, q, c, at, 0)
    refused(THIN_EINVAL, thin_q4_store, kv[:, :1], kv, c, at)
    refused(THIN_EDTYPE, thin_q4_store, kv, kv.bfloat16(), c, at)
    refused(THIN_EINVAL, thin_q4_load, c, at, 0)
    refused(THIN_EINVAL, thin_q4_load, c, at, 3, K=kv)
    for bad in (turns.float(), turns.cpu(), turns[:12], turns[::2]):
        refused(THIN_EINVAL, thin_rotary, q, at, bad)
    refused(THIN_EINVAL, thin_rotary, q, at, turns, layout="other")
    refused(THIN_EINVAL, thin_rotary, q, at, turns, Y=kv[:1].bfloat16())
    refused(THIN_EDTYPE, thin_rotary, q, at, turns, Y=kv)
    refused(THIN_EINVAL, thin_rotary, q, at, turns, out_Y=q)
    # the current device has not stopped working
    check_attention(c, q.cpu(), [10, 20], None, None, thin_q4_attention(q, c, at), "bf16")


def test_calls_on_a_stream_of_their_own():
    g = gen(18)
    c = filled(g, 1, 2, 1000, 64, [1000])
    q = randn(g, 1, 8, 1, 64, dtype="bf16").to(DEV)
    at = i32([999])
    want = thin_q4_attention(q, c, at, blocks=thin_q4_select(q, c, at, 5))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    blocks = thin_q4_select(q, c, at, 5, stream=side)
    got = thin_q4_attention(q, c, at, blocks=blocks, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_rows_of_the_cache_feed_the_coreset_path():
    """Cached rows, read back, are thinned and attended over as any rows are."""
    from paper_2606_10944_amd import thin_attention, thin_compress, thin_plan
    g = gen(19)
    c = filled(g, 1, 2, 512, 64, [512])
    k, v = thin_q4_load(c, i32([0]), 512)
    plan = thin_plan(1, 2, 512, 64, 512, 0)
    u = torch.rand(max(plan["uniforms_total"], 1), generator=g).to(DEV)
    idx = thin_compress(k, v, 512, 0, u)  # every row
    q = randn(g, 1, 2, 3, 64, dtype="bf16")
    got = thin_attention(q.to(DEV), k, v, idx)
    full = thin_q4_attention(q.to(DEV), c, i32([511]))[:, :, :1]
    for h in range(2):
        o, A, S = ref.attention(q[0, h, :1], k[0, h].cpu().double(), v[0, h].cpu().double(),
                                torch.ones(1, 512, dtype=torch.float64))
        assert ((got[0, h, :1].cpu().double() - o).abs() <= 2e-3).all()
        assert ((full[0, h].cpu().double() - o).abs() <= attention_bound(o, A, S, "bf16")).all()
