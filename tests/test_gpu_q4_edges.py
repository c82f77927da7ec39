"""The 4-bit cache's operators where rounding and ends of ranges show: outlier
channels, weights that sum to one, borders of a selection, many sequences."""
import math

import pytest
import torch

import q4_reference as ref
from paper_2606_10944_amd import Q4Cache, thin_q4_attention, thin_q4_load, thin_q4_select, thin_q4_store
from test_gpu_q4 import (DEV, attention_bound, check_attention, check_select_head, filled, fresh,
                         gen, i32, randn)

pytestmark = pytest.mark.gpu


# Calls (B, H, G, T, blocks listed) of the kernel for few query rows, over every row and
# over lists, and of the kernel for many.
KERNELS = {"few": (1, 1, 4, 1, False), "listed": (1, 2, 4, 2, True),
           "many": (16, 16, 4, 32, False)}


def two_kinds(kind, k, q, n_max=300):
    """Attention over rows that hold k[0] and k[1] in turn, whose values are 1 and -1: a
    cache, queries of the rows q, and the call's arguments."""
    B, H, G, T, listed = KERNELS[kind]
    d = q.numel()
    c = fresh(B, H, n_max, d)
    rows = torch.stack((k[0], k[1])).repeat(n_max // 2, 1).expand(B, H, n_max, d)
    vals = torch.tensor([1.0, -1.0]).repeat(n_max // 2).view(1, 1, n_max, 1).expand(B, H, n_max, d)
    thin_q4_store(rows.contiguous().to(DEV), vals.contiguous().to(DEV), c, i32([0] * B))
    assert torch.equal(ref.cached(c.k_codes[0, 0, :2], c.k_scales[0, 0, :2]),
                       torch.stack(k).double())  # the cache holds them exactly
    queries = q.view(1, 1, 1, d).expand(B, H * G, T, d).contiguous()
    blocks = None
    if listed:
        blocks = torch.arange((n_max + 63) // 64, dtype=torch.int32).expand(B, H, T, -1).contiguous()
    return c, queries, [n_max - T] * B, blocks


def check_two_kinds(kind, k, q):
    for dtype in (torch.bfloat16, torch.float32):
        c, queries, at, blocks = two_kinds(kind, k, q.to(dtype))
        got = thin_q4_attention(queries.to(DEV), c, i32(at),
                                blocks=None if blocks is None else blocks.to(DEV))
        one = Q4Cache.over(*[x[:1, :1].contiguous() for x in (c.k_codes, c.k_scales, c.v_codes,
                                                               c.v_scales, c.bounds)])
        G = KERNELS[kind][2]
        name = "bf16" if dtype == torch.bfloat16 else "fp32"
        check_attention(one, queries[:1, :G], at[:1], None,
                        None if blocks is None else blocks[:1, :1], got[:1, :G], name)
        B, H = c.B, c.H  # (the slices are alike)
        assert torch.equal(got.view(B, H, G, *got.shape[2:]),
                           got[:1, :G].view(1, 1, G, *got.shape[2:]).expand(B, H, -1, -1, -1))


@pytest.mark.parametrize("kind", list(KERNELS))
@pytest.mark.parametrize("d", [32, 64, 128])
def test_attention_keeps_small_products_beside_a_large_one(d, kind):
    """One channel of every key and query makes a product of 6144, the same for all keys;
    products of 1/8 of the others order them (2^-15.6 of it: below half a step of a sum in
    16 bits, 2^8 steps of one in float32)."""
    k = torch.zeros(2, d)
    q = torch.zeros(d)
    # beside it, under its scale, and under scales of their own
    k[0, 1:32], k[1, 1:32], q[1:32] = 8.0, -8.0, 2.0 ** -6
    k[0, 32:], k[1, 32:], q[32:] = 0.5, -0.5, 0.25
    k[:, 0] = 96.0
    q[0] = 64.0
    check_two_kinds(kind, list(k), q)


@pytest.mark.parametrize("kind", list(KERNELS))
@pytest.mark.parametrize("d", [32, 64, 128])
def test_attention_keeps_all_bits_of_small_query_channels(d, kind):
    """Channels 2^-12 of the row's largest that differ in their last bf16 bit alone, which
    decides between two kinds of keys; the largest meets zeros."""
    k = torch.zeros(2, d)
    k[0, 1::2], k[0, 2::2] = 0.5, -0.5
    q = torch.full((d,), 64.0)
    q[1::2] = 64.5
    q[0] = 2.0 ** 18
    check_two_kinds(kind, list(k), q)


# Weights are rounded, but their sum is that of the rounded ones: values that are all one
# number come back as it, whatever the weights (sums and quotient are off by 2^-18 at most,
# and the output's nearest bf16 is the number itself).
def ones_cache(k):
    B, H, n, d = k.shape
    c = fresh(B, H, n, d)
    thin_q4_store(k.to(DEV), torch.ones(B, H, n, d).to(DEV), c, i32([0] * B))
    return c


def test_constant_values_come_back_under_a_dominating_key():
    """One key with nearly all of the weight, found when the maximum stands 2^7 and more
    below it: its weight is no power of two."""
    for d in (32, 64, 128):
        n = 300
        k = torch.zeros(1, 1, n, d)
        k[..., 0] = -4.0
        k[0, 0, 0, 0] = 0.0
        k[0, 0, 256, 0] = 1.0
        c = ones_cache(k)
        bits = torch.linspace(7.02, 7.9, 60).view(1, 15, 4, 1)  # of the weight, to base 2
        q = torch.zeros(1, 15, 4, d)
        q[..., :1] = bits * math.sqrt(d) * math.log(2.0)
        got = thin_q4_attention(q.bfloat16().to(DEV), c, i32([n - 4]))
        assert (got == 1.0).all(), (d, got.unique())


@pytest.mark.parametrize("d,B,H,G,T,n,n_sel", [
    (128, 2, 3, 4, 1, 700, 0), (64, 1, 2, 5, 3, 9000, 0), (32, 2, 2, 2, 9, 900, 6),
    (128, 1, 1, 4, 1, 20000, 200), (64, 16, 16, 4, 33, 300, 0), (128, 1, 8, 4, 67, 5000, 0)])
def test_constant_values_come_back(d, B, H, G, T, n, n_sel):
    g = gen(30)
    c = ones_cache(randn(g, B, H, n, d) * 2)
    q = randn(g, B, H * G, T, d, dtype="bf16").to(DEV)
    at = i32([n - T] * B)
    blocks = thin_q4_select(q, c, at, n_sel) if n_sel else None
    got = thin_q4_attention(q, c, at, blocks=blocks)
    assert (got == 1.0).all(), got.unique()


def test_select_of_prompts_with_small_products_beside_a_large_one():
    """Blocks whose score is one large product and 126 products just under a float32 unit
    of it, all of one sign: a sum that cuts each of them is off by 2^-16, which is half of
    what two kinds of blocks differ by, and turns their order round."""
    H, T, d, nb = 64, 2, 128, 100
    c = fresh(1, H, 64 * nb, d)
    up = torch.arange(nb) % 2 == 1
    x = torch.zeros(nb, 2, d)
    x[:, 1] = torch.where(up, 123 / 128, -123 / 128).view(nb, 1)
    x[:, 1, 0] = 1.0
    x[:, 1, 1] = torch.where(up, 0.0, 0.875)  # less than the others make: `up` scores higher
    x[:, 0] = x[:, 1] - 1.0
    c.bounds.copy_(x.expand(1, H, nb, 2, d))
    q = torch.full((1, H, T, d), 2.0 ** -23)
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -15
    q = q.bfloat16()
    at = 64 * nb - T
    for n_sel in (7, 40, 60):
        got = thin_q4_select(q.to(DEV), c, i32([at]), n_sel, n_sinks=0, n_window=1).cpu()
        for h in (0, H - 1):
            check_select_head(c, q, at, n_sel, 0, 1, got, h)


def test_select_of_prompts_whose_products_underflow():
    """Scores of 2^-160 that are no float32 numbers, but differ."""
    g = gen(31)
    H, T, d, nb = 64, 3, 64, 200
    c = fresh(1, H, 64 * nb, d)
    x = torch.randn(1, H, nb, 2, d, generator=g) * 2.0 ** -100
    c.bounds.copy_(x.sort(-2)[0].bfloat16())
    q = (torch.randn(1, 2 * H, T, d, generator=g) * 2.0 ** -60).bfloat16()
    q[:, :, 1] = 0.0  # (a token whose scores are all 0)
    at = 64 * nb - T
    got = thin_q4_select(q.to(DEV), c, i32([at]), 20, n_sinks=1, n_window=2).cpu()
    for h in range(0, H, 9):
        check_select_head(c, q, at, 20, 1, 2, got, h)


@pytest.mark.parametrize("d", [32, 128])
@pytest.mark.parametrize("nb", [100, 500, 1500, 5000, 9000, 20000])
def test_select_border_in_the_last_bit(nb, d):
    """One token; scores of both signs, those around the border 1 and a few units of the
    last bit of a float64 more, some of them equal."""
    g = gen(32)
    c = Q4Cache(1, 1, 64 * nb, d, device=DEV)
    x = torch.zeros(1, 1, nb, 2, d)
    x[..., 1, 0] = torch.where(torch.rand(nb, generator=g) < 0.3, -1.0, 1.0)
    x[..., 1, 1] = torch.randint(0, 40, (nb,), generator=g) / 128.0
    x[..., 0, :] = x[..., 1, :] - 1.0
    c.bounds.copy_(x)
    q = torch.zeros(1, 1, 1, d)
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -45
    at = 64 * nb - 1
    for n_sel in (20, nb // 3, nb // 2):
        got = thin_q4_select(q.to(DEV), c, i32([at]), n_sel, n_sinks=1, n_window=2).cpu()
        check_select_head(c, q, at, n_sel, 1, 2, got, 0)


def test_select_over_short_sequences_of_a_large_cache_takes_few_launches():
    """Tokens that see few blocks cost no launches for the rows that the cache could hold."""
    from paper_2606_10944_amd import LaunchTimer
    g = gen(33)
    H, T, d, n = 64, 600, 32, 140000
    c = Q4Cache(1, H, n, d, device=DEV)
    c.bounds.copy_(torch.randn(1, H, (n + 63) // 64, 2, d, generator=g).sort(-2)[0])
    q = randn(g, 1, H, T, d, dtype="bf16")
    st = torch.cuda.current_stream()
    for at in (3000, 131072 - 300):  # none and half of the tokens see more than 2048 blocks
        with LaunchTimer(st) as lt:
            got = thin_q4_select(q.to(DEV), c, i32([at]), 9)
        torch.cuda.synchronize()
        assert len(lt.records()) <= 3
        for h in (0, 63):
            for t in (0, 299, 300, 301, 599):
                check_select_head_token(c, q, at, 9, 1, 2, got, h, t)


def check_select_head_token(c, q, at, n_sel, n_sinks, n_window, got, h, t):
    G = q.shape[1] // c.H
    sc = ref.block_scores(q[0, h * G:(h + 1) * G, t], c.bounds[0, h].cpu()).tolist()
    assert got[0, h, t].tolist() == ref.select(sc, at + t, n_sel, n_sinks, n_window), (h, t)


def test_selections_of_two_threads():
    """Prompts over a large and a small cache from two host threads: each has the LDS that
    its own scores need."""
    import threading
    g = gen(34)
    H, T, d = 64, 3, 32
    calls = []
    for nb in (2000, 1100):
        c = Q4Cache(1, H, 64 * nb, d, device=DEV)
        c.bounds.copy_(torch.randn(1, H, nb, 2, d, generator=g).sort(-2)[0])
        q = randn(g, 1, H, T, d, dtype="bf16").to(DEV)
        at = i32([64 * nb - T])
        calls.append((c, q, at, thin_q4_select(q, c, at, 9)))
    failed = []

    def work(c, q, at, want):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for _ in range(200):
                    if not torch.equal(thin_q4_select(q, c, at, 9), want):
                        failed.append("differs")
        except Exception as e:  # noqa: BLE001
            failed.append(repr(e))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=a) for a in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B", [65, 130, 256])
def test_attention_shares_of_more_sequences_than_lanes(dtype, B):
    """Keys shared out to workgroups over up to four sequences per lane, with nothing and
    long caches at the lanes' ends."""
    g = gen(40)
    n = 4200
    lengths = torch.randint(0, n + 1, (B,), generator=g).tolist()
    for i, x in zip((0, 62, 63, 64, 65, 126, 127, 128, 129, 191, 192, 254, 255),
                    (n, 0, 0, n, 1, 0, 33, 0, n, 0, 0, 32, n)):
        if i < B:
            lengths[i] = x
    c = filled(g, B, 1, n, 32, lengths)
    q = randn(g, B, 3, 2, 32, dtype=dtype)
    at = [x - 2 for x in lengths]
    check_attention(c, q, at, None, None, thin_q4_attention(q.to(DEV), c, i32(at)), dtype)


@pytest.mark.parametrize("n_out,g_", [(64, 1), (128, 0)])
def test_cached_rows_are_thinned(n_out, g_):
    """Rows of the cache, read back, thinned to a part of them and attended over: the
    coreset is that of the same rows as plain tensors, and its attention the definition's."""
    from paper_2606_10944_amd import thin_attention, thin_compress, thin_plan
    g = gen(50)
    H, n, d = 2, 512, 64
    c = filled(g, 1, H, n, d, [n])
    k, v = thin_q4_load(c, i32([0]), n)
    plan = thin_plan(1, H, n, d, n_out, g_)
    u = torch.rand(max(plan["uniforms_total"], 1), generator=g).to(DEV)
    idx = thin_compress(k, v, n_out, g_, u)
    rows = [x.cpu() for x in (k, v)]
    assert torch.equal(idx, thin_compress(*[x.to(DEV) for x in rows], n_out, g_, u))
    assert idx.shape[-1] == n_out < n
    q = randn(g, 1, H, 3, d, dtype="bf16")
    got = thin_attention(q.to(DEV), k, v, idx).cpu().double()
    for h in range(H):
        i = idx[0, h].cpu().long()
        assert i.unique().numel() == n_out and 0 <= int(i.min()) and int(i.max()) < n
        o, A, S = ref.attention(q[0, h], rows[0][0, h, i].double(), rows[1][0, h, i].double(),
                                torch.ones(3, n_out, dtype=torch.float64))
        # weights rounded to bf16 (half a step each) and float32 sums, as for the cache's
        # own kernels; the output is float32
        assert ((got[0, h] - o).abs() <= attention_bound(o, A, S, "bf16")).all()


def test_a_refused_step_stores_nothing():
    """Arguments that attention or the selection would refuse are refused before the rows
    are stored."""
    from paper_2606_10944_amd._lib import ThinError
    g = gen(60)
    c = filled(g, 2, 2, 300, 64, [100, 100])
    names = ("k_codes", "k_scales", "v_codes", "v_scales", "bounds")
    before = [getattr(c, x).clone() for x in names]
    q, k, v = (randn(g, 2, n, 3, 64, dtype="bf16").to(DEV) for n in (4, 2, 2))
    at = i32([100, 100])
    bad_q = [q[:, :3].contiguous(), q[:1], q[..., :32], q.half(), q.cpu()]
    bad = [dict(n_sel=2), dict(n_sel=-1), dict(n_sel=40000), dict(n_sel=5, n_sinks=4),
           dict(n_sel=5, n_window=0), dict(O=q.float()), dict(O=q[:1]), dict(O=q.cpu()),
           dict(O=q[:, :1].expand(2, 4, 3, 64))]
    wide = torch.zeros(2, 4, 3, 72, dtype=torch.bfloat16, device=DEV)
    bad_q.append(wide[..., 4:68])  # not 16-byte aligned
    bad.append(dict(O=wide[..., 4:68]))
    for a in [(x, {}) for x in bad_q] + [(q, x) for x in bad]:
        with pytest.raises(ThinError):
            c.step(a[0], k, v, at, **a[1])
        assert all(torch.equal(getattr(c, x), was) for x, was in zip(names, before)), a[1]
    c.step(q, k, v, at, n_sel=3)
    assert not torch.equal(c.k_codes, before[0])
