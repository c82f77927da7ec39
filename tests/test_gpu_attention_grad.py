"""The gradient of coreset attention on the GPU against its formulas in float64, and against
differences."""
import math

import pytest
import torch

import attention_grad_reference as ref
from paper_2606_10944_amd import (coreset_attention, thin_attention, thin_attention_backward,
                                  thin_compress, thin_plan, thin_rotary_axes, thin_rotary_turns)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("dQ", "dK", "dV", "dlogw")


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype="fp32", scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(DT[dtype])


def inputs(g, B, H, n_q, n, n_out, d, dtype, out, scale=1.0, weighted=False):
    """Q, K, V, idx, logw, dO on the CPU."""
    Q, K, V = (randn(g, B, H, r, d, dtype=dtype, scale=scale) for r in (n_q, n, n))
    idx = torch.rand(B, H, n, generator=g).argsort(-1)[..., :n_out].sort(-1)[0].to(torch.int32)
    logw = None
    if weighted:
        logw = torch.randn(B, H, n_out, generator=g) * 2
        logw[..., ::3] = 0.0
        if n_out > 4:
            logw[..., 4::5] = -math.inf
    return Q, K, V, idx.contiguous(), logw, randn(g, B, H, n_q, d, dtype=out)


def to(x):
    return None if x is None else x.to(DEV)


def backward(Q, K, V, idx, logw, dO, **kw):
    return thin_attention_backward(*(to(x) for x in (Q, K, V, idx, dO)), logw=to(logw),
                                   need_logw=True, **kw)


def check(args, got):
    want = ref.gradient(*args)
    for name, x in zip(NAMES, got):
        value, bound = want[name]
        err = (x.cpu().double() - value).abs()
        assert (err <= bound).all(), (name, float((err / bound).max()),
                                      (~(err <= bound)).nonzero()[:3].tolist())
        # where the gradient is 0 by its formula (rows off the coreset), it is exactly that
        assert (x.cpu()[bound <= 1e-37] == 0).all()


SHAPES = [
    # B, H, n_q, n, n_out, d: one key to one step past what a workgroup of each size holds
    (1, 1, 1, 1, 1, 32), (2, 1, 33, 5, 2, 64), (1, 3, 31, 40, 16, 128), (1, 1, 64, 17, 17, 32),
    (3, 2, 32, 50, 32, 64), (2, 2, 100, 33, 33, 128), (1, 2, 129, 64, 64, 32),
    (1, 1, 200, 100, 65, 64), (2, 1, 65, 128, 128, 128), (1, 2, 70, 300, 129, 64),
    (1, 1, 97, 200, 192, 32), (2, 1, 160, 300, 256, 128), (1, 2, 50, 257, 257, 64),
    (1, 1, 300, 700, 333, 128), (2, 1, 64, 600, 600, 32), (1, 1, 1, 300, 300, 128),
    (1, 2, 1, 90, 40, 64), (40, 9, 40, 20, 9, 32), (1, 1, 5000, 64, 48, 64),
    (1, 2, 2500, 400, 150, 128), (2, 2, 75, 300, 250, 32), (1, 2, 40, 90, 50, 32),
]
TYPES = [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")]


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("B,H,n_q,n,n_out,d", SHAPES)
def test_gradient(B, H, n_q, n, n_out, d, dtype, out):
    g = gen(201)
    args = inputs(g, B, H, n_q, n, n_out, d, dtype, out, weighted=n_out % 2 == 1)
    got = backward(*args)
    assert [x.dtype for x in got] == [DT[dtype]] * 3 + [torch.float32]
    check(args, got)
    again = backward(*args)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("B,H,n_q,n,n_out,d", [
    (33, 8, 20, 260, 257, 32), (16, 4, 200, 300, 260, 64), (32, 2, 193, 290, 288, 128),
    (2, 1, 37, 700, 513, 128), (1, 3, 31, 400, 290, 32)])
def test_waves_that_share_query_rows(B, H, n_q, n, n_out, d, dtype, out):
    """One, two (twice) and four (twice) waves per tile of rows."""
    g = gen(216)
    args = inputs(g, B, H, n_q, n, n_out, d, dtype, out, weighted=True)
    check(args, backward(*args))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_out", [40, 300])
def test_large_log_weights(n_out, dtype):
    """Weights whose exponential float32 does not hold, and rows of a step that are not there."""
    g = gen(218)
    args = inputs(g, 1, 2, 45, 400, n_out, 64, dtype, dtype, weighted=True)
    args[4][..., 2::5] += 200.0
    args[4][..., 3::5] -= 200.0
    check(args, backward(*args))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,H,n_q,n,n_out,d", [
    (1, 1, 3, 9001, 40, 128), (2, 3, 1, 16385, 1, 32), (1, 2, 7, 8003, 300, 64),
    (1, 5, 300, 9999, 130, 128)])
def test_many_rows_for_few_queries(B, H, n_q, n, n_out, d, dtype):
    """Their zeros come from a launch of their own; whatever the gradients held goes."""
    g = gen(217)
    Q, K, V, idx, logw, dO = args = inputs(g, B, H, n_q, n, n_out, d, dtype, dtype)
    dK, dV = (torch.full((B, H, n, d), math.nan, dtype=DT[dtype], device=DEV) for _ in range(2))
    got = backward(*args, dK=dK, dV=dV)
    assert got[1] is dK and got[2] is dV
    check(args, got)


@pytest.mark.parametrize("B,H,n_q,n,n_out,d", SHAPES)
def test_gradient_without_that_of_the_weights(B, H, n_q, n, n_out, d):
    """Products of a float32 dO with bf16 rows take fewer parts of it then."""
    g = gen(215)
    args = inputs(g, B, H, n_q, n, n_out, d, "bf16", "fp32", weighted=n_out % 2 == 0)
    Q, K, V, idx, logw, dO = args
    got = thin_attention_backward(*(to(x) for x in (Q, K, V, idx, dO)), logw=to(logw))
    assert len(got) == 3
    check(args, got)


@pytest.mark.parametrize("dtype,out", [("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("n_out", [7, 40, 300])
def test_gradient_against_differences(n_out, dtype, out):
    """Central differences of the forward's formula in float64: off by h^2 / 6 of the third
    derivative along a channel, below 1e-7 here for steps of 1e-4 (scores below 10, values below
    5), and by 1e-11 from rounding."""
    g = gen(202)
    args = inputs(g, 1, 1, 6, n_out + 3, n_out, 32, dtype, out, scale=0.8, weighted=True)
    Q, K, V, idx, logw, dO = args
    got = [x.cpu().double() for x in backward(*args)]
    bound = {k: b for k, (_, b) in ref.gradient(*args).items()}
    x = [Q.double(), K.double(), V.double(), logw.double()]

    def f():
        k, v, there = ref.coreset(x[1], x[2], idx, logw)
        return float((ref.forward(x[0], k, v, torch.where(there, x[3], -math.inf))[0]
                      * dO.double()).sum())
    for which, name in enumerate(NAMES):
        flat = x[which].view(-1)
        for i in torch.randperm(flat.numel(), generator=g)[:40].tolist():
            was, h = float(flat[i]), 1e-4
            if not math.isfinite(was):
                continue
            flat[i] = was + h
            up = f()
            flat[i] = was - h
            down = f()
            flat[i] = was
            diff = (up - down) / (2 * h)
            assert abs(float(got[which].view(-1)[i]) - diff) <= float(
                bound[name].view(-1)[i]) + 1e-6, (name, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_out", [20, 200, 400])
def test_keys_that_are_not_there(n_out, dtype):
    """Keys of weight 0 hold NaN and infinities, entries of the list lie outside the rows, one
    slice has no key at all."""
    g = gen(203)
    Q, K, V, idx, logw, dO = inputs(g, 2, 2, 70, 500, n_out, 64, dtype, dtype, weighted=True)
    dropped = logw == -math.inf
    idx[0, 0, 3], idx[1, 0, 0], idx[1, 0, n_out - 1] = -1, 500, 2 ** 31 - 1
    logw[0, 1] = -math.inf
    dropped = logw == -math.inf
    for b in range(2):
        for h in range(2):
            rows = idx[b, h][dropped[b, h]].long()
            rows = rows[(rows >= 0) & (rows < 500)]
            K[b, h, rows[::2]], K[b, h, rows[1::2]] = math.nan, math.inf
            V[b, h, rows[::2]], V[b, h, rows[1::2]] = -math.inf, math.nan
    args = (Q, K, V, idx, logw, dO)
    got = backward(*args)
    check(args, got)
    assert (got[0][0, 1] == 0).all() and (got[3][0, 1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_out", [6, 100, 300])
def test_rows_listed_more_than_once(n_out, dtype):
    g = gen(204)
    Q, K, V, idx, logw, dO = inputs(g, 1, 2, 50, 600, n_out, 128, dtype, "fp32", weighted=True)
    idx[0, 0, n_out // 2:] = idx[0, 0, 0]
    idx[0, 1] = idx[0, 1].flip(0)  # (any order)
    idx[0, 1, 1] = idx[0, 1, n_out - 1]
    args = (Q, K, V, idx, logw, dO)
    check(args, backward(*args))


@pytest.mark.parametrize("n_out", [12, 130, 290])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores_and_one_sided_rows(n_out, dtype):
    """Scores of several hundred: probabilities of 1 and 0; log-weights of +-60."""
    g = gen(205)
    Q, K, V, idx, logw, dO = inputs(g, 1, 1, 80, 300, n_out, 64, dtype, dtype, scale=6.0)
    logw = torch.where(torch.rand(1, 1, n_out, generator=g) < 0.5, 60.0, -60.0)
    args = (Q, K, V, idx, logw, dO)
    got = backward(*args)
    assert all(torch.isfinite(x).all() for x in got)
    check(args, got)


def test_equal_keys_share_equally():
    """One row listed everywhere: probabilities of 1 / n_out, so dV is the mean of dO's sums and
    ds is exactly what float32 leaves of 0."""
    g = gen(206)
    Q, K, V, _, _, dO = inputs(g, 1, 1, 64, 10, 4, 32, "fp32", "fp32")
    idx = torch.full((1, 1, 4), 7, dtype=torch.int32)
    got = backward(Q, K, V, idx, None, dO)
    check((Q, K, V, idx, None, dO), got)
    assert (got[1][0, 0, :7] == 0).all() and (got[1][0, 0, 8:] == 0).all()


def test_a_nan_row_stays_in_its_slice():
    g = gen(207)
    for n_out in (30, 300):
        args = list(inputs(g, 1, 2, 70, 400, n_out, 64, "bf16", "bf16"))
        clean = backward(*args)
        args[0] = args[0].clone()
        args[0][0, 0, 5, 3] = math.nan
        got = backward(*args)
        for a, b in zip(got, clean):
            assert torch.equal(a[0, 1], b[0, 1])
        rows = torch.arange(70) != 5
        assert torch.equal(got[0][0, 0].cpu()[rows], clean[0][0, 0].cpu()[rows])
        assert got[0][0, 0, 5].isnan().all()


def test_offsets_beyond_32_bits():
    """The third slice's rows lie 2^31 elements behind the first's."""
    g = gen(208)
    n, d, m = 1 << 23, 128, 64
    K = torch.zeros(3, 1, n, d, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    idx = torch.zeros(3, 1, m, dtype=torch.int32)
    rows = torch.randint(0, n, (m,), generator=g).unique()
    idx[2, 0] = torch.cat((torch.tensor([0, n - 1]), rows))[:m].to(torch.int32)[
        torch.arange(m) % min(m, rows.numel() + 2)]
    k, v = randn(g, m, d, dtype="bf16"), randn(g, m, d, dtype="bf16")
    K[2, 0, idx[2, 0].long().to(DEV)], V[2, 0, idx[2, 0].long().to(DEV)] = k.to(DEV), v.to(DEV)
    Q, dO = randn(g, 3, 1, 40, d, dtype="bf16").to(DEV), randn(g, 3, 1, 40, d, dtype="bf16").to(DEV)
    dQ, dK, dV = thin_attention_backward(Q, K, V, idx.to(DEV), dO)
    at = idx[2, 0].long().to(DEV)
    uniq = at.unique()
    small = torch.searchsorted(uniq, at).to(torch.int32).view(1, 1, m)
    want = thin_attention_backward(Q[2:], K[2:, :, uniq].contiguous(), V[2:, :, uniq].contiguous(),
                                   small, dO[2:])
    assert torch.equal(dQ[2:], want[0])
    for x, w in ((dK, want[1]), (dV, want[2])):
        assert torch.equal(x[2:, :, uniq], w)
        x[2:, :, uniq] = 0
        x[:2, :, 0] = 0  # (the other slices list row 0)
        assert not x.view(torch.int16).any()


# ---------------------------------------------------------------------------
# autograd, streams, graphs, together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("n_out", [30, 290])
def test_autograd_reaches_the_inputs(n_out):
    g = gen(209)
    args = inputs(g, 2, 2, 60, 400, n_out, 64, "bf16", "fp32", weighted=True)
    Q, K, V, idx, logw, _ = (to(x) for x in args)
    for t in (Q, K, V, logw):
        t.requires_grad_()
    O = coreset_attention(Q, K, V, idx, logw=logw)
    assert torch.equal(O, thin_attention(Q.detach(), K.detach(), V.detach(), idx,
                                         logw=logw.detach()))
    O.sum().backward()  # (the gradient of a sum is one number, expanded)
    want = thin_attention_backward(Q.detach(), K.detach(), V.detach(), idx, torch.ones_like(O),
                                   logw=logw.detach(), need_logw=True)
    for t, w in zip((Q, K, V, logw), want):
        assert torch.equal(t.grad, w)
    with pytest.raises(RuntimeError):
        x = coreset_attention(Q, K, V, idx)
        y, = torch.autograd.grad(x.sum(), Q, create_graph=True)
        y.sum().backward()


def test_autograd_of_strided_inputs_and_shared_heads():
    """Heads that share keys by expansion, rows between heads: the gradients add up."""
    g = gen(210)
    B, H, n, d = 2, 4, 50, 32
    q = randn(g, B, n, H, d).to(DEV).requires_grad_()
    k = randn(g, B, 1, n, d).to(DEV).requires_grad_()
    v = randn(g, B, 1, n, d).to(DEV).requires_grad_()
    idx = torch.arange(0, n, 3, dtype=torch.int32, device=DEV).expand(B, H, -1)
    w = randn(g, B, H, n, d).to(DEV)
    O = coreset_attention(q.transpose(1, 2), k.expand(B, H, n, d), v.expand(B, H, n, d), idx)
    (O * w).sum().backward()
    full = [x.detach().cpu() for x in (q.transpose(1, 2), k.expand(B, H, n, d),
                                       v.expand(B, H, n, d))]
    want = ref.gradient(*full, idx.cpu(), None, w.cpu())
    err = (q.grad.cpu().double() - want["dQ"][0].transpose(1, 2)).abs()
    assert (err <= want["dQ"][1].transpose(1, 2)).all()
    for x, name in ((k, "dK"), (v, "dV")):
        value, bound = want[name]
        err = (x.grad.cpu().double() - value.sum(1, keepdim=True)).abs()
        # four gradients, each within its bound, and three additions in float32
        size = (value.abs() + bound).sum(1, keepdim=True)
        assert (err <= bound.sum(1, keepdim=True) + 3 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("n_out", [30, 120, 290])
def test_replayed_gradient_follows_its_inputs(n_out):
    """Two captured calls with workspaces of the graphs' own, replayed with new inputs, eager
    calls and graphs of autograd alive between."""
    g = gen(211)
    shape = (1, 2, 90, 400, n_out, 64, "bf16", "bf16")
    Q, K, V, idx, logw, dO = (to(x) for x in inputs(g, *shape, weighted=True))
    leaf = Q.clone().requires_grad_()
    # (inputs of its own: autograd refuses those that changed since)
    alive = coreset_attention(leaf, K.clone(), V.clone(), idx.clone(), logw=logw.clone(),
                              out_dtype=torch.bfloat16)

    def call():
        return thin_attention_backward(Q, K, V, idx, dO, logw=logw, need_logw=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call())
        graphs.append(graph)
    for i in range(4):
        for x, y in zip((Q, K, V, idx, logw, dO), inputs(g, *shape, weighted=True)):
            x.copy_(y)
        for graph in graphs:
            graph.replay()
        want = call()
        torch.cuda.synchronize()
        for got in outs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    alive.sum().backward()
    assert torch.isfinite(leaf.grad).all()


def test_calls_on_streams_of_their_own():
    g = gen(212)
    args = [to(x) for x in inputs(g, 2, 2, 300, 400, 290, 64, "bf16", "fp32", weighted=True)]
    Q, K, V, idx, logw, dO = args
    want = thin_attention_backward(Q, K, V, idx, dO, logw=logw, need_logw=True)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [thin_attention_backward(Q, K, V, idx, dO, logw=logw, need_logw=True, stream=s)
           for s in streams]
    for s in streams:
        s.synchronize()
    for x in got:
        assert all(torch.equal(a, b) for a, b in zip(x, want))


def test_a_layer_of_image_tokens_as_it_is_trained():
    """Rows turned by positions with axes, thinned, attended to, and the way back: against the
    formulas' gradient through the same coreset."""
    g = gen(213)
    B, H, n, d, n_out = 1, 2, 256, 64, 16
    turns, _ = thin_rotary_turns(d)
    t, axis = turns.to(DEV), torch.arange(d // 2, dtype=torch.int32, device=DEV) % 3
    r = torch.arange(n)
    pos = torch.stack((r // 64, r // 8 % 8, r % 8), -1).to(torch.int32).expand(B, n, 3) \
        .contiguous().to(DEV)
    q, k, v, dO = (randn(g, B, H, n, d).to(DEV) for _ in range(4))
    qt, kt = thin_rotary_axes(q, pos, t, axis, Y=k)
    plan = thin_plan(B, H, n, d, n_out, 1)
    u = torch.rand(plan["uniforms_total"], generator=g).to(DEV)
    idx, logw = thin_compress(kt, v, n_out, 1, u, return_logw=True)
    dq, dk, dv = thin_attention_backward(qt, kt, v, idx, dO, logw=logw)
    dq, dk = thin_rotary_axes(dq, pos, t, axis, Y=dk, inverse=True)
    want = ref.gradient(*(x.cpu() for x in (qt, kt, v, idx, logw, dO)))
    assert ((dv.cpu().double() - want["dV"][0]).abs() <= want["dV"][1]).all()
    a = (pos.cpu().double()[..., axis.cpu().long()] * turns) % 1.0 * 2 * math.pi  # [B, n, d / 2]
    c, s = a.cos().unsqueeze(1), a.sin().unsqueeze(1)
    for x, name in ((dq, "dQ"), (dk, "dK")):
        (lo, hi), (el, eh) = want[name][0].chunk(2, -1), want[name][1].chunk(2, -1)
        back = torch.cat((lo * c + hi * s, hi * c - lo * s), -1)
        # the turn takes both channels' bounds along, and adds 3 2^-22 of both channels and a
        # rounding (cosines, sines, products and sums in float32)
        slack = (el + eh) + 3 * 2.0 ** -22 * (lo.abs() + hi.abs() + el + eh)
        bound = torch.cat((slack, slack), -1) + 2.0 ** -24 * back.abs()
        assert ((x.cpu().double() - back).abs() <= bound).all()


def test_binding_refuses_what_does_not_fit():
    from paper_2606_10944_amd._lib import THIN_EDTYPE, THIN_EINVAL, THIN_EWORKSPACE, ThinError
    g = gen(214)
    Q, K, V, idx, logw, dO = (to(x) for x in inputs(g, 2, 2, 8, 40, 9, 64, "bf16", "bf16",
                                                    weighted=True))

    def refused(status, *a, **kw):
        with pytest.raises(ThinError) as e:
            thin_attention_backward(*a, **kw)
        assert e.value.status == status

    for bad in (Q.cpu(), Q[:1], Q[..., :32], Q[0], Q.transpose(1, 2)):
        refused(THIN_EINVAL, bad, K, V, idx, dO)
    for bad in (dO.cpu(), dO[:, :, :7], dO[:, :, :1].expand_as(dO)):
        refused(THIN_EINVAL, Q, K, V, idx, bad)
    refused(THIN_EINVAL, Q, K, V[:, :, :39], idx, dO)
    refused(THIN_EDTYPE, Q, K, V.float(), idx, dO)
    refused(THIN_EDTYPE, Q, K, V, idx, dO.half())
    refused(THIN_EDTYPE, Q.half(), K.half(), V.half(), idx, dO)
    for bad in (idx.long(), idx[:1], idx.cpu(), idx[..., ::2], idx[..., :0]):
        refused(THIN_EINVAL, Q, K, V, bad, dO)
    for bad in (logw.double(), logw[:1], logw.cpu(), logw[..., :8]):
        refused(THIN_EINVAL, Q, K, V, idx, dO, logw=bad)
    refused(THIN_EINVAL, Q, K, V, idx, dO, dQ=Q.float())
    refused(THIN_EINVAL, Q, K, V, idx, dO, dK=K[:, :, :9])
    refused(THIN_EINVAL, Q, K, V, idx, dO, dlogw=logw[..., :8])
    refused(THIN_EWORKSPACE, Q, K, V, idx, dO,
            workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    for bad in (dict(dQ=Q), dict(dQ=dO), dict(dK=K), dict(dV=K), dict(dK=V)):
        refused(THIN_EINVAL, Q, K, V, idx, dO, **bad)
    same = torch.empty_like(K)
    refused(THIN_EINVAL, Q, K, V, idx, dO, dK=same, dV=same)
    for bad in ((Q.cpu(), K, V, idx), (Q, K, V, idx.cpu())):
        with pytest.raises(ThinError) as e:
            coreset_attention(*bad)
        assert e.value.status == THIN_EINVAL
    with pytest.raises(ThinError) as e:
        coreset_attention(Q.half(), K.half(), V.half(), idx)
    assert e.value.status == THIN_EDTYPE
    out = torch.full_like(K, 3.0)
    got = thin_attention_backward(Q, K, V, idx, dO, logw=logw, dK=out)
    assert got[1] is out and len(got) == 3
