"""Coreset attention and its gradient as a pair: lists that leave the rows, views at any offset,
sizes that one of them has not, and launch shapes beside those of the other tests."""
import math

import pytest
import torch

import attention_grad_reference as ref
import test_gpu_attention_grad as grad
from paper_2606_10944_amd import THIN_EINVAL, ThinError, coreset_attention, thin_attention
from test_gpu_attention_grad import DEV, NAMES, backward, check, gen, inputs, to

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")]


def list_that_leaves_the_rows(g, B, H, n, n_out):
    """A fifth of the entries outside [0, n), near it and far; some in range are the first and the
    last row, so that a row is listed by its number and by an entry outside."""
    idx = torch.randint(0, n, (B, H, n_out), generator=g, dtype=torch.int32)
    far = torch.tensor([-1, n, 2 ** 31 - 1, -2 ** 31, -7, n + 3], dtype=torch.int32)
    at = torch.rand(B, H, n_out, generator=g).argsort(-1)[..., :max(1, n_out // 5)]
    idx.scatter_(2, at, far[torch.arange(at.shape[-1]) % 6].expand_as(at).contiguous())
    if n_out > 6:
        idx[..., 2], idx[..., 5] = 0, n - 1
    return idx


def forward_bound(Q, K, V, idx, logw):
    """(O, bound).  Weights are off by r of themselves (see ref.gradient), and, of bf16 rows, by
    half a step where they round to bf16; their sum by r as well and by its own rounding."""
    n = K.shape[-2]
    k, v, there = ref.coreset(K, V, idx.clamp(0, n - 1), logw)
    lw = torch.zeros(idx.shape, dtype=torch.float64) if logw is None else logw.double()
    o, p, _ = ref.forward(Q.double(), k, v, torch.where(there, lw, -math.inf))
    S = (Q.double().abs() @ k.abs().transpose(-1, -2) / math.sqrt(Q.shape[-1])).amax(-1, True)
    big = torch.where(there, lw.abs(), 0.0).amax(-1, keepdim=True).unsqueeze(-1)
    r = 2.0 ** -18 * S + 2.0 ** -20 + 2.0 ** -22 * big
    m = idx.shape[-1]
    each = 2 * r + 2 * (m + 64) * 2.0 ** -24 + (2.0 ** -8 if Q.dtype == torch.bfloat16 else 0.0)
    return o, 1.01 * each * (p @ v.abs())


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("B,H,n_q,n,n_out,d", [
    (1, 1, 1, 1, 1, 32), (1, 2, 40, 5, 9, 64), (2, 2, 70, 90, 20, 64), (1, 1, 50, 300, 100, 32),
    (2, 1, 65, 400, 180, 128), (1, 2, 33, 300, 256, 64), (1, 2, 70, 500, 400, 128),
    (1, 1, 900, 60, 30, 128)])
@pytest.mark.parametrize("weighted", [False, True])
def test_entries_outside_are_the_nearest_rows(B, H, n_q, n, n_out, d, dtype, out, weighted):
    """The output and its gradients are those of one list: the one whose entries are clamped."""
    g = gen(301)
    Q, K, V, _, logw, dO = inputs(g, B, H, n_q, n, min(n, n_out), d, dtype, out)
    idx = list_that_leaves_the_rows(g, B, H, n, n_out)
    if weighted:
        logw = torch.randn(B, H, n_out, generator=g) * 2
        if n_out > 4:
            logw[..., 4::7] = -math.inf
    near = idx.clamp(0, n - 1)
    leaves = [to(x).requires_grad_() for x in (Q, K, V)] + [
        to(logw).requires_grad_() if weighted else None]
    O = coreset_attention(*leaves[:3], to(idx), logw=leaves[3], out_dtype=dO.dtype)
    assert torch.equal(O, thin_attention(to(Q), to(K), to(V), to(near), logw=to(logw),
                                         out_dtype=dO.dtype))
    want, bound = forward_bound(Q, K, V, idx, logw)
    err = (O.detach().cpu().double() - want).abs()
    assert (err <= bound + ref.HALF[dO.dtype] * (want.abs() + bound)).all()
    O.backward(to(dO))
    got = [x.grad for x in leaves if x is not None]
    check((Q, K, V, near, logw, dO), got)
    for a, b, name in zip(backward(Q, K, V, idx, logw, dO), backward(Q, K, V, near, logw, dO),
                          NAMES):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_out", [20, 200, 400])
def test_padded_lists(n_out, dtype):
    """Lists padded with -1 at weight 0: none of it is there, whatever the first row holds where
    nothing else lists it; rows that are listed by keys that are not there alone hold zeros."""
    g = gen(302)
    n = 500
    Q, K, V, idx, logw, dO = inputs(g, 2, 2, 70, n, n_out, 64, dtype, dtype, weighted=True)
    idx = idx.clamp(min=1)  # (row 0 is the padding's alone, but for one slice)
    idx[1, 1, 0], logw[1, 1, 0] = 0, 0.5
    idx[0, 0, n_out // 3:], logw[0, 0, n_out // 3:] = -1, -math.inf
    idx[1, 1, n_out // 2:], logw[1, 1, n_out // 2:] = -1, -math.inf
    idx[0, 1], logw[0, 1] = -1, -math.inf  # (no key at all)
    K[0, :, 0], V[0, :, 0] = math.nan, math.inf
    got = backward(Q, K, V, idx, logw, dO)
    check((Q, K, V, idx.clamp(min=0), logw, dO), got)
    assert (got[0][0, 1] == 0).all() and (got[3][0, 1] == 0).all()
    assert (got[1][0, :, 0] == 0).all() and (got[2][0, :, 0] == 0).all()
    gone = to(logw == -math.inf)
    assert (got[3][gone] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_out", [20, 200, 400])
def test_keys_without_weight_hold_anything(n_out, dtype):
    """Keys of weight 0 hold NaN and infinities, entries of the list lie outside the rows (with a
    weight and without), one slice has no key at all."""
    g = gen(203)
    Q, K, V, idx, logw, dO = inputs(g, 2, 2, 70, 500, n_out, 64, dtype, dtype, weighted=True)
    idx[0, 0, 3], idx[1, 0, 0], idx[1, 0, n_out - 1] = -1, 500, 2 ** 31 - 1
    logw[0, 1] = -math.inf
    near = idx.clamp(0, 499)
    there = logw != -math.inf
    for b in range(2):
        for h in range(2):
            rows = near[b, h][~there[b, h]].long()
            rows = rows[~torch.isin(rows, near[b, h][there[b, h]].long())]
            K[b, h, rows[::2]], K[b, h, rows[1::2]] = math.nan, math.inf
            V[b, h, rows[::2]], V[b, h, rows[1::2]] = -math.inf, math.nan
    got = backward(Q, K, V, idx, logw, dO)
    check((Q, K, V, near, logw, dO), got)
    assert (got[0][0, 1] == 0).all() and (got[3][0, 1] == 0).all()


# ---------------------------------------------------------------------------
# Views whose rows are not 16-byte aligned, through autograd
# ---------------------------------------------------------------------------
def at_offset(t, elements):
    """t's values, contiguous, `elements` into a buffer of their own."""
    flat = torch.empty(t.numel() + elements, dtype=t.dtype, device=t.device)
    flat[elements:] = t.flatten()
    view = flat[elements:].view(t.shape)
    assert view.is_contiguous() and view.data_ptr() % 16 == elements * t.element_size() % 16
    return view


@pytest.mark.parametrize("n_out", [30, 290])
@pytest.mark.parametrize("dtype,out", TYPES)
def test_gradient_that_arrives_at_an_offset(n_out, dtype, out):
    """The gradient of a concatenation is a view into that of the whole: here one element in."""
    g = gen(303)
    args = inputs(g, 1, 2, 45, 400, n_out, 64, dtype, out, weighted=True)
    Q, K, V, idx, logw, dO = (to(x) for x in args)
    leaves = [x.requires_grad_() for x in (Q, K, V, logw)]
    O = coreset_attention(Q, K, V, idx, logw=logw, out_dtype=dO.dtype)
    one = torch.ones(1, dtype=dO.dtype, device=dO.device)
    torch.cat((one, O.flatten())).backward(torch.cat((one, dO.flatten())))
    for x, want in zip(leaves, backward(*args)):
        assert torch.equal(x.grad, want)
    check(args, [x.grad for x in leaves])


@pytest.mark.parametrize("n_out", [30, 290])
@pytest.mark.parametrize("dtype,offset", [("bf16", 1), ("bf16", 2), ("bf16", 4), ("fp32", 1),
                                          ("fp32", 2), ("fp32", 3)])
def test_rows_at_an_offset(n_out, dtype, offset):
    """Queries, keys and values out of flat buffers: the output and gradients of aligned ones."""
    g = gen(304)
    args = inputs(g, 1, 2, 45, 400, n_out, 64, dtype, dtype, weighted=True)
    Q, K, V, idx, logw, dO = (to(x) for x in args)
    want = coreset_attention(Q, K, V, idx, logw=logw)
    leaves = [at_offset(x, offset).requires_grad_() for x in (Q, K, V)] \
        + [logw.clone().requires_grad_()]
    O = coreset_attention(*leaves[:3], idx, logw=leaves[3])
    assert torch.equal(O, want)
    O.backward(dO.float())
    exact = args[:5] + (args[5].float(),)
    for x, grad in zip(leaves, backward(*exact)):
        assert torch.equal(x.grad, grad)
    check(exact, [x.grad for x in leaves])


# ---------------------------------------------------------------------------
# Sizes that the output has and its gradient has not
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("H,n_out", [(1, (1 << 18) + 1), (256, (1 << 17) + 1)])
@pytest.mark.parametrize("which", ["Q", "K", "V", "logw"])
def test_sizes_without_a_gradient_are_refused_at_once(H, n_out, which):
    g = gen(305)
    x = {k: torch.randn(1, H, 2, 32, generator=g).to(DEV) for k in "QKV"}
    x["logw"] = torch.zeros(1, H, n_out, device=DEV)
    idx = torch.zeros(1, H, n_out, dtype=torch.int32, device=DEV)
    x[which].requires_grad_()
    with pytest.raises(ThinError) as e:
        coreset_attention(x["Q"], x["K"], x["V"], idx, logw=x["logw"])
    assert e.value.status == THIN_EINVAL


def test_sizes_without_a_gradient_have_an_output():
    """Nothing is recorded where nothing asks for a gradient: one row, listed 2^18 + 1 times."""
    g = gen(306)
    n_out = (1 << 18) + 1
    Q, K, V = (torch.randn(1, 1, r, 32, generator=g).to(DEV) for r in (3, 1, 1))
    idx = torch.zeros(1, 1, n_out, dtype=torch.int32, device=DEV)
    leaf = Q.clone().requires_grad_()
    with torch.no_grad():
        a = coreset_attention(leaf, K, V, idx)
    for O in (a, coreset_attention(Q, K, V, idx)):
        # equal weights: sums of n_out terms over their number, each off by n_out 2^-24 at most
        assert ((O - V).abs() <= 2 * n_out * 2.0 ** -24 * V.abs()).all()
        assert not O.requires_grad


# ---------------------------------------------------------------------------
# Launch shapes
# ---------------------------------------------------------------------------
SHAPES = [
    # B, H, n_q, n, n_out, d: 65 to 128 keys of 32 channels, four waves per row of the join
    (1, 2, 70, 200, 65, 32), (2, 1, 97, 150, 100, 32), (1, 1, 33, 128, 128, 32),
    (1, 1, 5000, 64, 48, 32),
    # one wave and two waves per tile of rows
    (33, 8, 20, 260, 257, 32), (33, 8, 20, 260, 257, 64), (33, 8, 20, 260, 257, 128),
    (16, 4, 200, 300, 260, 32), (16, 4, 200, 300, 260, 64), (32, 2, 193, 290, 288, 128),
]


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("B,H,n_q,n,n_out,d", SHAPES)
def test_gradient(B, H, n_q, n, n_out, d, dtype, out):
    grad.test_gradient(B, H, n_q, n, n_out, d, dtype, out)


@pytest.mark.parametrize("B,H,n_q,n,n_out,d", SHAPES)
def test_gradient_without_that_of_the_weights(B, H, n_q, n, n_out, d):
    grad.test_gradient_without_that_of_the_weights(B, H, n_q, n, n_out, d)
