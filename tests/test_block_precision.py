"""What the header promises of the projector block beyond its types' rounding: with up to 8 rows the gated feed-forward block
keeps twice the type's bits of h, and its gate bias's gradient sums values that are not rounded.  Inputs are made so that a
kernel that breaks the promise leaves the bound; that they do is shown on the CPU, with the mistake planted in the oracle."""
import pytest
import torch

import block_oracle as bo
import paper_2502_11490_amd as ann

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---- h in two parts


def _few_rows(M, F, act, dtype):
    """Rows that differ little, and a b_out that takes nearly all of out away: what is left is rounded finely."""
    g = torch.Generator().manual_seed(100 * M + F + act)
    D, O = 8, 24
    x = (torch.randn(1, D, generator=g) + torch.randn(M, D, generator=g) / 128).to(dtype)
    w_in, w_out = (torch.randn(2 * F, D, generator=g) * D ** -0.5).to(dtype), torch.randn(O, F, generator=g).to(dtype)
    b_in = torch.randn(2 * F, generator=g).to(dtype)
    b_out = -bo.ffn(x[:1], w_in, w_out, b_in, None, act, torch.float32)[0][0].to(dtype)
    return x, w_in, w_out, b_in, b_out


def _h(x, w_in, b_in, act):
    z = x.double() @ w_in.double().t() + b_in.double()
    F = z.shape[1] // 2
    return bo.act_of(act, z[:, :F])[0] * z[:, F:]


def _two_part_bound(x, w_in, w_out, b_in, b_out, act, dtype):
    """out and its bound before its rounding: that of an h in fp32, the rounding of what the first part leaves over, and
    as many sums again."""
    want, _, bound, _ = bo.ffn(x, w_in, w_out, b_in, b_out, act, torch.float32)
    h = _h(x, w_in, b_in, act).abs() * (1 + 2.0 ** -15)
    F = h.shape[1]
    left = bo.half_step(bo.half_step(h, dtype), dtype)
    return want, bound + (left + F * bo.U * h) @ w_out.double().abs().t()


SHAPES = [(M, F, act) for M in (1, 4, 5, 8) for F, act in ((16, 0), (40, 1), (16, 2), (40, 3))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,F,act", SHAPES)
def test_bound_of_two_parts_sees_an_h_of_one(M, F, act, dtype):
    t = TYPES[dtype]
    args = _few_rows(M, F, act, t)
    x, w_in, w_out, b_in, b_out = args
    want, bound = _two_part_bound(*args, act, t)
    h = _h(x, w_in, b_in, act)
    first = h.to(t)
    rest = (h - first.double()).to(t)
    out = lambda h: (h @ w_out.double().t() + b_out.double()).to(t)  # noqa: E731
    bo.assert_close(out(first.double() + rest.double()), want, bound)
    with pytest.raises(AssertionError):
        bo.assert_close(out(first.double()), want, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,F,act", SHAPES)
def test_few_rows_keep_h_in_two_parts(M, F, act, dtype):
    t = TYPES[dtype]
    args = [a.cuda() for a in _few_rows(M, F, act, t)]
    want, bound = _two_part_bound(*args, act, t)
    bo.assert_close(ann.ann_gated_ffn(*args, act), want, bound)


# ---- the gate bias's gradient


def _cancelling_rows(M, dtype):
    """One row of x many times, and rows of dout in threes a, b, -(a + b): every column of the gradient of gate and up sums to
    nothing, but not once it is rounded."""
    g = torch.Generator().manual_seed(M)
    D, F, O = 16, 40, 24
    x = torch.randn(1, D, generator=g).to(dtype).repeat(M, 1)
    w_in, w_out = (torch.randn(2 * F, D, generator=g) * D ** -0.5).to(dtype), torch.randn(O, F, generator=g).to(dtype)
    ab = torch.randint(-3, 4, (2, M // 3, O), generator=g)
    dout = torch.stack((ab[0], ab[1], -(ab[0] + ab[1])), 1).reshape(M, O).to(dtype)
    return x, w_in, w_out, dout


def _unrounded_bias_gradient(dout, x, pre, w_in, w_out, act):
    values, bounds = bo.ffn_grad(dout, x, pre, w_in, w_out, act, torch.float32)
    return values[3], bounds[3]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,act", [(30, 0), (30, 2), (300, 1)])
def test_bound_of_the_bias_gradient_sees_rounded_terms(M, act, dtype):
    t = TYPES[dtype]
    x, w_in, w_out, dout = _cancelling_rows(M, t)
    pre = (x.double() @ w_in.double().t()).float()
    want, bound = _unrounded_bias_gradient(dout, x, pre, w_in, w_out, act)
    F = w_out.shape[1]
    a, slope = bo.act_of(act, pre[:, :F].double())
    dh = dout.double() @ w_out.double()
    dz = torch.cat((dh * pre[:, F:].double() * slope, dh * a), 1)
    bo.assert_close(dz.sum(0).to(t), want, bound)
    with pytest.raises(AssertionError):
        bo.assert_close(dz.to(t).double().sum(0).to(t), want, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,act", [(30, 0), (30, 2), (300, 1)])
def test_bias_gradient_sums_what_is_not_rounded(M, act, dtype):
    x, w_in, w_out, dout = (a.cuda() for a in _cancelling_rows(M, TYPES[dtype]))
    _, pre = ann.ann_gated_ffn(x, w_in, w_out, act=act, save=True)
    db_in = ann.ann_gated_ffn_backward(dout, x, pre, w_in, w_out, act, bias=True)[3]
    bo.assert_close(db_in, *_unrounded_bias_gradient(dout, x, pre, w_in, w_out, act))
