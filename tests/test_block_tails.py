"""The activations of the gated feed-forward block far from zero, where what is small is the difference of what is not: the
values and slopes keep their leading bits there."""
import pytest
import torch

import block_oracle as bo
import paper_2502_11490_amd as ann

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NAMES = {ann.ANN_SILU: "silu", ann.ANN_GELU: "gelu", ann.ANN_SIGMOID: "sigmoid"}


def _relative(z):
    """Bound of an activation's relative error: the exponential's (and the normal distribution's) goes with the rounding of its
    argument, up to z^2 of it; 32 roundings for the functions and the operations around them."""
    return (2 * z * z + 32) * bo.U


def _one_unit(dtype):
    """z on a grid and a block of one hidden unit that answers act(z) * 1, its terms exact."""
    z = torch.arange(-96, 97, device="cuda", dtype=torch.float64)[:, None] / 8
    x, one = z.to(dtype), torch.ones(1, 1, dtype=dtype, device="cuda")
    w_in, b_in = torch.tensor([[1.0], [0.0]], device="cuda").to(dtype), torch.tensor([0.0, 1.0], device="cuda").to(dtype)
    assert torch.equal(x.double(), z)
    return z, x, w_in, one, b_in


@pytest.mark.parametrize("M", [1, 193], ids=["few rows", "tile"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", NAMES, ids=NAMES.values())
def test_values_in_the_tails(act, dtype, M):
    z, x, w_in, w_out, b_in = _one_unit(TYPES[dtype])
    want = bo.act_of(act, z)[0]
    h = 0.0 if M == 1 or dtype == "f32" else 1.0  # the rounding of h
    got = torch.cat([ann.ann_gated_ffn(rows, w_in, w_out, b_in, None, act) for rows in x.split(M)])
    bo.assert_close(got, want, want.abs() * _relative(z) + h * bo.half_step(want, TYPES[dtype]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", NAMES, ids=NAMES.values())
def test_slopes_in_the_tails(act, dtype):
    z, x, w_in, w_out, b_in = _one_unit(TYPES[dtype])
    pre = torch.cat((z, torch.ones_like(z)), 1).float()
    got = ann.ann_gated_ffn_backward(torch.ones_like(x), x, pre, w_in, w_out, act, need_dw=False)[0]
    want = bo.act_of(act, z)[1]
    # what the slope is the sum of: the function's own factor and z times that factor's derivative
    own = {ann.ANN_SILU: torch.sigmoid(z), ann.ANN_GELU: 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)}.get(act, want)
    bound = (own.abs() + (want - own).abs()) * _relative(z)
    h = 0.0 if dtype == "f32" else 1.0  # the rounding of dgate
    bo.assert_close(got, want, bound + h * bo.half_step(want.abs() + bound, TYPES[dtype]))
