"""silu and gelu keep their digits where they are small: relative errors over the whole range of the argument."""
import math

import pytest
import torch

from tests.operators_ref import U, within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
# include/agnes.h: with float32 results 2^-20 of the value (2^-142 where that is smaller), and of the two terms of the
# slope; with results of 16 bits 2^-16 and 2^-119
REL, ABS = 2.0 ** -20, 2.0 ** -142
REL16, ABS16 = 2.0 ** -16, 2.0 ** -119


@pytest.fixture(scope="module")
def ag():
    import paper_2601_01473_amd as m
    return m


def points():
    n = torch.linspace(-14.5, 14.5, 20001)
    return torch.cat([n, torch.linspace(-110, 110, 4001), torch.exp2(torch.linspace(-140, 6, 2001)),
                      -torch.exp2(torch.linspace(-140, 6, 2001)), torch.tensor([0.0, -0.0, 3e38, -3e38])])


def definition(kind, x):
    """(value, slope, magnitude of the slope's two terms) at x (float64)."""
    if kind == "silu":
        p, n = torch.sigmoid(x), torch.sigmoid(-x)
        return x * p, p * (1 + x * n), p * (1 + x.abs() * n)
    p = 0.5 * torch.special.erfc(-x / math.sqrt(2))
    d = torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return x * p, p + x * d, p + x.abs() * d


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_values_in_every_digit(ag, act):
    x = points()
    y, _, _ = definition(act, x.double())
    got, none = ag.mx8_activation(x.view(-1, 1).cuda(), act, keep=False)
    within(got.view(-1), y, REL * y.abs() + ABS, act)
    # a gate in front of it
    b = torch.full_like(x, 0.75)
    got, none = ag.mx8_activation(torch.stack([x, b], 1).cuda(), act, gated=True, keep=False)
    within(got.view(-1), 0.75 * y, 0.75 * (REL * y.abs() + ABS), act + " gated")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes_in_every_digit(ag, act):
    kept = ag.mx8_quantize(points().view(-1, 1).cuda())     # a block each
    k = ag.mx8_dequantize(kept).view(-1).cpu()
    y, slope, size = definition(act, k.double())
    one = torch.ones(len(k), 1, device="cuda")
    within(ag.mx8_activation_grad(one, kept, act).view(-1), slope, REL * size + ABS, act)
    both = ag.mx8_quantize(torch.stack([k, torch.full_like(k, 0.75)], 1).cuda())
    a, b = ag.mx8_dequantize(both).cpu().double().unbind(1)
    y, slope, size = definition(act, a)
    g = ag.mx8_activation_grad(one, both, act, gated=True).cpu()
    within(g[:, 0], b * slope, b.abs() * (REL * size + ABS) + U * (b * slope).abs(), act + " by the value")
    within(g[:, 1], y, REL * y.abs() + ABS, act + " by the gate")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_results_of_16_bits(ag, act, dtype):
    x = points()
    x = x[x.abs() < 1e6]
    y, _, _ = definition(act, x.double())
    got, kept = ag.mx8_activation(x.view(-1, 1).cuda(), act, dtype=dtype)
    within(got.view(-1), y, REL16 * y.abs() + ABS16, act)
    k = ag.mx8_dequantize(kept).view(-1).cpu().double()
    _, slope, size = definition(act, k)
    one = torch.ones(len(x), 1, device="cuda")
    within(ag.mx8_activation_grad(one, kept, act, dtype=dtype).view(-1), slope, REL16 * size + ABS16, act)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_undefined_arguments(ag, act):
    x = torch.tensor([[float("nan")], [float("inf")], [3e38], [-3e38]], device="cuda")
    got, kept = ag.mx8_activation(x, act)
    assert math.isnan(got[0]) and got[1] == float("inf") and got[2] == x[2] and got[3] == 0
    dx = ag.mx8_activation_grad(torch.ones_like(x), kept, act).view(-1).tolist()
    assert math.isnan(dx[0]) and math.isnan(dx[1]) and dx[2:] == [1.0, 0.0]
