"""The digits that the activations of a gated block in fp32 keep far from 0, on the GPU against 64 bits."""
import math

import pytest
import torch

from operator_reference import U, close
from paper_2205_05632_amd import operators as ops

pytestmark = pytest.mark.gpu

# How far from 0 an activation is neither 0 nor subnormal.
FAR = {"silu": 80.0, "sigmoid": 80.0, "gelu": 12.5, "gelu_tanh": 9.0}


def exact(a, act):
    """act(a), its slope, and the sizes of the terms that they are added up from."""
    if act in ("silu", "sigmoid"):
        q, p = torch.sigmoid(a), torch.sigmoid(-a)
        return (q, q * p, q, q * p) if act == "sigmoid" else (a * q, q + a * q * p, (a * q).abs(), q + (a * q * p).abs())
    if act == "gelu":
        q, density = 0.5 * torch.special.erfc(-a * math.sqrt(0.5)), torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    else:
        k = math.sqrt(2 / math.pi)
        u2 = 2 * k * (a + 0.044715 * a ** 3)
        q, p = torch.sigmoid(u2), torch.sigmoid(-u2)
        density = q * p * 2 * k * (1 + 3 * 0.044715 * a * a)
    return a * q, q + a * density, (a * q).abs(), q + (a * density).abs()


def entries(act, count):
    g = torch.Generator().manual_seed(count)
    far = FAR[act]
    return torch.cat([(torch.rand(count - 6, generator=g, dtype=torch.float64) * 2 - 1) * far,
                      torch.tensor([far, -far, 0.5, -0.5, 1e-3, -1e-3], dtype=torch.float64)]).float().double()


# exp 3 U, 1 + E, 1 / x and products a unit each (and U for each rounding of a sum): 12 U, and 4 U more for the rest of gelu_tanh's
# argument.  The normal distribution's integral besides: z and t 4 U, the polynomial 0.6 U of approximation and 10 of ten rounded
# steps, 1 / x twice 2 U, products 4 U.
UNITS = {"silu": 12, "sigmoid": 12, "gelu": 40, "gelu_tanh": 16}


@pytest.mark.parametrize("act", FAR)
def test_slopes_and_values_of_the_backward_pass(act):
    a = entries(act, 4000)
    value, slope, size, size_slope = exact(a, act)
    one = torch.ones((8, 500), device="cuda")
    got = ops.compams_gated_backward(one, a.float().cuda().view(8, 500), one, 2, act, bias=False)
    close(got[1].view(-1), value, UNITS[act] * U * size, "act")
    close(got[0].view(-1), slope, (UNITS[act] + 8) * U * size_slope, "slope")


@pytest.mark.parametrize("act", FAR)
@pytest.mark.parametrize("count", [60, 4000])
def test_values_of_the_forward_pass(act, count):
    """A gate that is picked out of x, an up projection of 1."""
    a = entries(act, count)
    x = torch.stack([a.float(), torch.ones(count)], 1).cuda()
    gate, up = torch.tensor([[1.0, 0.0]], device="cuda").repeat(5, 1), torch.tensor([[0.0, 1.0]], device="cuda").repeat(5, 1)
    m, kept, _ = ops.compams_gated_forward(x, gate, up, act)
    assert torch.equal(kept.cpu().double(), a[:, None].repeat(1, 5))
    value, _, size, _ = exact(a, act)
    close(m, value[:, None].repeat(1, 5), (UNITS[act] * U * size)[:, None].repeat(1, 5), "m")
