"""The gated block's activations far below 0, in fp32, against 64 bits."""

import math

import pytest
import torch

from paper_1606_00511_amd import hf as H
from tests import gated_util as G

pytestmark = pytest.mark.gpu


def exact(act, z):
    """By erfc and sigmoids: 1 + erf and 1 + tanh lose their digits in 64 bits too."""
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    w = z if act == "silu" else 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    return z * torch.exp(w) / (1 + torch.exp(w))


@pytest.mark.parametrize("act,end", [("silu", -87.0), ("gelu", -12.9), ("gelu_tanh", -10.0)])
@pytest.mark.parametrize("T", [50, 1000])
def test_far_below_zero(act, end, T):
    """Off by (of 2^-24): 32 by exp, erfc and the products around them; gelu's argument of
    erfc by 1.5 of itself, which erfc shows z^2 + 1 times; gelu_tanh's exponent by 6 of
    itself.  Past the end nothing is further from 0 than 2^-119."""
    z = torch.cat((torch.linspace(0, end, T // 2), torch.linspace(end, 4 * end, T - T // 2)))
    X = torch.stack((z, torch.ones(T)), 1).cuda()
    W = lambda *v: torch.tensor(v, device="cuda")       # noqa: E731
    n = H.HFGated(2, 1, T, act=act)
    Y = n.hf_gated_forward(X, W([1.0, 0.0]), W([0.0, 1.0]), W([1.0], [0.0]))[0][:, 0].double()
    z = X[:, 0].double()
    want = exact(act, z)
    few = {"silu": 0 * z, "gelu": 4 * (z * z + 1),
           "gelu_tanh": 6 * 1.6 * (z + 0.044715 * z ** 3).abs()}[act]
    near = z >= end
    assert ((Y - want).abs() <= (32 + few) * G.S * want.abs())[near].all()
    assert (Y.abs() <= 2.0 ** -119)[~near].all() and (Y <= 0).all()
