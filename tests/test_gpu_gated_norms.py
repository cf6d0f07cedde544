"""The gated block's results by their 2-norm against the definitions in 64 bits: bounds
element by element count every rounding at its worst, which a lost rounding can hide
behind; a norm shows it."""

import pytest
import torch

from paper_1606_00511_amd import hf as H
from tests import gated_util as G

pytestmark = pytest.mark.gpu


# around the forms of few rows: 17 to 64 rows with Wd in tiles (widths of 64) and in
# place, 65 to 128 rows
@pytest.mark.parametrize("T", [1, 16, 17, 24, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("D,F", [(320, 640), (301, 517), (320, 8256)])
def test_forward_rounds_once(T, D, F):
    """bf16 calls of up to 128 rows are off by the rounding of Y alone.  h in two terms
    is off by 2^-16 of itself at most, fp32 sums by less, 1% of the mean rounding of
    2^-9.2: with all of it along the rounding's error, 2% more than that.  (h in one term:
    41% more.)"""
    X, Wg, Wu, Wd, _ = G.inputs(T, D, F, torch.bfloat16, seed=T)
    n = H.HFGated(D, F, T, dtype="bf16")
    want = G.block("silu", X, Wg, Wu, Wd)[0]
    rounding = float((want.to(torch.bfloat16).double() - want).norm())
    for keep in (None, "full", "int8"):
        Y = n.hf_gated_forward(X, Wg, Wu, Wd, keep=keep)[0]
        assert float((Y.double() - want).norm()) <= 1.1 * rounding, keep
