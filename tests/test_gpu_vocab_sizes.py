"""The vocabulary calls at sizes that meet several of their limits, and on
values and arguments between the cases of the other tests."""

import math

import pytest

from paper_1606_00511_amd import hf as H
from tests.test_gpu_vocab import (E32, IGN, check_head, dt, gen, head_inputs, label_targets,
                                  list_targets, mask_rows, reference, teacher, unit, within)

pytestmark = pytest.mark.gpu


def T():
    import torch
    return torch


def test_embedding_past_a_million_workgroups():
    """Rows times strips of 1 KiB that take a second dimension of the grid;
    every element of the first and last rows and of every 997th."""
    torch = T()
    torch.cuda.empty_cache()
    rows, V, D = 65793, 5, 16500
    E = torch.randn(V, D, generator=gen(0), device="cuda")
    tok = mask_rows(torch.randint(0, V, (rows,), generator=gen(1), device="cuda").int(), "some")
    net = H.HFVocab(V, D, rows, "fp32")
    out = torch.full((rows, D), 7.0, device="cuda")
    net.hf_vocab_embed(E, tok, 2.0, out=out)
    assert -(-rows * -(-D // 256) // 4) > 1 << 20
    at = torch.cat([torch.arange(64), torch.arange(0, rows, 997), torch.arange(rows - 64, rows)])
    keep = (tok >= 0)[at, None]
    assert torch.equal(out[at], torch.where(keep, E[tok[at].long().clamp(min=0)] * 2, 0.0))
    assert int((out == 7).sum()) == 0
    net.hf_vocab_check()
    del net, out
    torch.cuda.empty_cache()
