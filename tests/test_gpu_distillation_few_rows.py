"""Distillation of up to 64 rows, whose backward pass finds the words, counts the rows that matter and moves them in one
launch: masked rows, rows without a weight and what stands in them, in every place among the workgroups' 16 rows."""
import math

import pytest
import torch

from oracle import model_oracle as mo
from test_gpu_distillation import DTYPES, NAMES, _inputs, _run
from test_gpu_model_ops import _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


def _left_out(rows, pattern):
    """Which rows are masked and which have no weight."""
    at = torch.arange(rows)
    gen = torch.Generator().manual_seed(rows)
    out, weightless = {"front": (at < 11, (at >= 11) & (at < 16)), "thirds": (at % 3 == 0, at % 3 == 1),
                       "all but the last": (at < rows - 1, at < 0), "weights of the first workgroup": (at < 0, at < 16),
                       "drawn": (torch.rand(rows, generator=gen) < 0.3, torch.rand(rows, generator=gen) < 0.3)}[pattern]
    return out.cuda(), weightless.cuda()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pattern", ["front", "thirds", "all but the last", "weights of the first workgroup", "drawn"])
@pytest.mark.parametrize("rows,vocab,entries", [(17, 500, 12), (33, 64, 1), (40, 5003, 12), (64, 300, 129), (64, 40003, 65), (16, 2000, 7)])
def test_masked_rows_reach_no_gradient(ops, dtype, pattern, rows, vocab, entries):
    x, w, index, logits, g = _inputs(rows, 64, vocab, entries, dtype, 6, unused=0.0, empty=0.0)
    out, weightless = _left_out(rows, pattern)
    half = torch.arange(rows, device="cuda") % 2 == 0
    index[out] = -7
    logits[out] = math.nan
    index[out & half] = 3
    logits[out & half] = -math.inf
    g[weightless] = 0.0
    left = out | weightless
    got = _run(ops, x, w, index, logits, torch.where(left, 0.0, g), 2.0)
    want = mo.distillation(x, w, index, logits, 2.0, torch.where(left, 0.0, g), 2 if dtype == torch.bfloat16 else 1)
    for name in NAMES:
        _check(name, got[name], *(t.cpu() for t in want[name]))
    # the rows that count alone, one behind the other: the same numbers
    keep = ~left
    alone = _run(ops, x[keep].contiguous(), w, index[keep].contiguous(), logits[keep].contiguous(), g[keep].contiguous(), 2.0)
    assert not got["dx"][left].any()
    if keep.any():
        assert torch.equal(alone["loss"], got["loss"][keep])
    # whatever stands in the rows that are left out, the results are the same
    x[out], x[weightless] = math.nan, math.inf
    g[out] = math.nan
    loss, lse, picked = ops.distillation(x, w, index, logits, 2.0)
    assert torch.equal(loss[~weightless], got["loss"][~weightless]) and not loss[out].any()
    dx, dw = ops.distillation_backward(g, x, w, index, logits, lse, picked, 2.0)
    assert not dx[left].any() and torch.equal(dx, got["dx"]) and torch.equal(dw, got["dw"])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 16, 17, 40, 64])
def test_all_rows_left_out(ops, dtype, rows):
    x, w, index, logits, g = _inputs(rows, 96, 333, 5, dtype, 4, unused=0.0, empty=0.0)
    for masked in (True, False):
        at, weight = (torch.full_like(index, -1), g) if masked else (index, torch.zeros_like(g))
        got = _run(ops, x, w, at, logits, weight, 1.0)
        for name in ("loss", "picked", "dx", "dw") if masked else ("dx", "dw"):
            assert not got[name].any(), name


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [17, 64])
def test_an_index_beyond_the_vocabulary(ops, dtype, rows):
    """In a row behind masked ones: it says so, the others do not know."""
    x, w, index, logits, g = _inputs(rows, 64, 400, 6, dtype, 9, unused=0.0, empty=0.0)
    index[:5] = -1
    clean = _run(ops, x, w, index, logits, g, 1.0)
    index[rows - 1, 2] = 400
    got = _run(ops, x, w, index, logits, g, 1.0)
    assert torch.isnan(got["loss"][rows - 1]) and torch.isnan(got["dx"][rows - 1]).all() and torch.isnan(got["dw"]).all()
    assert torch.equal(got["loss"][:rows - 1], clean["loss"][:rows - 1]) and torch.equal(got["dx"][:rows - 1], clean["dx"][:rows - 1])
