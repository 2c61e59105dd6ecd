"""Means of a layer norm's rows: rows of one value, rows far from zero, rows with a value far from the others.  What the
mean is off by goes into every value of a row and into its variance; the bounds (oracle/model_oracle.py) leave it one
rounding where it is stored and none where the forward pass uses it."""
import math

import pytest
import torch

from oracle import model_oracle as mo
from test_gpu_layer_norm import DTYPES, _compare, _inputs
from test_gpu_model_ops import _normal

pytestmark = pytest.mark.gpu
VALUES = (0.1, 1234.567, -7.3e-6, 3.1e7, 1.0 / 3, -2e38, 0.0)


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [8, 16, 72, 200, 512, 1000, 1600, 2056, 3000, 4104, 8200, 16384])
def test_rows_of_one_value(ops, dtype, width):
    """Their mean is the value and nothing is left of them: y is the bias, to the last bit, and r what eps says (two
    roundings of the root, one of eps in fp32)."""
    _, _, w, b, _, _ = (t.cuda() for t in _inputs(1, width, dtype, width))
    x = torch.tensor(VALUES).to(dtype)[:, None].expand(-1, width).contiguous().cuda()
    for eps in (1e-5, 1e-12):
        for residual in (None, x):                       # twice the value; -4e38 is beyond fp32
            rows = slice(None) if residual is None else [0, 1, 2, 3, 4, 6]
            given = x[rows]
            y, s, stats = ops.layer_norm(given, w, b, eps, None if residual is None else given)
            assert torch.equal(stats[0], s[:, 0].float())
            assert ((stats[1].double() * math.sqrt(eps) - 1).abs() <= 4 * mo.E).all()
            assert torch.equal(y, b.expand_as(y))
            assert not ops.layer_norm(given, w, None, eps)[0].any()
    y, _, stats = ops.layer_norm(x, w, b, 0.0)
    assert torch.isnan(y).all() and torch.isinf(stats[1]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width", [(40, 16), (33, 200), (40, 1000), (37, 1600), (21, 3000), (9, 4104), (9, 16384)])
def test_rows_far_from_zero(ops, dtype, rows, width):
    """Deviations of one around 1e3 to 1e6, deviations of a few of the type's steps, all other values around one that is far
    from them: forward and backward within the bounds."""
    x, r, w, b, dy, ds = _inputs(rows, width, dtype, 3)
    gen = torch.Generator().manual_seed(width)
    wide = x.double()
    for i, mean in enumerate((1e3, -1e4, 1e5, 1e6, 100.1)):
        wide[i::6] = wide[i::6] * (1.0 if i < 4 else 1e-4) + mean
    wide[5::6, 0] = 1e6                                  # the first value, or any other, far off
    wide[5, 0], wide[5, width - 3] = 0.5, -1e6
    x = wide.to(dtype)
    got = _compare(ops, x.cuda(), None, w.cuda(), b.cuda(), dy.cuda(), ds.cuda())
    _compare(ops, x.cuda(), (r * 3).cuda(), w.cuda(), None, dy.cuda(), None)
    # the norm does not know where zero is, as far as the type holds the moved rows: whole numbers
    if dtype == torch.float32:
        whole = torch.randint(-50, 50, (rows, width), generator=gen).float().cuda()
        whole[:, 0], whole[:, 1] = 50.0, -50.0
        moved = whole, whole + 2.0 ** 22
        near, far = (ops.layer_norm(t, w.cuda(), b.cuda())[0].double().cpu() for t in moved)
        assert ((near - far).abs() <= sum(mo.layer_norm(t.cpu(), w, b, 1e-5)["y"][1] for t in moved)).all()
    assert got[0].shape == x.shape


def test_the_mean_of_many_equal_steps(ops):
    """A mean that fp32 does not hold: rows of v and the number after v, three of four the latter.  n is -sqrt(3) and
    1 / sqrt(3) whatever v is, to what the bounds of a row next to zero give."""
    width, n = 1600, torch.arange(1600) % 4 > 0
    for v in (1.0, 1234.567, 2.0 ** 20):
        low = torch.tensor(v)
        high = torch.nextafter(low, torch.tensor(math.inf))
        x = torch.where(n, high, low).expand(3, width).contiguous()
        y = ops.layer_norm(x.cuda(), torch.ones(width, device="cuda"), None, 0.0)[0].cpu().double()
        want = torch.where(n, 1 / math.sqrt(3), -math.sqrt(3)).double()
        assert float(((y - want) / want).abs().max()) < 40 * mo.E, v
