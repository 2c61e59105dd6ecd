"""Residual sum and layer norm through the library against their definition in 64 bits (oracle/model_oracle.py), within
the bounds that rounding allows: every number of lanes a row, ragged widths, views, rows far from zero, masks."""
import pytest
import torch

from oracle import model_oracle as mo
from test_gpu_model_ops import _check, _normal

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


def _inputs(rows, width, dtype, seed, offset=0.0):
    gen = torch.Generator().manual_seed(seed)
    x = (_normal(gen, rows, width, dtype=torch.float64) + offset).to(dtype)
    r, dy, ds = (_normal(gen, rows, width, dtype=dtype) for _ in range(3))
    return x, r, _normal(gen, width, dtype=dtype, sigma=0.2, mean=1.0), _normal(gen, width, dtype=dtype, sigma=0.3), dy, ds


def _compare(ops, x, r, w, b, dy, ds, eps=1e-5):
    """Forward and backward; returns the results."""
    y, s, stats = ops.layer_norm(x, w, b, eps, r)
    dx, dw, db = ops.layer_norm_backward(dy, s, w, stats, ds, want=(True, b is not None))
    cpu = lambda t: None if t is None else t.detach().cpu()                # noqa: E731
    if r is not None:
        want = x.double().cpu() + r.double().cpu()
        # one rounding to fp32, one to the type
        _check("s", s, want, (mo.U[x.dtype] * 1.01 + mo.E) * want.abs())
    want = mo.layer_norm(cpu(s), cpu(w), cpu(b), eps, cpu(dy), cpu(ds))
    got = {"y": y, "mean": stats[0], "r": stats[1], "dx": dx, "dw": dw}
    if b is not None:
        got["db"] = db
    for name, t in got.items():
        _check(name, t, *want[name])
    return y, s, stats, dx, dw, db


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width", [(1, 8), (5, 16), (33, 40), (17, 128), (6, 136), (37, 256), (3, 264), (130, 512), (9, 520),
                                        (37, 1024), (4, 1032), (61, 1600), (2, 2048), (5, 2056), (7, 4096), (3, 5000), (1, 8192),
                                        (3, 8200), (2, 16384), (700, 1024), (2100, 72), (1100, 2048), (520, 4104)])
def test_layer_norm(ops, dtype, rows, width):
    x, r, w, b, dy, ds = (t.cuda() for t in _inputs(rows, width, dtype, rows + width, 0.5))
    got = _compare(ops, x, r, w, b, dy, ds)
    # without a residual, without a bias: the same norm of the same rows
    y, s, stats = ops.layer_norm(got[1], w, None)
    assert s is got[1] and torch.equal(stats, got[2])
    _compare(ops, x, None, w, None, dy, None)
    _compare(ops, x, None, w, b, dy, ds)
    # in place, forward and backward
    a, c = x.clone(), r.clone()
    y, s, stats = ops.layer_norm(a, w, b, residual=c, s=a, y=c)
    assert s is a and y is c and torch.equal(s, got[1]) and torch.equal(y, got[0])
    for place in ("dy", "ds"):
        given = {"dy": dy.clone(), "ds": ds.clone()}
        dx, dw, db = ops.layer_norm_backward(given["dy"], s, w, stats, given["ds"], dx=given[place])
        assert torch.equal(dx, got[3]) and torch.equal(dw, got[4]) and torch.equal(db, got[5])
    # one of the two sums over rows alone, or none
    for want in ((True, False), (False, True), (False, False)):
        dx, dw, db = ops.layer_norm_backward(dy, s, w, stats, ds, want=want)
        assert torch.equal(dx, got[3]) and (dw is None) == (not want[0]) and (db is None) == (not want[1])
        assert (dw is None or torch.equal(dw, got[4])) and (db is None or torch.equal(db, got[5]))


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_with_a_stride(ops, dtype):
    """Parts of wider rows, each array with its own stride; what lies between is left as it is."""
    rows, width = 45, 200
    dense = [t.cuda() for t in _inputs(rows, width, dtype, 3)]
    x, r, w, b, dy, ds = dense
    got = _compare(ops, x, r, w, b, dy, ds)

    def wide(t, extra):
        base = torch.full((rows, width + extra), 7.0, dtype=dtype, device="cuda")
        base[:, extra - 8:extra - 8 + width] = 0 if t is None else t
        return base, base[:, extra - 8:extra - 8 + width]

    views = [wide(t, 8 * n) for n, t in enumerate((x, r, None, None, dy, ds, None), 1)]
    vx, vr, vs, vy, vdy, vds, vdx = (v for _, v in views)
    y, s, stats = ops.layer_norm(vx, w, b, residual=vr, s=vs, y=vy)
    dx, dw, db = ops.layer_norm_backward(vdy, s, w, stats, vds, dx=vdx)
    for a, c in zip((y, s, stats, dx, dw, db), got):
        assert torch.equal(a, c)
    for n, (base, _) in enumerate(views, 1):
        assert (base[:, :8 * n - 8] == 7).all() and (base[:, 8 * n - 8 + width:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [64, 1024, 3000])
def test_rows_far_from_zero_and_rows_of_equal_values(ops, dtype, width):
    x, r, w, b, dy, ds = _inputs(20, width, dtype, 9)
    x[3] = 5.0
    x[4] = 0.0
    x[5:10] = (x[5:10].double() * 0.01 + 100).to(dtype)
    x[10:15] = (x[10:15].double() * 1e-12).to(dtype)
    x[15] = (x[15].double() * 1e10).to(dtype)
    y = _compare(ops, x.cuda(), None, w.cuda(), b.cuda(), dy.cuda(), ds.cuda())[0].cpu()
    assert torch.equal(y[3], b) and torch.equal(y[4], b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [72, 1024, 2504])
def test_non_finite_values_stay_in_their_row(ops, dtype, width):
    x, r, w, b, dy, ds = (t.cuda() for t in _inputs(21, width, dtype, 4))
    clean = ops.layer_norm(x, w, b, residual=r)
    bad = torch.zeros(21, dtype=torch.bool, device="cuda")
    bad[[0, 7, 20]] = True
    x[0, 5], x[7, 9], x[20] = float("nan"), float("inf"), -float("inf")
    y, s, stats = ops.layer_norm(x, w, b, residual=r)
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[0][~bad]) and torch.equal(stats[:, ~bad], clean[2][:, ~bad])
    dx = ops.layer_norm_backward(dy, s, w, stats, ds, want=(False, False))[0]
    want = ops.layer_norm_backward(dy, clean[1], w, clean[2], ds, want=(False, False))[0]
    assert torch.isnan(dx[bad]).all() and torch.equal(dx[~bad], want[~bad])


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(ops, dtype):
    w = torch.ones(64, dtype=dtype, device="cuda")
    x = torch.empty(0, 64, dtype=dtype, device="cuda")
    y, s, stats = ops.layer_norm(x, w, w, residual=x)
    assert y.shape == x.shape and stats.shape == (2, 0)
    dx, dw, db = ops.layer_norm_backward(x, s, w, stats, x)
    assert dx.shape == x.shape and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_beyond_32_bits(ops, dtype):
    """Rows 2^20 elements apart: the last ones begin more than 2^32 bytes after the first."""
    rows, width, far = 2300, 136, 1 << 20
    x, r, w, b, dy, ds = (t.cuda() for t in _inputs(rows, width, dtype, 1))
    got = _compare(ops, x, r, w, b, dy, ds)
    base = torch.empty(rows, far, dtype=dtype, device="cuda")
    parts = [base[:, n * 256:n * 256 + width] for n in range(7)]
    for p, t in zip(parts, (x, r, dy, ds)):
        p.copy_(t)
    y, s, stats = ops.layer_norm(parts[0], w, b, residual=parts[1], s=parts[4], y=parts[5])
    dx, dw, db = ops.layer_norm_backward(parts[2], s, w, stats, parts[3], dx=parts[6])
    for a, c in zip((y, s, stats, dx, dw, db), got):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_into_slices_of_an_arena(ops, dtype):
    """Gains' gradients beside each other in one buffer, on 4 bytes alone."""
    x, r, w, b, dy, ds = (t.cuda() for t in _inputs(50, 72, dtype, 2))
    y, s, stats = ops.layer_norm(x, w, b, residual=r)
    want = ops.layer_norm_backward(dy, s, w, stats, ds)
    arena = torch.full((2 + 72 + 2 + 72 + 2,), 3.0, dtype=dtype, device="cuda")
    got = ops.layer_norm_backward(dy, s, w, stats, ds, dw=arena[2:74], db=arena[76:148])
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    assert (arena[[0, 1, 74, 75, 148, 149]] == 3).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_are_those_of_the_definition(ops, dtype):
    """The classes against autograd on the definition in 64 bits: fp32 good to 1e-5 of a gradient's norm, bf16 to a
    rounding of the result and one of the residual stream on the way."""
    x, r, w, b, dy, ds = (t.cuda() for t in _inputs(40, 96, dtype, 8))
    ours = [t.clone().requires_grad_() for t in (x, r, w, b)]
    s, y = ops.AddLayerNorm.apply(*ours, 1e-5)
    z = ops.LayerNorm.apply(s, ours[2], None, 1e-5)
    torch.autograd.backward((s, y, z), (ds, dy, r))
    plain = [t.double().requires_grad_() for t in (x, r, w, b)]
    t = plain[0] + plain[1]
    n = (t - t.mean(1, keepdim=True)) / (t.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    torch.autograd.backward((t, n * plain[2] + plain[3], n * plain[2]), (ds.double(), dy.double(), r.double()))
    for a, c in zip(ours, plain):
        off = float((a.grad.double() - c.grad).norm() / c.grad.norm())
        assert off < (1e-5 if dtype == torch.float32 else 3 * 2.0 ** -8), off


def test_refusals(ops):
    from test_gpu_model_paths import _refused
    x, r, w, b, dy, ds = (t.cuda() for t in _inputs(6, 64, torch.bfloat16, 2))
    _refused(lambda: ops.layer_norm(x, w.float(), b), "w")
    _refused(lambda: ops.layer_norm(x, w[:32], b), "w")
    _refused(lambda: ops.layer_norm(x, w, b[::2]), "b")
    _refused(lambda: ops.layer_norm(x, w, b, residual=r[:5]), "residual")
    _refused(lambda: ops.layer_norm(x, w, b, residual=r.float()), "residual")
    _refused(lambda: ops.layer_norm(x, w, b, s=r), "s:")
    _refused(lambda: ops.layer_norm(x, w, b, residual=r, s=x, y=x), "eager_layer_norm")
    _refused(lambda: ops.layer_norm(x, w, b, eps=-1.0), "eager_layer_norm")
    _refused(lambda: ops.layer_norm(x[:, :60], w[:60], b[:60]), "eager_layer_norm")
    _refused(lambda: ops.layer_norm(x[:1].expand(6, -1), w, b), "eager_layer_norm")           # a broadcast view
    _refused(lambda: ops.layer_norm(x.t().contiguous().t(), w, b), "rows")
    y, s, stats = ops.layer_norm(x, w, b, residual=r)
    _refused(lambda: ops.layer_norm_backward(dy.float(), s, w, stats), "dy")
    _refused(lambda: ops.layer_norm_backward(dy, s, w, stats[:, :5]), "stats")
    _refused(lambda: ops.layer_norm_backward(dy, s, w, stats.t().contiguous().t()), "stats")
    _refused(lambda: ops.layer_norm_backward(dy, s, w, stats, ds[:5]), "ds")
    _refused(lambda: ops.layer_norm_backward(dy, s, w, stats, dw=w.float()), "dw")
    _refused(lambda: ops.layer_norm_backward(dy, s, w, stats, db=w[:8]), "db")
