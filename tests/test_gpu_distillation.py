"""Distillation through the library against its definition in 64 bits (oracle/model_oracle.py), within the bounds that
rounding allows: every shape of tiles and cut of the gradients, ragged and repeated entries, masks, confident rows."""
import math

import pytest
import torch

from oracle import model_oracle as mo
from test_gpu_model_ops import _check, _normal

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
NAMES = ("loss", "lse", "picked", "dx", "dw")


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


def _inputs(rows, width, vocab, entries, dtype, seed, unused=0.2, empty=0.1, repeats=False):
    """Words of a row differ from each other unless repeats are wanted."""
    gen = torch.Generator().manual_seed(seed)
    x, w = _normal(gen, rows, width, dtype=dtype), _normal(gen, vocab, width, dtype=dtype, sigma=1 / math.sqrt(width))
    if repeats:
        index = torch.randint(0, vocab, (rows, entries), generator=gen)
    else:
        index = torch.rand(rows, min(vocab, 4096), generator=gen).argsort(1)[:, :entries]
        index = index * (vocab // min(vocab, 4096))
    logits = _normal(gen, rows, entries, sigma=3.0)
    out = (torch.rand(rows, entries, generator=gen) < unused) | (torch.rand(rows, generator=gen) < empty)[:, None]
    index[out] = -1 - torch.randint(0, 5, (int(out.sum()),), generator=gen)
    logits[out] = math.nan
    return x.cuda(), w.cuda(), index.cuda(), logits.cuda(), _normal(gen, rows, sigma=0.1).cuda()


def _run(ops, x, w, index, logits, g, tau):
    loss, lse, picked = ops.distillation(x, w, index, logits, tau)
    dx, dw = ops.distillation_backward(g, x, w, index, logits, lse, picked, tau)
    return dict(zip(NAMES, (loss, lse, picked, dx, dw)))


def _compare(ops, x, w, index, logits, g, tau):
    pieces = 2 if x.dtype == torch.bfloat16 and (len(x) <= 128 or x.numel() * len(w) <= 2 ** 29) else 1
    got, want = _run(ops, x, w, index, logits, g, tau), mo.distillation(x, w, index, logits, tau, g, pieces)
    for name in NAMES:
        _check(name, got[name], *(t.cpu() for t in want[name]))
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width,vocab,entries,tau", [
    (1, 8, 1, 1, 1.0), (1, 64, 2, 2, 3.0), (5, 40, 129, 7, 0.5), (61, 128, 1000, 16, 1.0), (128, 64, 128, 64, 2.0),
    (129, 72, 257, 65, 1.0), (300, 136, 5003, 20, 4.0), (64, 1600, 101, 101, 1.5), (257, 256, 512, 256, 2.0), (17, 8, 300, 129, 1.0),
    (700, 64, 30001, 9, 2.0),        # large tiles
    (4000, 72, 130, 5, 1.0),         # dw in slices of the rows
    (8192, 8, 40003, 3, 1.0),        # several pieces
    (17003, 16, 300, 4, 2.0),        # rows counted by a kernel of their own
    (40, 1024, 2000, 33, 1.0),       # few rows: narrow tiles, dx in slices
    (2100, 328, 4097, 12, 0.7),
    (2100, 328, 4097, 128, 0.7),     # the same with all logits in the workspace
    (1500, 136, 13000, 256, 1.0), (1500, 64, 4097, 200, 3.0), (3000, 64, 4097, 256, 1.0), (4100, 136, 4097, 256, 1.0), (100, 8, 50257, 2, 1.0),   # in other tiles
    (1500, 8, 13000, 2, 1.0), (1500, 136, 4097, 1, 1.0),
    (129, 1600, 4097, 1, 1.0), (2600, 1600, 130, 2, 1.0),            # gradients with the weights' factor: large tiles, slices
    (129, 136, 30001, 2, 2.0)])      # gradients in two pieces: large tiles
def test_distillation(ops, dtype, rows, width, vocab, entries, tau):
    args = _inputs(rows, width, vocab, entries, dtype, rows + vocab)
    x, w, index, logits, g = args
    got = _compare(ops, *args, tau)
    rest = index, logits, got["lse"], got["picked"], tau
    assert torch.equal(ops.distillation_backward(g, x, w, *rest, want=(True, False))[0], got["dx"])
    assert torch.equal(ops.distillation_backward(g, x, w, *rest, want=(False, True))[1], got["dw"])
    for name, t in _run(ops, *args, tau).items():
        assert torch.equal(t, got[name]), name


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [3, 300, 20003])
def test_a_word_in_several_entries(ops, dtype, vocab):
    x, w, index, logits, g = _inputs(200, 64, vocab, 40, dtype, vocab, repeats=True)
    logits.nan_to_num_(0.0)
    index[:50, 1:] = index[:50, :1]                      # all entries of a row the same word
    index[50:60, 20:] = index[50:60, :20]
    _compare(ops, x, w, index, logits, g, 1.5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(300, 500), (20000, 64), (3001, 2000)])
def test_masked_rows_reach_no_gradient(ops, dtype, rows, vocab):
    """Whatever stands in rows without an entry or without a weight, and in entries that count nothing."""
    x, w, index, logits, g = _inputs(rows, 64, vocab, 12, dtype, 6, empty=0.0)
    gen = torch.Generator().manual_seed(1)
    out, weightless = ((torch.rand(rows, generator=gen) < share).cuda() for share in (0.3, 0.2))
    index[out] = -7
    half = torch.arange(rows, device="cuda") % 2 == 0
    index[out & half] = 3
    logits[out & half] = -math.inf                       # nothing left either way
    g[weightless] = 0.0
    left = out | weightless
    clean, weight = x.clone(), torch.where(left, 0.0, g)
    got = _run(ops, clean, w, index, logits, weight, 2.0)
    assert not got["loss"][out].any() and not got["picked"][(index < 0) | (logits == -math.inf)].any()
    x[out] = math.nan
    x[weightless] = math.inf
    g[out] = math.nan
    loss, lse, picked = ops.distillation(x, w, index, logits, 2.0)
    assert torch.equal(loss[~weightless], got["loss"][~weightless])
    dx, dw = ops.distillation_backward(g, x, w, index, logits, lse, picked, 2.0)
    assert not dx[left].any() and torch.equal(dx, got["dx"]) and torch.equal(dw, got["dw"])
    # an index beyond the vocabulary is not masked: the results say so
    index[0, 0], logits[0, 0], g[0] = vocab, 0.0, 1.0
    g[out] = 0.0
    loss, lse, picked = ops.distillation(clean, w, index, logits, 2.0)
    assert torch.isnan(loss[0]) and torch.isnan(picked[0, 0]) and torch.isfinite(loss).sum() == rows - 1
    dx, dw = ops.distillation_backward(g, clean, w, index, logits, lse, picked, 2.0)
    assert torch.isnan(dx[0]).all() and torch.isnan(dw).all() and torch.isfinite(dx[1:]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_all_rows_masked_and_no_rows(ops, dtype):
    x, w, index, logits, g = _inputs(90, 96, 333, 5, dtype, 4)
    index.fill_(-1)
    got = _run(ops, x, w, index, logits, g, 1.0)
    for name in ("loss", "picked", "dx", "dw"):
        assert not got[name].any(), name
    got = _run(ops, x[:0], w, index[:0], logits[:0], g[:0], 1.0)
    assert got["loss"].shape == (0,) and got["dx"].shape == (0, 96) and not got["dw"].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [200, 80000])
def test_numbers_that_are_none(ops, dtype, vocab):
    """NaN and infinities of a teacher that count: the row says so, the others do not know."""
    x, w, index, logits, g = _inputs(60, 64, vocab, 6, dtype, 11, unused=0.0, empty=0.0)
    clean = _run(ops, x, w, index, logits, g, 1.0)
    logits[4, 2], logits[9, 0], logits[11] = math.nan, math.inf, math.nan
    bad = torch.zeros(60, dtype=torch.bool, device="cuda")
    bad[[4, 9, 11]] = True
    dirty = _run(ops, x, w, index, logits, g, 1.0)
    assert torch.isnan(dirty["loss"][bad]).all() and torch.isnan(dirty["dx"][bad]).all()
    for name in ("loss", "dx"):
        assert torch.equal(dirty[name][~bad], clean[name][~bad]), name
    # a teacher without doubts: an infinity apart from one, all weight on one word
    logits[:] = -math.inf
    logits[:, 3] = 2.0
    got = _run(ops, x, w, index, logits, g, 1.0)
    loss, lse = ops.cross_entropy(x, w, index[:, 3].contiguous())
    assert ((got["loss"] - loss).abs() <= 8 * mo.E * (lse.abs() + loss.abs())).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_views(ops, dtype):
    rows, width, vocab = 90, 96, 333
    x, w, index, logits, g = _inputs(rows, width, vocab, 8, dtype, 5)
    xw, ww = torch.zeros(rows, width + 8, dtype=dtype, device="cuda"), torch.zeros(vocab, width + 16, dtype=dtype, device="cuda")
    xw[:, 8:], ww[:, :width] = x, w
    got = _run(ops, xw[:, 8:], ww[:, :width], index, logits, g, 2.0)
    for name, t in _run(ops, x, w, index, logits, g, 2.0).items():
        assert torch.equal(t, got[name]), name


def test_offsets_beyond_32_bits(ops):
    """Rows of the projection and of the hidden states 2^20 elements apart."""
    rows, width, vocab, far = 2200, 64, 2300, 1 << 20
    x, w, index, logits, g = _inputs(rows, width, vocab, 8, torch.bfloat16, 5)
    base = torch.empty(vocab, far, dtype=torch.bfloat16, device="cuda")
    wf, xf = base[:, -width:], base[:rows, :width]
    wf.copy_(w)
    xf.copy_(x)
    loss, lse, picked = ops.distillation(xf, wf, index, logits, 1.0)
    want = _run(ops, x, w, index, logits, g, 1.0)
    assert torch.equal(loss, want["loss"]) and torch.equal(picked, want["picked"])
    dx, dw = ops.distillation_backward(g, xf, wf, index, logits, lse, picked, 1.0, dx=base[:rows, 1024:1024 + width],
                                       dw=base[:, 2048:2048 + width])
    assert torch.equal(dx, want["dx"]) and torch.equal(dw, want["dw"])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(100, 100), (300, 129), (700, 1000), (257, 5003), (300, 40003)])
def test_confident_rows(ops, dtype, rows, vocab):
    """Student and teacher both all but sure of the same word: 1 - p and 1 - q about 1e-4.  Entries of dl are sums and
    exponentials of their own, good to the logits' error (8e-5 of the entry in fp32, see the cross entropy's test of the
    kind); formed as p - q they would be 5e-3 off.  bf16 inputs: dl is rounded, by up to 2^-8 of itself, and so is the
    result: the favourite's entry weighs as much as all others of a row together, so the two roundings may add up."""
    gen = torch.Generator().manual_seed(vocab)
    width, lead = 64, math.log(vocab) + 9
    w = _normal(gen, vocab, width, dtype=dtype, sigma=0.02).double()
    index = torch.rand(rows, vocab, generator=gen).argsort(1)[:, :8] if vocab < 10000 else torch.randint(0, vocab // 8, (rows, 8), generator=gen) * 8 + torch.arange(8)
    x = w[index[:, 2]] * (lead / w[index[:, 2]].square().sum(1, keepdim=True)) + 0.3 * _normal(gen, rows, width).double()
    logits = _normal(gen, rows, 8)
    logits[:, 2] = 11.5
    x, w, index, logits = x.to(dtype).cuda(), w.to(dtype).cuda(), index.cuda(), logits.cuda()
    index[5] = -1
    g = torch.rand(rows, generator=gen).cuda() + 0.1
    got, want = _run(ops, x, w, index, logits, g, 1.0), mo.distillation(x, w, index, logits, 1.0, g)
    for name in ("dx", "dw"):
        off = float((got[name].double() - want[name][0]).norm() / want[name][0].norm())
        assert off < (2e-4 if dtype == torch.float32 else 2 * 2.0 ** -8 + 2e-4), (name, off)


def test_gradients_are_those_of_the_definition(ops):
    """Against central differences of the definition in 64 bits, along random directions (h = 1e-4: good to about 1e-7
    of the gradient's size, the fp32 gradients to about 1e-5 of it), through the class."""
    x, w, index, logits, g = _inputs(45, 64, 77, 9, torch.float32, 8)
    leaf = {"x": x, "w": w}
    dev = {n: t.clone().requires_grad_() for n, t in leaf.items()}
    loss = ops.Distillation.apply(dev["x"], dev["w"], index, logits, 2.0)
    (loss.double() * g.double()).sum().backward()
    mo.U.setdefault(torch.float64, 0.0)
    gen = torch.Generator().manual_seed(3)
    for name, t in leaf.items():
        way, h = _normal(gen, *t.shape, dtype=torch.float64).cuda(), 1e-4
        value = []
        for sign in (1, -1):
            at = dict(leaf)
            at[name] = t.double() + sign * h * way
            value.append(float((mo.distillation(at["x"].double(), at["w"].double(), index, logits, 2.0)["loss"][0] * g.double()).sum()))
        slope, grad = (value[0] - value[1]) / (2 * h), dev[name].grad.double()
        assert abs(slope - float((grad * way).sum())) < 1e-4 * float(grad.norm() * way.norm()), name


@pytest.mark.parametrize("weight", [1 + 2.0 ** -8, -3.5e-4, 1e-40, 2.4e38])
def test_a_weight_of_all_rows_is_not_rounded(ops, weight):
    """A student that knows nothing, a teacher sure of one word: every row's dl there is all but the weight itself.  The
    weights' rounding to bf16 (up to 2^-8) would scale the gradients.  The gradients' own rounding is not counted: it may
    scale them as well (a word of one row has dw = x (1 + 2^-8) where x has 8 digits: always rounded up, by up to 2^-9).
    What else is rounded, to 2^-8 of itself at most, is so independently: along the gradient of n normal numbers that comes
    to 2^-8 sqrt(3 / n) at most (rms), 5e-5 for dx, a twentieth of the 2^-10 allowed.  bf16 numbers are 2^-133 apart at
    the least, so dl of 1e-40 is off by half of that, 0.46 of itself."""
    rows, width, vocab = 300, 64, 40003
    gen = torch.Generator().manual_seed(7)
    x, w = _normal(gen, rows, width, dtype=torch.bfloat16, sigma=1e-2).cuda(), _normal(gen, vocab, width, dtype=torch.bfloat16).cuda()
    index, logits = torch.randint(0, vocab, (rows, 1), generator=gen).cuda(), torch.zeros(rows, 1, device="cuda")
    g = torch.full((rows,), weight, device="cuda")
    if abs(weight) > 1e-30:
        g[::3] *= 0.25                                   # as others have it but for a power of two
    got, want = _run(ops, x, w, index, logits, g, 1.0), mo.distillation(x, w, index, logits, 1.0, g)
    for name in ("dx", "dw"):
        fits, unit = want[name][0].abs() < 3e38, abs(weight)     # (2.4e38 w is beyond what there is where w is above 1.4)
        value, here = want[name][0][fits].to(torch.bfloat16).double(), got[name][fits].double()
        if not value.any():                              # dw of 1e-40 x with x below 0.4
            assert not here.any(), name
            continue
        scale = float((here / unit * (value / unit)).sum() / (value / unit).square().sum())
        assert abs(scale - 1) < 2.0 ** -10 + 2.0 ** -134 / unit, (name, scale)


def test_the_cross_entropy_keeps_its_results(ops):
    """Its products are those of the distillation; their factor of the exponents is its own."""
    gen = torch.Generator().manual_seed(3)
    x, w = _normal(gen, 300, 64).cuda(), _normal(gen, 1000, 64, sigma=0.2).cuda()
    target = torch.randint(0, 1000, (300,), generator=gen).cuda()
    loss, lse = ops.cross_entropy(x, w, target)
    taught = ops.distillation(x, w, target[:, None].contiguous(), torch.zeros(300, 1, device="cuda"), 1.0)
    assert torch.equal(taught[1], lse) and torch.allclose(taught[0], loss, rtol=0, atol=1e-6)


def test_refusals(ops):
    from test_gpu_model_paths import _refused
    x, w, index, logits, g = _inputs(10, 64, 50, 5, torch.bfloat16, 2)
    _refused(lambda: ops.distillation(x, w[:, :32], index, logits), "expected x")
    _refused(lambda: ops.distillation(x, w.float(), index, logits), "expected")
    _refused(lambda: ops.distillation(x, w, index.int(), logits), "index")
    _refused(lambda: ops.distillation(x, w, index[:9], logits), "index")
    _refused(lambda: ops.distillation(x, w, index.t().contiguous().t(), logits), "index")
    _refused(lambda: ops.distillation(x, w, index, logits.bfloat16()), "logits")
    _refused(lambda: ops.distillation(x, w, index, logits[:, :4]), "logits")
    _refused(lambda: ops.distillation(x, w, index, logits, 0.0), "eager_distillation")
    _refused(lambda: ops.distillation(x, w, index[:, :0], logits[:, :0]), "eager_distillation")
    loss, lse, picked = ops.distillation(x, w, index, logits)
    rest = index, logits, lse, picked
    _refused(lambda: ops.distillation_backward(g[:5], x, w, *rest), "dloss")
    _refused(lambda: ops.distillation_backward(g, x, w, index, logits, lse, picked[:, :2]), "picked")
    _refused(lambda: ops.distillation_backward(g, x, w, *rest, dw=w.t().contiguous().t()), "dw")
    _refused(lambda: ops.distillation_backward(g, x, w, *rest, want=(False, False)), "eager_distillation_backward")
