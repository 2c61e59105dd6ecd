"""Rotation by position and its tables through the library against their definitions in 64 bits."""
import math

import pytest
import torch

from oracle import model_oracle as mo
from test_gpu_model_ops import _check, _normal, _table

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


# ---------------------------------------------------------------------------------- tables

@pytest.mark.parametrize("rows,part,kw", [
    (1, 8, {}), (7, 16, {}), (1024, 64, {}), (300, 40, {}), (97, 128, dict(magnitude=1.3)), (33, 96, dict(base=500000.0)),
    (20, 8, dict(base=1.0)), (500, 64, dict(scaling="linear", factor=8.0)), (700, 64, dict(scaling="base", factor=4.0)),
    (900, 128, dict(scaling="parts", factor=16.0, original=256)), (300, 24, dict(scaling="parts", factor=2.0, original=512, low=0.0, high=4.0)),
    (131072, 64, dict(scaling="parts", factor=64.0, original=2048, magnitude=1.4)), (50, 32, dict(scaling="base", factor=1.0))])
def test_table(ops, rows, part, kw):
    """Half a rounding of the value; 2e-10 that the series leave out; the angle's own rounding in 64 bits, three times."""
    cos, sin = ops.rotary_table(rows, part, **kw)
    size = kw.get("magnitude", 1.0)
    f = mo.frequencies(part, kw.get("base", 10000.0), kw.get("scaling", "none"), kw.get("factor", 1.0), kw.get("original", 0),
                       kw.get("low", 1.0), kw.get("high", 32.0))
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * f
    for name, got, want in (("cos", cos, angle.cos() * size), ("sin", sin, angle.sin() * size)):
        _check(name, got, want, mo.E * want.abs() * 1.001 + size * (3e-10 + 3 * 2.0 ** -52 * angle))


def test_far_positions(ops):
    """The last of many rows, beyond 2^24: positions that fp32 does not hold."""
    rows = (1 << 24) + 1000
    cos, sin = ops.rotary_table(rows, 8)
    f = mo.frequencies(8, 10000.0)
    angle = torch.arange(rows - 1000, rows, dtype=torch.float64)[:, None] * f
    for got, want in ((cos, angle.cos()), (sin, angle.sin())):
        _check("far", got[-1000:], want, mo.E * want.abs() * 1.001 + 3e-10 + 3 * 2.0 ** -52 * angle)


def test_tables_into_given_buffers(ops):
    cos, sin = torch.full((2, 12, 32), 9.0, device="cuda")
    a, b = ops.rotary_table(10, 64, cos=cos[:10], sin=sin[:10])
    c, d = ops.rotary_table(10, 64)
    assert torch.equal(a, c) and torch.equal(b, d) and (cos[10:] == 9).all() and (sin[10:] == 9).all()
    assert ops.rotary_table(0, 64)[0].shape == (0, 32)


# ---------------------------------------------------------------------------------- heads

HEADS = [(1, 1, 1, 8, 8), (3, 2, 1, 16, 16), (37, 16, 4, 64, 64), (37, 16, 4, 64, 32), (130, 25, 5, 64, 24), (65, 6, 3, 32, 8),
         (70, 10, 2, 80, 80), (33, 4, 1, 96, 40), (50, 2, 2, 40, 40), (257, 8, 2, 128, 128), (20, 8, 2, 128, 120), (5, 130, 13, 24, 16),
         (3, 900, 300, 16, 8), (1000, 1, 1, 8, 8), (4, 5, 5, 56, 48)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,part", HEADS)
def test_rotary(ops, dtype, interleaved, T, Hq, Hk, D, part):
    gen = torch.Generator().manual_seed(T * 1000 + part)
    qkv = _normal(gen, T, (Hq + 2 * Hk) * D, dtype=dtype)
    cos, sin = _table(T + 3, part)
    pos = torch.randint(0, T + 3, (T,), generator=gen, dtype=torch.int32)
    dev = qkv.cuda()
    table = cos.cuda(), sin.cuda(), pos.cuda(), interleaved
    q, k = qkv[:, :Hq * D].view(T, Hq, D), qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
    qd, kd = dev[:, :Hq * D].view(T, Hq, D), dev[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
    got = ops.rotary(qd, kd, *table)
    back = ops.rotary_backward(qd, kd, *table)
    assert torch.equal(dev.cpu(), qkv)
    for x, y, d in ((q, got[0], back[0]), (k, got[1], back[1])):
        _check("turned", y, *mo.rotary(x, cos, sin, pos, interleaved))
        _check("turned back", d, *mo.rotary(x, cos, sin, pos, interleaved, back=True))
        assert torch.equal(y.cpu()[..., part:], x[..., part:]) and torch.equal(d.cpu()[..., part:], x[..., part:])
    # in place, both or one of them, values left alone; heads outermost
    ops.rotary(qd, kd, *table, q_out=qd, k_out=kd)
    assert torch.equal(qd, got[0]) and torch.equal(kd, got[1])
    assert torch.equal(dev.cpu()[:, (Hq + Hk) * D:], qkv[:, (Hq + Hk) * D:])
    qh, kh = (t.transpose(0, 1).contiguous().transpose(0, 1).cuda() for t in (q, k))
    yq, yk = torch.empty_like(qh), kh
    ops.rotary(qh, kh, *table, q_out=yq, k_out=yk)
    assert torch.equal(yq, got[0]) and torch.equal(yk, got[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_position_outside_the_table(ops, dtype, interleaved):
    gen = torch.Generator().manual_seed(3)
    T, D, part = 40, 64, 48
    q, k = _normal(gen, T, 3, D, dtype=dtype).cuda(), _normal(gen, T, 1, D, dtype=dtype).cuda()
    cos, sin = (t.cuda() for t in _table(10, part))
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 10
    ok = ops.rotary(q, k, cos, sin, pos, interleaved)
    pos[7], pos[21], pos[22] = 10, -1, 2 ** 31 - 1
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[[7, 21, 22]] = True
    for x, a, b in zip((q, k), ok, ops.rotary(q, k, cos, sin, pos, interleaved)):
        assert torch.isnan(b[bad][..., :part]).all() and torch.equal(b[bad][..., part:], x[bad][..., part:])
        assert torch.equal(a[~bad], b[~bad])


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_beyond_32_bits(ops, dtype):
    T, far, D = 2300, 1 << 20, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    base = torch.empty(T, far, dtype=dtype, device="cuda")
    near = [torch.randn(T, H, D, device="cuda", generator=gen).to(dtype) for H in (2, 1)]
    views = [base[:, -n * 1024:-n * 1024 + H * D].view(T, H, D) for n, H in ((1, 2), (2, 1), (3, 2), (4, 1))]
    for v, t in zip(views, near):
        v.copy_(t)
    cos, sin = ops.rotary_table(100, 32)
    pos = torch.arange(T, device="cuda").int() % 100
    got = ops.rotary(*views[:2], cos, sin, pos, True, q_out=views[2], k_out=views[3])
    for a, b in zip(got, ops.rotary(*near, cos, sin, pos, True)):
        assert torch.equal(a, b)


def test_tables_of_the_library_in_the_head_norms(ops):
    """A table of the library's is one that qk_norm_rope takes: gains of one on heads of norm one are a rotation."""
    gen = torch.Generator().manual_seed(2)
    T, D = 50, 64
    q, k = _normal(gen, T, 2, D).cuda(), _normal(gen, T, 1, D).cuda()
    q, k = (t / t.square().mean(-1, keepdim=True).sqrt() for t in (q, k))
    cos, sin = ops.rotary_table(T, D)
    pos, w = torch.arange(T, device="cuda").int(), torch.ones(D, device="cuda")
    for a, b in zip(ops.rotary(q, k, cos, sin, pos), ops.qk_norm_rope(q, k, w, w, cos, sin, pos, eps=0.0)):
        # the norm divides by a one that is a few roundings off
        assert float((a - b).abs().max()) < 64 * mo.E * float(a.abs().max())


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_through_the_class(ops, interleaved):
    """q and k used twice, a broadcast and a transposed gradient from above; the rotation keeps scalar products."""
    gen = torch.Generator().manual_seed(5)
    T, D, part = 30, 32, 24
    q, k = (_normal(gen, T, h, D).cuda().requires_grad_() for h in (4, 2))
    cos, sin = (t.cuda() for t in _table(T, part))
    pos = torch.arange(T, device="cuda").int()
    yq, yk = ops.Rotary.apply(q, k, cos, sin, pos, interleaved)
    up = _normal(gen, D, T, 4).cuda().permute(1, 2, 0)
    torch.autograd.backward((yq, yk.sum()), (up, None))
    want = ops.rotary_backward(up.contiguous(), torch.ones_like(k), cos, sin, pos, interleaved)
    assert torch.equal(q.grad, want[0]) and torch.equal(k.grad, want[1])
    dot = lambda a, b: float((a.double() * b.double()).sum())              # noqa: E731
    off = abs(dot(yq.detach(), up) - dot(q.detach(), q.grad))
    assert off < 1e-6 * float(up.norm() * q.detach().norm()), off


def test_refusals(ops):
    from test_gpu_model_paths import _refused
    gen = torch.Generator().manual_seed(5)
    T, D = 8, 64
    q, k = _normal(gen, T, 4, D).cuda(), _normal(gen, T, 2, D).cuda()
    cos, sin = (t.cuda() for t in _table(T, D))
    pos = torch.arange(T, device="cuda").int()
    _refused(lambda: ops.rotary(q, k.bfloat16(), cos, sin, pos), "expected")
    _refused(lambda: ops.rotary(q, k[:7], cos, sin, pos), "expected")
    _refused(lambda: ops.rotary(q[:, :3], k, cos, sin, pos), "eager_rotary")
    _refused(lambda: ops.rotary(q, k, cos, sin[:5], pos), "sin")
    _refused(lambda: ops.rotary(q, k, cos.double(), sin, pos), "cos")
    _refused(lambda: ops.rotary(q, k, cos, sin, pos.long()), "positions")
    _refused(lambda: ops.rotary(q, k, cos[:, :30].contiguous(), sin[:, :30].contiguous(), pos), "eager_rotary")    # part 60
    _refused(lambda: ops.rotary(q[..., :56], k[..., :56], cos, sin, pos), "eager_rotary")                # more than a head
    _refused(lambda: ops.rotary(q, k, cos, sin, pos, q_out=k), "q_out")
    _refused(lambda: ops.rotary(q[:, :1].expand(-1, 4, -1), k, cos, sin, pos), "eager_rotary")           # a broadcast view
    _refused(lambda: ops.rotary_backward(q, k, cos, sin, pos, dk=q), "dk")
    _refused(lambda: ops.rotary_table(10, 60), "eager_rotary_table")
    _refused(lambda: ops.rotary_table(10, 64, base=0.0), "eager_rotary_table")
    _refused(lambda: ops.rotary_table(10, 64, scaling="parts", factor=2.0), "eager_rotary_table")        # no original context
    assert math.isfinite(float(ops.rotary(q, k, cos, sin, pos)[0].sum()))
