"""Layer norm, rotation and distillation without a GPU: the header from plain C, launch rules, what is refused before
any launch, and what the classes for torch's autograd add to the calls."""
import itertools
import math
import os
import subprocess

import pytest
import torch

from paper_1908_04207_amd import binding as eb
from paper_1908_04207_amd import model_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B, C = 0x10000, 0x20000, 0x30000          # aligned addresses that are never read
NAN, INF = float("nan"), float("inf")


def _refused(call, what=""):
    with pytest.raises(eb.EagerError) as e:
        call()
    assert e.value.status == eb.EINVAL and what in str(e.value), str(e.value)


def test_header_is_plain_c(tmp_path):
    exe = tmp_path / "hidden_header"
    lib_dir = os.path.dirname(eb.LIB_PATH)
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                           os.path.join(ROOT, "tests", "c", "hidden_header_is_plain_c.c"), "-o", str(exe), "-L", lib_dir,
                           "-leager", "-Wl,-rpath," + lib_dir])
    assert subprocess.run([str(exe)]).returncode == 0


def test_rules_on_the_cpu(tmp_path):
    exe = tmp_path / "norm_rules"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-static-libasan", "-Wall", "-Wextra", "-Werror",
                           os.path.join(ROOT, "tests", "c", "norm_rules_host.cpp"), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout[-500:], r.stderr[-2000:])


def test_what_the_calls_hand_over(tmp_path):
    """eager_model_api.cpp without the kernels, under both sanitizers: arguments of every launch, angles in long double."""
    exe = tmp_path / "hidden_api"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-static-libasan", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-isystem", "/opt/rocm/include",
                           os.path.join(ROOT, "tests", "c", "hidden_api_host.cpp"),
                           os.path.join(ROOT, "paper_1908_04207_amd", "csrc", "eager_model_api.cpp"), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout[-500:], r.stderr[-2000:])


def _rows(data=A, stride=256):
    return eb.Rows(data, stride)


VIEWS = [None, dict(data=None), dict(data=A + 8), dict(stride=0), dict(stride=248), dict(stride=258), dict(stride=-256),
         dict(stride=2 ** 22)]


@pytest.mark.parametrize("dtype", [eb.F32, eb.BF16])
def test_layer_norm_refusals(dtype):
    def forward(dtype=dtype, count=5, width=256, x=_rows(), residual=_rows(), w=A, b=A, eps=1e-5, sum=_rows(B), y=_rows(C), stats=A):
        eb.eager_layer_norm(dtype, count, width, x, residual, w, b, eps, sum, y, stats, stream=0)

    def backward(dtype=dtype, count=5, width=256, dy=_rows(), ds=_rows(), s=_rows(), w=A, stats=A, dx=_rows(), dw=A, db=A,
                 workspace=A, workspace_bytes=1 << 30):
        eb.eager_layer_norm_backward(dtype, count, width, dy, ds, s, w, stats, dx, dw, db, workspace, workspace_bytes, stream=0)

    for call in (forward, backward):
        _refused(lambda: call(dtype=2))
        for bad in (dict(count=-1), dict(count=2 ** 31 - 2 ** 15), dict(width=0), dict(width=-8), dict(width=252), dict(width=4),
                    dict(width=16392), dict(w=None), dict(w=A + 8), dict(stats=None), dict(stats=A + 2)):
            _refused(lambda: call(**bad))
    for eps in (-1e-6, NAN, INF):
        _refused(lambda: forward(eps=eps))
    _refused(lambda: forward(b=A + 2))
    _refused(lambda: forward(sum=None))                  # a residual whose sum goes nowhere
    _refused(lambda: forward(residual=None))             # a sum without a residual
    _refused(lambda: forward(y=_rows(B)))                # the sum and its norm in one place
    for bad in (dict(sum=_rows(A, 264)), dict(y=_rows(A, 264)), dict(residual=_rows(C, 264))):       # in an input's place, otherwise laid out
        _refused(lambda: forward(**bad))
    for bad in (dict(dy=_rows(B), dx=_rows(B, 264)), dict(ds=_rows(C), dx=_rows(C, 512))):
        _refused(lambda: backward(**bad))
    for name, bad in itertools.product(("x", "residual", "sum", "y"), VIEWS):
        _refused(lambda: forward(**{name: bad and _rows(**bad)}))
    for name, bad in itertools.product(("dy", "s", "dx"), VIEWS):
        _refused(lambda: backward(**{name: bad and _rows(**bad)}))
    for bad in VIEWS[1:]:
        _refused(lambda: backward(ds=_rows(**bad)))
    need = eb.eager_layer_norm_workspace_bytes(dtype, 500, 256)
    assert need > 0 and eb.eager_layer_norm_workspace_bytes(dtype, 5, 256) == 0
    for bad in (dict(dw=A + 2), dict(db=A + 2), dict(workspace=None), dict(workspace=A + 8), dict(workspace_bytes=need - 1)):
        _refused(lambda: backward(count=500, **bad))
    _refused(lambda: backward(workspace_bytes=-1))
    none = _rows(None)
    forward(count=0, x=none, residual=none, sum=none, y=none, stats=None)
    for bad in ((3, 5, 256), (dtype, -1, 256), (dtype, 5, 12)):
        _refused(lambda: eb.eager_layer_norm_workspace_bytes(*bad))


def test_table_refusals():
    def call(cos=A, sin=A, **kw):
        v = dict(positions=10, part=64, scaling=eb.ANGLES_PARTS, base=1e4, factor=4.0, original=2048.0, low=1.0, high=32.0, magnitude=1.0)
        eb.eager_rotary_table(eb.Angles(**{**v, **kw}), cos, sin, stream=0)

    for bad in (dict(positions=-1), dict(positions=2 ** 31), dict(part=0), dict(part=4), dict(part=12), dict(part=136), dict(scaling=-1),
                dict(scaling=4), dict(base=0.5), dict(base=NAN), dict(base=INF), dict(factor=0.5), dict(factor=NAN), dict(factor=INF),
                dict(original=0.0), dict(original=NAN), dict(original=INF), dict(low=-1.0), dict(low=NAN), dict(high=1.0), dict(high=INF),
                dict(high=NAN), dict(magnitude=INF), dict(magnitude=NAN), dict(cos=None), dict(sin=A + 4)):
        _refused(lambda: call(**bad))
    _refused(lambda: eb.eager_rotary_table(None, A, A, stream=0))
    # what a scaling does not use is not looked at; a table of no positions is none
    for scaling in (eb.ANGLES_PLAIN, eb.ANGLES_LINEAR, eb.ANGLES_BASE):
        call(positions=0, scaling=scaling, original=NAN, low=5.0, high=1.0, cos=None, sin=None)
    call(positions=0, scaling=eb.ANGLES_PLAIN, factor=0.0)
    _refused(lambda: ops.rotary_table(4, 64, scaling="other"), "scaling")
    _refused(lambda: ops.rotary_table(-1, 64), "positions")
    _refused(lambda: ops.rotary_table(4, 64, cos=torch.zeros(4, 32), sin=torch.zeros(4, 32)), "GPU")
    _refused(lambda: ops.rotary_table(4, 64, cos=torch.zeros(4, 16), sin=torch.zeros(4, 32)), "cos")


@pytest.mark.parametrize("dtype", [eb.F32, eb.BF16])
def test_rotary_refusals(dtype):
    def shape(**kw):
        return eb.Packed(**{**dict(tokens=10, q_heads=4, kv_heads=2, head_dim=64, sequences=0, cu_seqlens=None), **kw})

    def heads(**kw):
        return eb.Heads(**{**dict(data=A, row_stride=256, head_stride=64), **kw})

    def rot(**kw):
        return eb.Rotation(**{**dict(cos_table=A, sin_table=A, positions=A, table_rows=8), **kw})

    for entry in (eb.eager_rotary, eb.eager_rotary_backward):
        def call(dtype=dtype, shape=shape(), q=heads(), k=heads(), rotation=rot(), part=32, layout=0, q_out=heads(), k_out=heads()):
            entry(dtype, shape, q, k, rotation, part, layout, q_out, k_out, stream=0)

        _refused(lambda: call(dtype=9))
        _refused(lambda: call(shape=None))
        for bad in (dict(tokens=-1), dict(tokens=2 ** 31), dict(q_heads=0), dict(q_heads=3), dict(head_dim=60), dict(head_dim=136)):
            _refused(lambda: call(shape=shape(**bad)))
        for bad in (None, rot(cos_table=None), rot(sin_table=A + 4), rot(positions=None), rot(positions=A + 2), rot(table_rows=0)):
            _refused(lambda: call(rotation=bad))
        for part in (0, -8, 4, 12, 72):
            _refused(lambda: call(part=part))
        for layout in (-1, 2):
            _refused(lambda: call(layout=layout))
        views = [None, dict(data=None), dict(data=A + 8), dict(row_stride=0), dict(row_stride=261), dict(head_stride=0),
                 dict(head_stride=66), dict(row_stride=2 ** 22)]
        for name, bad in itertools.product(("q", "k", "q_out", "k_out"), views):
            _refused(lambda: call(**{name: bad and heads(**bad)}))
        for bad in (dict(row_stride=512), dict(head_stride=128, row_stride=512)):
            _refused(lambda: call(q_out=heads(**bad)))
            _refused(lambda: call(k_out=heads(**bad)))
        none = heads(data=None)
        call(shape=shape(tokens=0), q=none, k=none, q_out=none, k_out=none, rotation=rot(positions=None))


@pytest.mark.parametrize("dtype", [eb.F32, eb.BF16])
def test_distillation_refusals(dtype):
    def shape(**kw):
        return eb.Projection(**{**dict(rows=4, width=64, vocab=100, x_stride=64, w_stride=64), **kw})

    def teacher(**kw):
        return eb.Teacher(**{**dict(index=A, logits=A, entries=8, temperature=2.0), **kw})

    def forward(dtype=dtype, shape=shape(), x=A, w=A, teacher=teacher(), loss=A, lse=A, picked=A, workspace=A, workspace_bytes=1 << 30):
        eb.eager_distillation(dtype, shape, x, w, teacher, loss, lse, picked, workspace, workspace_bytes, stream=0)

    def backward(dtype=dtype, shape=shape(), x=A, w=A, teacher=teacher(), lse=A, picked=A, dloss=A, dx=A, dw=A, workspace=A,
                 workspace_bytes=1 << 40):
        eb.eager_distillation_backward(dtype, shape, x, w, teacher, lse, picked, dloss, dx, dw, workspace, workspace_bytes, stream=0)

    for call, backward_too in ((forward, False), (backward, True)):
        _refused(lambda: call(dtype=7))
        _refused(lambda: call(shape=None))
        _refused(lambda: call(teacher=None))
        for bad in (dict(rows=-1), dict(rows=2 ** 25 + 1), dict(width=0), dict(width=60), dict(vocab=0), dict(x_stride=56),
                    dict(w_stride=66), dict(w_stride=2 ** 22), dict(x_stride=0)):
            _refused(lambda: call(shape=shape(**bad)))
        for bad in (dict(index=None), dict(index=A + 4), dict(logits=None), dict(logits=A + 2), dict(entries=0), dict(entries=-1),
                    dict(entries=257), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF),
                    dict(temperature=2.0 ** -21), dict(temperature=2.0 ** 21)):
            _refused(lambda: call(teacher=teacher(**bad)))
        for name in ("x", "w", "lse", "picked", "workspace"):
            _refused(lambda: call(**{name: None}))
            _refused(lambda: call(**{name: A + 2}))
        need = eb.eager_distillation_workspace_bytes(dtype, shape(), 8, backward_too)
        _refused(lambda: call(workspace_bytes=need - 1))
    _refused(lambda: forward(loss=None))
    _refused(lambda: backward(dloss=None))
    _refused(lambda: backward(dx=None, dw=None))
    _refused(lambda: backward(dx=A + 8))
    _refused(lambda: backward(dw=A + 8))
    forward(shape=shape(rows=0), x=None, teacher=teacher(index=None, logits=None), loss=None, lse=None, picked=None)
    for bad in ((shape(rows=2 ** 25 + 1), 8), (shape(), 0), (shape(), 257), (None, 8)):
        _refused(lambda: eb.eager_distillation_workspace_bytes(dtype, *bad, False))


def test_tensors_off_the_gpu_are_refused():
    x, w = torch.zeros(3, 64), torch.ones(64)
    _refused(lambda: ops.layer_norm(x, w, w), "GPU")
    _refused(lambda: ops.layer_norm(x.double(), w.double()), "unsupported")
    _refused(lambda: ops.layer_norm(x[0], w), "rows")
    _refused(lambda: ops.layer_norm_backward(x, x, w, torch.zeros(2, 3)), "GPU")
    q, table, pos = torch.zeros(3, 2, 64), torch.zeros(4, 32), torch.zeros(3, dtype=torch.int32)
    _refused(lambda: ops.rotary(q, q, table, table, pos), "GPU")
    _refused(lambda: ops.rotary_backward(q, q, table, table, pos), "GPU")
    index = torch.zeros(3, 2, dtype=torch.int64)
    _refused(lambda: ops.distillation(x, torch.zeros(5, 64), index, torch.zeros(3, 2)), "GPU")


def test_the_stride_of_a_lone_row_counts_nothing():
    for t in (torch.zeros(64).expand(1, 64), torch.zeros(1, 3 << 21)[:, :64], torch.zeros(5, 67)[:1, :64]):
        assert eb.rows(t).stride == 64
    assert eb.rows(torch.zeros(5, 67)[:, :64]).stride == 67                      # refused later
    _refused(lambda: eb.rows(torch.zeros(64, 5).t()))


# ------------------------------------------------------------------------------ autograd

@pytest.fixture
def plain(monkeypatch):
    """The calls in plain torch on the CPU, without a graph, as the library's have none."""
    def gradients(fn, inputs, upstream):
        leaves = [t.detach().requires_grad_() for t in inputs]
        with torch.enable_grad():
            return tuple(g.detach() for g in torch.autograd.grad(fn(*leaves), leaves, upstream))

    def norm_of(s, w, b):
        c = s - s.mean(1, keepdim=True)
        y = c / (c.square().mean(1, keepdim=True) + 0.1).sqrt() * w
        return y if b is None else y + b

    def layer_norm(x, w, b=None, eps=0.1, residual=None, **_):
        with torch.no_grad():
            s = x if residual is None else x + residual
            return norm_of(s, w, b), s, torch.zeros(2, x.shape[0])

    def layer_norm_backward(dy, s, w, stats, ds=None, want=(True, True), **_):
        dx, dw = gradients(lambda s, w: norm_of(s, w, None), (s, w), dy)
        return dx if ds is None else dx + ds, dw if want[0] else None, dy.sum(0) if want[1] else None

    def turn(q, k, c, s, sign):
        def one(x):
            a, b = x.chunk(2, -1)
            return torch.cat((a * c - sign * b * s, b * c + sign * a * s), -1)
        return one(q), one(k)

    def rotary(q, k, c, s, positions, interleaved=False, **_):
        with torch.no_grad():
            return turn(q, k, c, s, 1)

    def rotary_backward(dq, dk, c, s, positions, interleaved=False, **_):
        return turn(dq, dk, c, s, -1)

    def divergence(x, w, index, logits, tau):
        q = torch.softmax(logits / tau, 1)
        return (q * (q.log() - torch.log_softmax(x @ w.t() / tau, 1).gather(1, index))).sum(1)

    def distillation(x, w, index, logits, temperature=1.0):
        with torch.no_grad():
            return divergence(x, w, index, logits, temperature), torch.zeros(len(x)), torch.zeros(index.shape)

    def distillation_backward(dloss, x, w, index, logits, lse, picked, temperature=1.0, want=(True, True), **_):
        grads = gradients(lambda x, w: divergence(x, w, index, logits, temperature), (x, w), dloss)
        return tuple(g if wanted else None for g, wanted in zip(grads, want))

    for fn in (layer_norm, layer_norm_backward, rotary, rotary_backward, distillation, distillation_backward):
        monkeypatch.setattr(ops, fn.__name__, fn)


def _cases():
    gen = torch.Generator().manual_seed(0)
    draw = lambda *s: torch.randn(*s, generator=gen).requires_grad_()      # noqa: E731
    x, r, w, b, head, q, k = draw(5, 8), draw(5, 8), draw(8), draw(8), draw(7, 8), draw(5, 4, 8), draw(5, 2, 8)
    angle, pos = torch.randn(4, generator=gen), torch.arange(5, dtype=torch.int32)
    index, logits = torch.arange(15).view(5, 3) % 7, torch.randn(5, 3, generator=gen)
    both = lambda t: t[0].square().sum() + t[1].sum()                      # noqa: E731
    return {"norm": ((x, w, b), lambda: ops.LayerNorm.apply(x, w, b, 0.1)),
            "norm without a bias": ((x, w), lambda: ops.LayerNorm.apply(x, w, None, 0.1)),
            "norm of a fixed gain": ((x, b), lambda: ops.LayerNorm.apply(x, w.detach(), b, 0.1)),
            "sum and norm": ((x, r, w, b), lambda: both(ops.AddLayerNorm.apply(x, r, w, b, 0.1))),
            "norm of a sum": ((x, r, w, b), lambda: ops.AddLayerNorm.apply(x, r, w, b, 0.1)[1]),
            "sum alone": ((x, r), lambda: ops.AddLayerNorm.apply(x, r, w, b, 0.1)[0]),
            "rotation": ((q, k), lambda: both(ops.Rotary.apply(q, k, angle.cos(), angle.sin(), pos, False))),
            "teacher": ((x, head), lambda: ops.Distillation.apply(x, head, index, logits, 2.0)),
            "teacher, fixed weights": ((x,), lambda: ops.Distillation.apply(x, head.detach(), index, logits, 2.0))}


@pytest.mark.parametrize("name", _cases())
def test_gradients_through_the_classes(plain, name):
    """Against central differences of the calls: h = 1e-2 in fp32 is good to about 1e-3."""
    leaves, call = _cases()[name]
    grads = torch.autograd.grad(call().square().sum(), leaves)
    again = torch.autograd.grad(call().square().sum(), leaves, create_graph=True)
    gen = torch.Generator().manual_seed(1)
    for leaf, grad, other in zip(leaves, grads, again):
        assert torch.equal(grad, other.detach()) and not grad.requires_grad
        way, h, at = torch.randn(leaf.shape, generator=gen), 1e-2, leaf.detach().clone()
        with torch.no_grad():
            leaf.copy_(at + h * way)
            up = call().double().square().sum()
            leaf.copy_(at - h * way)
            down = call().double().square().sum()
            leaf.copy_(at)
        slope = float((up - down) / (2 * h))
        assert abs(slope - float((grad * way).sum())) < 1e-2 * (1 + float(grad.norm() * way.norm())), name


@pytest.mark.parametrize("name", [n for n in _cases() if n != "sum alone"])
def test_second_derivatives_are_refused(plain, name):
    leaves, call = _cases()[name]
    grads = torch.autograd.grad(call().square().sum(), leaves, create_graph=True)
    with pytest.raises(eb.EagerError, match="second derivatives"):
        sum(g.square().sum() for g in grads).backward()


def test_gradients_of_x_and_residual_are_tensors_of_their_own(plain):
    x, r, w = torch.randn(5, 8).requires_grad_(), torch.randn(5, 8).requires_grad_(), torch.ones(8)
    s, y = ops.AddLayerNorm.apply(x, r, w, None, 0.1)
    (s.sum() + y.square().sum()).backward()
    assert torch.equal(x.grad, r.grad) and x.grad.data_ptr() != r.grad.data_ptr()


def test_what_the_angles_are():
    """The oracle's frequencies in closed form: the slowest pair of a stretched base is squeezed by the factor, the
    fastest kept; by parts both ends are what they should be."""
    from oracle import model_oracle as mo
    plain, n = mo.frequencies(64, 1e4), 64
    assert float(plain[0]) == 1.0 and abs(float(plain[-1]) - 1e4 ** (-62 / 64)) < 1e-15
    stretched = mo.frequencies(n, 1e4, "base", 8.0)
    assert float(stretched[0]) == 1.0 and abs(float(stretched[-1] / plain[-1]) - 1 / 8) < 1e-12
    parts = mo.frequencies(n, 1e4, "parts", 8.0, 2048)
    turns = 2048 * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32])
    assert torch.allclose(parts[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15, atol=0)
    assert (parts.diff() < 0).all()
