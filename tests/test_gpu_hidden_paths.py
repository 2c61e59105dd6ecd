"""Layer norm, rotation and distillation together as a step uses them: in graphs, on two streams, through both ways of
handing the arguments over, beside errors of other calls, captured backward passes."""
import pytest
import torch

from test_gpu_model_ops import _normal, _table

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
NAMES = ("layer_norm", "layer_norm_backward", "rotary_table", "rotary", "distillation")


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


def _state(dtype, seed, T=330):
    gen = torch.Generator().manual_seed(seed)
    s = {"x": _normal(gen, T, 256, dtype=dtype), "r": _normal(gen, T, 256, dtype=dtype), "dy": _normal(gen, T, 256, dtype=dtype),
         "ds": _normal(gen, T, 256, dtype=dtype), "w": _normal(gen, 256, dtype=dtype, mean=1.0, sigma=0.1),
         "b": _normal(gen, 256, dtype=dtype, sigma=0.1), "head": _normal(gen, 700, 256, dtype=dtype, sigma=0.1),
         "index": torch.randint(-20, 700, (T, 12), generator=gen), "logits": _normal(gen, T, 12, sigma=2.0), "g": _normal(gen, T),
         "pos": torch.randint(0, 90, (T,), generator=gen, dtype=torch.int32)}
    s["index"][: 3 + seed] = -1
    return {n: t.cuda() for n, t in s.items()}


def _step(ops, s):
    """What a step does with them: sum and norm, heads turned, loss, and back."""
    cos, sin = ops.rotary_table(90, 48, scaling="parts", factor=4.0, original=128.0)
    y, total, stats = ops.layer_norm(s["x"], s["w"], s["b"], residual=s["r"])
    heads = y.view(-1, 4, 64)
    q, k = ops.rotary(heads[:, :2], heads[:, 2:], cos, sin, s["pos"], True)
    loss, lse, picked = ops.distillation(y, s["head"], s["index"], s["logits"], 2.0)
    dx, dhead = ops.distillation_backward(s["g"], y, s["head"], s["index"], s["logits"], lse, picked, 2.0)
    dq, dk = ops.rotary_backward(q, k, cos, sin, s["pos"], True)
    back = ops.layer_norm_backward(s["dy"], total, s["w"], stats, s["ds"])
    return (cos, sin, y, total, stats, q, k, loss, lse, picked, dx, dhead, dq, dk, *back)


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_two_graphs_replayed_between_eager_work(ops, dtype):
    states = [_state(dtype, 0), _state(dtype, 0, T=90)]
    for s in states:
        _step(ops, s)
    torch.cuda.synchronize()
    graphs, captured = [], []
    for s in states:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            captured.append(_step(ops, s))
    for seed in range(1, 5):
        for s, T in zip(states, (330, 90)):
            for n, t in _state(dtype, seed, T).items():
                s[n].copy_(t)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for i, (s, got) in enumerate(zip(states, captured)):
            eager = _step(ops, s)
            torch.cuda.synchronize()
            for n, (a, b) in enumerate(zip(got, eager)):
                assert torch.equal(a, b), (seed, i, n)


@pytest.mark.parametrize("dtype", DTYPES)
def test_two_calls_at_once(ops, dtype):
    """On two streams, each with workspaces of its own."""
    states = [_state(dtype, 1), _state(dtype, 2)]
    want = [_step(ops, s) for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    got = [[], []]
    for _ in range(4):
        for i, (s, side) in enumerate(zip(states, streams)):
            with torch.cuda.stream(side):
                got[i].append(_step(ops, s))
    torch.cuda.synchronize()
    for runs, each in zip(got, want):
        for run in runs:
            for n, (a, b) in enumerate(zip(run, each)):
                assert torch.equal(a, b), n


@pytest.mark.parametrize("dtype", DTYPES)
def test_through_the_module_and_through_ctypes(ops, dtype, monkeypatch):
    from paper_1908_04207_amd import binding as eb
    s = _state(dtype, 3)
    _step(ops, s)                                        # from here on the current stream is known
    taken = []

    class Counting:
        def __getattr__(self, name):
            fn = getattr(real, name)

            def call(*args):
                result = fn(*args)
                if name in NAMES:
                    taken.append(result is not NotImplemented)
                return result
            return call

    real = eb._marshal
    monkeypatch.setattr(eb, "_marshal", Counting())
    through_module = _step(ops, s)
    assert taken == [True] * 7
    monkeypatch.setattr(eb, "_marshal", eb._CtypesOnly)
    for a, b in zip(through_module, _step(ops, s)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("through", ["module", "ctypes"])
def test_lone_rows_of_any_stride_and_arguments_left_out(ops, through, monkeypatch):
    from paper_1908_04207_amd import binding as eb
    s = _state(torch.float32, 4)
    if through == "ctypes":
        monkeypatch.setattr(eb, "_marshal", eb._CtypesOnly)
    wide = torch.cat([s["x"], s["r"][:, :3]], 1)                       # rows of 259 elements
    lone = wide[:1, :256]
    for r in (None, s["r"][0].expand(1, 256)):
        a, b = (ops.layer_norm(t, s["w"], residual=r) for t in (lone, lone.clone()))
        for u, v in zip(a[:1] + a[2:], b[:1] + b[2:]):
            assert torch.equal(u, v)
        c, d = (ops.layer_norm_backward(t, a[1], s["w"], a[2], want=(True, False)) for t in (lone, lone.clone()))
        assert torch.equal(c[0], d[0]) and torch.equal(c[1], d[1]) and c[2] is None
    one = s["index"][5:6, :1], s["logits"][5:6, :1]                    # a list of one entry out of a longer one
    loss, lse, picked = ops.distillation(lone, s["head"], *one, 1.0)
    for u, v in zip((loss, lse, picked), ops.distillation(lone.clone(), s["head"], one[0].clone(), one[1].clone(), 1)):
        assert torch.equal(u, v)
    # an int for a float, a table of ints
    for u, v in zip(ops.rotary_table(20, 16, 500), ops.rotary_table(20, 16, 500.0)):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", DTYPES)
def test_an_error_of_another_call_is_not_an_operator_s(ops, dtype):
    import ctypes
    from paper_1908_04207_amd import binding as eb
    s = _state(dtype, 5)
    _step(ops, s)
    torch.cuda.synchronize()
    hip = ctypes.CDLL(eb.LIB_PATH)                  # the runtime that the library is linked with
    left = hip.hipSetDevice(1 << 20)
    assert left != 0
    try:
        _step(ops, s)
    finally:
        assert hip.hipGetLastError() == left
        assert hip.hipGetLastError() == 0
    torch.cuda.synchronize()


def test_upstream_gradients_off_a_boundary_and_broadcast(ops):
    s = _state(torch.bfloat16, 6)
    x, w = s["x"].clone().requires_grad_(), s["w"].clone().requires_grad_()
    flat = torch.cat([s["dy"].flatten(), s["dy"][0, :1]])[1:].view(330, 256)       # contiguous, two bytes off
    y = ops.LayerNorm.apply(x, w, None, 1e-5)
    for up in (flat, s["dy"].t().contiguous().t(), s["dy"][:1].expand(330, 256)):
        for a, b in zip(torch.autograd.grad(y, (x, w), up, retain_graph=True),
                        torch.autograd.grad(y, (x, w), up.contiguous().clone(), retain_graph=True)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_captured_backward_pass(ops, dtype):
    """Gradients of a whole step through the classes, captured with leaves of their own and replayed with other inputs."""
    s = _state(dtype, 7)
    cos, sin = (t.cuda() for t in _table(90, 64))

    def step(s):
        leaves = [s[n].detach().requires_grad_() for n in ("x", "r", "w", "b", "head")]
        total, y = ops.AddLayerNorm.apply(*leaves[:4], 1e-5)
        h = y.view(-1, 4, 64)
        q, k = ops.Rotary.apply(h[:, :2], h[:, 2:], cos, sin, s["pos"], False)
        z = ops.LayerNorm.apply(torch.cat((q, k), 1).reshape(-1, 256) + total, leaves[2], None, 1e-5)
        loss = ops.Distillation.apply(z, leaves[4], s["index"], s["logits"], 2.0)
        return torch.autograd.grad(loss, leaves, s["g"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(s)
    for seed in (8, 9, 10):
        for n, t in _state(dtype, seed).items():
            s[n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, step(s)):
            assert torch.isfinite(a).all() and torch.equal(a, b)
        torch.cuda.synchronize()
