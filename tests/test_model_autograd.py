"""The model operators' classes for torch's autograd without a GPU: the calls they make are replaced by plain
torch, so that what is tested is what the classes add to them."""
import pytest
import torch

from paper_1908_04207_amd import binding as eb
from paper_1908_04207_amd import model_ops as ops

T, Hq, Hk, D, V = 5, 4, 2, 8, 7


def _softmax(q, k, v):
    group = q.shape[1] // k.shape[1]
    s = torch.einsum("thd,shd->hts", q, k.repeat_interleave(group, 1))
    p = torch.softmax(s.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), -1e9), -1)
    return torch.einsum("hts,shd->thd", p, v.repeat_interleave(group, 1))


def _gradients(fn, inputs, upstream):
    leaves = [t.detach().requires_grad_() for t in inputs]
    with torch.enable_grad():
        grads = torch.autograd.grad(fn(*leaves), leaves, upstream)
    return tuple(g.detach() for g in grads)


@pytest.fixture
def plain(monkeypatch):
    """The six calls in plain torch on the CPU, without a graph, as the library's have none."""
    def norm(q, k, wq, wk, cos, sin, positions, eps=1e-6, **kw):
        with torch.no_grad():
            return q * wq, k * wk

    def norm_backward(dq_out, dk_out, q, k, wq, wk, *rest, **kw):
        return _gradients(lambda *a: (a[0] * a[2], a[1] * a[3]), (q, k, wq, wk), (dq_out, dk_out))

    def attention(q, k, v, cu, scale=None, **kw):
        with torch.no_grad():
            return _softmax(q, k, v), torch.zeros(Hq, T)

    def attention_backward(dout, q, k, v, out, lse, cu, scale=None, **kw):
        return _gradients(_softmax, (q, k, v), dout)

    def losses(x, w, target):
        return torch.logsumexp(x @ w.t(), 1) - (x @ w.t())[torch.arange(T), target]

    def loss(x, w, target):
        with torch.no_grad():
            return losses(x, w, target), torch.zeros(T)

    def loss_backward(dloss, x, w, target, lse, dx=None, dw=None, want=(True, True), **kw):
        grads = _gradients(lambda x, w: losses(x, w, target), (x, w), dloss)
        return tuple(g if wanted else None for g, wanted in zip(grads, want))

    for name, fn in (("qk_norm_rope", norm), ("qk_norm_rope_backward", norm_backward), ("attention", attention),
                     ("attention_backward", attention_backward), ("cross_entropy", loss),
                     ("cross_entropy_backward", loss_backward)):
        monkeypatch.setattr(ops, name, fn)


def _cases():
    gen = torch.Generator().manual_seed(0)
    draw = lambda *s: torch.randn(*s, generator=gen).requires_grad_()      # noqa: E731
    q, k, v, wq, wk, x, w = (draw(T, Hq, D), draw(T, Hk, D), draw(T, Hk, D), draw(D), draw(D), draw(T, D), draw(V, D))
    cu, table, pos = torch.tensor([0, T], dtype=torch.int32), torch.ones(T, D // 2), torch.arange(T, dtype=torch.int32)
    target = torch.arange(T) % V
    return {"norm": ((q, k, wq, wk), lambda: ops.QKNormRope.apply(q, k, wq, wk, table, table, pos, 1e-6)[0]),
            "attention": ((q, k, v), lambda: ops.Attention.apply(q, k, v, cu, None)),
            "loss": ((x, w), lambda: ops.CrossEntropy.apply(x, w, target)),
            "loss of fixed weights": ((x,), lambda: ops.CrossEntropy.apply(x, w.detach(), target))}


@pytest.mark.parametrize("name", _cases())
def test_first_gradients_with_and_without_a_graph(plain, name):
    leaves, call = _cases()[name]
    once = torch.autograd.grad(call().square().sum(), leaves, allow_unused=True)
    again = torch.autograd.grad(call().square().sum(), leaves, create_graph=True, allow_unused=True)
    for a, b in zip(once, again):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b.detach()))
    assert all(g is None or not g.requires_grad for g in once)


@pytest.mark.parametrize("linear", [False, True])
@pytest.mark.parametrize("name", _cases())
def test_second_derivatives_are_refused(plain, name, linear):
    """A penalty on the gradients beside the loss itself: their own derivatives are not formed, so they may not
    be left out in silence either - whether or not the upstream gradient (here of a sum: ones, and of a sum of
    squares) depends on anything."""
    leaves, call = _cases()[name]
    y = call()
    value = y.sum() if linear else y.square().sum()
    grads = torch.autograd.grad(value, leaves, create_graph=True, allow_unused=True)
    penalty = sum(g.square().sum() for g in grads if g is not None)
    with pytest.raises(eb.EagerError, match="second derivatives"):
        (value + penalty).backward()


def _views():
    """Upstream gradients [T, heads, D] as torch may hand them over, and whether the kernels take them as they are."""
    def contiguous(h):
        return torch.randn(T, h, D)

    def part_of_a_row(h):
        return torch.randn(T, h * D + 24)[:, 8:8 + h * D].view(T, h, D)

    def heads_first(h):
        return torch.randn(h, T, D).transpose(0, 1)

    def off_a_boundary(h):
        return torch.randn(T * h * D + 1)[1:].view(T, h, D)

    def odd_rows(h):
        return torch.randn(T, h * D + 1)[:, :h * D].view(T, h, D)

    def broadcast(h):
        return torch.randn(1, 1, D).expand(T, h, D)

    def one_number(h):
        return torch.ones(()).expand(T, h, D)

    def dims_first(h):
        return torch.randn(T, D, h).transpose(1, 2)

    return [(contiguous, True), (part_of_a_row, True), (heads_first, True), (off_a_boundary, False), (odd_rows, False),
            (broadcast, False), (one_number, False), (dims_first, False)]


@pytest.mark.parametrize("view,taken", _views(), ids=lambda x: getattr(x, "__name__", None))
@pytest.mark.parametrize("name", ["attention", "norm"])
def test_upstream_gradients_reach_the_kernels_in_a_form_they_take(plain, monkeypatch, name, view, taken):
    handed = []
    for fn in ("attention_backward", "qk_norm_rope_backward"):
        call = getattr(ops, fn)

        def spy(*a, call=call, n=1 if fn[0] == "a" else 2, **kw):
            handed.extend(a[:n])
            return call(*a, **kw)
        monkeypatch.setattr(ops, fn, spy)
    if name == "norm":
        q, k, w = (torch.randn(*s).requires_grad_() for s in ((T, Hq, D), (T, Hk, D), (D,)))
        table, pos = torch.ones(T, D // 2), torch.arange(T, dtype=torch.int32)
        outs, leaves = ops.QKNormRope.apply(q, k, w, w, table, table, pos, 1e-6), (q, k)
        ups = [view(Hq), view(Hk)]
    else:
        q, k, v = (torch.randn(T, h, D).requires_grad_() for h in (Hq, Hk, Hk))
        outs, leaves = (ops.Attention.apply(q, k, v, torch.tensor([0, T], dtype=torch.int32), None),), (q, k, v)
        ups = [view(Hq)]
    torch.autograd.grad(outs, leaves, ups)
    assert len(handed) == len(ups)
    for up, got in zip(ups, handed):
        assert torch.equal(up, got)
        assert got.data_ptr() % 16 == 0 and got.stride(2) == 1 and all(s % 4 == 0 and s >= D for s in got.stride()[:2])
        assert (got.data_ptr() == up.data_ptr()) == taken
