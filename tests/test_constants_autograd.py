"""Inputs of the operators' classes that have no gradient, where a graph asks for one: the calls are replaced by plain
torch, so that what is tested is what the classes say."""
import pytest
import torch

from paper_1908_04207_amd import binding as eb
from paper_1908_04207_amd import model_ops as ops
from test_hidden_host import plain                       # noqa: F401  (a fixture)


def _student():
    gen = torch.Generator().manual_seed(0)
    x, w = torch.randn(5, 8, generator=gen).requires_grad_(), torch.randn(7, 8, generator=gen).requires_grad_()
    return x, w, torch.arange(15).view(5, 3) % 7, torch.randn(5, 3, generator=gen)


@pytest.mark.parametrize("fixed", [(), ("x",), ("x", "w")])
def test_a_teacher_that_is_trained_along_is_refused(plain, fixed):                  # noqa: F811
    """The loss depends on the teacher's logits too; without a word their part of the gradient would be missing."""
    x, w, index, logits = _student()
    x, w = x.detach() if "x" in fixed else x, w.detach() if "w" in fixed else w
    loss = ops.Distillation.apply(x, w, index, logits.requires_grad_(), 2.0)
    with pytest.raises(eb.EagerError, match="teacher's logits") as e:
        loss.sum().backward()
    assert e.value.status == eb.EINVAL and x.grad is None and w.grad is None and logits.grad is None


def test_a_teacher_out_of_the_graph(plain):                                         # noqa: F811
    """Detached, or made without one, as Teacher's lists are."""
    x, w, index, logits = _student()
    ops.Distillation.apply(x, w, index, (logits.requires_grad_() * 2).detach(), 2.0).sum().backward()
    assert x.grad.any() and w.grad.any() and logits.grad is None
    with torch.no_grad():
        loss = ops.Distillation.apply(x, w, index, logits, 2.0)
    assert not loss.requires_grad


def _heads():
    gen = torch.Generator().manual_seed(1)
    q, k = torch.randn(5, 4, 8, generator=gen).requires_grad_(), torch.randn(5, 2, 8, generator=gen).requires_grad_()
    angle = torch.randn(4, generator=gen)
    return q, k, angle.cos(), angle.sin(), torch.arange(5, dtype=torch.int32)


@pytest.mark.parametrize("which", [(2,), (3,), (2, 3)])
@pytest.mark.parametrize("fixed", [False, True])
def test_tables_that_are_trained_along_are_refused(plain, which, fixed):            # noqa: F811
    args = list(_heads())
    if fixed:
        args[:2] = args[0].detach(), args[1].detach()
    for n in which:
        args[n].requires_grad_()
    q, k = ops.Rotary.apply(*args, False)
    with pytest.raises(eb.EagerError, match="tables") as e:
        (q.sum() + k.sum()).backward()
    assert e.value.status == eb.EINVAL and args[0].grad is None and args[2].grad is None


def test_tables_out_of_the_graph(plain):                                            # noqa: F811
    q, k, cos, sin, pos = _heads()
    sum(t.sum() for t in ops.Rotary.apply(q, k, (cos.requires_grad_() * 1).detach(), sin, pos, False)).backward()
    assert q.grad.any() and k.grad.any() and cos.grad is None
