"""packed_lm.py with layer norms, rotation of a part of every head, and a student that learns from a teacher: gradients
against torch's autograd on the same model written with plain operations in 64 bits, training through the library's
rounds bit-identical to the oracle."""
import math
from dataclasses import replace

import numpy as np
import pytest
import torch

from harness import bits
from oracle import eager_oracle as eo
from paper_1908_04207_amd import packed_lm as lm

SMALL = lm.Model(vocab=211, width=64, layers=2, q_heads=4, kv_heads=2, head_dim=16, ffn=96, positions=64)
LAYER = replace(SMALL, layer_norm=True, rotary_part=8)


def test_layouts():
    """The model of before has the tensors of before; gains and biases come in pairs."""
    assert [n for n, _ in SMALL.tensors()] == ["embedding", "h0.qkv", "h0.q_gain", "h0.k_gain", "h0.out", "h0.fc1", "h0.fc2", "h1.qkv",
                                               "h1.q_gain", "h1.k_gain", "h1.out", "h1.fc1", "h1.fc2", "head"]
    names = [n for n, _ in LAYER.tensors()]
    assert sum(n.endswith(".gain") for n in names) == sum(n.endswith(".bias") for n in names) == 5
    assert not any("q_gain" in n for n in names)
    off, num, arena = LAYER.layout()
    assert all(o % 8 == 0 for o in off) and off[-1] + num[-1] <= arena


def _plain_hidden(m, weights, tokens, cu, positions, cos, sin):
    def norm(x, name):
        c = x - x.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * weights[name + ".gain"] + weights[name + ".bias"]

    def rotate(x):
        n = m.rotary_part
        c, s = cos[positions.long()][:, None].double(), sin[positions.long()][:, None].double()
        a, b = x[..., :n // 2], x[..., n // 2:n]
        return torch.cat((a * c - b * s, b * c + a * s, x[..., n:]), -1)

    x = weights["embedding"][tokens]
    T, D, group = tokens.numel(), m.head_dim, m.q_heads // m.kv_heads
    for n in range(m.layers):
        q, k, v = (t.view(T, -1, D) for t in (norm(x, f"h{n}.norm1") @ weights[f"h{n}.qkv"].t()).split(
            (m.q_heads * D, m.kv_heads * D, m.kv_heads * D), 1))
        q, k, v = rotate(q), rotate(k).repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        out = []
        for a, b in zip(cu[:-1], cu[1:]):
            s = (q[a:b].transpose(0, 1) @ k[a:b].permute(1, 2, 0).contiguous()) / math.sqrt(D)
            later = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
            out.append((torch.softmax(s.masked_fill(later, -math.inf), -1) @ v[a:b].transpose(0, 1).contiguous()).transpose(0, 1))
        x = x + torch.cat(out).reshape(T, -1) @ weights[f"h{n}.out"].t()
        x = x + torch.nn.functional.gelu(norm(x, f"h{n}.norm2") @ weights[f"h{n}.fc1"].t()) @ weights[f"h{n}.fc2"].t()
    return norm(x, "norm")


def _weights(m, gen, dtype):
    return {n: (torch.randn(*s, device="cuda", generator=gen) * (0.2 if len(s) == 2 else 0.1) +
                (len(s) == 1 and not n.endswith("bias"))).to(dtype) for n, s in m.tensors()}


@pytest.mark.gpu
@pytest.mark.parametrize("taught", [False, True])
@pytest.mark.parametrize("dtype,most", [(torch.float32, 2e-5), (torch.bfloat16, 0.06)])
def test_gradients_of_the_model(dtype, most, taught):
    """Relative error of every tensor's gradient, with the limits of the model of before (test_packed_lm.py): as many
    roundings on the way."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    data = lm.Batches(LAYER, 5)
    tokens, targets, cu, positions = data.batch([2, 17, 40, 33, 64])
    cos, sin = lm.rotation_table(LAYER)
    start = _weights(LAYER, gen, dtype)
    ours = {n: t.clone().requires_grad_() for n, t in start.items()}
    plain = {n: t.double().requires_grad_() for n, t in start.items()}
    y = _plain_hidden(LAYER, plain, tokens, cu.tolist(), positions, cos, sin)
    logits = y @ plain["head"].t()
    if taught:
        top, index = logits.detach().float().topk(9, dim=1)
        index[targets < 0] = -1
        top = top * 0.7 + 0.5 * torch.randn(top.shape, device="cuda", generator=gen)
        from paper_1908_04207_amd import model_ops as ops
        a = ops.Distillation.apply(lm.hidden_of(LAYER, ours, tokens, cu, positions, cos, sin), ours["head"], index, top, 2.0).sum()
        q = torch.log_softmax(top.double() / 2, 1)
        b = (q.exp() * (q - torch.log_softmax(logits / 2, 1).gather(1, index.clamp(min=0)))).sum(1)[targets >= 0].sum()
    else:
        a = lm.loss_of(LAYER, ours, tokens, targets, cu, positions, cos, sin).sum()
        b = torch.where(targets >= 0, torch.logsumexp(logits, 1) - logits.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0).sum()
    a.backward()
    b.backward()
    assert abs(float(a.detach()) - float(b.detach())) < most * abs(float(b.detach()))
    for n in ours:
        off = float((ours[n].grad.double() - plain[n].grad).norm() / plain[n].grad.norm())
        assert off < most, (n, off)


@pytest.mark.gpu
def test_what_a_teacher_says():
    """Its lists are the largest logits of its own hidden states, none where a target is masked."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    weights = _weights(LAYER, gen, torch.float32)
    off, num, arena = LAYER.layout()
    flat = torch.zeros(arena, device="cuda")
    for (n, _), o, c in zip(LAYER.tensors(), off, num):
        flat[o:o + c] = weights[n].flatten()
    tokens, targets, cu, positions = lm.Batches(LAYER, 6).batch([5, 30, 64, 2])
    index, logits = lm.Teacher(LAYER, flat, entries=7).lists(tokens, targets, cu, positions, torch.float32)
    cos, sin = lm.rotation_table(LAYER)
    y = _plain_hidden(LAYER, {n: t.double() for n, t in weights.items()}, tokens, cu.tolist(), positions, cos, sin)
    want = (y @ weights["head"].double().t()).topk(7, dim=1)
    keep = targets >= 0
    assert (index[~keep] == -1).all() and (index[keep] >= 0).all()
    assert float((logits.double() - want.values).norm() / want.values.norm()) < 2e-5
    assert float((index[keep] == want.indices[keep]).float().mean()) > 0.99


@pytest.mark.gpu
@pytest.mark.parametrize("model,mode,bf16,taught", [(LAYER, "solo", False, False), (LAYER, "majority", True, False),
                                                    (SMALL, "majority", False, True), (LAYER, "majority", True, True)])
def test_training_run_bit_identical_to_oracle(model, mode, bf16, taught):
    off, num, arena = model.layout()
    teacher = None
    if taught:
        big = replace(LAYER, width=96)
        teacher = lm.Teacher(big, torch.randn(big.layout()[2], device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) * 0.1)
    oracle = None

    def on_round(t, plan, G, w, v):
        nonlocal oracle
        if t < 0:
            oracle = eo.OracleState(4, off, num, arena, w.cpu().numpy(), 0.1, 0.9)
            return
        grads = [g.cpu().view(torch.int16).numpy().view(np.uint16) if bf16 else g.cpu().numpy() for g in G]
        assert all(np.isfinite(g.float().cpu().numpy()).all() and g.any() for g in G)
        oracle.round(plan.mask, grads)
        for name, ours, theirs in (("w", w.cpu().numpy(), oracle.w), ("v", v.cpu().numpy(), oracle.v)):
            for o, n in zip(off, num):
                assert np.array_equal(bits(ours[o:o + n]), bits(theirs[o:o + n])), (t, name, o)

    r = lm.train(mode, 4, P=4, model=model, sentences=6, mean=20.0, lr=0.1, mu=0.9, bf16=bf16, on_round=on_round, teacher=teacher)
    assert oracle is not None and all(math.isfinite(x) for x in r.loss) and r.weights.shape == (arena,)


@pytest.mark.gpu
def test_the_commands(capsys, monkeypatch):
    for more in ([], ["--layer-norm", "--bf16", "--distill"]):
        monkeypatch.setattr("sys.argv", ["packed_lm", "--steps", "2", *more])
        lm.main()
        lines = capsys.readouterr().out.splitlines()
        assert len(lines) == (6 if more else 3) and all("nan" not in line for line in lines)
