"""The small language model of packed_lm.py: its gradients against torch's autograd on the same model written
with plain operations in 64 bits, training through the library's rounds bit-identical to the oracle,
and the loss going down."""
import math

import numpy as np
import pytest
import torch

from harness import bits
from oracle import eager_oracle as eo
from paper_1908_04207_amd import packed_lm as lm

pytestmark = pytest.mark.gpu
SMALL = lm.Model(vocab=211, width=64, layers=2, q_heads=4, kv_heads=2, head_dim=16, ffn=96, positions=64)


def _plain_loss(m, weights, tokens, targets, cu, positions, cos, sin):
    """loss_of with elementary operations, sequence by sequence."""
    def rms(x):
        return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def rotate(x, gain):
        x = rms(x) * gain
        c, s = cos[positions.long()][:, None].double(), sin[positions.long()][:, None].double()
        a, b = x.chunk(2, -1)
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    x = weights["embedding"][tokens]
    T, D, group = tokens.numel(), m.head_dim, m.q_heads // m.kv_heads
    for n in range(m.layers):
        q, k, v = (t.view(T, -1, D) for t in (rms(x) @ weights[f"h{n}.qkv"].t()).split(
            (m.q_heads * D, m.kv_heads * D, m.kv_heads * D), 1))
        q, k = rotate(q, weights[f"h{n}.q_gain"]), rotate(k, weights[f"h{n}.k_gain"])
        k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        out = []
        for a, b in zip(cu[:-1], cu[1:]):
            s = (q[a:b].transpose(0, 1) @ k[a:b].permute(1, 2, 0).contiguous()) / math.sqrt(D)
            later = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
            out.append((torch.softmax(s.masked_fill(later, -math.inf), -1) @ v[a:b].transpose(0, 1).contiguous()).transpose(0, 1))
        x = x + torch.cat(out).reshape(T, -1) @ weights[f"h{n}.out"].t()
        x = x + torch.nn.functional.gelu(rms(x) @ weights[f"h{n}.fc1"].t()) @ weights[f"h{n}.fc2"].t()
    logits = rms(x) @ weights["head"].t()
    return torch.where(targets >= 0, torch.logsumexp(logits, 1) - logits.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)


@pytest.mark.parametrize("dtype,most", [(torch.float32, 2e-5), (torch.bfloat16, 0.06)])
def test_gradients_of_the_model(dtype, most):
    """Relative error of every tensor's gradient: fp32 roundings through a dozen operations; in bf16 about
    twenty roundings of 2^-8 on the way, added as a random walk and three times that allowed."""
    m = SMALL
    gen = torch.Generator(device="cuda").manual_seed(0)
    data = lm.Batches(m, 5)
    tokens, targets, cu, positions = data.batch([2, 17, 40, 33, 64])
    cos, sin = lm.rotation_table(m)
    start = {n: (torch.randn(*s, device="cuda", generator=gen) * (0.2 if len(s) == 2 else 0.1) + (len(s) == 1)).to(dtype)
             for n, s in m.tensors()}
    ours = {n: t.clone().requires_grad_() for n, t in start.items()}
    plain = {n: t.double().requires_grad_() for n, t in start.items()}
    a = lm.loss_of(m, ours, tokens, targets, cu, positions, cos, sin).sum()
    b = _plain_loss(m, plain, tokens, targets, cu.tolist(), positions, cos, sin).sum()
    a.backward()
    b.backward()
    assert abs(float(a) - float(b)) < most * abs(float(b))
    for n in ours:
        off = float((ours[n].grad.double() - plain[n].grad).norm() / plain[n].grad.norm())
        assert off < most, (n, off)


@pytest.mark.parametrize("mode,bf16", [("solo", False), ("majority", True)])
def test_training_run_bit_identical_to_oracle(mode, bf16):
    off, num, arena = SMALL.layout()
    oracle = None

    def on_round(t, plan, G, w, v):
        nonlocal oracle
        if t < 0:
            oracle = eo.OracleState(4, off, num, arena, w.cpu().numpy(), 0.1, 0.9)
            return
        grads = [g.cpu().view(torch.int16).numpy().view(np.uint16) if bf16 else g.cpu().numpy() for g in G]
        oracle.round(plan.mask, grads)
        for name, ours, theirs in (("w", w.cpu().numpy(), oracle.w), ("v", v.cpu().numpy(), oracle.v)):
            for o, n in zip(off, num):
                assert np.array_equal(bits(ours[o:o + n]), bits(theirs[o:o + n])), (t, name, o)

    lm.train(mode, 6, P=4, model=SMALL, sentences=6, mean=20.0, lr=0.1, mu=0.9, bf16=bf16, on_round=on_round)
    assert oracle is not None


@pytest.mark.parametrize("mode,bf16", [("sync", False), ("majority", False), ("solo", False), ("majority", True)])
def test_loss_goes_down(mode, bf16):
    """From the logarithm of the vocabulary (and more at the start, with random weights) by well over half of
    what can be learnt in 40 rounds; fewer processes wait than in a synchronous run."""
    r = lm.train(mode, 40, model=lm.Model(vocab=101, positions=128), sentences=12, mean=30.0, bf16=bf16)
    assert all(math.isfinite(x) for x in r.loss)
    assert sum(r.loss[-5:]) / 5 < r.loss[0] - 1.0, r.loss
    assert r.nap_mean == 4 if mode == "sync" else r.nap_mean < 4
