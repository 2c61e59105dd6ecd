"""The operators of a transformer training step, as cases that can be timed and compared.

Three operators make the gradients that the rounds of this library reduce:

    qk_norm_rope    RMS norm of every query and key head with a learned gain, then the rotation by
                    position, and its gradients (inputs and gains)
    attention       causal attention over packed sequences of different lengths with grouped heads,
                    and its gradients
    cross_entropy   output projection and softmax cross entropy over the vocabulary without keeping
                    the logits, and its gradients (hidden states and projection)

Fields of a case
    op         the operator
    dtype      "bf16" or "f32": inputs, outputs and gradients (losses, log-sum-exps and the
               rotation's table are always fp32)
    backward   False: the forward pass alone (validation); True: a training step, forward and
               gradients
    tokens     rows of the packed batch
    q_heads, kv_heads, head_dim      attention and qk_norm_rope
    seqs, spread, padding            sequences of the batch, standard deviation of the logarithm of
               their lengths, rows after the last sequence that belong to none
    vocab, width, ignored            cross_entropy: vocabulary, width of the model, share of the rows
               whose target is masked

With `own` False a pass is computed by elementary torch operations in 32 bits, rounded once at the
end; with `own` True by the library's kernels.
"""
import math
import random

import torch

own = False

EPS = 1e-6
IGNORE = -100
PARAM_SIGMA = 0.02
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One short sequence of a validation batch: launches and the host path.
        _heads("qk_norm_rope", "norm_rope_37tok_bf16_fwd", "bf16", False, 37, 16, 4, 64),
        # A process's share of a batch of the 24-layer model (width 1024 = 16 heads of 64), grouped keys.
        _heads("qk_norm_rope", "norm_rope_8k_bf16_train", "bf16", True, 8192, 16, 4, 64),
        # The 48-layer model's heads (width 1600 = 25 heads of 64), every head with its own keys, fp32,
        # a ragged number of rows.
        _heads("qk_norm_rope", "norm_rope_20k_f32_train", "f32", True, 20011, 25, 25, 64),
        # A handful of sentences: launches, lengths that fill no tile.
        _packed("attn_3short_bf16_fwd", "bf16", False, 113, 3, 0.5, 0, 16, 4, 64),
        # Sentences of very different lengths packed into one batch of the 24-layer model, a padded end.
        _packed("attn_16seq_8k_bf16_train", "bf16", True, 8192, 16, 0.8, 77, 16, 4, 64),
        # The same in fp32, the type of the 24-layer model's gradients.
        _packed("attn_9seq_4k_f32_train", "f32", True, 4099, 9, 0.7, 0, 16, 8, 64),
        # Full contexts of the 48-layer model (1024 positions each), no grouping.
        _packed("attn_8seq_8k_25h_bf16_train", "bf16", True, 8192, 8, 0.0, 0, 25, 25, 64),
        # One long document, heads of 128: the largest attention.
        _packed("attn_1seq_16k_d128_bf16_train", "bf16", True, 16384, 1, 0.0, 0, 8, 2, 128),
        # Validation loss of a few rows over the whole vocabulary: bound by reading the projection.
        _loss("loss_61tok_bf16_fwd", "bf16", False, 61, 1024, 50257, 0.0),
        # A training step of the 24-layer model's last layer on a packed batch, some targets masked.
        _loss("loss_4k_w1024_bf16_train", "bf16", True, 4096, 1024, 50257, 0.1),
        # The same in fp32 on a smaller ragged batch.
        _loss("loss_1k_w1024_f32_train", "f32", True, 1019, 1024, 50257, 0.1),
        # The 48-layer model's last layer on a large batch: the largest case.
        _loss("loss_8k_w1600_bf16_train", "bf16", True, 8191, 1600, 50257, 0.05),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _heads(op, name, dtype, backward, tokens, q_heads, kv_heads, head_dim):
    return _named(name, dict(op=op, dtype=dtype, backward=backward, tokens=tokens, q_heads=q_heads,
                             kv_heads=kv_heads, head_dim=head_dim, seqs=max(1, tokens // 700), spread=0.5,
                             padding=0))


def _packed(name, dtype, backward, tokens, seqs, spread, padding, q_heads, kv_heads, head_dim):
    return _named(name, dict(op="attention", dtype=dtype, backward=backward, tokens=tokens, seqs=seqs,
                             spread=spread, padding=padding, q_heads=q_heads, kv_heads=kv_heads,
                             head_dim=head_dim))


def _loss(name, dtype, backward, tokens, width, vocab, ignored):
    return _named(name, dict(op="cross_entropy", dtype=dtype, backward=backward, tokens=tokens, width=width,
                             vocab=vocab, ignored=ignored))


# q heads, kv heads, head dim: widths of the transformer configurations and smaller ones
HEADS = ((16, 4, 64), (16, 8, 64), (25, 5, 64), (25, 25, 64), (8, 2, 128), (8, 4, 128), (6, 3, 32), (10, 2, 80),
         (4, 1, 96), (2, 2, 40))


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        op = rng.choice(("qk_norm_rope", "attention", "attention", "cross_entropy", "cross_entropy"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        backward = rng.random() < 0.7
        if op == "qk_norm_rope":
            case = _heads(op, None, dtype, backward, _log_uniform(rng, 1, 20011), *rng.choice(HEADS))
        elif op == "attention":
            tokens = _log_uniform(rng, 1, 16384)
            # a training step has sequences of more than one token: the gradients of queries and keys of
            # a lone token are zero, and what rounding leaves of them says nothing
            tokens += backward and tokens == 1
            seqs = min(tokens // 2 if backward else tokens, _log_uniform(rng, 1, 64))
            padding = rng.choice((0, 0, rng.randint(0, 100)))
            case = _packed(None, dtype, backward, tokens + padding, seqs, rng.uniform(0.0, 1.2), padding,
                           *rng.choice(HEADS))
        else:
            case = _loss(None, dtype, backward, _log_uniform(rng, 1, 8191), 8 * _log_uniform(rng, 8, 200),
                         _log_uniform(rng, 2, 50257), rng.choice((0.0, 0.1, 0.6)))
        largest = max(_cost(c) for c in listed() if c["dtype"] == dtype and c["op"] == op)
        if _cost(case) <= largest and not _excluded(case):
            return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _excluded(case):
    """A width that none of the configurations stands for, and batches whose padded scores in 32 bits
    would not leave the plain form room on the card."""
    sizes = [v for v in case.values() if isinstance(v, int)]
    if "q_heads" in case:
        sizes += [(case["q_heads"] + 2 * case["kv_heads"]) * case["head_dim"]]
    if case["op"] == "attention":
        n = _lengths(case)
        if case["q_heads"] * len(n) * max(n) ** 2 > 8 * 16384 ** 2:
            return True
    return 3072 in sizes


# ------------------------------------------------------------------------------------- its data

def _lengths(case):
    """Lengths of the sequences: at least one token each, log-normal around their mean."""
    rng = random.Random(1000003 * case["seqs"] + case["tokens"])
    total, n = case["tokens"] - case["padding"], case["seqs"]
    weight = [math.exp(rng.gauss(0.0, case["spread"])) for _ in range(n)]
    lens = [1 + int((total - n) * w / sum(weight)) for w in weight]
    lens[rng.randrange(n)] += total - sum(lens)
    return lens


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    T = case["tokens"]

    def normal(*shape, sigma=1.0, mean=0.0, to=dtype):
        return (torch.randn(*shape, device="cuda", generator=gen) * sigma + mean).to(to)

    s = {"case": case}
    if case["op"] == "cross_entropy":
        d, V = case["width"], case["vocab"]
        w = normal(V, d, sigma=PARAM_SIGMA)
        target = torch.randint(0, V, (T,), device="cuda", generator=gen)
        # hidden states after the last norm, leaning towards their target as in a half-trained model
        x = (torch.randn(T, d, device="cuda", generator=gen) + w[target].float() * (8 / (d * PARAM_SIGMA ** 2))).to(dtype)
        masked = torch.rand(T, device="cuda", generator=gen) < case["ignored"]
        target[masked] = IGNORE
        s.update(x=x, w=w, target=target)
        # upstream gradient of the mean over the rows that count
        s["dloss"] = (~masked).float() / (~masked).sum().clamp(min=1)
        return s
    Hq, Hk, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    lens = _lengths(case)
    s["lens"] = lens
    s["cu"] = torch.tensor([0] + lens, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
    # queries, keys and values as the projection leaves them: parts of one row per token
    qkv = normal(T, (Hq + 2 * Hk) * D)
    s["q"], s["k"], s["v"] = _parts(qkv, Hq, Hk, D)
    if case["op"] == "attention":
        s["dout"] = normal(T, Hq, D)
        s["scale"] = D ** -0.5
        return s
    s["wq"], s["wk"] = normal(D, sigma=0.1, mean=1.0), normal(D, sigma=0.1, mean=1.0)
    s["dq_out"], s["dk_out"] = normal(T, Hq, D), normal(T, Hk, D)
    s["positions"] = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).cuda()
    angle = torch.arange(max(lens), dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, D, 2, dtype=torch.float64) / D)
    s["cos"], s["sin"] = angle.cos().float().cuda(), angle.sin().float().cuda()
    return s


def _parts(qkv, Hq, Hk, D):
    T = qkv.shape[0]
    q, k, v = qkv.split((Hq * D, Hk * D, Hk * D), dim=1)
    return q.view(T, Hq, D), k.view(T, Hk, D), v.view(T, Hk, D)


# ------------------------------------------------------------------------------------- a pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"qk_norm_rope": _own_norm_rope, "attention": _own_attention, "cross_entropy": _own_loss}[op](state)
    return {"qk_norm_rope": _plain_norm_rope, "attention": _plain_attention, "cross_entropy": _plain_loss}[op](state)


def _own_norm_rope(s):
    from paper_1908_04207_amd import model_ops as ops
    table = (s["cos"], s["sin"], s["positions"])
    q, k = ops.qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], *table, eps=EPS)
    if not s["case"]["backward"]:
        return {"q": q, "k": k}
    Hq, Hk, D = s["q"].shape[1], s["k"].shape[1], s["q"].shape[2]
    dqkv = torch.empty(s["q"].shape[0], (Hq + 2 * Hk) * D, dtype=s["q"].dtype, device=s["q"].device)
    dq, dk, _ = _parts(dqkv, Hq, Hk, D)
    dwq, dwk = torch.empty_like(s["wq"]), torch.empty_like(s["wk"])
    ops.qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["wq"], s["wk"], *table, eps=EPS,
                              dq=dq, dk=dk, dwq=dwq, dwk=dwk)
    return {"q": q, "k": k, "dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def _own_attention(s):
    from paper_1908_04207_amd import model_ops as ops
    out, lse = ops.attention(s["q"], s["k"], s["v"], s["cu"], scale=s["scale"])
    if not s["case"]["backward"]:
        return {"out": out, "lse": lse}
    Hq, Hk, D = s["q"].shape[1], s["k"].shape[1], s["q"].shape[2]
    dqkv = torch.empty(s["q"].shape[0], (Hq + 2 * Hk) * D, dtype=s["q"].dtype, device=s["q"].device)
    dq, dk, dv = _parts(dqkv, Hq, Hk, D)
    ops.attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, s["cu"], scale=s["scale"],
                           dq=dq, dk=dk, dv=dv)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_loss(s):
    from paper_1908_04207_amd import model_ops as ops
    loss, lse = ops.cross_entropy(s["x"], s["w"], s["target"])
    if not s["case"]["backward"]:
        return {"loss": loss, "lse": lse}
    dx, dw = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    ops.cross_entropy_backward(s["dloss"], s["x"], s["w"], s["target"], lse, dx=dx, dw=dw)
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def _rotate(u, cos, sin):
    a, b = u.chunk(2, dim=-1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)


def _plain_norm_rope(s):
    at = s["positions"].long()
    cos, sin = s["cos"][at][:, None, :], s["sin"][at][:, None, :]
    out = {}
    for name in "qk":
        x, w = s[name].float(), s["w" + name].float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        n = x * r
        out[name] = _rotate(n * w, cos, sin).to(s[name].dtype)
        if s["case"]["backward"]:
            du = _rotate(s["d%s_out" % name].float(), cos, -sin)
            dn = du * w
            out["d" + name] = (r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(s[name].dtype)
            out["dw" + name] = (du * n).sum((0, 1)).to(s[name].dtype)
    return out


def _plain_attention(s):
    """The sequences padded to the longest one, the keys repeated for the heads that share them."""
    c, cu, lens = s["case"], s["cu"].long(), s["lens"]
    T, Hq, D = s["q"].shape
    Hk, B, L = s["k"].shape[1], len(lens), max(lens)
    group = Hq // Hk
    within = torch.arange(L, device="cuda")
    real = within < (cu[1:] - cu[:-1])[:, None]                        # B, L
    at = torch.where(real, cu[:-1, None] + within, T)                  # rows of the packed batch; T: none

    def pad(x):                                                        # T, H, D -> B * H, L, D
        x = torch.cat((x.float(), x.new_zeros(1, *x.shape[1:], dtype=torch.float32)))
        return x[at].transpose(1, 2).reshape(-1, L, D)

    def unpad(x):                                                      # B * H, L, D -> T, H, D
        x = x.view(B, -1, L, D).transpose(1, 2)
        y = x.new_zeros(T + 1, x.shape[2], D)
        y[at.reshape(-1)] = x.reshape(B * L, -1, D)
        return y[:T].to(s["q"].dtype)

    def shared(x):                                                     # B * Hk, L, D -> B * Hq, L, D
        return x.view(B, Hk, 1, L, D).expand(B, Hk, group, L, D).reshape(-1, L, D)

    q, k, v = pad(s["q"]), shared(pad(s["k"])), shared(pad(s["v"]))
    p = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(s["scale"])
    p.masked_fill_(within[None, :] > within[:, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top).exp_()
    norm = p.sum(-1, keepdim=True)
    p = p.div_(norm)
    out = torch.bmm(p, v)
    lse = torch.full((T + 1, Hq), -math.inf, device="cuda")
    lse[at.reshape(-1)] = (top + norm.log()).view(B, Hq, L).transpose(1, 2).reshape(B * L, Hq)
    result = {"out": unpad(out), "lse": lse[:T].t().contiguous()}
    if not c["backward"]:
        return result
    dout = pad(s["dout"])

    def grouped(x):                                                    # gradients of the heads that share
        return unpad(x.view(B, Hk, group, L, D).sum(2).view(-1, L, D))

    result["dv"] = grouped(torch.bmm(p.transpose(1, 2).contiguous(), dout))
    dp = torch.bmm(dout, v.transpose(1, 2).contiguous())
    ds = dp.sub_((dout * out).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    del p
    result["dq"] = unpad(torch.bmm(ds, k))
    result["dk"] = grouped(torch.bmm(ds.transpose(1, 2).contiguous(), q))
    return result


def _plain_loss(s):
    x, w = s["x"].float(), s["w"].float()
    target = s["target"]
    counted = target >= 0
    at = torch.where(counted, target, 0)[:, None]
    p = x @ w.t()
    right = p.gather(1, at)[:, 0]
    top = p.amax(1, keepdim=True)
    p = p.sub_(top).exp_()
    norm = p.sum(1, keepdim=True)
    lse = (top + norm.log())[:, 0]
    out = {"loss": torch.where(counted, lse - right, 0.0), "lse": lse}
    if not s["case"]["backward"]:
        return out
    p = p.div_(norm)
    p.scatter_add_(1, at, torch.full_like(p[:, :1], -1.0))
    p.mul_(torch.where(counted, s["dloss"], 0.0)[:, None])
    out["dx"] = (p @ w).to(s["x"].dtype)
    out["dw"] = (p.t() @ x).to(s["w"].dtype)
    return out


# ------------------------------------------------------------------------------------- its measure

def work(case):
    """Inputs read once, outputs written once; products that the mathematics needs (nothing computed
    again in the backward pass)."""
    g = 2 if case["dtype"] == "bf16" else 4
    T, train = case["tokens"], case["backward"]
    if case["op"] == "cross_entropy":
        d, V = case["width"], case["vocab"]
        io = g * (T * d + V * d)
        return {"bytes": io * (2 if train else 1) + T * (8 + 8) + (4 * T if train else 0),
                "flops": (6 if train else 2) * T * V * d}
    Hq, Hk, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "qk_norm_rope":
        rows = T * (Hq + Hk)
        return {"bytes": rows * D * g * (4 if train else 2) + T * 4 + 4 * D * max(_lengths(case)),
                "flops": rows * D * (22 if train else 8)}
    pairs = sum(n * (n + 1) // 2 for n in _lengths(case))
    io = T * D * g * (2 * Hq + 2 * Hk)
    return {"bytes": io * (2 if train else 1) + 4 * T * Hq, "flops": (14 if train else 4) * D * Hq * pairs}


# ------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in 64 bits, sequence by sequence and head by head."""
    s = prepare(case, seed)
    f64 = torch.float64
    train = case["backward"]
    if case["op"] == "cross_entropy":
        x, w, t = s["x"].to(f64), s["w"].to(f64), s["target"]
        n = x.shape[0]
        loss, lse = torch.zeros(n, dtype=f64, device="cuda"), torch.zeros(n, dtype=f64, device="cuda")
        dx, dw = torch.zeros_like(x), torch.zeros_like(w)
        for r in range(0, n, 1024):
            rows = slice(r, min(n, r + 1024))
            logits = x[rows] @ w.t()
            lse[rows] = torch.logsumexp(logits, 1)
            use = torch.nonzero(t[rows] >= 0)[:, 0]
            loss[rows][use] = lse[rows][use] - logits[use, t[rows][use]]
            if train:
                grad = torch.softmax(logits, 1)
                grad[use, t[rows][use]] -= 1.0
                weight = torch.zeros(grad.shape[0], dtype=f64, device="cuda")
                weight[use] = s["dloss"][rows][use].to(f64)
                grad *= weight[:, None]
                dx[rows] = grad @ w
                dw += grad.t() @ x[rows]
        return {"loss": loss, "lse": lse, "dx": dx, "dw": dw} if train else {"loss": loss, "lse": lse}
    if case["op"] == "qk_norm_rope":
        at = s["positions"].long()
        turn = torch.complex(s["cos"][at].to(f64), s["sin"][at].to(f64))[:, None, :]
        half = case["head_dim"] // 2
        out = {}
        for name in "qk":
            x, w = s[name].to(f64), s["w" + name].to(f64)
            root = torch.sqrt((x * x).sum(-1, keepdim=True) / (2 * half) + EPS)
            u = w * x / root
            z = torch.complex(u[..., :half].contiguous(), u[..., half:].contiguous()) * turn
            out[name] = torch.cat((z.real, z.imag), -1)
            if train:
                dy = s["d%s_out" % name].to(f64)
                z = torch.complex(dy[..., :half].contiguous(), dy[..., half:].contiguous()) * turn.conj()
                du = torch.cat((z.real, z.imag), -1)
                out["dw" + name] = (du * x / root).sum(1).sum(0)
                along = (du * w * x).sum(-1, keepdim=True) / (2 * half)
                out["d" + name] = du * w / root - x * along / root ** 3
        return out
    T, Hq, D = s["q"].shape
    group = Hq // s["k"].shape[1]
    out = {"out": torch.zeros(T, Hq, D, dtype=f64, device="cuda"),
           "lse": torch.full((Hq, T), -math.inf, dtype=f64, device="cuda")}
    if train:
        out["dq"] = torch.zeros(T, Hq, D, dtype=f64, device="cuda")
        out["dk"], out["dv"] = (torch.zeros(s["k"].shape, dtype=f64, device="cuda") for _ in range(2))
    start = 0
    for n in s["lens"]:
        rows = slice(start, start + n)
        later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        for h in range(Hq):
            q, k, v = s["q"][rows, h].to(f64), s["k"][rows, h // group].to(f64), s["v"][rows, h // group].to(f64)
            score = s["scale"] * (q @ k.t())
            score[later] = -math.inf
            out["lse"][h, rows] = torch.logsumexp(score, 1)
            p = torch.softmax(score, 1)
            del score
            o = p @ v
            out["out"][rows, h] = o
            if train:
                do = s["dout"][rows, h].to(f64)
                out["dv"][rows, h // group] += p.t() @ do
                p *= do @ v.t() - (do * o).sum(1, keepdim=True)
                out["dq"][rows, h] = s["scale"] * (p @ k)
                out["dk"][rows, h // group] += s["scale"] * (p.t() @ q)
            del p
        start += n
    return out
