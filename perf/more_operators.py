"""More operators of a transformer training step, as cases that can be timed and compared.

    layer_norm      sum with the residual stream, norm of every row with gain and bias, and its gradients (inputs,
                    gain and bias)
    rotary_table    cosines and sines of every position's angles, plain or scaled for contexts longer than those
                    of training
    rotary          rotation of query and key heads, or of the first part of each, pairs side by side
                    (interleaved) or half a part away, and its gradients
    distillation    output projection and the divergence of a student's softmax from that of a teacher's top
                    logits, without keeping the student's, and its gradients (hidden states and projection)

Fields of a case
    op         the operator
    dtype      "bf16" or "f32": inputs, outputs and gradients (statistics, tables, the teacher's logits, losses
               and log-sum-exps are always fp32)
    backward   False: the forward pass alone (validation); True: a training step, forward and gradients
    tokens     rows of the packed batch
    width      of the hidden states (layer_norm, distillation)
    residual, bias                       layer_norm: whether there is a residual stream to add, a bias
    q_heads, kv_heads, head_dim          rotary
    part, interleaved                    rotary, rotary_table: elements of a head that are rotated; layout of pairs
    positions, scaling, factor           rotary_table; `positions` also of the table that rotary reads
    vocab, entries, temperature          distillation: vocabulary, teacher's logits a row
    ignored, unused                      distillation: share of rows without any entry, of entries that hold none

With `own` False a pass is computed by elementary torch operations in 32 bits (angles in 64), rounded once at
the end; with `own` True by the library's kernels.
"""
import math
import random

import torch

own = False

EPS = 1e-5
PARAM_SIGMA = 0.02
ORIGINAL = 2048                     # positions that a scaled table's model was trained on
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One short sequence of a validation batch: launches and the host path.
        _norm("norm_37x1024_bf16_fwd", "bf16", False, 37, 1024, True, True),
        # A process's share of a batch of the 24-layer model: residual sum and norm before every product.
        _norm("norm_8k_w1024_bf16_train", "bf16", True, 8192, 1024, True, True),
        # The 48-layer model's width in fp32, a ragged number of rows.
        _norm("norm_20k_w1600_f32_train", "f32", True, 20011, 1600, True, True),
        # Wide rows without a bias or a residual stream: more than one wavefront holds a row.
        _norm("norm_2k_w8192_bf16_train", "bf16", True, 2047, 8192, False, False),
        # The table of the 24-layer model's positions.
        _table("table_1k_d64", 1024, 64, "none", 1.0),
        # A table for contexts 64 times as long as the model was trained on, frequencies scaled by parts.
        _table("table_131k_d128_parts", 131072, 128, "parts", 64.0),
        # One short sequence: launches and the host path.
        _rotary("rotary_61tok_bf16_fwd", "bf16", False, 61, 16, 4, 64, 64, False),
        # A process's share of a batch of the 24-layer model, half of every head rotated, pairs side by side.
        _rotary("rotary_8k_bf16_train", "bf16", True, 8192, 16, 4, 64, 32, True),
        # The 48-layer model's heads, rotated whole, fp32.
        _rotary("rotary_20k_f32_train", "f32", True, 20011, 25, 25, 64, 64, False),
        # Validation of a student on a few rows: bound by reading the projection.
        _distill("distill_61tok_bf16_fwd", "bf16", False, 61, 1024, 50257, 16, 1.0, 0.0, 0.0),
        # A training step of a student of the 24-layer model's size, 64 of the teacher's logits a row.
        _distill("distill_4k_w1024_bf16_train", "bf16", True, 4096, 1024, 50257, 64, 2.0, 0.1, 0.1),
        # The same in fp32 on a smaller ragged batch.
        _distill("distill_1k_w1024_f32_train", "f32", True, 1019, 1024, 50257, 32, 1.0, 0.1, 0.0),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _norm(name, dtype, backward, tokens, width, residual, bias):
    return _named(name, dict(op="layer_norm", dtype=dtype, backward=backward, tokens=tokens, width=width,
                             residual=residual, bias=bias))


def _table(name, positions, part, scaling, factor):
    return _named(name, dict(op="rotary_table", dtype="f32", backward=False, positions=positions, part=part,
                             scaling=scaling, factor=factor))


def _rotary(name, dtype, backward, tokens, q_heads, kv_heads, head_dim, part, interleaved):
    return _named(name, dict(op="rotary", dtype=dtype, backward=backward, tokens=tokens, q_heads=q_heads,
                             kv_heads=kv_heads, head_dim=head_dim, part=part, interleaved=interleaved,
                             positions=1024))


def _distill(name, dtype, backward, tokens, width, vocab, entries, temperature, ignored, unused):
    return _named(name, dict(op="distillation", dtype=dtype, backward=backward, tokens=tokens, width=width,
                             vocab=vocab, entries=entries, temperature=temperature, ignored=ignored, unused=unused))


# q heads, kv heads, head dim: widths of the transformer configurations and smaller ones
HEADS = ((16, 4, 64), (16, 8, 64), (25, 5, 64), (25, 25, 64), (8, 2, 128), (8, 4, 128), (6, 3, 32), (10, 2, 80),
         (4, 1, 96), (2, 2, 40))


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        op = rng.choice(("layer_norm", "layer_norm", "layer_norm", "rotary", "rotary", "rotary_table", "distillation",
                         "distillation", "distillation"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        backward = rng.random() < 0.7
        if op == "layer_norm":
            case = _norm(None, dtype, backward, _log_uniform(rng, 1, 65536), 8 * _log_uniform(rng, 2, 1024),
                         rng.random() < 0.6, rng.random() < 0.7)
        elif op == "rotary_table":
            scaling = rng.choice(("none", "linear", "base", "parts"))
            case = _table(None, _log_uniform(rng, 1, 131072), 8 * rng.randint(1, 16), scaling,
                          1.0 if scaling == "none" else float(_log_uniform(rng, 2, 64)))
            dtype = "f32"
        elif op == "rotary":
            q_heads, kv_heads, head_dim = rng.choice(HEADS)
            part = rng.choice((head_dim, 8 * rng.randint(1, head_dim // 8)))
            case = _rotary(None, dtype, backward, _log_uniform(rng, 1, 20011), q_heads, kv_heads, head_dim, part,
                           rng.random() < 0.5)
        else:
            vocab = _log_uniform(rng, 2, 50257)
            case = _distill(None, dtype, backward, _log_uniform(rng, 1, 8191), 8 * _log_uniform(rng, 8, 200), vocab,
                            min(vocab, _log_uniform(rng, 1, 128)), rng.choice((1.0, 2.0, round(rng.uniform(0.5, 4.0), 2))),
                            rng.choice((0.0, 0.1, 0.6)), rng.choice((0.0, 0.1, 0.5)))
        if _cost(case) <= max(_cost(c) for c in listed() if c["dtype"] == dtype and c["op"] == op):
            return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ------------------------------------------------------------------------------------- its data

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape, sigma=1.0, mean=0.0, to=dtype):
        return (torch.randn(*shape, device="cuda", generator=gen) * sigma + mean).to(to)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    s = {"case": case}
    if case["op"] == "rotary_table":
        # what a program has in hand are numbers; another seed is a model of another base
        s["base"] = 10000.0 + seed % 1000
        return s
    T = case["tokens"]
    if case["op"] == "layer_norm":
        d = case["width"]
        # a residual stream has columns that stand out in every row
        x = torch.randn(T, d, device="cuda", generator=gen) * 0.7 + torch.randn(d, device="cuda", generator=gen)
        s["x"] = x.to(dtype)
        s["residual"] = normal(T, d) if case["residual"] else None
        s["w"] = normal(d, sigma=0.1, mean=1.0)
        s["b"] = normal(d, sigma=0.1) if case["bias"] else None
        s["dy"] = normal(T, d)
        s["ds"] = normal(T, d) if case["residual"] else None
        return s
    if case["op"] == "rotary":
        Hq, Hk, D = case["q_heads"], case["kv_heads"], case["head_dim"]
        # queries, keys and values as the projection leaves them: parts of one row per token
        s["q"], s["k"], _ = _parts(normal(T, (Hq + 2 * Hk) * D), Hq, Hk, D)
        s["dq_out"], s["dk_out"] = normal(T, Hq, D), normal(T, Hk, D)
        # sequences packed one behind the other, each from position 0
        at = torch.arange(T, device="cuda")
        begins = (uniform(T) < 1 / 300) | (at == 0)
        first = torch.where(begins, at, 0).cummax(0).values
        s["positions"] = ((at - first) % case["positions"]).int()
        angle = torch.arange(case["positions"], dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(0, case["part"], 2, dtype=torch.float64) / case["part"])
        s["cos"], s["sin"] = angle.cos().float().cuda(), angle.sin().float().cuda()
        return s
    d, V, K = case["width"], case["vocab"], case["entries"]
    s["w"] = normal(V, d, sigma=PARAM_SIGMA)
    # which entries a row's teacher favours: few of them often, as words are; all of a row differ
    each = torch.arange(K, device="cuda")
    index = (float(V) ** uniform(T, K)).long().clamp_(max=V) - 1
    index = (index.sort(1).values - each).cummax(1).values + each
    index = torch.minimum(index, V - K + each)
    index = index.gather(1, uniform(T, K).argsort(1))
    # their logits, the largest first, as a search for the top of a row leaves them
    gaps = -torch.log(uniform(T, K).clamp_(min=1e-6)) * 0.4
    s["teacher"] = (12.0 - gaps.cumsum(1)).contiguous()
    # hidden states that lean towards the first two, as in a half-trained student
    x = torch.randn(T, d, device="cuda", generator=gen)
    for k, lean in enumerate((6.0, 3.0)):
        if k < K:
            x += s["w"][index[:, k]].float() * (lean / (d * PARAM_SIGMA ** 2))
    s["x"] = x.to(dtype)
    empty = (uniform(T) < case["ignored"])[:, None] | (uniform(T, K) < case["unused"])
    index[empty] = -1
    s["teacher"][empty] = math.nan                      # nothing stands there
    s["index"] = index.contiguous()
    counted = (index >= 0).any(1)
    s["dloss"] = counted.float() / counted.sum().clamp(min=1)
    return s


def _parts(qkv, Hq, Hk, D):
    T = qkv.shape[0]
    q, k, v = qkv.split((Hq * D, Hk * D, Hk * D), dim=1)
    return q.view(T, Hq, D), k.view(T, Hk, D), v.view(T, Hk, D)


# ------------------------------------------------------------------------------------- a pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"layer_norm": _own_norm, "rotary_table": _own_table, "rotary": _own_rotary, "distillation": _own_distill}[op](state)
    return {"layer_norm": _plain_norm, "rotary_table": _plain_table, "rotary": _plain_rotary,
            "distillation": _plain_distill}[op](state)


def _own_norm(s):
    from paper_1908_04207_amd import model_ops as ops
    y, total, stats = ops.layer_norm(s["x"], s["w"], s["b"], EPS, residual=s["residual"])
    out = {"y": y, "stats": stats}
    if s["residual"] is not None:
        out["sum"] = total
    if s["case"]["backward"]:
        dx, dw, db = ops.layer_norm_backward(s["dy"], total, s["w"], stats, ds=s["ds"], want=(True, s["b"] is not None))
        out.update(dx=dx, dw=dw)
        if s["b"] is not None:
            out["db"] = db
    return out


def _own_table(s):
    from paper_1908_04207_amd import model_ops as ops
    c = s["case"]
    cos, sin = ops.rotary_table(c["positions"], c["part"], s["base"], scaling=c["scaling"], factor=c["factor"],
                                original=ORIGINAL, device="cuda")
    return {"cos": cos, "sin": sin}


def _own_rotary(s):
    from paper_1908_04207_amd import model_ops as ops
    table = (s["cos"], s["sin"], s["positions"], s["case"]["interleaved"])
    q, k = ops.rotary(s["q"], s["k"], *table)
    if not s["case"]["backward"]:
        return {"q": q, "k": k}
    Hq, Hk, D = s["q"].shape[1], s["k"].shape[1], s["q"].shape[2]
    dqkv = torch.empty(s["q"].shape[0], (Hq + 2 * Hk) * D, dtype=s["q"].dtype, device=s["q"].device)
    dq, dk, _ = _parts(dqkv, Hq, Hk, D)
    ops.rotary_backward(s["dq_out"], s["dk_out"], *table, dq=dq, dk=dk)
    return {"q": q, "k": k, "dq": dq, "dk": dk}


def _own_distill(s):
    from paper_1908_04207_amd import model_ops as ops
    tau = s["case"]["temperature"]
    loss, lse, picked = ops.distillation(s["x"], s["w"], s["index"], s["teacher"], tau)
    out = {"loss": loss, "lse": lse, "picked": picked}
    if s["case"]["backward"]:
        out["dx"], out["dw"] = ops.distillation_backward(s["dloss"], s["x"], s["w"], s["index"], s["teacher"], lse, picked, tau)
    return out


def _plain_norm(s):
    dtype, w = s["x"].dtype, s["w"].float()
    total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dtype)
    x = total.float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    r = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    n = x * r
    y = n * w if s["b"] is None else n * w + s["b"].float()
    out = {"y": y.to(dtype), "stats": torch.cat((mean, r), 1).t().contiguous()}
    if s["residual"] is not None:
        out["sum"] = total
    if s["case"]["backward"]:
        dy = s["dy"].float()
        dn = dy * w
        dx = r * (dn - dn.mean(1, keepdim=True) - n * (dn * n).mean(1, keepdim=True))
        out["dx"] = (dx if s["ds"] is None else dx + s["ds"].float()).to(dtype)
        out["dw"] = (dy * n).sum(0).to(dtype)
        if s["b"] is not None:
            out["db"] = dy.sum(0).to(dtype)
    return out


def _plain_table(s):
    c, base = s["case"], s["base"]
    n, scaling, factor = c["part"], c["scaling"], c["factor"]
    if scaling == "base":
        base = base * factor ** (n / max(n - 2, 1))
    freq = base ** (-torch.arange(0, n, 2, dtype=torch.float64, device="cuda") / n)
    if scaling == "linear":
        freq = freq / factor
    if scaling == "parts":
        # frequencies of more than 32 turns over the original context stay, those of less than one are divided
        keep = ((ORIGINAL * freq / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        freq = freq * (keep + (1 - keep) / factor)
    angle = torch.arange(c["positions"], dtype=torch.float64, device="cuda")[:, None] * freq
    return {"cos": angle.cos().float(), "sin": angle.sin().float()}


def _turn(x, cos, sin, interleaved):
    """The first 2 * cos.shape[-1] elements of every head turned, the rest as it is."""
    n = 2 * cos.shape[-1]
    head, rest = x[..., :n], x[..., n:]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else head.chunk(2, dim=-1)
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(turned, -1).flatten(-2) if interleaved else torch.cat(turned, -1)
    return torch.cat((turned, rest), -1)


def _plain_rotary(s):
    c = s["case"]
    at = s["positions"].long()
    cos, sin = s["cos"][at][:, None, :], s["sin"][at][:, None, :]
    out = {}
    for name in "qk":
        out[name] = _turn(s[name].float(), cos, sin, c["interleaved"]).to(s[name].dtype)
        if c["backward"]:
            out["d" + name] = _turn(s["d%s_out" % name].float(), cos, -sin, c["interleaved"]).to(s[name].dtype)
    return out


def _plain_distill(s):
    x, w, tau = s["x"].float(), s["w"].float(), s["case"]["temperature"]
    used = s["index"] >= 0
    counted = used.any(1)
    at = torch.where(used, s["index"], 0)
    p = x @ w.t()
    picked = torch.where(used, p.gather(1, at), 0.0)
    p.div_(tau)
    top = p.amax(1, keepdim=True)
    p = p.sub_(top).exp_()
    norm = p.sum(1, keepdim=True)
    lse = (top + norm.log())[:, 0]
    t = torch.where(used, s["teacher"] / tau, -math.inf)
    t_top = torch.where(counted, t.amax(1), 0.0)[:, None]
    q = torch.where(used, (t - t_top).exp(), 0.0)
    q_norm = torch.where(counted, q.sum(1), 1.0)[:, None]
    q = q / q_norm
    logs = torch.where(used, t - t_top - q_norm.log() - (picked / tau - lse[:, None]), 0.0)
    out = {"loss": (q * logs).sum(1), "lse": lse, "picked": picked}
    if not s["case"]["backward"]:
        return out
    p = p.div_(norm)
    p.scatter_add_(1, at, -q)
    p.mul_((torch.where(counted, s["dloss"], 0.0) / tau)[:, None])
    out["dx"] = (p @ w).to(s["x"].dtype)
    out["dw"] = (p.t() @ x).to(s["w"].dtype)
    return out


# ------------------------------------------------------------------------------------- its measure

def work(case):
    """Inputs read once, outputs written once; products that the mathematics needs (nothing computed again in
    the backward pass)."""
    g = 2 if case["dtype"] == "bf16" else 4
    train = case["backward"]
    if case["op"] == "rotary_table":
        pairs = case["positions"] * case["part"] // 2
        return {"bytes": 8 * pairs, "flops": 30 * pairs}
    T = case["tokens"]
    if case["op"] == "layer_norm":
        d = case["width"]
        arrays = (4 if case["residual"] else 2) + ((4 if case["residual"] else 3) if train else 0)
        vectors = (2 if case["bias"] else 1) * (2 if train else 1)
        return {"bytes": g * T * d * arrays + g * d * vectors + 8 * T, "flops": T * d * (22 if train else 9)}
    if case["op"] == "rotary":
        rows = T * (case["q_heads"] + case["kv_heads"])
        return {"bytes": rows * case["head_dim"] * g * (4 if train else 2) + 4 * T + 4 * case["part"] * min(T, case["positions"]),
                "flops": rows * case["part"] * (6 if train else 3)}
    d, V, K = case["width"], case["vocab"], case["entries"]
    io = g * (T * d + V * d)
    return {"bytes": io * (2 if train else 1) + T * K * (8 + 4 + 4) + T * 8 + (4 * T if train else 0),
            "flops": (6 if train else 2) * T * V * d}


# ------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    return {"layer_norm": _exact_norm, "rotary_table": _exact_table, "rotary": _exact_rotary,
            "distillation": _exact_distill}[case["op"]](s)


def _exact_norm(s):
    f64, d = torch.float64, s["x"].shape[1]
    x, w = s["x"].to(f64), s["w"].to(f64)
    out = {}
    if s["residual"] is not None:
        # the norm is that of the residual stream as it is stored
        out["sum"] = x + s["residual"].to(f64)
        x = out["sum"].to(s["x"].dtype).to(f64)
    mean = x.sum(1) / d
    root = torch.sqrt((x - mean[:, None]).pow(2).sum(1) / d + EPS)
    out["stats"] = torch.stack((mean, 1 / root))
    out["y"] = (x - mean[:, None]) / root[:, None] * w + (0 if s["b"] is None else s["b"].to(f64))
    if s["case"]["backward"]:
        dy = s["dy"].to(f64)
        centred = x - mean[:, None]
        along = (dy * w * centred).sum(1, keepdim=True) / d
        even = (dy * w).sum(1, keepdim=True) / d
        out["dx"] = (dy * w - even) / root[:, None] - centred * along / root[:, None] ** 3
        if s["ds"] is not None:
            out["dx"] = out["dx"] + s["ds"].to(f64)
        out["dw"] = torch.einsum("rd,rd->d", dy, centred / root[:, None])
        if s["b"] is not None:
            out["db"] = dy.sum(0)
    return out


def _exact_table(s):
    c = s["case"]
    n, how, factor = c["part"], c["scaling"], c["factor"]
    freq = []
    for i in range(n // 2):
        base = s["base"] * (factor ** (n / (n - 2)) if how == "base" else 1.0)
        f = math.exp(-2 * i / n * math.log(base))
        if how == "linear":
            f /= factor
        elif how == "parts":
            turns = ORIGINAL * f / math.tau
            if turns <= 1:
                f /= factor
            elif turns < 32:
                share = (turns - 1) / 31
                f = share * f + (1 - share) * f / factor
        freq.append(f)
    at = torch.arange(c["positions"], dtype=torch.float64, device="cuda")
    turned = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                         torch.outer(at, torch.tensor(freq, dtype=torch.float64, device="cuda")))
    return {"cos": turned.real.contiguous(), "sin": turned.imag.contiguous()}


def _exact_rotary(s):
    f64, n = torch.float64, s["case"]["part"]
    at = s["positions"].long()
    turn = torch.complex(s["cos"][at].to(f64), s["sin"][at].to(f64))[:, None, :]

    def through(x, by):
        x = x.to(f64).clone()
        if s["case"]["interleaved"]:
            z = torch.view_as_complex(x[..., :n].reshape(*x.shape[:2], n // 2, 2).contiguous()) * by
            x[..., :n] = torch.view_as_real(z).reshape(*x.shape[:2], n)
        else:
            z = torch.complex(x[..., :n // 2].contiguous(), x[..., n // 2:n].contiguous()) * by
            x[..., :n // 2], x[..., n // 2:n] = z.real, z.imag
        return x

    out = {name: through(s[name], turn) for name in "qk"}
    if s["case"]["backward"]:
        out.update({"d" + name: through(s["d%s_out" % name], turn.conj()) for name in "qk"})
    return out


def _exact_distill(s):
    f64, tau, train = torch.float64, s["case"]["temperature"], s["case"]["backward"]
    x, w = s["x"].to(f64), s["w"].to(f64)
    T, K = s["index"].shape
    loss, lse = torch.zeros(T, dtype=f64, device="cuda"), torch.zeros(T, dtype=f64, device="cuda")
    picked = torch.zeros(T, K, dtype=f64, device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    for r in range(0, T, 1024):
        rows = slice(r, min(T, r + 1024))
        logits = x[rows] @ w.t()
        log_p = torch.log_softmax(logits / tau, 1)
        lse[rows] = torch.logsumexp(logits / tau, 1)
        row, slot = torch.nonzero(s["index"][rows] >= 0, as_tuple=True)
        at = s["index"][rows][row, slot]
        picked[rows][row, slot] = logits[row, at]
        t = torch.full(s["index"][rows].shape, -math.inf, dtype=f64, device="cuda")
        t[row, slot] = s["teacher"][rows][row, slot].to(f64) / tau
        log_q = t[row, slot] - torch.logsumexp(t, 1)[row]
        loss[rows].index_add_(0, row, log_q.exp() * (log_q - log_p[row, at]))
        if train:
            grad = log_p.exp()
            grad.index_put_((row, at), -log_q.exp(), accumulate=True)
            weight = torch.zeros(grad.shape[0], dtype=f64, device="cuda")
            weight[row] = s["dloss"][rows].to(f64)[row] / tau
            grad *= weight[:, None]
            dx[rows] = grad @ w
            dw += grad.t() @ x[rows]
    out = {"loss": loss, "lse": lse, "picked": picked}
    return dict(out, dx=dx, dw=dw) if train else out
