"""The model operators where their launches take another form: every shape of tiles and cut of the backward
pass, many rows, strides whose offsets pass 32 bits, masked rows, graphs, and both ways of handing the
arguments over.  The oracle runs in 64 bits on the GPU here (the sizes are too large for the CPU)."""
import math

import pytest
import torch

from oracle import model_oracle as mo
from test_gpu_model_ops import _attention_inputs, _check, _normal, _run_attention, _table

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


def _on_gpu(pairs):
    return {n: tuple(t.cpu() for t in p) for n, p in pairs.items()}


# rows, width, vocabulary: one shape of tiles or one cut of the gradients each (see eager_model_rules.h)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width,vocab", [(700, 64, 30001),        # large tiles
                                              (4000, 72, 130),         # dw in slices of the rows
                                              (8192, 8, 40003),        # several pieces
                                              (17003, 16, 300),        # rows counted by a kernel of their own
                                              (40, 1024, 2000),        # few rows: narrow tiles, dx in slices
                                              (2100, 328, 4097)])
def test_cross_entropy_cuts(ops, dtype, rows, width, vocab):
    gen = torch.Generator().manual_seed(rows)
    x, w = _normal(gen, rows, width, dtype=dtype).cuda(), _normal(gen, vocab, width, dtype=dtype, sigma=1 / math.sqrt(width)).cuda()
    target = torch.randint(0, vocab, (rows,), generator=gen)
    target[torch.rand(rows, generator=gen) < 0.3] = -1
    target, dloss = target.cuda(), _normal(gen, rows, sigma=0.1).cuda()
    loss, lse = ops.cross_entropy(x, w, target)
    dx, dw = ops.cross_entropy_backward(dloss, x, w, target, lse)
    want = _on_gpu(mo.cross_entropy(x, w, target, dloss))
    for name, t in (("loss", loss), ("lse", lse), ("dx", dx), ("dw", dw)):
        _check(name, t, *want[name])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(300, 500), (20000, 64)])
def test_masked_rows_reach_no_gradient(ops, dtype, rows, vocab):
    """Whatever stands in rows without a target or without a weight."""
    gen = torch.Generator().manual_seed(6)
    width = 64
    x, w = _normal(gen, rows, width, dtype=dtype), _normal(gen, vocab, width, dtype=dtype, sigma=0.1).cuda()
    target, dloss = torch.randint(0, vocab, (rows,), generator=gen), _normal(gen, rows)
    out = torch.rand(rows, generator=gen) < 0.4
    weightless = torch.rand(rows, generator=gen) < 0.2
    target[out] = -100
    dloss[weightless] = 0.0
    left = out | weightless
    clean = x.clone()
    x[out] = float("nan")
    x[weightless] = float("inf")
    dloss[out] = float("nan")
    args = x.cuda(), w, target.cuda()
    lse = ops.cross_entropy(*args)[1]
    dx, dw = ops.cross_entropy_backward(dloss.cuda(), *args, lse)
    assert not dx.cpu()[left].any() and torch.isfinite(dx).all() and torch.isfinite(dw).all()
    lse = ops.cross_entropy(clean.cuda(), *args[1:])[1]
    same = ops.cross_entropy_backward(torch.where(left, 0.0, dloss).cuda(), clean.cuda(), *args[1:], lse)
    assert torch.equal(dx, same[0]) and torch.equal(dw, same[1])
    # a target beyond the vocabulary is not masked: its gradient says so
    target[0], dloss[0] = vocab + 5, 1.0
    dx, dw = ops.cross_entropy_backward(dloss.cuda(), clean.cuda(), w, target.cuda(), lse)
    assert torch.isnan(dx[0]).all() and torch.isnan(dw).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_many_tiles(ops, dtype):
    """Several tiles of queries and keys, the last ones ragged, heads that share keys in parts."""
    q, k, v, dout, cu = _attention_inputs([1100, 7, 515], 6, 2, 128, dtype, 1, 3, 77)
    got = _run_attention(ops, q, k, v, dout, cu)
    want = _on_gpu(mo.attention(q.cuda(), k.cuda(), v.cuda(), cu, 128 ** -0.5, dout.cuda()))
    for name in got:
        _check(name, got[name], *want[name])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,kv", [(64, 6), (64, 2), (40, 2), (128, 6), (128, 3), (104, 1)])
@pytest.mark.parametrize("empty", [0, 120])
def test_attention_backward_in_one_launch_and_in_two(ops, dtype, D, kv, empty):
    """The same sequences with and without many empty ones among them, which give the launches more
    workgroups (all of which find nothing): one launch for all gradients, or one for dq's alone first."""
    q, k, v, dout, cu = _attention_inputs([130] + [0] * empty + [1, 300, 64], 6, kv, D, dtype, 1, 3, 78)
    got = _run_attention(ops, q, k, v, dout, cu)
    want = _on_gpu(mo.attention(q.cuda(), k.cuda(), v.cuda(), cu, D ** -0.5, dout.cuda()))
    for name in got:
        _check(name, got[name], *want[name])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,kv", [(300, 1), (70000, 1)])
def test_attention_parts_agree(ops, dtype, T, kv):
    """Heads that share keys, summed in parts (few tokens) or by one workgroup (many): as with the keys
    repeated for every head and the gradients added up."""
    gen = torch.Generator().manual_seed(1)
    lens = [100] * (T // 100)
    cu = torch.tensor([0] + lens, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
    group, D = 4, 16
    q, dout = (_normal(gen, T, kv * group, D, dtype=dtype).cuda() for _ in range(2))
    k, v = (_normal(gen, T, kv, D, dtype=dtype).cuda() for _ in range(2))
    out, lse = ops.attention(q, k, v, cu)
    dq, dk, dv = ops.attention_backward(dout, q, k, v, out, lse, cu)
    kr, vr = (t.repeat_interleave(group, 1) for t in (k, v))
    out_r, lse_r = ops.attention(q, kr, vr, cu)
    dq_r, dk_r, dv_r = ops.attention_backward(dout, q, kr, vr, out_r, lse_r, cu)
    assert torch.equal(out, out_r) and torch.equal(lse, lse_r) and torch.equal(dq, dq_r)
    for got, each in ((dk, dk_r), (dv, dv_r)):
        each = each.double().view(T, kv, group, D)
        # one rounding of the result and one of each of the four that are added here
        bound = mo.U[dtype] * (each.abs().sum(2) * 2.01) + 64 * mo.E * each.abs().sum(2) + 1e-6 * each.abs().amax()
        assert ((got.double() - each.sum(2)).abs() <= bound).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_beyond_32_bits(ops, dtype):
    """Rows 2^20 elements apart: the last ones begin more than 2^32 bytes after the first."""
    T, far = 2500, 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(3)

    def wide(heads, D):
        base = torch.empty(T, far, dtype=dtype, device="cuda")
        view = base[:, far - heads * D:].view(T, heads, D)
        return view.copy_(torch.randn(T, heads, D, device="cuda", generator=gen))

    q, k, v, dout = wide(2, 64), wide(1, 64), wide(1, 64), wide(2, 64)
    cu = torch.tensor([5, 2300, 2499], dtype=torch.int32, device="cuda")
    out, dq, dk, dv = wide(2, 64), wide(2, 64), wide(1, 64), wide(1, 64)
    _, lse = ops.attention(q, k, v, cu, out=out)
    ops.attention_backward(dout, q, k, v, out, lse, cu, dq=dq, dk=dk, dv=dv)
    near = [t.contiguous() for t in (q, k, v, dout)]
    out_n, lse_n = ops.attention(*near[:3], cu)
    grads_n = ops.attention_backward(near[3], *near[:3], out_n, lse_n, cu)
    for a, b in zip((out, lse, dq, dk, dv), (out_n, lse_n, *grads_n)):
        assert torch.equal(a, b)

    w = torch.ones(64, dtype=dtype, device="cuda")
    cos, sin = (t.cuda() for t in _table(T, 64))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    ops.qk_norm_rope(q, k, w, w, cos, sin, pos, q_out=dq, k_out=dk)
    for a, b in zip((dq, dk), ops.qk_norm_rope(*near[:2], w, w, cos, sin, pos)):
        assert torch.equal(a, b)
    ops.qk_norm_rope_backward(dout, v, q, k, w, w, cos, sin, pos, dq=dq, dk=dk)
    for a, b in zip((dq, dk), ops.qk_norm_rope_backward(near[3], near[2], *near[:2], w, w, cos, sin, pos)):
        assert torch.equal(a, b)

    x, head = q[:, 0], out[:, 1]
    target = torch.randint(0, T, (T,), device="cuda", generator=gen)
    g = torch.rand(T, device="cuda", generator=gen)
    dx, dw = dq[:, 0], dout[:, 1]
    loss, lse = ops.cross_entropy(x, head, target)
    ops.cross_entropy_backward(g, x, head, target, lse, dx=dx, dw=dw)
    xn, hn = x.contiguous(), head.contiguous()
    loss_n, lse_n = ops.cross_entropy(xn, hn, target)
    for a, b in zip((loss, lse, dx, dw), (loss_n, lse_n, *ops.cross_entropy_backward(g, xn, hn, target, lse_n))):
        assert torch.equal(a, b)


def _step(ops, s):
    """One pass through all of it on static buffers."""
    table = s["cos"], s["sin"], s["pos"]
    q, k = ops.qk_norm_rope(s["q"], s["k"], s["w"], s["w"], *table)
    out, lse = ops.attention(q, k, s["v"], s["cu"])
    x = out.flatten(1)
    loss, lse2 = ops.cross_entropy(x, s["head"], s["target"])
    dx, dhead = ops.cross_entropy_backward(s["g"], x, s["head"], s["target"], lse2)
    dq, dk, dv = ops.attention_backward(dx.view_as(out), q, k, s["v"], out, lse, s["cu"])
    return (loss, dhead, dv, *ops.qk_norm_rope_backward(dq, dk, s["q"], s["k"], s["w"], s["w"], *table))


def _state(dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    T = 333
    cos, sin = _table(T, 64)
    s = {"q": _normal(gen, T, 4, 64, dtype=dtype), "k": _normal(gen, T, 2, 64, dtype=dtype), "v": _normal(gen, T, 2, 64, dtype=dtype),
         "w": _normal(gen, 64, dtype=dtype, mean=1.0, sigma=0.1), "head": _normal(gen, 700, 256, dtype=dtype, sigma=0.1),
         "target": torch.randint(-100, 700, (T,), generator=gen), "g": _normal(gen, T), "cos": cos, "sin": sin,
         "pos": torch.randint(0, T, (T,), generator=gen, dtype=torch.int32),
         "cu": torch.tensor([0, 60 + seed, 200, 330], dtype=torch.int32)}
    return {n: t.cuda() for n, t in s.items()}


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_a_graph_replayed_between_eager_work(ops, dtype):
    s = _state(dtype, 0)
    for _ in range(2):
        _step(ops, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _step(ops, s)
    for seed in range(1, 5):
        other = _state(dtype, seed)
        for n in s:
            s[n].copy_(other[n])
        graph.replay()
        torch.cuda.synchronize()
        eager = _step(ops, s)
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(captured, eager)):
            assert torch.equal(a, b), (seed, i)


@pytest.mark.parametrize("dtype", DTYPES)
def test_through_the_module_and_through_ctypes(ops, dtype, monkeypatch):
    """The same bits, and the module does take the usual calls."""
    from paper_1908_04207_amd import binding as eb
    s = _state(dtype, 3)
    _step(ops, s)                                        # from here on the current stream is known
    taken = []

    class Counting:
        def __getattr__(self, name):
            fn = getattr(real, name)

            def call(*args):
                result = fn(*args)
                if name in ("qk_norm_rope", "attention", "cross_entropy"):
                    taken.append(result is not NotImplemented)
                return result
            return call

    real = eb._marshal
    monkeypatch.setattr(eb, "_marshal", Counting())
    through_module = _step(ops, s)
    assert taken == [True] * 6
    monkeypatch.setattr(eb, "_marshal", eb._CtypesOnly)
    for a, b in zip(through_module, _step(ops, s)):
        assert torch.equal(a, b)


def _refused(call, what):
    from paper_1908_04207_amd import binding as eb
    with pytest.raises(eb.EagerError) as e:
        call()
    assert e.value.status == eb.EINVAL and what in str(e.value), str(e.value)


def test_refusals(ops):
    s = _state(torch.bfloat16, 0)
    q, k, v, cu = s["q"], s["k"], s["v"], s["cu"]
    _refused(lambda: ops.attention(q, k, v.float(), cu), "expected")
    _refused(lambda: ops.attention(q, k, v[:, :1], cu), "v:")
    _refused(lambda: ops.attention(q, k[:, :1].expand(-1, 2, -1), v, cu), "eager_attention")    # a broadcast view
    _refused(lambda: ops.attention(q[:, :3], k, v, cu), "eager_attention")                      # 3 heads over 2
    _refused(lambda: ops.attention(q, k, v, cu.long()), "cu_seqlens")
    _refused(lambda: ops.attention(q, k, v, cu[:1]), "cu_seqlens")
    _refused(lambda: ops.attention(q[..., :60], k[..., :60], v[..., :60], cu), "eager_attention")
    _refused(lambda: ops.attention(q, k, v, cu, scale=-1.0), "eager_attention")
    _refused(lambda: ops.attention(q.transpose(1, 2), k, v, cu), "expected")
    _refused(lambda: ops.attention(q[0], k, v, cu), "expected q")
    out, lse = ops.attention(q, k, v, cu)
    _refused(lambda: ops.attention_backward(out, q, k, v, out, lse.t().contiguous(), cu), "lse")
    _refused(lambda: ops.attention_backward(out, q, k, v, out, lse, cu, dk=torch.empty_like(q)), "dk")
    w, table = s["w"], (s["cos"], s["sin"], s["pos"])
    _refused(lambda: ops.qk_norm_rope(q, k, w[:32], w, *table), "wq")
    _refused(lambda: ops.qk_norm_rope(q, k, w, w, s["cos"].double(), s["sin"], s["pos"]), "cos")
    _refused(lambda: ops.qk_norm_rope(q, k, w, w, s["cos"], s["sin"][:5], s["pos"]), "sin")
    _refused(lambda: ops.qk_norm_rope(q, k, w, w, s["cos"], s["sin"], s["pos"].long()), "positions")
    _refused(lambda: ops.qk_norm_rope(q, k, w, w, *table, eps=-1.0), "eager_qk_norm_rope")
    x, head, target = out.flatten(1), s["head"], s["target"]
    _refused(lambda: ops.cross_entropy(x, head[:, :128], target), "expected x")
    _refused(lambda: ops.cross_entropy(x, head, target.int()), "target")
    _refused(lambda: ops.cross_entropy(x, head.float(), target), "expected")
    _refused(lambda: ops.cross_entropy(x[:, :4], head[:, :4], target), "eager_cross_entropy")   # width 4
    loss, lse = ops.cross_entropy(x, head, target)
    _refused(lambda: ops.cross_entropy_backward(loss[:5], x, head, target, lse), "dloss")
    _refused(lambda: ops.cross_entropy_backward(loss, x, head, target, lse, dw=head.t().contiguous().t()), "dw")
    _refused(lambda: ops.cross_entropy_backward(loss, x, head, target, lse, want=(False, False)), "eager_cross_entropy_backward")


@pytest.mark.parametrize("rows,vocab", [(50, 2), (300, 20), (130, 128), (1000, 101)])
def test_cross_entropy_of_confident_rows(ops, rows, vocab):
    """Few classes and targets that lead by 12: losses and 1 - p of about vocab e^-12.  The loss comes from a sum
    of 1 + vocab e^-12 in fp32, so it is good to vocab 2^-24 of a one; dl's entries are sums and
    exponentials of their own, good to the logits' error (|l| 2^-24 times a few tens of products' roundings)
    relative to themselves - and neither loses more to log-sum-exps that are held in fp32."""
    gen = torch.Generator().manual_seed(vocab)
    width = 64
    w = _normal(gen, vocab, width, sigma=0.02).double()
    target = torch.randint(0, vocab, (rows,), generator=gen)
    x = (w[target] * (12 / (w[target].square().sum(1, keepdim=True))) + _normal(gen, rows, width).double()).float().cuda()
    w, target, g = w.float().cuda(), target.cuda(), torch.rand(rows, generator=gen).cuda()
    loss, lse = ops.cross_entropy(x, w, target)
    dx, dw = ops.cross_entropy_backward(g, x, w, target, lse)
    want = mo.cross_entropy(x, w, target, g)
    assert ((loss.double() - want["loss"][0]).abs() <= 4 * vocab * mo.E + 2e-5 * want["loss"][0]).all()
    for name, t in (("dx", dx), ("dw", dw)):
        off = float((t.double() - want[name][0]).norm() / want[name][0].norm())
        assert off < 1e-4, (name, off)
