"""The model operators where kernels share memory between steps, where statistics are joined over many tiles,
and where calls come in forms that torch makes by itself; against the definitions in 64 bits."""
import math

import pytest
import torch

from oracle import model_oracle as mo
from test_gpu_model_ops import _check, _normal

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    from paper_1908_04207_amd import model_ops
    return model_ops


def _on_gpu(pairs):
    return {n: tuple(t.cpu() for t in p) for n, p in pairs.items()}


# widths of an odd number of 128-byte steps (32 values in fp32, 64 in bf16), so that the loads under way after the
# last step go to the tile in shared memory that the epilogue uses next
@pytest.mark.parametrize("dtype,rows,width,vocab", [(torch.float32, 300, 96, 100), (torch.float32, 500, 800, 100),
                                                    (torch.float32, 2000, 96, 64), (torch.float32, 200, 32, 100),
                                                    (torch.float32, 3656, 160, 3), (torch.float32, 130, 72, 128),
                                                    (torch.bfloat16, 300, 192, 100), (torch.bfloat16, 500, 64, 100),
                                                    (torch.bfloat16, 3656, 320, 3), (torch.bfloat16, 130, 136, 128)])
def test_cross_entropy_one_tile_of_vocabulary_odd_steps(ops, dtype, rows, width, vocab):
    gen = torch.Generator().manual_seed(rows + width)
    x, w = _normal(gen, rows, width, dtype=dtype).cuda(), _normal(gen, vocab, width, dtype=dtype, sigma=1 / math.sqrt(width)).cuda()
    target = torch.randint(0, vocab, (rows,), generator=gen)
    target[torch.rand(rows, generator=gen) < 0.1] = -1
    target, dloss = target.cuda(), _normal(gen, rows, sigma=0.1).cuda()
    loss, lse = ops.cross_entropy(x, w, target)
    dx, dw = ops.cross_entropy_backward(dloss, x, w, target, lse)
    want = _on_gpu(mo.cross_entropy(x, w, target, dloss))
    for name, t in (("loss", loss), ("lse", lse), ("dx", dx), ("dw", dw)):
        _check(name, t, *want[name])
    for _ in range(5):
        for a, b in zip((dx, dw), ops.cross_entropy_backward(dloss, x, w, target, lse)):
            assert torch.equal(a, b)


def test_second_derivatives_of_the_library_s_own_are_refused(ops):
    from paper_1908_04207_amd import binding as eb
    gen = torch.Generator().manual_seed(2)
    x, w = (_normal(gen, n, 64).cuda().requires_grad_() for n in (20, 30))
    loss = ops.CrossEntropy.apply(x, w, torch.arange(20, device="cuda")).sum()
    grads = torch.autograd.grad(loss, (x, w), create_graph=True)
    with pytest.raises(eb.EagerError, match="second derivatives"):
        (loss + sum(g.square().sum() for g in grads)).backward(retain_graph=True)
    loss.backward()                                      # the graph of the loss itself is still there
    assert torch.equal(x.grad, grads[0]) and torch.equal(w.grad, grads[1])


@pytest.mark.parametrize("n,centre", [(2048, 50), (16384, 50), (16384, 200), (16384, -120)])
def test_attention_statistics_over_many_tiles(ops, n, centre):
    """Rows whose scores lie around `centre` beside rows whose maximum moves in every tile of keys, fp32.  Inputs
    are multiples of 1/16, so the scores (up to 2^11) are exact; what is left is rounding of the result and of the
    logarithm (a unit of each, relative to it), of exponentials, and of a sum whose roundings have random
    signs: 64 E covers 4096 tiles of it.  A factor per tile that is not exactly 1 would add up beyond."""
    gen = torch.Generator().manual_seed(centre)
    D, scale = 64, 0.125
    grid = lambda *s: (torch.randint(-24, 25, s, generator=gen) / 16).float()      # noqa: E731
    q, k, v = grid(n, 1, D) / 2, grid(n, 1, D) / 2, _normal(gen, n, 1, D)
    q = (q * 16).round() / 16
    k = (k * 16).round() / 16
    q[..., 0], k[..., 0] = centre / scale, 1.0
    k[:, 0, 1] = torch.arange(n) * 64 // n / 8                     # a ramp from 0 to 8 that every 32nd row looks at
    q[..., 1] = 0.0
    q[7::32, :, 1] = 16.0
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    out, lse = ops.attention(q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), scale)
    first = n - 256
    later = torch.arange(n, device="cuda") > torch.arange(first, n, device="cuda")[:, None]
    s = (scale * (q[first:, 0].double() @ k[:, 0].double().t())).masked_fill(later, -math.inf)
    want = torch.logsumexp(s, 1)
    off = (lse[0, first:].double() - want).abs()
    assert (off <= 2 * mo.E * want.abs() + 64 * mo.E).all(), float(off.max())
    p = torch.exp(s - want[:, None])
    off = (out[first:, 0].double() - p @ v[:, 0].double()).abs()
    assert (off <= 64 * mo.E * (p @ v[:, 0].double().abs())).all(), float(off.max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(100, 100), (300, 129), (130, 300), (700, 1000), (257, 5003), (300, 40003), (2500, 3001)])
def test_cross_entropy_gradients_of_confident_rows_any_vocabulary(ops, dtype, rows, vocab):
    """Targets that lead by so much that 1 - p is about 1e-4, whatever the number of tiles.  Entries of dl are sums and
    exponentials of their own, good to the logits' error: of width 64 at most 66 E of products that add up to
    about the lead (up to 20), 8e-5 of the entry, in fp32; an entry 1 - p formed from a log-sum-exp in fp32
    would be 5e-3 off.  bf16 inputs: 2^-8 of dl and of the result."""
    gen = torch.Generator().manual_seed(vocab)
    width, lead = 64, math.log(vocab) + 9
    w = _normal(gen, vocab, width, dtype=dtype, sigma=0.02).double()
    target = torch.randint(0, vocab, (rows,), generator=gen)
    x = w[target] * (lead / w[target].square().sum(1, keepdim=True)) + 0.3 * _normal(gen, rows, width).double()
    x, w = x.to(dtype).cuda(), w.to(dtype).cuda()
    target[5], target = -1, target.cuda()
    g = torch.rand(rows, generator=gen).cuda() + 0.1
    lse = ops.cross_entropy(x, w, target)[1]
    dx, dw = ops.cross_entropy_backward(g, x, w, target, lse)
    want = mo.cross_entropy(x, w, target, g)
    for name, t in (("dx", dx), ("dw", dw)):
        off = float((t.double() - want[name][0]).norm() / want[name][0].norm())
        assert off < (1e-4 if dtype == torch.float32 else 2.0 ** -8 + 1e-4), (name, off)


@pytest.mark.parametrize("dtype", DTYPES)
def test_an_error_of_another_call_is_not_an_operator_s(ops, dtype):
    """The runtime keeps the last error of a thread until somebody asks.  One that an unrelated call has left there
    (a device that does not exist) is not reported by any operator as its own, nor taken away."""
    import ctypes
    from paper_1908_04207_amd import binding as eb
    gen = torch.Generator().manual_seed(1)
    T, D = 40, 64
    q, k, v = (_normal(gen, T, h, D, dtype=dtype).cuda() for h in (4, 2, 2))
    w, table, pos = torch.ones(D, dtype=dtype, device="cuda"), torch.ones(T, D // 2, device="cuda"), torch.arange(T, device="cuda").int()
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    out, lse = ops.attention(q, k, v, cu)
    x, target, g = q.flatten(1), torch.arange(T, device="cuda"), torch.ones(T, device="cuda")
    of_loss = {n: ops.cross_entropy(x[:, :64], head, target)[1] for n, head in (("one", k[:, 0]), ("many", torch.cat([x[:, :64]] * 10)))}
    heads = {"one": k[:, 0], "many": torch.cat([x[:, :64]] * 10)}
    many_q, many_k = q.repeat(200, 1, 1), k.repeat(200, 1, 1)
    many_cu = torch.arange(0, 200 * T + 1, T, device="cuda").int()
    many_out, many_lse = ops.attention(many_q, many_k, many_k, many_cu)
    torch.cuda.synchronize()
    hip = ctypes.CDLL(eb.LIB_PATH)                  # the runtime that the library is linked with
    calls = {
        "norm": lambda: ops.qk_norm_rope(q, k, w, w, table, table, pos),
        "norm, gradients": lambda: ops.qk_norm_rope_backward(q, k, q, k, w, w, table, table, pos),
        "attention": lambda: ops.attention(q, k, v, cu),
        "attention, gradients": lambda: ops.attention_backward(q, q, k, v, out, lse, cu),
        "attention, gradients of many": lambda: ops.attention_backward(many_q, many_q, many_k, many_k, many_out, many_lse, many_cu),
        "loss": lambda: ops.cross_entropy(x[:, :64], heads["one"], target)}
    for n, head in heads.items():
        calls["loss, gradients, " + n] = lambda n=n, head=head: ops.cross_entropy_backward(g, x[:, :64], head, target, of_loss[n])
    for call in calls.values():
        call()                                      # what torch allocates is there from here on
    for name, call in calls.items():
        left = hip.hipSetDevice(1 << 20)
        assert left != 0
        try:
            call()
        finally:
            assert hip.hipGetLastError() == left, name
            assert hip.hipGetLastError() == 0
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", DTYPES)
def test_upstream_gradients_off_a_boundary(ops, dtype):
    """Contiguous, but not on 16 bytes: as a part of a flat buffer that other gradients share may be."""
    gen = torch.Generator().manual_seed(5)
    T, D = 50, 64
    q, k, v = (_normal(gen, T, h, D, dtype=dtype).cuda().requires_grad_() for h in (4, 2, 2))
    w, table, pos = torch.ones(D, dtype=dtype, device="cuda"), torch.ones(T, D // 2, device="cuda"), torch.arange(T, device="cuda").int()
    flat = _normal(gen, T * 4 * D + 1, dtype=dtype).cuda()
    up = flat[1:].view(T, 4, D)
    out = ops.Attention.apply(q, k, v, torch.tensor([0, T], dtype=torch.int32, device="cuda"), None)
    for a, b in zip(torch.autograd.grad(out, (q, k, v), up, retain_graph=True), torch.autograd.grad(out, (q, k, v), up.clone())):
        assert torch.equal(a, b)
    out = ops.QKNormRope.apply(q, k, w, w, table, table, pos, 1e-6)
    for a, b in zip(torch.autograd.grad(out, (q, k), (up, up[:, :2]), retain_graph=True),
                    torch.autograd.grad(out, (q, k), (up.clone(), up[:, :2].clone()))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("through", ["module", "ctypes"])
def test_a_lone_token_or_head_of_any_stride(ops, dtype, through, monkeypatch):
    from paper_1908_04207_amd import binding as eb
    gen = torch.Generator().manual_seed(7)
    D = 64
    w, table, pos = torch.ones(D, dtype=dtype, device="cuda"), torch.ones(9, D // 2, device="cuda"), torch.arange(9, device="cuda").int()
    base = _normal(gen, 9, 2, D, dtype=dtype).cuda()
    odd = _normal(gen, 3, 2 * D + 3, dtype=dtype).cuda()
    views = [base[0].expand(1, 2, D),                              # a token out of a row: stride 0
             odd[:1, :2 * D].view(1, 2, D),                        # the first of rows of an odd length
             base[:, 0].as_strided((9, 1, D), (2 * D, 1, 1))]      # a head whose stride is a leftover
    if through == "ctypes":
        monkeypatch.setattr(eb, "_marshal", eb._CtypesOnly)
    for q in views:
        T, H, near = q.shape[0], q.shape[1], q.contiguous().clone()
        cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        out, lse = ops.attention(q, q, q, cu)
        want, lse_n = ops.attention(near, near, near, cu)
        assert torch.equal(out, want) and torch.equal(lse, lse_n)
        for a, b in zip(ops.attention_backward(q, q, q, q, out, lse, cu), ops.attention_backward(near, near, near, near, out, lse, cu)):
            assert torch.equal(a, b)
        rest = w, w, table, table, pos[:T]
        for a, b in zip(ops.qk_norm_rope_backward(q, q, q, q, *rest), ops.qk_norm_rope_backward(near, near, near, near, *rest)):
            assert torch.equal(a, b)
        for a, b in zip(ops.qk_norm_rope(q, q, *rest), ops.qk_norm_rope(near, near, *rest)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,group", [(70000, 4), (66000, 3)])
def test_attention_shared_keys_summed_by_one_workgroup(ops, dtype, T, group):
    """Enough tiles that the heads that share keys are not split into parts (checked with the launch rules on the
    CPU): as with the keys repeated for every head and the gradients added up."""
    gen = torch.Generator().manual_seed(3)
    kv, D = 2, 16
    cu = torch.tensor([0] + [100] * (T // 100), dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
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
        # one rounding of the result and one of each of those that are added here
        bound = mo.U[dtype] * (each.abs().sum(2) * 2.01) + 64 * mo.E * each.abs().sum(2) + 1e-6 * each.abs().amax()
        assert ((got.double() - each.sum(2)).abs() <= bound).all()


@pytest.mark.parametrize("rows,width,vocab,sigma", [(1, 24, 2715, 0.2), (5, 24, 1077, 0.2), (3, 8, 300, 1.0), (2, 40, 4000, 0.02)])
def test_cross_entropy_gradients_of_few_rows_without_favourites(ops, rows, width, vocab, sigma):
    """Rows whose targets have next to no weight, one by one: there p - 1 is as good as a rounding of one, and the sum of the
    others, as far off as their common log-sum-exp, is not."""
    for seed in range(60):
        gen = torch.Generator().manual_seed(seed)
        x, w = _normal(gen, rows, width), _normal(gen, vocab, width, sigma=sigma)
        target, g = torch.randint(0, vocab, (rows,), generator=gen), _normal(gen, rows)
        xd, wd, td, gd = (t.cuda() for t in (x, w, target, g))
        lse = ops.cross_entropy(xd, wd, td)[1]
        want = mo.cross_entropy(x, w, target, g)
        for name, t in zip(("dx", "dw"), ops.cross_entropy_backward(gd, xd, wd, td, lse)):
            _check(f"{name} {seed}", t, *want[name])
