"""The model operators' host side without a GPU: the header from plain C, what is refused before any
launch, workspace sizes, and the rules that cut a backward pass into pieces."""
import ctypes
import itertools
import os
import subprocess

import pytest

from paper_1908_04207_amd import binding as eb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000                      # an aligned address that is never read


def test_header_is_plain_c(tmp_path):
    exe = tmp_path / "model_header"
    lib_dir = os.path.dirname(eb.LIB_PATH)
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                           os.path.join(ROOT, "tests", "c", "model_header_is_plain_c.c"), "-o", str(exe), "-L", lib_dir,
                           "-leager", "-Wl,-rpath," + lib_dir])
    assert subprocess.run([str(exe)]).returncode == 0


def test_rules_on_the_cpu(tmp_path):
    """Pieces cover the vocabulary, slices and parts divide what they should, workspaces hold what the
    layout says, under AddressSanitizer and UndefinedBehaviorSanitizer."""
    exe = tmp_path / "model_rules"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-static-libasan", "-Wall", "-Wextra", "-Werror",
                           os.path.join(ROOT, "tests", "c", "model_rules_host.cpp"), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout[-500:], r.stderr[-2000:])


def _refused(call):
    with pytest.raises(eb.EagerError) as e:
        call()
    assert e.value.status == eb.EINVAL


SHAPES = [dict(tokens=-1), dict(tokens=2 ** 31 - 2 ** 15), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=6, kv_heads=4),
          dict(head_dim=4), dict(head_dim=12), dict(head_dim=136)]


def _shape(**kw):
    return eb.Packed(**{**dict(tokens=10, q_heads=4, kv_heads=2, head_dim=64, sequences=2, cu_seqlens=A), **kw})


def _heads(**kw):
    return eb.Heads(**{**dict(data=A, row_stride=256, head_stride=64), **kw})


VIEWS = [None, dict(data=None), dict(data=A + 8), dict(row_stride=0), dict(row_stride=260 + 1), dict(head_stride=0),
         dict(head_stride=66), dict(row_stride=2 ** 22), dict(row_stride=-256)]


@pytest.mark.parametrize("dtype", [eb.F32, eb.BF16])
def test_attention_refusals(dtype):
    def forward(dtype=dtype, shape=_shape(), q=_heads(), k=_heads(), v=_heads(), scale=0.1, out=_heads(), lse=A):
        eb.eager_attention(dtype, shape, q, k, v, scale, out, lse, stream=0)

    def backward(dtype=dtype, shape=_shape(), q=_heads(), k=_heads(), v=_heads(), out=_heads(), lse=A, dout=_heads(),
                 scale=0.1, dq=_heads(), dk=_heads(), dv=_heads(), workspace=A, workspace_bytes=1 << 30):
        eb.eager_attention_backward(dtype, shape, q, k, v, out, lse, dout, scale, dq, dk, dv, workspace, workspace_bytes, stream=0)

    for call in (forward, backward):
        _refused(lambda: call(dtype=2))
        _refused(lambda: call(shape=None))
        for bad in SHAPES + [dict(sequences=0), dict(sequences=-1), dict(cu_seqlens=None), dict(cu_seqlens=A + 2),
                             dict(tokens=2 ** 31 - 2 ** 16, q_heads=1 << 20, kv_heads=1)]:
            _refused(lambda: call(shape=_shape(**bad)))
        for scale in (0.0, -1.0, float("nan"), float("inf")):
            _refused(lambda: call(scale=scale))
        _refused(lambda: call(lse=None))
        _refused(lambda: call(lse=A + 1))
    for name, bad in itertools.product(("q", "k", "v", "out"), VIEWS):
        _refused(lambda: forward(**{name: bad and _heads(**bad)}))
    for name, bad in itertools.product(("q", "k", "v", "out", "dout", "dq", "dk", "dv"), VIEWS):
        _refused(lambda: backward(**{name: bad and _heads(**bad)}))
    need = eb.eager_attention_workspace_bytes(dtype, _shape())
    for kw in (dict(workspace=None), dict(workspace=A + 8), dict(workspace_bytes=need - 1), dict(workspace_bytes=-1)):
        _refused(lambda: backward(**kw))
    forward(shape=_shape(tokens=0), q=_heads(data=None), k=_heads(data=None), v=_heads(data=None), out=_heads(data=None), lse=None)


@pytest.mark.parametrize("dtype", [eb.F32, eb.BF16])
def test_qk_norm_rope_refusals(dtype):
    def rot(**kw):
        return eb.Rotation(**{**dict(cos_table=A, sin_table=A, positions=A, table_rows=8), **kw})

    def forward(dtype=dtype, shape=_shape(), q=_heads(), k=_heads(), wq=A, wk=A, rotation=rot(), eps=1e-6, q_out=_heads(),
                k_out=_heads()):
        eb.eager_qk_norm_rope(dtype, shape, q, k, wq, wk, rotation, eps, q_out, k_out, stream=0)

    def backward(dtype=dtype, shape=_shape(), dq_out=_heads(), dk_out=_heads(), q=_heads(), k=_heads(), wq=A, wk=A,
                 rotation=rot(), eps=1e-6, dq=_heads(), dk=_heads(), dwq=A, dwk=A, workspace=A, workspace_bytes=1 << 30):
        eb.eager_qk_norm_rope_backward(dtype, shape, dq_out, dk_out, q, k, wq, wk, rotation, eps, dq, dk, dwq, dwk, workspace,
                                       workspace_bytes, stream=0)

    for call in (forward, backward):
        _refused(lambda: call(dtype=-1))
        for bad in SHAPES:
            _refused(lambda: call(shape=_shape(**bad)))
        for eps in (-1e-6, float("nan"), float("inf")):
            _refused(lambda: call(eps=eps))
        for bad in (None, rot(cos_table=None), rot(sin_table=A + 4), rot(positions=None), rot(table_rows=0)):
            _refused(lambda: call(rotation=bad))
        for name in ("wq", "wk"):
            _refused(lambda: call(**{name: None}))
            _refused(lambda: call(**{name: A + 2}))
    for name, bad in itertools.product(("q", "k", "q_out", "k_out"), VIEWS):
        _refused(lambda: forward(**{name: bad and _heads(**bad)}))
    for name, bad in itertools.product(("dq_out", "dk_out", "q", "k", "dq", "dk"), VIEWS):
        _refused(lambda: backward(**{name: bad and _heads(**bad)}))
    need = eb.eager_qk_norm_rope_workspace_bytes(dtype, _shape())
    for kw in (dict(dwq=None), dict(dwk=None), dict(workspace=None), dict(workspace_bytes=need - 1)):
        _refused(lambda: backward(**kw))


@pytest.mark.parametrize("dtype", [eb.F32, eb.BF16])
def test_cross_entropy_refusals(dtype):
    def shape(**kw):
        return eb.Projection(**{**dict(rows=4, width=64, vocab=100, x_stride=64, w_stride=64), **kw})

    def forward(dtype=dtype, shape=shape(), x=A, w=A, target=A, loss=A, lse=A, workspace=A, workspace_bytes=1 << 30):
        eb.eager_cross_entropy(dtype, shape, x, w, target, loss, lse, workspace, workspace_bytes, stream=0)

    def backward(dtype=dtype, shape=shape(), x=A, w=A, target=A, lse=A, dloss=A, dx=A, dw=A, workspace=A, workspace_bytes=1 << 40):
        eb.eager_cross_entropy_backward(dtype, shape, x, w, target, lse, dloss, dx, dw, workspace, workspace_bytes, stream=0)

    for call, backward_too in ((forward, False), (backward, True)):
        _refused(lambda: call(dtype=7))
        _refused(lambda: call(shape=None))
        for bad in (dict(rows=-1), dict(width=0), dict(width=60), dict(vocab=0), dict(x_stride=56), dict(w_stride=66),
                    dict(w_stride=2 ** 22), dict(x_stride=0), dict(rows=2 ** 31 - 2 ** 15), dict(rows=1 << 30, vocab=1 << 30)):
            _refused(lambda: call(shape=shape(**bad)))
        for name in ("x", "w", "target", "lse", "workspace"):
            _refused(lambda: call(**{name: None}))
            _refused(lambda: call(**{name: A + 2}))
        need = eb.eager_cross_entropy_workspace_bytes(dtype, shape(), backward_too)
        _refused(lambda: call(workspace_bytes=need - 1))
    _refused(lambda: forward(loss=None))
    _refused(lambda: backward(dloss=None))
    _refused(lambda: backward(dx=None, dw=None))
    _refused(lambda: backward(dx=A + 8))
    _refused(lambda: backward(dw=A + 8))
    forward(shape=shape(rows=0), x=None, target=None, loss=None, lse=None)


def test_workspace_queries_refuse_too():
    n = ctypes.c_int64()
    lib = eb.lib
    assert lib.eager_attention_workspace_bytes(eb.F32, _shape(), None) == eb.EINVAL
    assert lib.eager_attention_workspace_bytes(5, _shape(), ctypes.byref(n)) == eb.EINVAL
    assert lib.eager_qk_norm_rope_workspace_bytes(eb.F32, _shape(head_dim=7), ctypes.byref(n)) == eb.EINVAL
    assert lib.eager_cross_entropy_workspace_bytes(eb.F32, eb.Projection(1, 8, 1, 8, 8), 2, ctypes.byref(n)) == eb.EINVAL
    for rows in (0, 1, 5, 1 << 20):
        assert lib.eager_cross_entropy_workspace_bytes(eb.F32, eb.Projection(rows, 8, 1, 8, 8), 1, ctypes.byref(n)) == eb.OK
        assert n.value > 0


def test_tensors_off_the_gpu_are_refused():
    import torch
    from paper_1908_04207_amd import model_ops as ops
    q, k, cu = torch.zeros(3, 2, 64), torch.zeros(3, 1, 64), torch.tensor([0, 3], dtype=torch.int32)
    w, pos, table = torch.ones(64), torch.zeros(3, dtype=torch.int32), torch.zeros(4, 32)
    _refused(lambda: ops.attention(q, k, k, cu))
    _refused(lambda: ops.qk_norm_rope(q, k, w, w, table, table, pos))
    _refused(lambda: ops.cross_entropy(torch.zeros(3, 64), torch.zeros(5, 64), torch.zeros(3, dtype=torch.int64)))
    _refused(lambda: ops.attention(q.double(), k.double(), k.double(), cu))


def test_the_stride_of_a_lone_token_or_head_counts_nothing():
    """Nothing is stepped over there, and torch may give it any stride."""
    import torch
    for t in (torch.zeros(2, 64).expand(1, 2, 64), torch.zeros(5, 64)[:, None], torch.zeros(64).expand(1, 1, 64),
              torch.zeros(1, 2, 3 << 21)[:, :, :64], torch.zeros(3, 1, 64).as_strided((3, 1, 64), (64, 1, 1))):
        h = eb.heads(t)
        assert h.data == t.data_ptr()
        assert h.row_stride == (t.stride(0) if t.shape[0] > 1 else 64)
        assert h.head_stride == (t.stride(1) if t.shape[1] > 1 else 64)
    assert eb.heads(torch.zeros(3, 64)[:, None].expand(3, 2, 64)).head_stride == 0       # a broadcast view: refused later


def test_places_in_tiles_on_the_cpu(tmp_path):
    """The chunks of a tile's rows have places of their own, by arithmetic that stays in its types (under
    UndefinedBehaviorSanitizer)."""
    exe = tmp_path / "model_tiles"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-static-libasan", "-Wall", "-Wextra", "-Werror",
                           os.path.join(ROOT, "tests", "c", "model_tiles_host.cpp"), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout[-500:], r.stderr[-2000:])


@pytest.mark.parametrize("dtype", [eb.F32, eb.BF16])
def test_scales_that_leave_the_range_of_fp32_are_refused(dtype):
    """lse / scale and scale * log2(e) have to be numbers: log-sum-exps of 2^31 equal scores reach 21.5, and 21.5 / 6e-38 is
    none (keys' gradients would be zeros)."""
    none = _heads(data=None)

    def forward(scale):
        eb.eager_attention(dtype, _shape(tokens=0), none, none, none, scale, none, None, stream=0)

    def backward(scale):
        eb.eager_attention_backward(dtype, _shape(tokens=0), none, none, none, none, None, none, scale, none, none, none, A, 1 << 30, stream=0)

    for call in (forward, backward):
        for scale in (1e-38, 1e-45, 2.0 ** -121, 2.0 ** 121, 3e38):
            _refused(lambda: call(scale))
        for scale in (2.0 ** -120, 1e-6, 1.0, 2.0 ** 120):
            call(scale)
