"""Tables that begin on 16 bytes and on no larger boundary, as a part of a buffer does: what a table of its own gives."""
import os
import re
import subprocess

import pytest
import torch

from test_gpu_model_ops import _normal, _table

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FLAGS = ["--offload-arch=gfx950", "-O1", "-std=c++17", "-ffp-contract=off", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", "-x", "hip", "--cuda-device-only", "-S", "-emit-llvm"]


@pytest.mark.parametrize("source", ["eager_rotary.hip", "eager_norm_rope.hip", "eager_layer_norm.hip"])
def test_what_the_compiler_is_told(source, tmp_path):
    """No load from or store to global memory is said to be on more than 16 bytes, which is what the calls check."""
    out = tmp_path / "device.ll"
    subprocess.check_call(["/opt/rocm/bin/hipcc", *FLAGS, os.path.join(ROOT, "paper_1908_04207_amd", "csrc", source), "-o", str(out)])
    over = [line for line in out.read_text().splitlines()
            if re.search(r"\b(load|store)\b.*(ptr addrspace\(1\)|ptr %)", line) and int((re.search(r"align (\d+)", line) or [0, 0])[1]) > 16]
    assert not over, over[:4]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("part", [16, 40, 64, 128])
def test_tables_on_16_bytes(dtype, interleaved, part):
    from paper_1908_04207_amd import model_ops as ops
    gen = torch.Generator().manual_seed(part)
    T, rows = 70, 90
    q, k = _normal(gen, T, 4, 128, dtype=dtype).cuda(), _normal(gen, T, 2, 128, dtype=dtype).cuda()
    pos = torch.randint(0, rows, (T,), generator=gen, dtype=torch.int32).cuda()
    own = [t.cuda() for t in _table(rows, part)]
    parts = []
    for n, t in zip((4, 12), own):
        buffer = torch.empty(t.numel() + 16, device="cuda")
        at = buffer[n:n + t.numel()].view(t.shape)
        assert at.data_ptr() % 32 == 16
        parts.append(at.copy_(t))
    for call in (ops.rotary, ops.rotary_backward):
        for a, b in zip(call(q, k, *own, pos, interleaved), call(q, k, *parts, pos, interleaved)):
            assert torch.equal(a, b)
    # made there as well
    into = [torch.empty(rows * part // 2 + 16, device="cuda")[4:4 + rows * part // 2].view(rows, part // 2) for _ in range(2)]
    for a, b in zip(ops.rotary_table(rows, part), ops.rotary_table(rows, part, cos=into[0], sin=into[1])):
        assert torch.equal(a, b)
    if part == 128:
        w = torch.ones(128, dtype=dtype, device="cuda")
        for a, b in zip(ops.qk_norm_rope(q, k, w, w, *own, pos), ops.qk_norm_rope(q, k, w, w, *parts, pos)):
            assert torch.equal(a, b)
