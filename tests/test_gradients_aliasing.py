"""Gradient calls whose buffers are the same memory: what the header allows is right, what it does not is refused."""
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2509_25041_amd as grace
from paper_2509_25041_amd import asm_hazards

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def kernel_parameters(source, kernel):
    """Of each instance of the kernel its parameters as the compiler takes them, with their attributes."""
    done = subprocess.run(["hipcc", "-O3", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                           "-I", os.path.join(asm_hazards.ROOT, "include"), "-I", asm_hazards.CSRC, "-S", "-emit-llvm", "--cuda-device-only",
                           os.path.join(asm_hazards.CSRC, source), "-o", "-"], check=True, stdout=subprocess.PIPE, stderr=subprocess.DEVNULL, text=True)
    lists = re.findall(rf"^define [^\n]*amdgpu_kernel[^\n]*@\w*{kernel}\w*\((.*?)\) local_unnamed_addr", done.stdout, re.M)
    return [re.split(r", (?=ptr|i32|i64)", line) for line in lists]


def test_buffers_that_may_be_the_same_are_not_taken_to_be_apart():
    """dy may be y, dx may be dx_shared: without a promise that they are apart the compiler keeps a row's loads ahead of its stores."""
    combine, permute = (kernel_parameters("rows_backward.hip", name) for name in ("combine_backward_kernel", "permute_backward_kernel"))
    assert len(combine) == 4 and len(permute) == 2
    for parameters, same in [(p, (1, 10)) for p in combine] + [(p, (8, 9)) for p in permute]:
        assert "noalias" in parameters[0]                   # (the attribute is there to be found)
        for i in same:
            assert parameters[i].startswith("ptr") and "noalias" not in parameters[i], (i, parameters[i])


def normal(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vectors", [1, 63, 64, 65, 200, 256, 257, 700])      # of 16 bytes a row: one and four a lane, and several rounds of four
@pytest.mark.parametrize("T,k", [(37, 4), (5, 70)])
def test_rows_backward_in_place(T, k, vectors, dtype):
    """The same bits as with buffers of their own."""
    rng = np.random.default_rng(vectors + k)
    dt = DTYPES[dtype]
    d = vectors * (8 if dtype == "bf16" else 4)
    pos = torch.from_numpy(rng.permutation(T * k).astype(np.int32)).cuda()
    y, dout, w = normal(rng, (T * k, d), dt), normal(rng, (T, d), dt), torch.rand((T, k), device="cuda")
    dy, dw = grace.grace_combine_backward(dout, y, pos, w)
    over = y.clone()
    _, dw_over = grace.grace_combine_backward(dout, over, pos, w, dy=over)
    assert torch.equal(over, dy) and torch.equal(dw_over, dw)
    more = normal(rng, (T, d), dt)
    dx = grace.grace_permute_backward(y, pos, k, more)
    assert torch.equal(grace.grace_permute_backward(y, pos, k, more, dx=more), dx)
