"""Gradient calls whose buffers are the same memory: what the header allows is right, what it does not is refused."""
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2509_25041_amd as grace
from paper_2509_25041_amd import asm_hazards
from test_launch_limits import HERE, PRELUDE, run

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


# ---- clipping: (gradient, output, elements) of fp32 tensors, as offsets in bytes
OVERLAPS = {
    "one gradient twice, in place": [(0, 0, 64), (0, 0, 64)],
    "views of one another, in place": [(0, 0, 64), (128, 128, 64)],
    "one inside the other, in place": [(0, 0, 1000), (400, 400, 2)],
    "an output over another gradient": [(0, 4096, 64), (4100, 8192, 64)],
    "an output over a later gradient that is in place": [(0, 4096, 64), (4096, 4096, 64)],
    "two outputs": [(0, 4096, 64), (512, 4096 + 252, 64)],
    "one output twice": [(0, 4096, 64), (512, 4096, 64)],
    "an output over its own gradient in part": [(0, 128, 64)],
    "far apart in the list": [(0, 0, 64)] + [(1024 * i, 1024 * i, 128) for i in range(1, 200)] + [(4, 4, 1)],
    "the norm": [(0, 0, 64), (1 << 29, 1 << 29, 4)],
    "the norm, in an output": [(0, (1 << 29) - 252, 64)],
    "the workspace": [(0, 0, 64), ((1 << 30) + 16376, (1 << 30) + 16376, 1)],
}
APART = {
    "in place": [(0, 0, 64), (256, 256, 64)],
    "neighbours": [(256, 0, 64), (512, 768, 64)],
    "one gradient twice, with outputs of its own": [(0, 4096, 64), (0, 8192, 64), (128, 12288, 64)],
    "nothing in one of them": [(0, 0, 64), (0, 0, 0), (4, 4, 0)],
    "many": [(1024 * i, 1024 * i, 256) for i in range(300)],
    "right ahead of the norm and the workspace": [((1 << 29) - 256, (1 << 29) - 256, 64), ((1 << 29) + 4, (1 << 29) + 4, 1), ((1 << 30) - 4, (1 << 30) - 4, 1)],
}
CLIP = PRELUDE + r"""
sys.path.insert(0, sys.argv[3])
from test_gradients_aliasing import APART, OVERLAPS
base = 1 << 20
lib.grace_clip_grad_norm.argtypes = [C.c_void_p] * 3 + [i32, C.c_float] + [C.c_void_p] * 4
lib.grace_clip_grads.argtypes = [C.c_void_p] * 3 + [i32, C.c_void_p, C.c_float] + [C.c_void_p] * 2
for cases in (OVERLAPS, APART):
    for name, tensors in cases.items():
        n = len(tensors)
        grads, out = ((C.c_void_p * n)(*[base + t[i] for t in tensors]) for i in (0, 1))
        numel, dtypes = (C.c_int64 * n)(*[t[2] for t in tensors]), (i32 * n)()
        norm, ws = base + (1 << 29), base + (1 << 30)
        C.c_int.in_dll(recorder, "n_recorded").value = 0
        rc = [lib.grace_clip_grad_norm(grads, numel, dtypes, n, 1.0, out, norm, ws, None)]
        rc.append(lib.grace_clip_grads(grads, numel, dtypes, n, norm, 1.0, out, None))
        print(cases is APART, *rc, C.c_int.in_dll(recorder, "n_recorded").value, name, lib.grace_last_error().decode(), sep="|")
"""


def test_clipping_refuses_memory_that_is_written_and_used_twice(tmp_path):
    """Workgroups would scale the same values in any order.  Gradients that are only read may overlap."""
    lines = [line.split("|") for line in run(tmp_path, CLIP, HERE).splitlines()]
    assert len(lines) == len(OVERLAPS) + len(APART)
    for apart, joint, scaling, launches, name, said in lines:
        if apart == "True":
            assert (joint, scaling) == ("0", "0") and int(launches) >= 3, (name, said)
        elif name == "the workspace":                  # (the scaling alone has none)
            assert joint == "-1" and scaling == "0", name
        else:
            assert (joint, scaling, launches) == ("-1", "-1", "0") and "overlaps" in said, (name, said)


@pytest.mark.gpu
def test_clipping_of_a_gradient_that_is_in_the_list_twice():
    """In place it is refused and left as it was; into outputs of their own both are what one would be, and both count towards the norm."""
    rng = np.random.default_rng(1)
    for dtype in DTYPES.values():
        g, other = normal(rng, (70001,), dtype), normal(rng, (33,), dtype)
        kept = g.clone()
        norm = torch.empty((), device="cuda")
        for again in (g, g[1:], g.view(-1)[5:9]):
            with pytest.raises(grace.GraceError, match="overlaps"):
                grace.grace_clip_grad_norm([g, other, again], 0.5, norm=norm)
            with pytest.raises(grace.GraceError, match="overlaps"):
                grace.grace_clip_grads([g, other, again], torch.ones((), device="cuda"), 0.5)
        assert torch.equal(g, kept)
        out = [torch.empty_like(v) for v in (g, other, g)]
        grace.grace_clip_grad_norm([g, other, g], 0.5, out, norm)
        want = (2 * g.double().square().sum() + other.double().square().sum()).sqrt().item()
        assert abs(norm.item() / want - 1) < 2.0 ** -22
        assert torch.equal(out[0], out[2]) and torch.equal(g, kept)
        off = (out[0].double() - g.double() * (0.5 / want)).abs()
        assert bool((off <= g.double().abs() * (0.5 / want) * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -21) * 1.01).all())
