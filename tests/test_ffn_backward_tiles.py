"""Large tiles of the FFN's backward products, with shared experts and with more experts than lanes: which sizes take them, and what they give."""
import re

import numpy as np
import pytest
import torch

import paper_2509_25041_amd as grace
from test_gpu_gradients import check_grads, normal, swiglu_grads, table_of
from test_launch_limits import PRELUDE, run

SHAPES = {(256, 256): "large", (192, 256): "lower", (128, 128): "medium", (64, 64): "small"}
# (experts, rows, d, f, shared) and the tiles of dh, of the gates, of dx and of the weights' gradients.  Few experts: their row offsets in one register
# of a wavefront, more than 64: in four.
FEW = [
    ((3, 3001, 1032, 1000, True), "lower lower lower large"),
    ((2, 2501, 136, 3000, True), "large large small medium"),
    ((3, 3000, 72, 3800, False), "lower lower small medium"),
    ((16, 1847, 2040, 1016, False), "medium medium lower large"),
    ((1, 4000, 264, 4000, False), "large large small medium"),
]
MANY = [
    ((66, 16000, 136, 1000, False), "lower large lower large"),
    ((65, 20000, 72, 1000, False), "large large medium medium"),
]
CHOICE = PRELUDE + r"""
class Launch(C.Structure):
    _fields_ = [("kernel", C.c_void_p), ("groups", C.c_uint32), ("threads", C.c_uint32), ("lds", C.c_uint64)]
class Info(C.Structure):
    _fields_ = [("file", C.c_char_p), ("base", C.c_void_p), ("symbol", C.c_char_p), ("symbol_at", C.c_void_p)]
dladdr, info = C.CDLL(None).dladdr, Info()
dladdr.argtypes = [C.c_void_p, C.POINTER(Info)]
S, rows, d, f, shared = map(int, sys.argv[3].split())
if shared:
    rc = lib.grace_shared_ffn_backward(at, at, rows, d, f, S, 1, *[at] * 8, None)
else:
    rc = lib.grace_expert_ffn_backward(table(S, 1), 0, at, at, at, rows, 1, d, f, 1, *[at] * 8, None)
assert rc == 0, lib.grace_last_error()
assert recorder.launches_refused() == 0
for launch in (Launch * C.c_int.in_dll(recorder, "n_recorded").value).in_dll(recorder, "recorded"):
    assert dladdr(launch.kernel, C.byref(info))
    print(info.symbol.decode())
"""


@pytest.mark.parametrize("sizes,tiles", FEW + MANY, ids=str)
def test_sizes_take_the_tiles_that_they_are_tested_for(tmp_path, sizes, tiles):
    """The kernels that a call launches, by their names: template arguments are the product, the registers of row offsets, and the tile shapes."""
    names = run(tmp_path, CHOICE, " ".join(str(int(v)) for v in sizes)).split()
    assert len(names) == 3
    taken = []
    for product, name in enumerate(names):
        if product < 2:
            assert "bf16_kernel" in name and f"ProductE{product}E" in name
        else:
            assert "bf16_input_weights_kernel" in name
        assert f"Li{4 if sizes[0] > 64 else 1}ENS" in name
        shapes = [SHAPES[int(m), int(n)] for m, n in re.findall(r"Li(\d+)ELi(\d+)ELi64E", name)]
        taken += shapes if product < 2 else [shapes[0], shapes[-1]]      # (a name holds one shape that is both once)
    assert " ".join(taken) == tiles


def random_inputs(rng, S, rows, d, f):
    bf16 = torch.bfloat16
    return (normal(rng, (rows, d), bf16), normal(rng, (rows, d), bf16),
            (normal(rng, (S, f, d), bf16, d ** -0.5), normal(rng, (S, f, d), bf16, d ** -0.5), normal(rng, (S, d, f), bf16, f ** -0.5)))


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [c for c, _ in FEW if c[4]], ids=str)
def test_shared_ffn_backward_on_large_tiles(sizes):
    """Every expert over all rows, odd rows and widths that end inside a tile; dx sums over the experts' columns one after the other."""
    S, rows, d, f, _ = sizes
    x, dy, w = random_inputs(np.random.default_rng(rows), S, rows, d, f)
    got = grace.grace_shared_ffn_backward(x, dy, *w)
    want = size = 0.0
    for e in range(S):
        grads, sizes = swiglu_grads(x, dy, *(v[e] for v in w))
        want, size = want + grads[0], size + sizes[0]
        check_grads((got[0],) + tuple(v[e] for v in got[1:]), (got[0].double(),) + grads[1:], sizes, torch.bfloat16, f"expert {e}")
    check_grads(got[:1], (want,), (size,), torch.bfloat16, "sum over the experts")
    again = grace.grace_shared_ffn_backward(x, dy, *w)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [c for c, _ in MANY], ids=str)
def test_expert_ffn_backward_of_more_experts_than_lanes_on_large_tiles(sizes):
    """Some experts without rows, some that end at a tile's edge and beside it, one with many."""
    S, rows, d, f, _ = sizes
    rng = np.random.default_rng(rows)
    some = [0, 1, 191, 192, 193, 255, 256, 257, 0, 0, 64, 384, 512, 7] + list(rng.integers(0, 300, S - 15))
    edges = np.concatenate([[0], np.cumsum(some)])
    edges = np.append(np.minimum(edges, rows - 100), rows).astype(np.int32)      # the last expert has the rest
    x, dy, w = random_inputs(rng, S, rows, d, f)
    got = grace.grace_expert_ffn_backward(table_of([S]), 0, x, dy, torch.from_numpy(edges).cuda(), rows, 1, *w)
    for e, (a, b) in enumerate(zip(edges, edges[1:])):
        mine = (got[0][a:b],) + tuple(v[e] for v in got[1:])
        if a == b:
            assert all(bool((v == 0).all()) for v in mine[1:]), e
            continue
        check_grads(mine, *swiglu_grads(x[a:b], dy[a:b], *(v[e] for v in w)), torch.bfloat16, f"expert {e}")
