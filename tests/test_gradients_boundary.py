"""What the gradient calls refuse, on the host: nothing is launched, the status says why."""
import ctypes as C

import pytest
import torch

import paper_2509_25041_amd as grace
from paper_2509_25041_amd import asm_hazards, binding

AT, ODD = 1 << 20, (1 << 20) + 2   # (nothing is behind the device addresses)
F32, BF16 = grace.GRACE_F32, grace.GRACE_BF16
OK, EINVAL, ESHAPE = 0, -1, -2


@pytest.fixture(scope="module")
def lib():
    return grace.load_library()


@pytest.mark.parametrize("over,status", [
    (dict(T=-1), EINVAL), (dict(k=0), EINVAL), (dict(d=0), EINVAL), (dict(dt=7), EINVAL), (dict(d=12), ESHAPE), (dict(d=3, dt=F32), ESHAPE),
    (dict(T=1 << 30, k=4), ESHAPE), (dict(d=1 << 30), ESHAPE), (dict(T=1 << 28, k=1, d=4096), ESHAPE), (dict(rank=-1, off=AT), EINVAL),
    (dict(rank=5000, off=AT), EINVAL), (dict(a=None), EINVAL), (dict(b=None), EINVAL), (dict(pos=None), EINVAL), (dict(out=None), EINVAL),
    (dict(a=ODD), EINVAL), (dict(out=ODD), EINVAL), (dict(T=0, a=None, b=None, pos=None, out=None), OK)])
def test_rows_backward_refusals(lib, over, status):
    c = dict(T=4, k=2, d=64, dt=BF16, off=None, rank=0, a=AT, b=AT, pos=AT, out=AT)
    c.update(over)
    if "b" not in over or c["T"] == 0:
        got = lib.grace_permute_backward(c["a"], c["pos"], c["T"], c["k"], c["d"], c["dt"], c["off"], c["rank"], None, c["out"], None)
        if not (status == ESHAPE and c["T"] == 1 << 28):    # (as many wavefronts as a launch takes: rows of a piece more)
            assert got == status
    if c["T"] != 1 << 28:
        assert lib.grace_combine_backward(c["a"], c["b"], c["pos"], AT, c["T"], c["k"], c["d"], c["dt"], c["off"], c["rank"], c["out"], AT,
                                          None) == status
    if status != OK:
        assert grace.grace_last_error() != ""


@pytest.mark.parametrize("over,status", [
    (dict(T=-1), EINVAL), (dict(E=0), EINVAL), (dict(k=0), EINVAL), (dict(E=257), ESHAPE), (dict(k=9), ESHAPE), (dict(E=200, k=65), ESHAPE),
    (dict(T=1 << 30), ESHAPE), (dict(logits=None), EINVAL), (dict(out=None), EINVAL), (dict(T=0, logits=None, out=None), OK)])
def test_route_backward_refusals(lib, over, status):
    c = dict(T=4, E=8, k=2, logits=AT, out=AT)
    c.update(over)
    assert lib.grace_route_backward(c["logits"], AT, AT, AT, c["T"], c["E"], c["k"], 1, c["out"], None) == status


@pytest.mark.parametrize("over,status", [
    (dict(T=-1), EINVAL), (dict(n=0), EINVAL), (dict(d=0), EINVAL), (dict(f=-8), EINVAL), (dict(dt=2), EINVAL), (dict(d=12), ESHAPE),
    (dict(f=20), ESHAPE), (dict(d=(1 << 20) + 8), ESHAPE), (dict(n=2, f=1 << 20), ESHAPE), (dict(x=None), EINVAL), (dict(w=None), EINVAL),
    (dict(ws=None), EINVAL), (dict(x=ODD), EINVAL), (dict(w=ODD), EINVAL), (dict(T=1 << 30, d=1 << 20), ESHAPE)])
def test_shared_ffn_backward_refusals(lib, over, status):
    c = dict(T=4, d=64, f=64, n=1, dt=BF16, x=AT, w=AT, ws=AT)
    c.update(over)
    assert lib.grace_shared_ffn_backward(c["x"], AT, c["T"], c["d"], c["f"], c["n"], c["dt"], c["w"], AT, AT, AT, AT, AT, AT, c["ws"],
                                         None) == status


def test_expert_ffn_backward_refusals(lib):
    call = lambda table, rank=0, T=4: lib.grace_expert_ffn_backward(table, rank, AT, AT, AT, T, 1, 64, 64, BF16, AT, AT, AT, AT, AT, AT, AT, AT, None)
    assert call(None) == EINVAL


def test_workspace_sizes():
    size = grace.grace_ffn_backward_workspace_bytes
    assert size(-1, 8, 8) == size(1, 0, 8) == size(1, 8, 0) == size(1, 8, 8, -1) == size(1, 8, 8, 0, 9) == 0
    assert size(0, 8, 8) > 0
    assert size(1000, 64, 128, 0, BF16) >= 3 * 1000 * 128 * 2 and size(1000, 64, 128, 3, F32) >= 3 * 1000 * 128 * 3 * 4
    assert size(1 << 20, 64, 1 << 14) >= 3 << 35                       # past 32 bits
    norm = grace.grace_grad_norm_workspace_bytes
    assert norm(-1) == 0 and 0 < norm(0) <= norm(1) <= norm(1000)


def test_clip_refusals(lib):
    def arrays(ptrs, numel, dtypes):
        n = len(ptrs)
        return (C.c_void_p * n)(*ptrs), (C.c_int64 * n)(*numel), (C.c_int32 * n)(*dtypes), n

    def clip(ptrs=(AT,), numel=(8,), dtypes=(F32,), out=None, max_norm=1.0, norm=AT, ws=AT):
        a = arrays(ptrs, numel, dtypes)
        dst = a[0] if out is None else (C.c_void_p * len(out))(*out)
        first = lib.grace_clip_grad_norm(*a, max_norm, dst, norm, ws, None)
        if ws:
            assert lib.grace_clip_grads(*a, norm, max_norm, dst, None) == first
        return first

    assert clip(numel=(-1,)) == clip(dtypes=(5,)) == clip(ptrs=(None,)) == clip(ptrs=(ODD,)) == clip(ptrs=(AT + 1,), dtypes=(BF16,)) == EINVAL
    assert clip(max_norm=-1.0) == clip(max_norm=float("nan")) == clip(max_norm=float("inf")) == clip(norm=None) == clip(ws=None) == EINVAL
    assert clip(out=(None,)) == clip(out=(AT + 2,)) == clip(out=(AT + 16,)) == clip(out=(AT - 16,)) == EINVAL      # overlaps in part
    assert lib.grace_grad_norm(None, None, None, 1, AT, AT, None) == EINVAL
    assert lib.grace_grad_norm(None, None, None, -1, AT, AT, None) == EINVAL
    assert lib.grace_clip_grad_norm(*arrays((AT,), (1 << 41,), (BF16,)), 1.0, (C.c_void_p * 1)(AT), AT, AT, None) == EINVAL


@pytest.mark.parametrize("native", [True, False])
def test_binding_refuses_shapes_before_the_library_sees_them(native, monkeypatch):
    if not native:
        monkeypatch.setattr(binding, "_calls", False)     # through Python, as where the native calls cannot be built
    elif not binding._native():
        pytest.skip("no native calls here")
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
    i32 = lambda *shape: z(*shape, dtype=torch.int32)
    with pytest.raises(ValueError, match="dout"):
        grace.grace_combine_backward(z(3, 8), z(8, 8), i32(8), z(4, 2))
    with pytest.raises(ValueError, match="perm_pos"):
        grace.grace_combine_backward(z(4, 8), z(8, 8), i32(7), z(4, 2))
    with pytest.raises(ValueError, match="dy"):
        grace.grace_combine_backward(z(4, 8), z(8, 8), i32(8), z(4, 2), dy=z(8, 4))
    with pytest.raises(ValueError, match="multiple of k"):
        grace.grace_permute_backward(z(7, 8), i32(7), 2)
    with pytest.raises(ValueError, match="dx_shared"):
        grace.grace_permute_backward(z(8, 8), i32(8), 2, z(3, 8))
    with pytest.raises(ValueError, match="rank=2"):
        grace.grace_permute_backward(z(8, 8), i32(8), 2, None, i32(3), 2, z(4, 8))
    with pytest.raises(ValueError, match="topk_expert"):
        grace.grace_route_backward(z(4, 8), i32(3, 2), z(4, 2), z(4, 2))
    with pytest.raises(ValueError, match="dtopk_weight"):
        grace.grace_route_backward(z(4, 8), i32(4, 2), z(4, 2), z(4, 3))
    with pytest.raises(ValueError, match="weights"):
        grace.grace_shared_ffn_backward(z(4, 8), z(4, 8), z(1, 16, 8), z(1, 16, 8), z(1, 16, 8))
    with pytest.raises(ValueError, match="dw"):
        grace.grace_shared_ffn_backward(z(4, 8), z(4, 8), z(1, 16, 8), z(1, 16, 8), z(1, 8, 16), dw=(z(1, 16, 8), z(1, 16, 8)))
    with pytest.raises(ValueError, match="workspace too small"):
        grace.grace_shared_ffn_backward(z(4, 8), z(4, 8), z(1, 16, 8), z(1, 16, 8), z(1, 8, 16), ws=z(10))
    with pytest.raises(ValueError, match="out"):
        grace.grace_clip_grad_norm([z(4)], 1.0, [z(5)])
    with pytest.raises(ValueError, match="no gradients"):
        grace.grace_grad_norm([])
    with pytest.raises(ValueError, match="live on the GPU"):
        grace.grace_clip_grad_norm([z(4)], 1.0)


def test_ffn_backward_assembly_keeps_its_wait_states():
    n, found = asm_hazards.check("ffn_backward.hip")
    assert n > 30
    assert found == [], "\n".join(found)


def test_rows_backward_refuses_more_wavefronts_than_a_launch_takes(lib):
    """T * k fits its range and a row its own, the launch's work-items do not: the entry of T = 1 << 28 above, whose statuses are not looked at there."""
    T, d = 1 << 28, 4096
    for k in (1, 2, 7):
        for dt in (F32, BF16):
            assert lib.grace_permute_backward(AT, AT, T, k, d, dt, None, 0, None, AT, None) == ESHAPE
            assert lib.grace_combine_backward(AT, AT, AT, AT, T, k, d, dt, None, 0, AT, AT, None) == ESHAPE
            assert "too many rows" in grace.grace_last_error()
