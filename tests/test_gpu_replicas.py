"""Gradients where experts have instances on several ranks: what the ranks' calls give has to be summed, and is then the layer's gradient."""
import numpy as np
import pytest
import torch

import paper_2509_25041_amd as grace

pytestmark = pytest.mark.gpu


def test_instances_gradients_sum_to_the_experts_and_the_norm_is_that_of_the_sums():
    """fp32, tolerance of the norm of a tensor: some 10 sums of up to 1024 terms, each 2^-24 of sqrt(1024) terms' size, sqrt(10 * 1024) 2^-24 = 6e-6, twice."""
    T, E, R, k, d, f = 300, 6, 3, 2, 72, 56
    hosts = [[0, 1, 2], [0], [1], [1, 2], [2], [0, 2]]                       # experts 0, 3 and 5 are replicated
    table = grace.GraceTable(E, R, 1, [0] * R, [1, 2, 1], np.cumsum([0] + [len(h) for h in hosts]).tolist(), sum(hosts, []))
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *shape, scale=1.0, mean=0.0: torch.randn(shape, generator=gen, device="cuda") * scale + mean
    logits, x, dout = rand(T, E), rand(T, d, mean=0.5), rand(T, d, mean=0.5)   # (means: the instances' gradients of an expert are alike)
    w = rand(E, f, d, scale=d ** -0.5), rand(E, f, d, scale=d ** -0.5), rand(E, d, f, scale=f ** -0.5)
    (expert, weight, inst, _), (pos, _, inst_off, rank_off, _, xp) = grace.grace_route_permute(table, 0, logits, k, x, policy=grace.GRACE_POLICY_WRR)
    counts = inst_off.diff().tolist()
    inst_expert, _, rank_ptr = table.instances()
    assert all(n > 0 for n in counts)

    y = torch.zeros_like(xp)
    for rank in range(R):
        mine = [v[torch.as_tensor(table.local_experts(rank).astype(np.int64), device="cuda")].contiguous() for v in w]
        part = grace.grace_expert_ffn(table, rank, xp, inst_off, T, k, *mine)
        lo, hi = rank_off[rank].item(), rank_off[rank + 1].item()
        y[lo:hi] = part[lo:hi]

    dy, dw_gate, dx = torch.zeros_like(xp), torch.zeros((T, k), device="cuda"), torch.zeros_like(x)
    by_expert = [torch.zeros_like(v) for v in w]
    squares_of_parts = 0.0
    for rank in range(R):
        experts = table.local_experts(rank).astype(np.int64)
        mine = [v[torch.as_tensor(experts, device="cuda")].contiguous() for v in w]
        dw_gate += grace.grace_combine_backward(dout, y, pos, weight, rank_off, rank, dy=dy)[1]
        dxp, *parts = grace.grace_expert_ffn_backward(table, rank, xp, dy, inst_off, T, k, *mine)
        dx += grace.grace_permute_backward(dxp, pos, k, None, rank_off, rank)
        for total, part in zip(by_expert, parts):
            for slot, e in enumerate(experts):
                total[e] += part[slot]
        squares_of_parts += grace.grace_grad_norm(parts).item() ** 2
    dlogits = grace.grace_route_backward(logits, expert, weight, dw_gate, 1)

    l64, x64 = logits.double().requires_grad_(), x.double().requires_grad_()
    w64 = [v.double().requires_grad_() for v in w]
    gate = torch.softmax(l64.gather(1, expert.long()), 1)
    out = torch.zeros_like(x64)
    for e in range(E):
        t, j = (expert == e).nonzero(as_tuple=True)
        rows = x64[t]
        out = out.index_add(0, t, gate[t, j][:, None] * ((torch.nn.functional.silu(rows @ w64[0][e].t()) * (rows @ w64[1][e].t())) @ w64[2][e].t()))
    want = torch.autograd.grad(out, [x64, l64] + w64, dout.double())
    for got, ref in zip([dx, dlogits] + by_expert, want):
        assert (got.double() - ref).norm().item() <= 1.2e-5 * ref.norm().item()
    norm = sum(v.square().sum().item() for v in want[2:]) ** 0.5
    assert abs(grace.grace_grad_norm(by_expert).item() / norm - 1) <= 1.2e-5
    assert abs(squares_of_parts ** 0.5 / norm - 1) > 1.2e-5                  # a norm of the parts is another one
