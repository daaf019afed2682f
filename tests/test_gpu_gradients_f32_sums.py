"""Long sums of the fp32 FFN's gradients: their error does not grow as that of one running sum.

Roundings of a sum are taken to be independent, with an rms of 2^-24 / sqrt(3) = 3.4e-8 of the partial sum.  One running sum of K terms of random signs is then off by sqrt(K / 2)
times that, of its result: 2.2e-6 for K = 8192 (some 1.5e-6 for the mean mantissa).  Sums of 256 terms that are added up are off by sqrt(128) = 11.3 times it for the
parts, whose errors are as independent as their values, and sqrt(32 / 2) = 4 times for their sum: 4.1e-7 together.  What goes into a sum has an error of its own: from sums of
64 terms sqrt(32) = 5.7 times, 1.9e-7, twice or three times over (g, u, dh) with some units in the last place of the sigmoid: 4e-7 at most.  So 6e-7 of the norm where
the terms come from short sums; where all three of them come from sums of 8192, sqrt(3 * 4.1^2 + 4^2) = 8.2e-7 and, for the slope that multiplies g's
error, up to half as much again: 1.2e-6."""
import numpy as np
import pytest
import torch

import paper_2509_25041_amd as grace
from test_gpu_gradients import normal, swiglu_grads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d,f,tolerance,what", [
    (8192, 64, 64, 6e-7, "dw"), (8191, 66, 67, 6e-7, "dw"),           # sums over the rows; odd widths take loads of single values
    (64, 64, 4096, 6e-7, "dx"), (63, 65, 4095, 6e-7, "dx"),           # over the hidden columns, of dg and of du
    (64, 8192, 64, 1.2e-6, "dx dw"), (65, 8190, 66, 1.2e-6, "dx dw"),  # of g, u and dh, over d
])
def test_long_sums(rows, d, f, tolerance, what):
    rng = np.random.default_rng(rows + d + f)
    x, dy = normal(rng, (rows, d)), normal(rng, (rows, d))
    w = normal(rng, (1, f, d), scale=d ** -0.5), normal(rng, (1, f, d), scale=d ** -0.5), normal(rng, (1, d, f), scale=f ** -0.5)
    got = grace.grace_shared_ffn_backward(x, dy, *w)
    want, _ = swiglu_grads(x, dy, *(v[0] for v in w))
    for name, a, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), (got[0],) + tuple(v[0] for v in got[1:]), want):
        if name[:2] in what.split():
            off = (a.double() - b).norm().item() / b.norm().item()
            assert off <= tolerance, (name, off)
