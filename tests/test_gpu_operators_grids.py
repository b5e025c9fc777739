"""Calls whose launches would pass 2^32 threads in the tiles that smaller ones take."""

import pytest
import torch

from gated_util import check, reference
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_f32_backward_of_8_billion_elements():
    T, D, F = (1 << 22) - 1, 2040, 8
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GB")
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *s: torch.empty(s, device=DEV).normal_(generator=g)
    w = {"gate_up_w": rnd(2 * F, D) * D ** -0.5, "down_w": rnd(D, F) * F ** -0.5, "gate_up_b": rnd(2 * F), "down_b": rnd(D)}
    x, dy = rnd(T, D), rnd(T, D)
    op = B.GatedMLP("f32", D, F, max_tokens=T, use_bias=True, training=True)
    y, saved = op.forward(w, x, save=True)
    grads = op.backward(w, x, dy, saved)
    rows = torch.unique(torch.cat([torch.randint(0, T, (300,), generator=torch.Generator().manual_seed(2)), torch.arange(70), torch.arange(T - 70, T)])).to(DEV)
    want = reference("swiglu", w, x[rows], dy[rows])
    check({"y": y[rows], "dx": grads["dx"][rows]}, {n: want[n] for n in ("y", "dx")})
    del y, grads["dx"]
    sums = {}
    for r in range(0, T, 1 << 18):                                     # rows' shares of the sums, in float64
        part = reference("swiglu", w, x[r:r + (1 << 18)], dy[r:r + (1 << 18)])
        for n in grads:
            sums[n] = sums.get(n, 0.0) + part[n][0]
    # a sum of T terms of random signs: each addition is off by 2^-24 of a partial sum, which grows as the root of the terms: the root of the
    # sum of (2^-24)^2 k / 3 over k <= T is 2^-24 T / sqrt(6), of a sum of sqrt(T): 0.4 2^-24 sqrt(T), and twice that for all before it
    for n in grads:
        assert float((grads[n].double() - sums[n]).norm() / sums[n].norm()) <= 2.0 ** -24 * T ** 0.5, n
    del x, dy, saved, op, grads
    torch.cuda.empty_cache()
