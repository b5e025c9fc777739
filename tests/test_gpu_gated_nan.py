"""A NaN that only a gate holds -- from its weights, from its bias, from infinities that cancel in its sum -- is not lost: every output
that the channel enters is NaN, all others keep their bits."""

import numpy as np
import pytest
import torch

from gated_util import make
from paper_2601_11590_amd import binding as B, workloads as W
from parity_util import run_gpu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def spoil(w, x, how, c):
    """The weights with a NaN gate in channel c, and nothing else that is not finite behind the first product."""
    w = {n: t.clone() for n, t in w.items()}
    if how == "weight":
        w["gate_up_w"][c, 3] = float("nan")
    elif how == "bias":
        w["gate_up_b"][c] = float("nan")
    else:                                                              # x[:, 0] and x[:, 1] are positive: inf - inf
        w["gate_up_w"][c, 0], w["gate_up_w"][c, 1] = float("inf"), -float("inf")
    return w


@pytest.mark.parametrize("act", W.GATED_ACTS)
@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 9), ("bf16", 40), ("bf16", 300), ("bf16", 3000), ("f32", 1), ("f32", 40), ("f32", 1500)])
@pytest.mark.parametrize("how", ["weight", "bias", "infinities"])
def test_a_gate_of_nan(how, dtype, T, act):
    D, F, c = 128, 264, 37
    w, x, dy = make(T, D, F, DT[dtype], True, T)
    x[:, :2] = x[:, :2].abs() + 0.5
    op = B.GatedMLP(dtype, D, F, act=act, max_tokens=T, use_bias=True, training=True)
    _, saved = op.forward(w, x, save=True)
    good = op.backward(w, x, dy, saved)
    bad_w = spoil(w, x, how, c)
    y, saved = op.forward(bad_w, x, save=True)
    assert torch.isnan(y).all() and torch.isnan(op.forward(bad_w, x)).all()
    bad = op.backward(bad_w, x, dy, saved)
    assert torch.isnan(bad["dx"]).all()
    rest = torch.tensor([i for i in range(F) if i != c], device=DEV)
    for n, own in (("gate_up_w", [c, F + c]), ("gate_up_b", [c, F + c])):
        assert torch.isnan(bad[n][own]).all(), n                       # of the gate, and of the up half by act(NaN)
        both = torch.cat([rest, rest + F])
        assert torch.equal(bad[n][both], good[n][both]), n
    assert torch.isnan(bad["down_w"][:, c]).all() and torch.equal(bad["down_w"][:, rest], good["down_w"][:, rest])
    assert torch.equal(bad["down_b"], good["down_b"])


@pytest.mark.parametrize("act", W.GATED_ACTS)
@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 9), ("bf16", 300), ("f32", 40)])
def test_a_gate_of_infinity(dtype, T, act):
    # act(g) = g * (0 .. 1) of the formulas: -infinity * 0 is NaN, +infinity stays
    D, F = 128, 264
    w, x, _ = make(T, D, F, DT[dtype], True, T)
    op = B.GatedMLP(dtype, D, F, act=act, max_tokens=T, use_bias=True, training=True)
    for value in (-float("inf"), float("inf")):
        w["gate_up_b"][37] = value
        y, _ = op.forward(w, x, save=True)
        assert (torch.isnan(y) if value < 0 else ~torch.isfinite(y)).all(), value
        y = op.forward(w, x)
        assert (torch.isnan(y) if value < 0 else ~torch.isfinite(y)).all(), value


@pytest.mark.parametrize("act", W.GATED_ACTS)
@pytest.mark.parametrize("dtype,tile", [("f32", -1)] + [("bf16", t) for t in (0, 2, 4, 5, 7, 8)])
def test_a_gate_of_nan_in_the_encoder(dtype, tile, act):
    cfg = W.EncoderConfig(name="nan", dtype=dtype, num_layers=1, hidden=256, num_heads=4, head_dim=64, mlp_dim=264, patch=4, temporal_patch=1,
                          norm="rmsnorm", rope="2d", rope_pairs=(0, 16, 16), out_dim=192, act=act)
    grids = [(1, 14, 18), (1, 2, 2)]
    gw, layers = W.all_weights(cfg)
    cu, grid = W.metadata(grids)
    kw = {} if tile < 0 else dict(gemm_tile=tile)
    run = lambda l: run_gpu(cfg, gw, l, W.packed_patches(cfg, grids), cu, grid, **kw)
    assert np.isfinite(run(layers)).all()
    fc1_b = layers[0]["fc1_b"].copy()
    fc1_b[37] = float("nan")                                           # gate rows come first
    assert np.isnan(run([dict(layers[0], fc1_b=fc1_b)])).all()
