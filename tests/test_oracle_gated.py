"""The oracle's encoder with gated MLPs: the two independent paths agree, and planted mistakes are seen."""

import numpy as np
import pytest

from oracle import brute_force as BF, vit_encode as O
from paper_2601_11590_amd import workloads as W


def tiny(act, **kw):
    return W.EncoderConfig(name="gated", dtype="f32", num_layers=2, hidden=8, num_heads=2, head_dim=4, mlp_dim=6, patch=2, temporal_patch=1,
                           norm="rmsnorm", rope="2d", rope_pairs=(0, 1, 1), out_dim=5, act=act, **kw)


def both(cfg):
    grids = [(1, 2, 4), (1, 2, 2)]
    gw, layers = W.all_weights(cfg, std=0.4)
    patches = W.packed_patches(cfg, grids)
    cu, grid = W.metadata(grids)
    return O.encode(cfg, gw, layers, patches, cu, grid), np.array(BF.encode(cfg, gw, layers, patches.tolist(), cu.tolist(), grid.tolist())), (gw, layers, patches, cu, grid)


@pytest.mark.parametrize("act", W.GATED_ACTS)
@pytest.mark.parametrize("bias", [True, False])
def test_two_paths_agree(act, bias):
    a, b, _ = both(tiny(act, use_bias=bias))
    assert np.abs(a - b).max() <= 1e-10


def test_halves_exchanged_are_seen():
    cfg = tiny("swiglu")
    a, _, (gw, layers, patches, cu, grid) = both(cfg)
    for lw in layers:
        lw["fc1_w"] = np.concatenate([lw["fc1_w"][6:], lw["fc1_w"][:6]])
    assert np.abs(O.encode(cfg, gw, layers, patches, cu, grid) - a).max() > 1e-3


def test_closed_forms():
    x = np.array([[0.0, 1.0, -2.0, 3.0, 5.0, 7.0]])
    sig = 1 / (1 + np.exp(-x[:, :3]))
    assert np.allclose(O.gated_activation(tiny("swiglu"), x), x[:, :3] * sig * x[:, 3:], rtol=1e-14)
    assert np.allclose(O.gated_activation(tiny("geglu_erf"), x), O.gelu_erf(x[:, :3]) * x[:, 3:], rtol=1e-14)
    assert np.allclose(O.gated_activation(tiny("geglu_tanh"), x), O.gelu_tanh(x[:, :3]) * x[:, 3:], rtol=1e-14)


def test_weight_shapes():
    cfg = tiny("geglu_erf")
    lw = W.layer_weights(cfg, 0)
    assert lw["fc1_w"].shape == (12, 8) and lw["fc1_b"].shape == (12,) and lw["fc2_w"].shape == (8, 6)
