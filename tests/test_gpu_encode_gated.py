"""Encoders with gated MLPs through epd_encode, against the oracle: both dtypes, both norms (RMSNorm is folded into the
products), every tile, and a block of a multimodal model made of the operators beside the encoder."""

import math

import numpy as np
import pytest
import torch

from oracle import vit_encode as O
from paper_2601_11590_amd import binding as B, workloads as W
from parity_util import check, run_gpu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def small(dtype, **kw):
    base = dict(name="gated-" + dtype, dtype=dtype, num_layers=2, hidden=256, num_heads=4, head_dim=64, mlp_dim=512, patch=4,
                temporal_patch=1, norm="rmsnorm", rope="2d", rope_pairs=(0, 16, 16), out_dim=192, act="swiglu")
    base.update(kw)
    return W.EncoderConfig(**base)


RAGGED = [(1, 6, 10), (1, 14, 18), (2, 4, 4), (1, 2, 2)]


def parity(cfg, grids, std=0.02, **kw):
    gw, layers = W.all_weights(cfg, std)
    patches = W.packed_patches(cfg, grids)
    cu, grid = W.metadata(grids)
    check(cfg, run_gpu(cfg, gw, layers, patches, cu, grid, **kw), O.encode(cfg, gw, layers, patches, cu, grid))


@pytest.mark.parametrize("act", W.GATED_ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("extra", [dict(), dict(norm="layernorm", use_bias=False), dict(mlp_dim=328, rope="3d", rope_pairs=(8, 12, 12)),
                                   dict(num_heads=2, head_dim=72, hidden=144, mlp_dim=304, rope_pairs=(0, 18, 18), norm="layernorm"),
                                   dict(num_heads=3, head_dim=72, hidden=216, mlp_dim=200, rope_pairs=(0, 18, 18))])
def test_ragged_batches(dtype, act, extra):
    parity(small(dtype, act=act, **extra), RAGGED)


@pytest.mark.parametrize("tile", [0, 2, 4, 5, 7, 8])
def test_every_tile(tile):
    parity(small("bf16", num_layers=1, mlp_dim=712), [(1, 26, 40), (1, 14, 18)], gemm_tile=tile)


def test_hidden_1024_takes_the_sums_of_squares_from_either_tile():
    for grids in ([(1, 14, 14)], [(1, 40, 64)]):
        parity(small("bf16", hidden=1024, num_heads=16, mlp_dim=1024), grids)


def test_wide_gates():
    for act in W.GATED_ACTS:
        parity(small("bf16", num_layers=1, act=act), RAGGED, std=0.1)


def test_fc1_is_the_operator_with_the_same_weights():
    # one block without attention's share: both entries round H once and add in fp32
    cfg = small("bf16", num_layers=1, use_bias=False, norm="layernorm")
    gw, layers = W.all_weights(cfg)
    grids = [(1, 16, 20)]
    patches = W.packed_patches(cfg, grids)
    cu, grid = W.metadata(grids)
    layers[0]["proj_w"] = np.zeros_like(layers[0]["proj_w"])
    _, hidden = run_gpu(cfg, gw, layers, patches, cu, grid, want_hidden=True)
    no_mlp = [dict(layers[0], fc2_w=np.zeros_like(layers[0]["fc2_w"]))]
    _, before = run_gpu(cfg, gw, no_mlp, patches, cu, grid, want_hidden=True)
    x = torch.from_numpy(O.layer_norm(before, layers[0]["norm2_g"], layers[0]["norm2_b"], cfg.norm_eps)).to(DEV).to(torch.bfloat16)
    up = lambda a: torch.from_numpy(a).to(DEV).to(torch.bfloat16)
    y = B.GatedMLP("bf16", 256, 512, max_tokens=320).forward({"gate_up_w": up(layers[0]["fc1_w"]), "down_w": up(layers[0]["fc2_w"])}, x)
    diff = hidden - before - y.double().cpu().numpy()
    # y is rounded once more than the residual's share, and x may be rounded the other way here and there: 2^-8 of each
    # of the two products' operands in the mean square, and of y
    assert np.sqrt((diff ** 2).mean()) <= 3 * 2 ** -8 / math.sqrt(3) * np.sqrt((y.double().cpu().numpy() ** 2).mean())


# ------------------------------------------------------------------ the operators together

def test_a_block_over_visual_and_text_tokens_and_its_gradients():
    """Visual tokens and texts of two sequences: positions from the grids, q and k turned, causal attention, gated MLP -- forward and
    back to the gradients of the block's input and of the MLP's weights, against float64 autograd on the same values."""
    spans, cu = [(7, 0, 0), (1, 6, 10), (5, 0, 0), (9, 0, 0), (2, 4, 4), (11, 0, 0)], [0, 3, 6]
    D, H, KV, d, F = 128, 4, 2, 32, 264
    pos, after = B.rope_positions(spans, cu, t_step=2)
    T = pos.shape[1]
    assert T == 7 + 60 + 5 + 9 + 32 + 11 and after.tolist() == [22, 9 + 4 + 11]
    g = torch.Generator(device=DEV).manual_seed(3)
    rnd = lambda *s, std=1.0: torch.randn(s, generator=g, device=DEV) * std
    x, dy = rnd(T, D), rnd(T, D)
    wqkv = rnd((H + 2 * KV) * d, D, std=D ** -0.5)
    wo = rnd(D, H * d, std=D ** -0.5)
    w = {"gate_up_w": rnd(2 * F, D, std=D ** -0.5), "down_w": rnd(D, F, std=F ** -0.5)}
    rope = B.Rope("f32", d, (6, 5, 5), layout="interleaved", ladder="head")
    mlp = B.GatedMLP("f32", D, F, max_tokens=T, training=True)
    ends = [72, T]
    mask = torch.ones(T, T, dtype=torch.bool, device=DEV).tril()
    mask[72:, :72] = False

    def attend(q, k, v):
        k, v = k.repeat_interleave(H // KV, dim=1), v.repeat_interleave(H // KV, dim=1)
        s = (q.transpose(0, 1) @ k.transpose(0, 1).transpose(1, 2).contiguous()) * d ** -0.5
        p = torch.softmax(s.masked_fill(~mask, float("-inf")), dim=-1)
        return (p @ v.transpose(0, 1).contiguous()).transpose(0, 1).reshape(T, H * d)

    # with the operators
    qkv = (x @ wqkv.t()).view(T, H + 2 * KV, d)
    q, k = rope.apply([qkv[:, :H], qkv[:, H:H + KV]], pos)
    q.requires_grad_(True)
    k.requires_grad_(True)
    v = qkv[:, H + KV:].clone().requires_grad_(True)
    o = attend(q, k, v)
    r = (x + o.detach() @ wo.t())
    y, saved = mlp.forward(w, r, save=True)
    grads = mlp.backward(w, r, dy, saved)
    dr = dy + grads["dx"]                                # y + r leaves the block
    dq, dk, dv = torch.autograd.grad(o, [q, k, v], dr @ wo)
    dqk = rope.apply([dq.contiguous(), dk.contiguous()], pos, inverse=True)
    dx = dr + torch.cat(dqk + [dv], dim=1).reshape(T, -1) @ wqkv

    # in float64 by autograd
    X = x.double().requires_grad_(True)
    W64 = {n: t.double().requires_grad_(True) for n, t in w.items()}
    QKV = (X @ wqkv.double().t()).view(T, H + 2 * KV, d)
    rounds = sorted((j, a) for a, n in enumerate((6, 5, 5)) for j in range(n))
    axis = torch.tensor([a for _, a in rounds], device=DEV)
    f = 10000.0 ** (-torch.arange(16, dtype=torch.float64, device=DEV) / 16)
    ang = (pos.double()[axis].t() * f)[:, None]
    turn = lambda z: torch.cat([z[..., :16] * ang.cos() - z[..., 16:] * ang.sin(), z[..., :16] * ang.sin() + z[..., 16:] * ang.cos()], dim=-1)
    R = X + attend(turn(QKV[:, :H]), turn(QKV[:, H:H + KV]), QKV[:, H + KV:]) @ wo.double().t()
    gu = R @ W64["gate_up_w"].t()
    Y = (torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]) @ W64["down_w"].t()
    want = torch.autograd.grad(Y + R, [X, W64["gate_up_w"], W64["down_w"]], dy.double())
    # fp32 throughout: each of the ten or so products in a row adds sqrt(K) 2^-24 of its result, K <= 264; ten of them 1e-5
    for got, ref in zip([y, dx, grads["gate_up_w"], grads["down_w"]], [Y] + list(want)):
        assert float((got.double() - ref.detach()).norm() / ref.detach().norm()) <= 1e-5
    assert ends[1] == T
