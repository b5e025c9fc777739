"""The gated MLP in every kernel its planner knows, and both operators on arrays that pass 2^31 elements."""

import numpy as np
import pytest
import torch

from gated_util import check, make, reference
from paper_2601_11590_amd import binding as B
from test_gpu_rope import check as check_rope

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# Together with those in parts below and the smaller ones of test_gpu_gated_mlp.py these reach each tile with each epilogue (plain, gated, gated
# and kept, backward), operands as they stand and turned, read along their rows and across them, in one launch and cut into two.
@pytest.mark.parametrize("T,D,F", [(530, 4624, 1928), (585, 1112, 10104), (2091, 824, 10000), (4692, 1192, 1872), (7259, 1168, 3344), (9754, 792, 1880), (13071, 1648, 280),
                                   (13600, 1792, 1304), (20118, 848, 72)])
def test_every_kernel_of_the_products(T, D, F):
    w, x, dy = make(T, D, F, torch.bfloat16, True, T)
    op = B.GatedMLP("bf16", D, F, act="geglu_tanh", max_tokens=T, use_bias=True, training=True)
    y, saved = op.forward(w, x, save=True)
    check({"y": y, **op.backward(w, x, dy, saved)}, reference("geglu_tanh", w, x, dy))
    assert torch.equal(op.forward(w, x), y)


# Few rows: the long products' K in parts (in each of their tiles, two to eight parts, the last one shorter or not), joined
@pytest.mark.parametrize("T,D,F", [(65, 1024, 4096), (130, 1160, 4312), (333, 1024, 4096), (600, 2048, 6152), (784, 3200, 12808), (1024, 2056, 6144), (1500, 1024, 8192),
                                   (3000, 1024, 4096)])
@pytest.mark.parametrize("bias", [False, True])
def test_products_in_parts(T, D, F, bias):
    w, x, dy = make(T, D, F, torch.bfloat16, bias, T)
    op = B.GatedMLP("bf16", D, F, act="swiglu", max_tokens=T + 9, use_bias=bias, training=True)
    op.workspace.fill_(0xFF)                                           # nothing is read that was not written
    wide = torch.full((T, D + 24), 7.0, dtype=torch.bfloat16, device=DEV)
    y, saved = op.forward(w, x, save=True, out=wide[:, 8:8 + D])
    op.workspace.fill_(0xFF)
    grads = op.backward(w, x, dy, saved)
    check({"y": y, **grads}, reference("swiglu", w, x, dy))
    assert torch.equal(op.backward(w, x, dy, saved, want=["dx"])["dx"], grads["dx"])
    assert (wide[:, :8] == 7).all() and (wide[:, 8 + D:] == 7).all()
    again = B.GatedMLP("bf16", D, F, act="swiglu", max_tokens=T, use_bias=bias)
    assert torch.equal(again.forward(w, x), y) and torch.equal(again.forward(w, x, out=x), y)


def some_channels(w, channels):
    F = w["down_w"].shape[1]
    both = torch.cat([channels, channels + F])
    return both, {"gate_up_w": w["gate_up_w"][both], "down_w": w["down_w"][:, channels], "gate_up_b": w["gate_up_b"][both], "down_b": w["down_b"]}


@pytest.mark.parametrize("dtype,T,D,F", [("bf16", 168_007, 64, 12_808), ("f32", 168_007, 16, 12_808), ("bf16", 4_194_303, 8, 8), ("bf16", 131_075, 16_392, 8)])
def test_mlp_of_more_than_2_31_elements(dtype, T, D, F):
    w, x, dy = make(T, D, F, torch.bfloat16 if dtype == "bf16" else torch.float32, True, 1)
    op = B.GatedMLP(dtype, D, F, max_tokens=T, use_bias=True, training=True)
    y, saved = op.forward(w, x, save=True)
    grads = op.backward(w, x, dy, saved)
    # rows: y and dx of a row need no other
    rows = torch.unique(torch.cat([torch.randint(0, T, (300,), generator=torch.Generator().manual_seed(2)), torch.arange(20), torch.arange(T - 20, T)])).to(DEV)
    want = reference("swiglu", w, x[rows], dy[rows])
    check({"y": y[rows], "dx": grads["dx"][rows]}, {n: want[n] for n in ("y", "dx")})
    # channels: their weights' gradients need no other.  (The norm's limit is for gradients as large as those of random signs.)
    channels = torch.unique(torch.cat([torch.randint(0, F, (8,), generator=torch.Generator().manual_seed(3)), torch.tensor([0, F - 1])])).to(DEV)
    if T * D < 1 << 29:
        both, part = some_channels(w, channels)
        want = reference("swiglu", part, x, dy)
        check({"gate_up_w": grads["gate_up_w"][both], "gate_up_b": grads["gate_up_b"][both], "down_w": grads["down_w"][:, channels], "down_b": grads["down_b"]},
              {n: want[n] for n in ("gate_up_w", "gate_up_b", "down_w", "down_b")}, norms=False)


def test_mlp_rows_2_22_apart():
    T, D, F, ld = 700, 64, 72, (1 << 22) - 8
    for dtype, torch_dtype in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        w, x, dy = make(T, D, F, torch_dtype, False, 4)
        far = torch.empty((T, ld), dtype=torch_dtype, device=DEV)
        far[:, 8:8 + D], far[:, 80:80 + D] = x, dy
        op = B.GatedMLP(dtype, D, F, max_tokens=T, training=True)
        y, saved = op.forward(w, far[:, 8:8 + D], save=True, out=far[:, 160:160 + D])
        check({"y": y, **op.backward(w, far[:, 8:8 + D], far[:, 80:80 + D], saved)}, reference("swiglu", w, x, dy))
        few = op.forward(w, far[:33, 8:8 + D], out=far[:33, 240:240 + D])
        check({"y": few}, reference("swiglu", w, x[:33]))
        del far, y, few


@pytest.mark.parametrize("dtype,pairing,T,H,d,pairs", [("bf16", "half", 70_001, 256, 128, (24, 20, 20)), ("f32", "adjacent", 70_001, 256, 128, (24, 20, 20)),
                                                       ("bf16", "half", 9_000_001, 1, 256, (128,))])
def test_rotation_of_more_than_2_31_elements(dtype, pairing, T, H, d, pairs):
    op = B.Rope(dtype, d, pairs, pairing=pairing)
    x = torch.empty((H, T, d), dtype=op.dtype, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(5)).transpose(0, 1)     # head by head, as in a cache
    pos = torch.randint(0, 1 << 20, (len(pairs), T), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV, dtype=torch.int32)
    y = op.apply([x], pos)[0]
    op.apply([x], pos, out=[x])
    assert torch.equal(x, y)
    op.apply([y], pos, inverse=True, out=[y])                          # back, from rows rounded once: checked below in float64
    rows = torch.unique(torch.cat([torch.randint(0, T, (100,), generator=torch.Generator().manual_seed(7)), torch.arange(3), torch.arange(T - 3, T)])).to(DEV)
    check_rope(y[rows], x[rows], pos[:, rows], pairs, "sections", "axis", pairing, inverse=True)


@pytest.mark.parametrize("T,D,F", [(2001, 1024, 2048), (130, 1024, 4096), (5000, 328, 1288)])
def test_a_gradient_alone_has_the_bits_of_the_whole_call(T, D, F):
    w, x, dy = make(T, D, F, torch.bfloat16, True, T)
    op = B.GatedMLP("bf16", D, F, max_tokens=T, use_bias=True, training=True)
    _, saved = op.forward(w, x, save=True)
    whole = op.backward(w, x, dy, saved)
    for want in ([n] for n in whole):
        assert torch.equal(op.backward(w, x, dy, saved, want=want)[want[0]], whole[want[0]]), want
    some = op.backward(w, x, dy, saved, want=["down_w", "dx"])
    assert torch.equal(some["down_w"], whole["down_w"]) and torch.equal(some["dx"], whole["dx"])


@pytest.mark.parametrize("dtype,T,D,F", [("bf16", 130, 1024, 4096), ("bf16", 1, 2056, 4104), ("bf16", 40, 512, 2048), ("f32", 1024, 256, 1024)])
def test_two_objects_in_graphs_on_two_streams(dtype, T, D, F):
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    w, x, dy = make(T, D, F, t, True, 8)
    ops = [B.GatedMLP(dtype, D, F, act="geglu_erf", max_tokens=T, use_bias=True, training=True) for _ in range(2)]

    def step(op):
        y, saved = op.forward(w, x, save=True)
        return {"y": y, **op.backward(w, x, dy, saved)}

    step(ops[0])
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in ops]
    for op in ops:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(op))
        graphs.append(graph)
    for seed in (30, 31, 32):
        _, x1, dy1 = make(T, D, F, t, True, seed)
        x.copy_(x1)
        dy.copy_(dy1)
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        eager = step(B.GatedMLP(dtype, D, F, act="geglu_erf", max_tokens=T, use_bias=True, training=True))
        torch.cuda.synchronize()
        for got in outs:
            assert all(torch.equal(got[n], eager[n]) for n in eager)
