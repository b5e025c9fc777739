"""Gated MLP, forward and backward, against float64: every size class of the kernels, odd row counts, strides, and what is
allowed around them (streams, graphs, calls in place, empty calls)."""

import numpy as np
import pytest
import torch

from gated_util import act_of, check, make, reference
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def op_for(dtype, D, F, act, T, bias, training=True):
    return B.GatedMLP(dtype, D, F, act=act, max_tokens=T, use_bias=bias, training=training)


SIZES = [(1, 8, 8), (2, 64, 72), (5, 72, 8), (15, 256, 40), (16, 320, 16), (17, 264, 136), (31, 1024, 128), (33, 128, 1032), (63, 200, 64),
         (64, 1152, 200), (65, 1152, 200), (100, 64, 24), (129, 328, 648), (257, 1152, 264), (300, 1024, 1024), (777, 640, 1288)]


@pytest.mark.parametrize("act,bias", [("swiglu", False), ("geglu_erf", True), ("geglu_tanh", True)])
@pytest.mark.parametrize("T,D,F", SIZES)
def test_bf16_training_step(T, D, F, act, bias):
    w, x, dy = make(T, D, F, torch.bfloat16, bias, T + D + F)
    op = op_for("bf16", D, F, act, T, bias)
    y, saved = op.forward(w, x, save=True)
    got = {"y": y, **op.backward(w, x, dy, saved)}
    check(got, reference(act, w, x, dy))
    assert torch.equal(op.forward(w, x), y)                            # with and without saving, the same bits


@pytest.mark.parametrize("act,bias", [("swiglu", True), ("geglu_erf", False), ("geglu_tanh", True)])
@pytest.mark.parametrize("T,D,F", [(1, 1, 1), (1, 256, 1024), (3, 7, 5), (33, 255, 129), (64, 256, 64), (257, 256, 1024), (1000, 33, 65), (130, 510, 301)])
def test_f32_training_step(T, D, F, act, bias):
    w, x, dy = make(T, D, F, torch.float32, bias, T + D + F)
    op = op_for("f32", D, F, act, T, bias)
    y, saved = op.forward(w, x, save=True)
    check({"y": y, **op.backward(w, x, dy, saved)}, reference(act, w, x, dy))
    assert torch.equal(op.forward(w, x), y)


# tiles through LDS for some or all products: whole and ragged K, edges across and along, a K below one step, rows apart
@pytest.mark.parametrize("T,D,F", [(700, 1024, 1030), (1111, 517, 643), (2049, 350, 1030), (40_000, 20, 30), (1024, 512, 2048), (3000, 255, 129), (6001, 128, 64)])
def test_f32_many_tokens(T, D, F):
    w, x, dy = make(T, D, F, torch.float32, True, T)
    op = op_for("f32", D, F, "geglu_erf", T, True)
    wide = torch.full((T, D + 3), 5.0, device=DEV)
    y, saved = op.forward(w, x, save=True, out=wide[:, 1:1 + D])
    grads = op.backward(w, x, dy, saved)
    check({"y": y, **grads}, reference("geglu_erf", w, x, dy))
    assert torch.equal(op.forward(w, x), y) and (wide[:, 0] == 5).all() and (wide[:, 1 + D:] == 5).all()
    for n in ("dx", "down_w"):
        assert torch.equal(op.backward(w, x, dy, saved, want=[n])[n], grads[n])


# sizes whose first product is planned in each of the large tiles, with rows behind whole tiles, channels that no tile
# divides and inner dimensions that are and are not whole K steps
LARGE = [(2049, 1024, 1024), (3000, 1152, 4304), (5003, 1160, 2056), (6273, 320, 1288), (9001, 256, 2560), (12545, 64, 136)]


@pytest.mark.parametrize("T,D,F", LARGE)
def test_bf16_many_tokens(T, D, F):
    w, x, dy = make(T, D, F, torch.bfloat16, True, T)
    op = op_for("bf16", D, F, "swiglu", T, True)
    y, saved = op.forward(w, x, save=True)
    check({"y": y, **op.backward(w, x, dy, saved)}, reference("swiglu", w, x, dy))


@pytest.mark.parametrize("act,bias", [("swiglu", True), ("geglu_erf", False), ("geglu_tanh", True)])
@pytest.mark.parametrize("T", [1, 2])
@pytest.mark.parametrize("D,F", [(8, 4096), (2048, 2056), (2056, 2048), (4104, 72), (72, 12808), (3200, 8200), (520, 1032)])
def test_bf16_one_and_two_tokens(T, D, F, act, bias):
    w, x, dy = make(T, D, F, torch.bfloat16, bias, D + F)
    op = op_for("bf16", D, F, act, T, bias)
    y, saved = op.forward(w, x, save=True)
    check({"y": y, **op.backward(w, x, dy, saved)}, reference(act, w, x, dy))
    assert torch.equal(op.forward(w, x), y)
    one = op.forward(w, x[:1].clone())
    assert torch.equal(op.forward(w, x[:1], out=x[:1]), one) and torch.equal(x[:1], one)                 # in place


@pytest.mark.parametrize("T", [16, 17, 32, 33, 64])
@pytest.mark.parametrize("D,F,act,bias", [(512, 2048, "swiglu", True), (1024, 4096, "geglu_tanh", False), (1152, 4304, "geglu_erf", True), (2056, 4104, "swiglu", True),
                                          (8200, 2048, "swiglu", False)])
def test_bf16_few_tokens(T, D, F, act, bias):
    # where one or both products change from the kernels for few tokens to the tiles
    w, x, dy = make(T, D, F, torch.bfloat16, bias, D + F)
    op = op_for("bf16", D, F, act, T, bias)
    y, saved = op.forward(w, x, save=True)
    check({"y": y, **op.backward(w, x, dy, saved)}, reference(act, w, x, dy))
    assert torch.equal(op_for("bf16", D, F, act, T, bias, training=False).forward(w, x), y)
    assert torch.equal(op_for("bf16", D, F, act, 4 * T, bias).forward(w, x), y)


def test_the_large_sizes_reach_every_tile():
    plans = set()
    for T, D, F in LARGE + SIZES:
        for M, N, K in ((T, (F + 15) // 16 * 32, D), (T, D, F), (T, F, D), (2 * F, D, (T + 63) // 64 * 64), (D, F, (T + 63) // 64 * 64)):
            plans.add(B.epd_probe_gemm_plan(M, N, K)[:2])
    assert {(256, 256), (320, 256), (128, 128), (64, 64), (64, 128)} <= plans, plans


def test_rows_apart_and_what_lies_between_them():
    for dtype, T in (("bf16", 5), ("bf16", 150), ("f32", 70)):
        D, F = 136, 200
        w, x, dy = make(T, D, F, DT[dtype], True, 3)
        wide = torch.full((T, 2 * D + 8), 7.0, dtype=DT[dtype], device=DEV)
        wide[:, 8:8 + D] = x
        far = torch.full((T + 1, 3 * D), -3.0, dtype=DT[dtype], device=DEV)
        op = op_for(dtype, D, F, "geglu_erf", T, True)
        y = op.forward(w, wide[:, 8:8 + D], out=far[:T, D:2 * D])
        check({"y": y}, reference("geglu_erf", w, x))
        assert (far[:, :D] == -3).all() and (far[:, 2 * D:] == -3).all() and (far[T] == -3).all()
        assert torch.equal(y, op.forward(w, x))


def test_in_place():
    for dtype, T in (("bf16", 3), ("bf16", 300), ("f32", 40)):
        w, x, _ = make(T, 128, 256, DT[dtype], False, 4)
        op = op_for(dtype, 128, 256, "swiglu", T, False, training=False)
        y = op.forward(w, x)
        assert torch.equal(op.forward(w, x, out=x), y) and torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_gradients_have_the_bits_of_the_whole_call(dtype):
    T, D, F = 200, 136, 72
    w, x, dy = make(T, D, F, DT[dtype], True, 5)
    op = op_for(dtype, D, F, "geglu_tanh", T, True)
    _, saved = op.forward(w, x, save=True)
    whole = op.backward(w, x, dy, saved)
    for n in whole:
        assert torch.equal(op.backward(w, x, dy, saved, want=[n])[n], whole[n]), n
    assert op.backward(w, x, dy, saved, want=[]) == {}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_tokens(dtype):
    w, x, dy = make(0, 64, 72, DT[dtype], True, 6)
    op = op_for(dtype, 64, 72, "swiglu", 10, True)
    y, saved = op.forward(w, x, save=True)
    assert y.shape == (0, 64)
    g = op.backward(w, x, dy, saved)
    assert all(not v.any() for v in g.values()) and g["gate_up_w"].shape == (144, 64)


def test_fewer_tokens_than_before_in_the_same_workspace():
    # what a longer call left in the workspace is not seen by a shorter one (pads of K steps among it)
    D, F = 136, 40
    op = op_for("bf16", D, F, "swiglu", 500, True)
    for T in (500, 67, 3, 130, 1):
        w, x, dy = make(T, D, F, torch.bfloat16, True, T)
        if T == 500:
            x = x * float("inf")
        y, saved = op.forward(w, x, save=True)
        got = {"y": y, **op.backward(w, x, dy, saved)}
        if T < 500:
            check(got, reference("swiglu", w, x, dy))


def test_a_workspace_of_nan_is_never_read():
    for T in (4, 200):
        D, F = 72, 24
        w, x, dy = make(T, D, F, torch.bfloat16, True, 8)
        op = op_for("bf16", D, F, "geglu_erf", T, True)
        op.workspace.fill_(0xFF)
        y, saved = op.forward(w, x, save=True)
        op.workspace.fill_(0xFF)
        check({"y": y, **op.backward(w, x, dy, saved)}, reference("geglu_erf", w, x, dy))


def test_a_bad_row_stays_alone():
    for T in (9, 300):
        w, x, _ = make(T, 128, 256, torch.bfloat16, False, 9)
        op = op_for("bf16", 128, 256, "swiglu", T, False)
        good = op.forward(w, x)
        x = x.clone()
        x[4] = float("nan")
        x[T - 1, 3] = float("inf")
        bad = op.forward(w, x)
        rows = [i for i in range(T) if i not in (4, T - 1)]
        assert torch.equal(bad[rows], good[rows]) and torch.isnan(bad[4]).all()


@pytest.mark.parametrize("act", ["swiglu", "geglu_erf", "geglu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_from_tiny_to_huge(dtype, act):
    # gates of every size through one channel each: identity-like weights, up factor 1 through its bias
    vals = [0.0, 1e-30, -1e-30, 1e-4, -1e-4, 9e-4, -9e-4, 2e-3, 0.3, -0.3, 1.0, -1.0, 3.0, -3.0, 7.4, -7.4, 20.0, -20.0, 300.0, -300.0, 1e5, -1e5, 1e20, -1e20]
    D = F = 24
    T = 70
    w = {"gate_up_w": torch.zeros(2 * F, D, device=DEV), "gate_up_b": torch.cat([torch.zeros(F), torch.ones(F)]).to(DEV),
         "down_w": torch.eye(F, device=DEV), "down_b": torch.zeros(D, device=DEV)}
    w["gate_up_w"][:F] = torch.eye(D, device=DEV)
    w = {n: t.to(DT[dtype]) for n, t in w.items()}
    x = torch.tensor(vals, device=DEV).repeat(T, 1).to(DT[dtype])
    op = op_for(dtype, D, F, act, T, True)
    y, saved = op.forward(w, x, save=True)
    dx = op.backward(w, x, torch.ones_like(x), saved, want=["dx"])["dx"]
    a, d = act_of(act, x.double())
    half = torch.finfo(DT[dtype]).eps / 2
    lost = 4e-6 if dtype == "bf16" else 6e-7
    for got, want in ((y, a), (dx, d)):
        assert torch.isfinite(got).all()
        # two roundings (H and y; dG and dX) and the arithmetic, relative to the gate where it is large
        big = torch.where(x.double() > 0, x.double(), x.double().abs().clamp(max=10.0)) if got is y else torch.full_like(a, 10.0)
        assert ((got.double() - want).abs() <= 2.1 * half * want.abs() + lost * (1 + big)).all(), (got[0], want[0])


def test_gradients_by_differences():
    T, D, F = 6, 16, 24
    w, x, dy = make(T, D, F, torch.float32, True, 10)
    op = op_for("f32", D, F, "geglu_erf", T, True)
    _, saved = op.forward(w, x, save=True)
    g = op.backward(w, x, dy, saved)
    step = 1e-2
    loss = lambda: float((op.forward(w, x).double() * dy.double()).sum())
    for name, t, at in [("dx", x, (2, 5)), ("dx", x, (5, 15)), ("gate_up_w", w["gate_up_w"], (3, 7)), ("gate_up_w", w["gate_up_w"], (F + 4, 2)),
                        ("down_w", w["down_w"], (9, 20)), ("gate_up_b", w["gate_up_b"], (1,)), ("gate_up_b", w["gate_up_b"], (F + 1,)), ("down_b", w["down_b"], (3,))]:
        v = float(t[at])
        t[at] = v + step
        hi = loss()
        t[at] = v - step
        lo = loss()
        t[at] = v
        # central difference: step^2 / 6 of the third derivative (of the order of the loss's terms), roundings 1e-5 / step
        assert abs((hi - lo) / (2 * step) - float(g[name][at])) <= 2e-2 * max(1.0, abs(float(g[name][at]))), name


def test_another_stream_and_graphs():
    D, F = 128, 264
    for T in (7, 200):
        w, x, dy = make(T, D, F, torch.bfloat16, True, 11)
        op = op_for("bf16", D, F, "swiglu", T, True)
        y, saved = op.forward(w, x, save=True)
        want = op.backward(w, x, dy, saved)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            y2, saved2 = op.forward(w, x, save=True)
            got = op.backward(w, x, dy, saved2)
        s.synchronize()
        assert torch.equal(y, y2) and all(torch.equal(want[n], got[n]) for n in want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y3, saved3 = op.forward(w, x, save=True)
            g3 = op.backward(w, x, dy, saved3)
        for seed in (20, 21, 22):
            _, x1, dy1 = make(T, D, F, torch.bfloat16, True, seed)
            x.copy_(x1)
            dy.copy_(dy1)
            graph.replay()
            torch.cuda.synchronize()
            ye, se = op.forward(w, x, save=True)
            ge = op.backward(w, x, dy, se)
            torch.cuda.synchronize()
            assert torch.equal(y3, ye) and all(torch.equal(g3[n], ge[n]) for n in ge)


def test_two_objects_at_once_on_two_streams():
    T, D, F = 500, 256, 512
    w, x, _ = make(T, D, F, torch.bfloat16, False, 12)
    ops = [op_for("bf16", D, F, "swiglu", T, False, training=False) for _ in range(2)]
    want = ops[0].forward(w, x)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(5):
        for op, s in zip(ops, streams):
            with torch.cuda.stream(s):
                outs.append(op.forward(w, x))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_calls_are_deterministic():
    for dtype, T in (("bf16", 13), ("bf16", 1500), ("f32", 300)):
        w, x, dy = make(T, 320, 648, DT[dtype], True, 13)
        op = op_for(dtype, 320, 648, "geglu_tanh", T, True)
        runs = []
        for _ in range(2):
            y, saved = op.forward(w, x, save=True)
            runs.append({"y": y, **op.backward(w, x, dy, saved)})
        assert all(torch.equal(runs[0][n], runs[1][n]) for n in runs[0])
