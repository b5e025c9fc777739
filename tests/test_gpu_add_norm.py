"""AddNorm.forward / backward, quant_rows and dequant_rows against the definitions in 64 bits.

Tolerances.  A row's sums go through at most 64 additions in a thread, 6 between lanes and 16 between waves: 88 half steps of fp32,
relative to the sum of magnitudes, with the rounding of what is added.  rstd takes half of that and four roundings more (48); s one
half step of its own, so y is within 52 half steps, then rounded.  Backward: mean(g n) 88 + 48 + 4 half steps of mean |g n|, n 49, so
n mean(g n) 190, all of dx within 200 of |ds| + rstd (|g| + |n| mean |g n|).  The gradient of gain adds T values that are 51 off.
8 bits: half a step of the scale, plus what y is off (at most 127 steps of 54 half steps of fp32 each)."""

import numpy as np
import pytest
import torch

from entry_util import DEV, KINDS, U32, Gapped, generator, randn, replays, unit, within
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
EPS = 1e-6
LEAST = 2.0 ** -100
# every width of rows that eight lanes, a wave or a block take in chunks of eight: full, one less and one more
SIZES = [(1, 1), (3, 7), (2, 8), (70, 64), (33, 65), (5, 511), (4, 512), (7, 513), (9, 1024), (3, 1100), (6, 2048), (5, 2049), (16, 3200), (2, 4096), (3, 4100), (2, 8192), (3, 8200), (2, 16384), (3, 16385),
         (2, 32768), (3, 32769), (2, 65535), (1, 65536), (257, 1152), (1031, 72)]


def inputs(T, D, dtype, residual, seed=0):
    gen = generator(T * 7 + D + seed)
    return randn(gen, T, D, dtype=KINDS[dtype]), randn(gen, T, D, dtype=KINDS[residual], std=3.0), (1 + 0.3 * randn(gen, D)).to(KINDS[dtype]), gen


def check_q(q, scale, y, off):
    """q and scale stand for y, which the kernel has within off |y|."""
    m = y.abs().amax(dim=1, keepdim=True).clamp(min=LEAST)
    within(scale[:, None], m / 127, m / 127 * (off + 3 * U32))
    step = scale.double()[:, None]
    within(q.double() * step, y, step * (0.5 + 128 * (off + 3 * U32)))
    assert (q != -128).all()


@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("T,D", SIZES)
def test_forward(dtype, residual, T, D):
    x, r, gain, _ = inputs(T, D, dtype, residual)
    op = B.AddNorm(dtype, D, residual=residual, eps=EPS, max_tokens=T)
    eps = op.cfg.eps
    got = op.forward(gain, x, r, want=("sum", "y", "q"))
    assert set(got) == {"sum", "y", "q", "scale"}
    s = x.double() + r.double()
    y = s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt() * gain.double()
    ur, ut = (unit(KINDS[k]) if k == "bf16" else 0.0 for k in (residual, dtype))
    within(got["sum"], s, s.abs() * (ur + 2 * U32))
    within(got["y"], y, y.abs() * (ut + 54 * U32))
    check_q(got["q"], got["scale"], y, 54 * U32)
    # each output alone, and without one of the inputs
    for n in ("sum", "y", "q"):
        one = op.forward(gain, x, r, want=(n,))
        assert all(torch.equal(one[k], got[k]) for k in one)
    for kw, h in (({"x": x}, x.double()), ({"residual": r}, r.double())):
        o = op.forward(gain, want=("sum", "y"), **kw)
        y = h / (h.square().mean(dim=1, keepdim=True) + eps).sqrt() * gain.double()
        within(o["y"], y, y.abs() * (ut + 54 * U32))
        within(o["sum"], h, h.abs() * ur)


@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("T,D", SIZES + [(4097, 40), (5000, 1024)])
def test_backward(dtype, residual, T, D):
    s, ds, gain, gen = inputs(T, D, residual, residual, 1)
    gain = gain.to(KINDS[dtype])
    dy = randn(gen, T, D, dtype=KINDS[dtype])
    op = B.AddNorm(dtype, D, residual=residual, eps=EPS, max_tokens=T, training=True)
    h = s.double()
    rstd = 1 / (h.square().mean(dim=1, keepdim=True) + op.cfg.eps).sqrt()
    n, g = h * rstd, dy.double() * gain.double()
    dgain = (dy.double() * n).sum(dim=0)
    dgain_off = (60 + T) * U32 * (dy.double() * n).abs().sum(dim=0)
    for with_ds in (True, False):
        got = op.backward(gain, s, dy, dsum=ds if with_ds else None, want=("dx", "dresidual", "gain"))
        d0 = ds.double() if with_ds else torch.zeros_like(h)
        dx = d0 + rstd * (g - n * (g * n).mean(dim=1, keepdim=True))
        off = 200 * U32 * (d0.abs() + rstd * (g.abs() + n.abs() * (g * n).abs().mean(dim=1, keepdim=True)))
        for name in ("dx", "dresidual"):
            u = unit(got[name].dtype)
            within(got[name], dx, dx.abs() * u + off * (1 + u))
        u = unit(KINDS[dtype])
        within(got["gain"], dgain, dgain.abs() * u + dgain_off * (1 + u))
        for name in got:                                     # alone, the same bits
            assert torch.equal(op.backward(gain, s, dy, dsum=ds if with_ds else None, want=[name])[name], got[name])


@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("T,D", [(2100, 1100), (1100, 2049), (1030, 8192), (530, 16384), (530, 16392), (261, 65536)])
def test_several_rows_a_block_and_in_place(dtype, residual, T, D):
    """Loads of the next row ahead of its turn, and wide rows that are read twice, where the results take the inputs' places."""
    s, ds, gain, gen = inputs(T, D, residual, residual, 2)
    gain = gain.to(KINDS[dtype])
    dy = randn(gen, T, D, dtype=KINDS[dtype])
    op = B.AddNorm(dtype, D, residual=residual, eps=EPS, max_tokens=T, training=True)
    got = op.backward(gain, s, dy, dsum=ds, want=("dx", "dresidual", "gain"))
    h = s.double()
    rstd = 1 / (h.square().mean(dim=1, keepdim=True) + op.cfg.eps).sqrt()
    n, g = h * rstd, dy.double() * gain.double()
    within(got["gain"], (dy.double() * n).sum(dim=0), (60 + T) * U32 * (dy.double() * n).abs().sum(dim=0) + unit(KINDS[dtype]) * (dy.double() * n).sum(dim=0).abs())
    dx = ds.double() + rstd * (g - n * (g * n).mean(dim=1, keepdim=True))
    off = 200 * U32 * (ds.double().abs() + rstd * (g.abs() + n.abs() * (g * n).abs().mean(dim=1, keepdim=True)))
    for k, kind in (("dx", dtype), ("dresidual", residual)):
        within(got[k], dx, off + unit(KINDS[kind]) * (dx.abs() + off))
    here = op.backward(gain, s, dy, dsum=ds, want=("dx", "dresidual", "gain"), out={"dx": dy, "dresidual": ds})
    assert here["dx"] is dy and here["dresidual"] is ds and all(torch.equal(here[k], got[k]) for k in got)


def test_gradients_against_differences():
    T, D = 6, 200
    x, r, gain, gen = inputs(T, D, "f32", "f32", 2)
    dy, ds, vs, vg = (randn(gen, *shape) for shape in ((T, D), (T, D), (T, D), (D,)))
    op = B.AddNorm("f32", D, eps=EPS, max_tokens=T, training=True)
    o = op.forward(gain, x, r)
    got = op.backward(gain, o["sum"], dy, dsum=ds)

    def loss(s, g):
        return (s / (s.square().mean(dim=1, keepdim=True) + EPS).sqrt() * g * dy.double()).sum() + (s * ds.double()).sum()

    s, g, e = o["sum"].double(), gain.double(), 1e-5
    for slope, grad, v in (((loss(s + e * vs.double(), g) - loss(s - e * vs.double(), g)) / (2 * e), got["dx"], vs),
                           ((loss(s, g + e * vg.double()) - loss(s, g - e * vg.double())) / (2 * e), got["gain"], vg)):
        # the difference is off by e^2 times a third derivative, of the order of the sizes here, and fp64 roundings of the loss over e
        size = (grad.double().abs() * v.double().abs()).sum()
        assert abs(slope - (grad.double() * v.double()).sum()) <= 1e-6 * size


def fp32_rows(x):
    """The definition of rows in 8 bits, operation by operation in fp32 (IEEE on the host)."""
    x = x.float().cpu().numpy()
    m = np.maximum(np.abs(x).max(axis=1), np.float32(LEAST)).astype(np.float32)
    return np.rint(x * (np.float32(127) / m)[:, None]).astype(np.int8), m * np.float32(1.0 / 127.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D", SIZES)
def test_quant_and_back(dtype, T, D):
    gen = generator(T + D)
    x = randn(gen, T, D, dtype=KINDS[dtype], std=0.02)
    q, scale = B.quant_rows(x)
    wq, ws = fp32_rows(x)
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(scale.cpu().numpy(), ws)
    for out in ("bf16", "f32"):
        v = B.dequant_rows(q, scale, out)
        assert torch.equal(v, (q.float() * scale[:, None]).to(KINDS[out]))


def test_quant_of_rows_apart_makes_dense_outputs():
    gen = generator(31)
    base = randn(gen, 12, 40)
    for x in (base[:, 3:20], base[::2, :1], base[5:6], base[5:6, 7:8], base.t()[:1, :1], base[4:5, :9].expand(1, 9)):
        q, scale = B.quant_rows(x)
        wq, ws = B.quant_rows(x.contiguous().clone(memory_format=torch.contiguous_format))
        assert q.is_contiguous() and q.dtype == torch.int8 and q.shape == x.shape and torch.equal(q, wq) and torch.equal(scale, ws)
        wide = torch.full((x.shape[0], x.shape[1] + 3), 99, dtype=torch.int8, device=DEV)
        wide[:, 1:-2] = q
        back = B.dequant_rows(wide[:, 1:-2], scale, "f32")
        assert back.is_contiguous() and torch.equal(back, q.float() * scale[:, None])


def test_quant_of_odd_values():
    inf, nan = float("inf"), float("nan")
    rows = [[0.0, -0.0, 0.0], [1e-38, -1e-38, 0.0], [3e38, -3e38, 1.0], [1.0, inf, 2.0], [1.0, -inf, nan], [nan, 1.0, 2.0], [127.0, 0.5, 1.5], [-127.0, 2.5, -0.5], [1.0, 1.0, 1.0]]
    x = torch.tensor(rows, device=DEV)
    q, scale = B.quant_rows(x)
    ok = torch.tensor([all(np.isfinite(r)) for r in rows])
    wq, ws = fp32_rows(x[ok.to(DEV)])
    assert np.array_equal(q.cpu().numpy()[ok.numpy()], wq) and np.array_equal(scale.cpu().numpy()[ok.numpy()], ws)
    assert (q.cpu()[~ok] == 0).all() and torch.isnan(scale.cpu()[~ok]).all()
    assert q[6].tolist() == [127, 0, 2] and q[7].tolist() == [-127, 2, 0] and q[1].tolist() == [0, 0, 0]
    # ... wherever in a long row they stand
    for D in (500, 5000, 40000):
        x = torch.ones(3, D, device=DEV)
        x[0, D - 1], x[2, 0] = nan, -inf
        q, scale = B.quant_rows(x)
        assert torch.isnan(scale[[0, 2]]).all() and (q[[0, 2]] == 0).all() and (q[1] == 127).all() and not torch.isnan(scale[1])
    op = B.AddNorm("f32", 8, max_tokens=2)
    x = torch.ones(2, 8, device=DEV)
    x[0, 3] = inf
    o = op.forward(torch.ones(8, device=DEV), x, want=("y", "q"))
    assert torch.isnan(o["y"][0, 3]) and torch.isnan(o["scale"][0]) and (o["q"][0] == 0).all() and (o["q"][1] == 127).all()


def test_a_row_that_is_not_finite_stays_alone():
    T, D = 40, 3200
    x, r, gain, gen = inputs(T, D, "bf16", "f32", 5)
    op = B.AddNorm("bf16", D, residual="f32", max_tokens=T, training=True)
    want, wq = op.forward(gain, x, r, want=("sum", "y", "q")), B.quant_rows(x)
    dy = randn(gen, T, D, dtype=torch.bfloat16)
    wdx = op.backward(gain, want["sum"], dy)["dx"]
    x[7, 3000], x[9, 0], x[30, 17] = float("nan"), float("inf"), float("-inf")
    got, gq = op.forward(gain, x, r, want=("sum", "y", "q")), B.quant_rows(x)
    bad = torch.zeros(T, dtype=torch.bool, device=DEV)
    bad[[7, 9, 30]] = True
    for n in ("sum", "y", "q", "scale"):
        assert torch.equal(got[n][~bad], want[n][~bad]), n
    assert torch.isnan(got["scale"][bad]).all() and (got["q"][bad] == 0).all() and torch.isnan(got["y"][7]).all()
    for a, b in zip(gq, wq):
        assert torch.equal(a[~bad], b[~bad])
    assert torch.isnan(gq[1][bad]).all() and torch.isnan(B.dequant_rows(*gq)[bad]).all()
    back = op.backward(gain, got["sum"], dy)
    assert torch.equal(back["dx"][~bad], wdx[~bad]) and torch.isnan(back["dx"][bad].float()).any(dim=1).all()


def test_a_sum_alone_needs_no_gain():
    x, r, _, _ = inputs(5, 100, "bf16", "f32", 6)
    op = B.AddNorm("bf16", 100, residual="f32", max_tokens=5)
    assert torch.equal(op.forward(None, x, r, want=("sum",))["sum"], x.float() + r)
    for want in ((), ("dx",), ("sum", "scale")):
        with pytest.raises((ValueError, B.EpdError)):
            op.forward(None, x, r, want=want)


def test_zero_rows():
    op = B.AddNorm("bf16", 40, max_tokens=3, training=True)
    z, gain = torch.zeros(3, 40, dtype=torch.bfloat16, device=DEV), torch.ones(40, dtype=torch.bfloat16, device=DEV)
    o = op.forward(gain, z, z, want=("sum", "y", "q"))
    assert all((o[n] == 0).all() for n in ("sum", "y", "q")) and torch.isfinite(o["scale"]).all()
    g = op.backward(gain, z, torch.ones_like(z), want=("dx", "gain"))
    assert torch.isfinite(g["dx"].float()).all() and (g["gain"] == 0).all()


@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("D", [77, 1153, 3200, 9001])
def test_rows_apart_in_place_and_rows_behind(dtype, residual, D):
    T = 13
    x, r, gain, gen = inputs(T, D, dtype, residual, 3)
    op = B.AddNorm(dtype, D, residual=residual, max_tokens=20, training=True)
    want = op.forward(gain, x, r, want=("sum", "y", "q"))
    gx, gr = Gapped(T, D, KINDS[dtype], gap=3, offset=1, values=x), Gapped(T, D, KINDS[residual], gap=1, offset=5, values=r)
    outs = {"sum": Gapped(T, D, KINDS[residual], gap=9, offset=2), "y": Gapped(T, D, KINDS[dtype], gap=2, offset=1), "q": Gapped(T, D, torch.int8, gap=1, offset=1)}
    got = op.forward(gain, gx.view, gr.view, want=("sum", "y", "q"), out={n: g.view for n, g in outs.items()})
    for n in outs:
        assert torch.equal(got[n], want[n]) and outs[n].untouched()
    assert torch.equal(got["scale"], want["scale"]) and gx.untouched() and gr.untouched()
    got = op.forward(gain, gx.view, gr.view, out={"sum": gr.view, "y": gx.view})       # in place
    assert torch.equal(gr.view, want["sum"]) and torch.equal(gx.view, want["y"]) and gx.untouched() and gr.untouched()
    dy, ds = randn(gen, T, D, dtype=KINDS[dtype]), randn(gen, T, D, dtype=KINDS[residual])
    back = op.backward(gain, want["sum"], dy, dsum=ds, want=("dx", "dresidual", "gain"))
    gs, gy, gd = Gapped(T, D, KINDS[residual], values=want["sum"]), Gapped(T, D, KINDS[dtype], gap=1, offset=1, values=dy), Gapped(T, D, KINDS[residual], gap=7, values=ds)
    got = op.backward(gain, gs.view, gy.view, dsum=gd.view, want=("dx", "dresidual", "gain"), out={"dx": gy.view, "dresidual": gd.view})
    assert all(torch.equal(got[n], back[n]) for n in back) and gs.untouched() and gy.untouched() and gd.untouched()
    q, scale = B.quant_rows(Gapped(T, D, KINDS[dtype], gap=1, offset=1, values=x).view)
    assert torch.equal(q, B.quant_rows(x)[0])
    gq, go = Gapped(T, D, torch.int8, gap=5, offset=1, values=q), Gapped(T, D, KINDS[dtype], gap=3, offset=1)
    assert torch.equal(B.dequant_rows(gq.view, scale, dtype, out=go.view), B.dequant_rows(q, scale, dtype)) and go.untouched()
    # every row the same: a stride of no elements is refused by the outputs, and a broadcast input too
    with pytest.raises(B.EpdError):
        op.forward(gain, x[:1].expand(T, D), r)


def test_no_rows_and_one_row_of_any_stride():
    op = B.AddNorm("bf16", 24, max_tokens=4, training=True)
    gain = torch.ones(24, dtype=torch.bfloat16, device=DEV)
    none = torch.empty(0, 24, dtype=torch.bfloat16, device=DEV)
    assert op.forward(gain, none, none)["y"].shape == (0, 24)
    g = op.backward(gain, none, none, want=("dx", "gain"))
    assert (g["gain"] == 0).all() and g["dx"].shape == (0, 24)
    q, scale = B.quant_rows(none)
    assert q.shape == (0, 24) and scale.shape == (0,) and B.dequant_rows(q, scale).shape == (0, 24)
    one = torch.randn(1, 24, device=DEV).to(torch.bfloat16).as_strided((1, 24), (3, 1))
    assert torch.equal(op.forward(gain, one, one)["sum"], one + one)


@pytest.mark.parametrize("D", [320, 3200])
def test_captured_and_replayed(D):
    T = 100
    x, r, gain, gen = inputs(T, D, "bf16", "f32")
    op = B.AddNorm("bf16", D, residual="f32", max_tokens=T, training=True)
    dy = randn(gen, T, D, dtype=torch.bfloat16)

    def change(i):
        x.copy_(randn(generator(i), T, D, dtype=torch.bfloat16))

    def call():
        o = op.forward(gain, x, r, want=("sum", "y", "q"))
        b = op.backward(gain, o["sum"], dy, dsum=o["sum"])
        return [*o.values(), *b.values(), *B.quant_rows(x), B.dequant_rows(o["q"], o["scale"])]

    replays(call, lambda v: v, change)


def test_two_objects_on_two_streams():
    T, D = 2000, 1024
    ops = [B.AddNorm("bf16", D, max_tokens=T, training=True) for _ in range(2)]
    data = [inputs(T, D, "bf16", "bf16", 10 + k) for k in range(2)]
    want = [op.backward(g, x, r)["gain"].clone() for op, (x, r, g, _) in zip(ops, data)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got.append((k, ops[k].backward(data[k][2], data[k][0], data[k][1])["gain"]))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[k]) for k, g in got)


def test_arrays_beyond_2_31_elements():
    T, D = 33000, 65536                                      # 2^31 + 15 million
    op = B.AddNorm("bf16", D, max_tokens=T, training=True)
    gain = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    x = torch.ones(T, D, dtype=torch.bfloat16, device=DEV)
    x[-1] = 2.0
    x[-1, ::2] = -2.0
    o = op.forward(gain, x, x, want=("sum", "q"))
    assert (o["sum"][0] == 2).all() and torch.equal(o["sum"][-1], 2 * x[-1]) and torch.equal(o["q"][-1].float(), 127 * torch.sign(x[-1].float()))
    assert (o["q"][T // 2] == 127).all()
    v = B.dequant_rows(o["q"], o["scale"])
    assert torch.equal(v[-1], torch.sign(x[-1]))
    del v, x
    q, scale = B.quant_rows(o["sum"])
    assert torch.equal(q[-1], o["q"][-1]) and abs(scale[-1].item() * 127 - 4) < 1e-6
    g = op.backward(gain, o["sum"], o["sum"], want=("dx", "gain"))
    # dy along s: dx = rstd (g - n mean(g n)) is s eps / (mean s^2 + eps) and less, at most 2^-20 here with its roundings; gain's is sum dy n = sum |s|
    assert g["dx"][-1].float().abs().max() < 2e-5 * 4
    assert ((g["gain"].float() / (2.0 * (T - 1) + 4.0) - 1).abs() <= 2.0 ** -8 + (T + 60) * U32).all()
