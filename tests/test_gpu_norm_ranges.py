"""AddNorm on rows whose squares, or their sum, leave fp32 while the rows and their norms do not: far apart magnitudes, one in each row, against
the definition in 64 bits.

Tolerances.  As in test_gpu_add_norm.py, whose roundings are the same: powers of two that a row is multiplied by for its sums round nothing that
counts there (at most 2^-149 of values of which one is beyond 2^-30).  One rounding is added where 1 / rms is below the normal numbers, of half of
2^-149, and 1 / rms is at least 2^-128: 4 half steps of fp32.  So y is within 58 half steps, dx within 204."""

import pytest
import torch

from entry_util import DEV, KINDS, U32, generator, randn, unit, within
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
WIDTHS = [7, 64, 300, 1000, 1500, 3200, 5000, 12000, 20000, 50000]          # every kernel that by_width chooses
LEAST = 2.0 ** -100
EXPONENTS = {0.0: [0, 58, 60, 62, 63, 64, 65, 90, 120, 126, -20, -45, -50, -51, -55, -63, -64, -75, -100, -120, -126],
             2.0 ** -120: [0, 62, 64, 126, -50, -55, -58, -60, -62, -64, -75, -100, -130],
             1e-6: [0, 8, 58, 60, 62, 63, 64, 65, 90, 126, -10, -20, -64, -75, -130]}


def rows(gen, exponents, D, dtype):
    """Normal values, cut at 3, times 2^e in row e."""
    e = torch.tensor(exponents, dtype=torch.float64, device=DEV)
    v = torch.randn(len(exponents), D, generator=gen, device=DEV).clamp(-3, 3).double()
    v[:, 0] = 1.5                                            # (no row of zeros, however short)
    return (v * torch.exp2(e)[:, None]).to(KINDS[dtype])


def normed(s, gain, eps):
    return s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt() * gain.double()


@pytest.mark.parametrize("eps", EXPONENTS)
@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(dtype, residual, D, eps):
    gen, e = generator(D), EXPONENTS[eps]
    gain = (1 + 0.3 * randn(gen, D)).to(KINDS[dtype])
    op = B.AddNorm(dtype, D, residual=residual, eps=eps, max_tokens=len(e))
    x, r = rows(gen, [k - 1 for k in e], D, dtype), rows(gen, [k - 1 for k in e], D, residual)
    for kw, s in (({"residual": r}, r.double()), ({"x": x, "residual": r}, x.double() + r.double())):
        got = op.forward(gain, want=("sum", "y", "q"), **kw)
        assert torch.isfinite(s.float()).all()
        y = normed(s, gain, op.cfg.eps)
        within(got["y"], y, y.abs() * ((unit(KINDS[dtype]) if dtype == "bf16" else 0.0) + 58 * U32))
        within(got["sum"], s, s.abs() * ((unit(KINDS[residual]) if residual == "bf16" else 0.0) + 2 * U32))
        m, step, off = y.abs().amax(dim=1, keepdim=True).clamp(min=LEAST), got["scale"].double()[:, None], 61 * U32
        within(step, m / 127, m / 127 * off)
        within(got["q"].double() * step, y, step * (0.5 + 128 * off))
        for k in range(len(e)):                              # a row's bits do not depend on its neighbours
            one = op.forward(gain, want=("y", "q"), **{n: t[k:k + 1] for n, t in kw.items()})
            assert all(torch.equal(one[n], got[n][k:k + 1]) for n in one)


@pytest.mark.parametrize("eps", EXPONENTS)
@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(dtype, residual, D, eps):
    gen = generator(D + 1)
    gain = (1 + 0.3 * randn(gen, D)).to(KINDS[dtype])
    T, u = 3, unit(KINDS[dtype])
    op = B.AddNorm(dtype, D, residual=residual, eps=eps, max_tokens=T, training=True)
    for e in EXPONENTS[eps]:
        if not -120 <= e <= 120:                             # (gradients of such rows leave fp32 themselves)
            continue
        s = rows(gen, [e] * T, D, residual)
        h = s.double()
        rstd = 1 / (h.square().mean(dim=1, keepdim=True) + op.cfg.eps).sqrt()
        half = (e / 2) if eps == 0.0 else max(e / 2, 0)      # gradients whose dx is of the size of 1 / sqrt(rms)
        dy, ds = rows(gen, [half] * T, D, dtype), rows(gen, [half + float(rstd.log2().mean())] * T, D, residual)
        got = op.backward(gain, s, dy, dsum=ds, want=("dx", "dresidual", "gain"))
        n, g = h * rstd, dy.double() * gain.double()
        dgain = (dy.double() * n).sum(dim=0)
        within(got["gain"], dgain, dgain.abs() * u + (64 + T) * U32 * (dy.double() * n).abs().sum(dim=0) * (1 + u))
        dx = ds.double() + rstd * (g - n * (g * n).mean(dim=1, keepdim=True))
        off = 204 * U32 * (ds.double().abs() + rstd * (g.abs() + n.abs() * (g * n).abs().mean(dim=1, keepdim=True)))
        for name, kind in (("dx", dtype), ("dresidual", residual)):
            within(got[name], dx, dx.abs() * unit(KINDS[kind]) + off * (1 + unit(KINDS[kind])))


@pytest.mark.parametrize("D", [300, 3200, 20000])
def test_rows_without_a_norm_stay_as_they_are(D):
    """Zeros over zero are NaN, an infinity is NaN beside zeros, and neither touches the rows of extreme sizes beside it."""
    gen = generator(D + 2)
    e = [100, 0, -100, 0, 64, 0]
    x = rows(gen, e, D, "f32")
    gain = torch.ones(D, device=DEV)
    op = B.AddNorm("f32", D, eps=0.0, max_tokens=len(e))
    want = op.forward(gain, x, want=("y",))["y"]
    x[1], x[3, 5], x[5, D - 1] = 0.0, float("inf"), float("nan")
    got = op.forward(gain, x, want=("y", "q"))
    y = got["y"]
    assert torch.equal(y[[0, 2, 4]], want[[0, 2, 4]]) and torch.isnan(y[1]).all() and torch.isnan(y[5]).all()
    assert torch.isnan(y[3, 5]) and (y[3, :5] == 0).all() and (y[3, 6:] == 0).all()
    assert torch.isnan(got["scale"][[1, 3, 5]]).all() and (got["q"][[1, 3, 5]] == 0).all()
    x = torch.full((1, D), 2.0 ** -140, device=DEV)          # 1 / rms is 2^140: the largest number stands for it
    assert torch.equal(op.forward(gain, x, want=("y",))["y"], x * torch.finfo(torch.float32).max)
    assert B.AddNorm("f32", D, eps=2.0 ** -120, max_tokens=1).forward(gain, torch.zeros(1, D, device=DEV), want=("y",))["y"].abs().max() == 0
