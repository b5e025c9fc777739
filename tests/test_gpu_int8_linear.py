"""Int8Linear (epd_int8_linear) against the definition in 64 bits.  Tolerance: the sum is exact in int32; fp32 rounds it once, both products
with scales once each and the bias' addition once, and the result is rounded to its type."""

import pytest
import torch

from entry_util import DEV, KINDS, U32, Gapped, generator, randn, replays, unit, within
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu


def operands(T, K, N, seed=0, full=False):
    gen = generator(T + 3 * K + 5 * N + seed)
    lo, hi = (-128, 128) if full else (-40, 41)
    x, w = (torch.randint(lo, hi, s, generator=gen, device=DEV, dtype=torch.int32).to(torch.int8) for s in ((T, K), (N, K)))
    return x, 0.01 + torch.rand(T, generator=gen, device=DEV), {"w": w, "scale": 0.001 + torch.rand(N, generator=gen, device=DEV), "bias": randn(gen, N, std=20.0)}


def check(y, x, xs, w, bias):
    acc = x.double() @ w["w"].double().t()                   # whole numbers below 2^53: exact
    prod = acc * xs.double()[:, None] * w["scale"].double()
    b = w["bias"].double() if bias else torch.zeros_like(w["scale"]).double()
    exact, u = prod + b, unit(y.dtype) if y.dtype != torch.float32 else 0.0
    within(y, exact, exact.abs() * u + 5 * U32 * (prod.abs() + b.abs()) * (1 + u))


SIZES = [(1, 16, 8), (1, 3200, 136), (1, 2064, 4096), (1, 1040, 72), (2, 32, 16), (3, 48, 24), (5, 128, 8), (15, 1024, 40), (16, 3200, 264), (17, 144, 136), (31, 272, 72), (32, 1024, 128), (33, 400, 64),
         (63, 1152, 200), (64, 2048, 512), (65, 112, 320), (100, 640, 1032), (128, 128, 256), (129, 1136, 264), (255, 64, 520), (257, 1152, 304), (300, 4112, 64),
         (513, 528, 776), (640, 16, 640), (1000, 80, 1000), (2049, 336, 264)]

# a size for every tile, whole, cut behind its whole rounds, and in parts (test_entry_host_logic.py counts them)
PLANS = [(1, 5008, 8), (2, 16, 8328), (35, 16, 5160), (61, 1040, 8192), (64, 8192, 264), (64, 8208, 264), (65, 6272, 3736), (1340, 896, 14648), (4256, 8416, 72), (5697, 14816, 392), (6160, 544, 4208), (10362, 7360, 72),
         (16779, 5200, 80), (18230, 8336, 136), (19241, 144, 680), (25656, 16, 648), (28671, 96, 432), (32410, 3952, 648), (32554, 992, 160), (33870, 7072, 168),
         (36136, 16, 424), (38188, 16, 8), (44024, 3008, 312), (45731, 1840, 88)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("T,K,N", SIZES + PLANS)
def test_product(out, T, K, N):
    for bias, full in ((False, False), (True, True)):
        x, xs, w = operands(T, K, N, full=full)
        y = B.Int8Linear(K, N, out=out, max_tokens=T, use_bias=bias).forward(w, x, xs)
        assert y.dtype == KINDS[out]
        check(y, x, xs, w, bias)


def test_largest_sums():
    # K at its largest, every product the largest there is: 131056 * 2^14 < 2^31
    for K, T in ((131056, 1), (131056, 3), (131056, 70), (131056, 300)):
        x = torch.full((T, K), -128, dtype=torch.int8, device=DEV)
        w = {"w": torch.full((16, K), -128, dtype=torch.int8, device=DEV), "scale": torch.ones(16, device=DEV)}
        w["w"][3] = 127
        y = B.Int8Linear(K, 16, out="f32", max_tokens=T).forward(w, x, torch.ones(T, device=DEV))
        want = torch.full((16,), 128.0 * 128 * K, device=DEV)
        want[3] = -128.0 * 127 * K
        assert torch.equal(y, want.expand(T, 16)), (K, T)


@pytest.mark.parametrize("T", [1, 7, 40, 65, 300, 1100])
def test_rows_apart_and_rows_behind(T):
    K, N = 144, 136
    x, xs, w = operands(T, K, N, 1)
    for out in ("bf16", "f32"):
        op = B.Int8Linear(K, N, out=out, max_tokens=2000, use_bias=True)
        want = op.forward(w, x, xs)
        gx, y = Gapped(T, K, torch.int8, gap=16, offset=16, values=x), Gapped(T, N, KINDS[out], gap=8, offset=8)
        op.forward(w, gx.view, xs, out=y.view)
        assert torch.equal(y.view, want) and y.untouched()


@pytest.mark.parametrize("T", [1, 4, 33, 200, 700])
def test_a_row_of_nan_stays_alone(T):
    K, N = 320, 264
    x, xs, w = operands(T, K, N, 2)
    op = B.Int8Linear(K, N, max_tokens=T)
    want = op.forward(w, x, xs)
    xs[T // 2] = float("nan")
    y = op.forward(w, x, xs)
    assert torch.isnan(y[T // 2]).all()
    keep = torch.arange(T, device=DEV) != T // 2
    assert torch.equal(y[keep], want[keep])


@pytest.mark.parametrize("T,K,N", [(1, 3200, 264), (20, 1024, 264), (90, 4096, 128), (700, 256, 520)])
def test_captured_and_replayed(T, K, N):
    x, xs, w = operands(T, K, N)
    op = B.Int8Linear(K, N, max_tokens=T, use_bias=True)

    def change(i):
        a, s, _ = operands(T, K, N, 10 + i)
        x.copy_(a)
        xs.copy_(s)

    replays(lambda: [op.forward(w, x, xs)], lambda v: v, change)


def test_no_tokens():
    op = B.Int8Linear(32, 16, max_tokens=4)
    _, _, w = operands(1, 32, 16)
    assert op.forward(w, torch.empty(0, 32, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV)).shape == (0, 16)


def test_outputs_beyond_2_31_elements():
    T, K, N = 262144, 16, 8328
    x, xs, w = operands(T, K, N, 4)
    y = B.Int8Linear(K, N, max_tokens=T).forward(w, x, xs)
    for a in (0, 130000, T - 300):
        check(y[a:a + 300], x[a:a + 300], xs[a:a + 300], w, False)
