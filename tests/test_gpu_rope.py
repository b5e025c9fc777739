"""Rotary positions with several axes as an operator of its own: rotation, inverse, positions of mixed
sequences, against plain float64 / integer implementations."""

import numpy as np
import pytest
import torch

from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# One rounding to the type is off by at most eps / 2 of the value; the fp32 arithmetic before it: cos and sin within 1e-7
# (polynomials 2e-9, their roundings, the reduced angle's), two products and a sum, 4 * 2^-24 of |x| + |y| in all.
ARITH = 5e-7


def tables(pairs, layout, ladder, base):
    order = [(a, j) for a, n in enumerate(pairs) for j in range(n)]
    if layout == "interleaved":
        order.sort(key=lambda e: (e[1], e[0]))
    P = len(order)
    f = [base ** (-(j / pairs[a]) if ladder == "axis" else -(p / P)) for p, (a, j) in enumerate(order)]
    return np.array([a for a, _ in order]), np.array(f)


def plain(x, pos, pairs, layout, ladder, pairing, base=10000.0, inverse=False):
    """x [T, H, d] float64, pos [axes, T] int: the definition, and |x| + |y| of every element's pair."""
    axis, f = tables(pairs, layout, ladder, base)
    P = len(axis)
    ang = pos.astype(np.float64)[axis].T * f
    if inverse:
        ang = -ang
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    i = np.arange(P)
    lo, hi = (i, i + P) if pairing == "half" else (2 * i, 2 * i + 1)
    y, size = x.copy(), np.abs(x)
    y[..., lo], y[..., hi] = x[..., lo] * c - x[..., hi] * s, x[..., lo] * s + x[..., hi] * c
    size[..., lo] = size[..., hi] = np.abs(x[..., lo]) + np.abs(x[..., hi])
    return y, size


def check(got, x, pos, pairs, layout, ladder, pairing, **kw):
    want, size = plain(x.double().cpu().numpy(), pos.cpu().numpy(), pairs, layout, ladder, pairing, **kw)
    err = np.abs(got.double().cpu().numpy() - want)
    half = torch.finfo(got.dtype).eps / 2
    # the value that is rounded is off by ARITH * size, so the rounding is of that value
    tol = half * np.abs(want) + (1 + half) * ARITH * size
    assert (err <= tol).all(), (err - tol).max()


def rand(*shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV, dtype=torch.float32).to(dtype)


def positions(axes, T, far, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(0, far, (axes, T), generator=g, device=DEV, dtype=torch.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,ladder,pairing", [("sections", "axis", "half"), ("interleaved", "head", "half"), ("sections", "head", "adjacent"), ("interleaved", "axis", "adjacent")])
@pytest.mark.parametrize("T,hq,hk,d,pairs", [(1, 1, 1, 2, (1,)), (5, 3, 1, 72, (0, 18, 18)), (33, 32, 8, 128, (24, 20, 20)), (257, 4, 2, 64, (3, 5, 7)),
                                            (2, 5, 5, 80, (7, 6, 0, 7)), (300, 7, 7, 96, (48,)), (1500, 2, 1, 256, (100, 20, 8)), (3, 256, 1, 256, (1,))])
def test_rotation_and_inverse(dtype, layout, ladder, pairing, T, hq, hk, d, pairs):
    op = B.Rope(dtype, d, pairs, layout=layout, ladder=ladder, pairing=pairing)
    q, k = (rand(T, h, d, dtype=op.dtype, seed=s) for s, h in ((1, hq), (2, hk)))
    pos = positions(len(pairs), T, 5000, 3)
    for inverse in (False, True):
        for x, y in zip((q, k), op.apply([q, k], pos, inverse=inverse)):
            check(y, x, pos, pairs, layout, ladder, pairing, inverse=inverse)


def test_views_in_place_and_head_major_outputs():
    T, hq, hk, d, pairs = 37, 6, 2, 72, (4, 14, 14)
    op = B.Rope("bf16", d, pairs, layout="interleaved")
    packed = rand(T, (hq + 2 * hk) * d, dtype=torch.bfloat16, seed=5)
    q, k = packed[:, :hq * d].view(T, hq, d), packed[:, hq * d:(hq + hk) * d].view(T, hk, d)
    pos = positions(3, T + 9, 900, 6)[:, 4:4 + T]                     # rows of a longer table
    a, b = op.apply([q, k], pos)
    check(a, q, pos, pairs, "interleaved", "axis", "half")
    major = torch.zeros(hq, T + 3, d, dtype=torch.bfloat16, device=DEV)   # [heads, tokens, d] of a cache with room
    op.apply([q], pos, out=[major[:, :T].transpose(0, 1)])
    assert torch.equal(major[:, :T].transpose(0, 1), a) and not major[:, T:].any()
    before = packed.clone()
    op.apply([q, k], pos, out=[q, k])
    assert torch.equal(q, a) and torch.equal(k, b)
    assert torch.equal(packed[:, (hq + hk) * d:], before[:, (hq + hk) * d:])        # v stays


@pytest.mark.parametrize("shift", [0, 1, 2, 3, 4])
def test_rows_at_any_alignment(shift):
    T, h, d, pairs = 19, 3, 64, (10, 11, 11)
    for pairing in ("half", "adjacent"):
        op = B.Rope("bf16", d, pairs, pairing=pairing)
        wide = rand(T, h * (d + 5) + 8, dtype=torch.bfloat16, seed=7)
        x = torch.as_strided(wide, (T, h, d), (wide.stride(0), d + 5, 1), shift)
        pos = positions(3, T, 100, 8)
        check(op.apply([x], pos)[0], x, pos, pairs, "sections", "axis", pairing)


def test_a_broadcast_input_turns_by_every_position():
    d, pairs, T = 32, (8, 4, 4), 11
    op = B.Rope("f32", d, pairs)
    x = rand(1, 1, d, dtype=torch.float32, seed=9).expand(T, 3, d)
    pos = positions(3, T, 50, 10)
    check(op.apply([x], pos)[0], x, pos, pairs, "sections", "axis", "half")


def test_far_and_negative_positions_keep_their_phase():
    d, pairs = 64, (16, 8, 8)
    op = B.Rope("f32", d, pairs)
    pos = torch.tensor([[0, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, 123456789]] * 3, dtype=torch.int32, device=DEV)
    x = rand(6, 2, d, dtype=torch.float32, seed=11)
    y = op.apply([x], pos)[0]
    # 2^31 radians at 2^-53: 2.4e-7 both in the reference and here, on top of the fp32 arithmetic
    want, size = plain(x.double().cpu().numpy(), pos.cpu().numpy(), pairs, "sections", "axis", "half")
    assert (np.abs(y.double().cpu().numpy() - want) <= 2 ** -24 * np.abs(want) + (ARITH + 5e-7) * size).all()
    assert torch.equal(op.apply([x], torch.zeros_like(pos))[0], x)


def test_the_inverse_is_the_gradient_also_by_differences():
    d, pairs, T, h = 16, (3, 2, 3), 4, 2
    op = B.Rope("f32", d, pairs, pairing="adjacent")
    x, dy, pos = rand(T, h, d, dtype=torch.float32, seed=12), rand(T, h, d, dtype=torch.float32, seed=13), positions(3, T, 40, 14)
    grad = op.apply([dy], pos, inverse=True)[0].double()
    # the map is linear: the difference over a step of one is the derivative, but for roundings
    for t, hh, e in [(0, 0, 0), (1, 1, 3), (3, 0, 15), (2, 1, 8)]:
        step = torch.zeros_like(x)
        step[t, hh, e] = 1.0
        diff = (op.apply([x + step], pos)[0].double() - op.apply([x], pos)[0].double()) * dy.double()
        assert abs(float(diff.sum() - grad[t, hh, e])) <= 16 * 1e-6 * float(dy.abs().max())


def test_infinities_and_nan_stay_in_their_pair():
    d, pairs = 64, (16, 8, 8)
    op = B.Rope("bf16", d, pairs)
    x = rand(3, 2, d, dtype=torch.bfloat16, seed=15)
    x[1, 0, 5], x[1, 1, 40] = float("nan"), float("inf")
    y = op.apply([x], positions(3, 3, 50, 16))[0]
    bad = ~torch.isfinite(y)
    allowed = torch.zeros_like(bad)
    allowed[1, 0, [5, 37]] = True
    allowed[1, 1, [40, 8]] = True
    assert not (bad & ~allowed).any() and bad[1, 0, 5] and bad[1, 0, 37]


def test_empty_calls_write_nothing():
    op = B.Rope("bf16", 64, (32,))
    x = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    assert op.apply([x], torch.empty(1, 0, dtype=torch.int32, device=DEV))[0].shape == (0, 4, 64)
    none = torch.empty(3, 0, 64, dtype=torch.bfloat16, device=DEV)
    y = rand(3, 2, 64, dtype=torch.bfloat16, seed=17)
    pos = positions(1, 3, 9, 18)
    a, b = op.apply([none, y], pos)
    assert a.shape == (3, 0, 64)
    check(b, y, pos, (32,), "sections", "axis", "half")


def test_another_stream_and_a_graph_replayed_on_new_data():
    op = B.Rope("bf16", 128, (24, 20, 20), layout="interleaved", ladder="head")
    q, k = rand(65, 8, 128, dtype=torch.bfloat16, seed=19), rand(65, 2, 128, dtype=torch.bfloat16, seed=20)
    pos = positions(3, 65, 4000, 21)
    out = [torch.empty_like(q), torch.empty_like(k)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        op.apply([q, k], pos, out=out)
    s.synchronize()
    check(out[0], q, pos, (24, 20, 20), "interleaved", "head", "half")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op.apply([q, k], pos, out=out)
    for seed in (30, 31, 32):
        q.copy_(rand(65, 8, 128, dtype=torch.bfloat16, seed=seed))
        pos.copy_(positions(3, 65, 4000, seed))
        out[0].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], op.apply([q, k], pos)[0])


# ------------------------------------------------------------------ positions

def walk(spans, cu, start, t_step):
    cols, after = [], []
    for s in range(len(cu) - 1):
        p = int(start[s])
        for t, h, w in spans[cu[s]:cu[s + 1]]:
            if h == 0:
                cols += [(p + i,) * 3 for i in range(t)]
                p += t
            else:
                cols += [(p + t_step * ti, p + r, p + c) for ti in range(t) for r in range(h) for c in range(w)]
                p += max(t_step * (t - 1) + 1, h, w)
        after.append(p)
    return np.array(cols, dtype=np.int32).reshape(-1, 3).T, np.array(after, dtype=np.int32)


def random_spans(seed, n_seq, most):
    rng = np.random.default_rng(seed)
    spans, cu = [], [0]
    for _ in range(n_seq):
        for _ in range(int(rng.integers(0, most + 1))):
            if rng.random() < 0.5:
                spans.append((int(rng.integers(0, 40)), 0, 0))
            else:
                spans.append(tuple(int(v) for v in rng.integers(1, 9, 3)))
        cu.append(len(spans))
    return spans, cu, rng.integers(0, 1000, n_seq)


@pytest.mark.parametrize("seed,n_seq,most,t_step", [(0, 1, 1, 1), (1, 1, 7, 0), (2, 9, 5, 3), (3, 70, 9, 2), (4, 240, 3, 1), (5, 2, 700, 1)])
def test_positions_of_mixed_sequences(seed, n_seq, most, t_step):
    spans, cu, start = random_spans(seed, n_seq, most)
    want, after = walk(spans, cu, start, t_step)
    got, nxt = B.rope_positions(spans, cu, start=start, t_step=t_step)
    assert np.array_equal(got.cpu().numpy(), want) and np.array_equal(nxt, after)


@pytest.mark.parametrize("n", [0, 1, 239, 240, 241, 480, 481])
def test_positions_over_several_launches(n):
    spans = [((i % 5) + 1, 0, 0) if i % 3 else (1, 2, i % 4 + 1) for i in range(n)]
    want, after = walk(spans, [0, n], [7], 1)
    room = torch.full((3, want.shape[1] + 5), -9, dtype=torch.int32, device=DEV)
    got, nxt = B.rope_positions(spans, [0, n], start=[7], out=room)
    assert np.array_equal(got.cpu().numpy()[:, :want.shape[1]], want) and np.array_equal(nxt, after)
    assert (got[:, want.shape[1]:] == -9).all()


def test_a_conversation_goes_on_where_it_stopped():
    spans = [(5, 0, 0), (2, 4, 6), (3, 0, 0), (1, 8, 2), (4, 0, 0)]
    whole, end = B.rope_positions(spans, [0, 5])
    a, mid = B.rope_positions(spans[:2], [0, 2])
    b, last = B.rope_positions(spans[2:], [0, 3], start=mid)
    assert torch.equal(torch.cat([a, b], dim=1), whole) and last[0] == end[0]
    alone, _ = B.rope_positions([(2, 4, 6)], [0, 1])                  # an item alone: the raster coordinates of the encoder
    want = np.indices((2, 4, 6)).reshape(3, -1)
    assert np.array_equal(alone.cpu().numpy(), want)


def test_positions_in_a_graph():
    spans, cu = [(3, 0, 0), (1, 5, 5), (9, 0, 0)], [0, 3]
    out = torch.zeros(3, 37, dtype=torch.int32, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.rope_positions(spans, cu, out=out)
    want, _ = walk(spans, cu, [0], 1)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), want)
