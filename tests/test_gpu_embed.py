"""Embedding.forward / backward (epd_embed, epd_embed_backward) against the definition in 64 bits.

Tolerances.  Forward: one fp32 product and one rounding.  Backward: n values added in fp32 in any order are within (n - 1) half steps of the
sum of their magnitudes, then one product and one rounding."""

import pytest
import torch

from entry_util import DEV, KINDS, U32, Gapped, generator, randn, replays, unit, within
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
NONE = 2 ** 31 - 1


def some_ids(gen, T, V, R, hot=0.2, none=0.1):
    ids = torch.randint(0, V, (T,), generator=gen, device=DEV)
    draw = torch.rand(T, generator=gen, device=DEV)
    ids = torch.where(draw < hot, torch.full_like(ids, V // 3), ids)
    if R:
        ids = torch.where(draw > 0.6, -1 - torch.randint(0, R, (T,), generator=gen, device=DEV), ids)
    ids = torch.where((draw > hot) & (draw < hot + none), torch.full_like(ids, NONE), ids)
    for i, odd in enumerate((V, -R - 1, -2 ** 31)):          # nearest ids of no row, and the lowest
        if T > 40 + i:
            ids[20 + i] = odd
    return ids.to(torch.int32)


def keys_of(ids, V, R):
    i = ids.long()
    return torch.where((i >= 0) & (i < V), i, torch.where((i < 0) & (i >= -R), V - 1 - i, torch.full_like(i, V + R)))


def check_forward(out, table, rows, ids, scale, V, R):
    every = torch.cat([table.double() * scale] + ([rows.double()] if R else []) + [table.new_zeros(1, table.shape[1]).double()])
    exact = every[keys_of(ids, V, R)]
    within(out, exact, exact.abs() * ((unit(out.dtype) if out.dtype != torch.float32 else 0.0) + 2 * U32))


def check_backward(got, dout, ids, scale, V, R, dtype):
    D, key = dout.shape[1], keys_of(ids, V, R)
    n = torch.bincount(key, minlength=V + R + 1)[:, None].double()
    sums, mags = (torch.zeros(V + R + 1, D, dtype=torch.float64, device=DEV).index_add_(0, key, d) for d in (dout.double(), dout.double().abs()))
    for name, a, b, s in (("table", 0, V, scale), ("rows", V, V + R, 1.0)):
        if name not in got:
            continue
        exact = sums[a:b] * s
        within(got[name], exact, exact.abs() * unit(KINDS[dtype]) + (n[a:b] + 2) * U32 * mags[a:b] * abs(s) * (1 + unit(KINDS[dtype])))
        assert (got[name][n[a:b, 0] == 0] == 0).all()


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("T,V,D,R", [(1, 1, 1, 0), (1, 7, 8, 0), (2, 3, 5, 2), (5, 100, 513, 0), (32, 1000, 3200, 0), (63, 64, 1024, 17), (128, 50, 2049, 64), (129, 50, 2049, 64),
                                     (1000, 300, 130, 400), (4099, 999, 40, 1000), (300, 30, 5, 7)])
def test_forward_and_gradients(dtype, out, T, V, D, R):
    gen = generator(T + V + D)
    ids = some_ids(gen, T, V, R)
    table, rows = randn(gen, V, D, dtype=KINDS[dtype]), randn(gen, R, D, dtype=KINDS[dtype])
    op = B.Embedding(dtype, V, D, out=out, scale=1.7, max_tokens=T, training=True)
    got = op.forward(table, ids, rows if R else None)
    check_forward(got, table, rows, ids, op.cfg.scale, V, R)
    dout = randn(gen, T, D, dtype=KINDS[out])
    grads = op.backward(ids, dout, num_rows=R)
    assert set(grads) == ({"table", "rows"} if R else {"table"})
    check_backward(grads, dout, ids, op.cfg.scale, V, R, dtype)
    for name in grads:                                       # alone, the same bits
        assert torch.equal(op.backward(ids, dout, num_rows=R, want=[name])[name], grads[name])


# (beyond 4096 pieces of 2048 elements a wave takes such a piece, not a quarter of it)
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("T,D", [(4100, 520), (2050, 2056), (4096, 2047)])
def test_rows_of_many_tokens(dtype, out, T, D):
    gen, V, R = generator(T + D), 100, 50
    ids = some_ids(gen, T, V, R)
    table, rows = randn(gen, V, D, dtype=KINDS[dtype]), randn(gen, R, D, dtype=KINDS[dtype])
    op = B.Embedding(dtype, V, D, out=out, scale=0.3, max_tokens=T)
    check_forward(op.forward(table, ids, rows), table, rows, ids, op.cfg.scale, V, R)


# lists of 4096 that are merged: one full, two, the eighth full, one more than eight, three rounds of merging; tables of one to four digits of nine bits
@pytest.mark.parametrize("T,V,D,hot", [(4096, 300, 8, 0.0), (4097, 40000, 8, 0.9), (8192, 500, 8, 0.0), (8193, 40000, 8, 0.9), (32768, 1000, 8, 0.1), (32769, 1000, 8, 0.1), (262145, 3000, 4, 0.3), (16384, 131072, 16, 0.1), (16385, 131072, 8, 0.5), (65536, 70, 8, 0.2),
                                       (65537, 262143, 8, 0.3), (150001, 1 << 20, 4, 0.99),
                                       # rows of no token cleared beside the sums: few rows, many, one wave's last ones, and odd lengths
                                       (8300, 300, 3200, 0.4), (10007, 5000, 2601, 0.1), (9001, 4099, 2804, 0.0), (400, 70, 65536, 0.3)])
def test_gradients_of_many_tokens(T, V, D, hot):
    gen = generator(T)
    R = 100
    ids = some_ids(gen, T, V, R, hot)
    op = B.Embedding("bf16", V, D, out="f32", scale=0.5, max_tokens=T, training=True)
    dout = randn(gen, T, D)
    got = op.backward(ids, dout, num_rows=R)
    check_backward(got, dout, ids, 0.5, V, R, "bf16")
    for name in got:
        assert torch.equal(op.backward(ids, dout, num_rows=R, want=[name])[name], got[name])


def test_one_object_and_calls_of_every_size():
    """Sizes on both sides of every border -- one launch or several, tokens of a piece, rounds of the sort, lists that are merged -- through one
    object, whose workspace holds what the calls before left; rows of dout apart."""
    V, D, R, most = 40, 9, 11, 33000
    op = B.Embedding("bf16", V, D, out="f32", scale=0.25, max_tokens=most, training=True)
    for T in (33000, 1, 7, 8, 9, 16, 17, 24, 25, 127, 128, 129, 136, 137, 1023, 1024, 1025, 2049, 4095, 4096, 4097, 8191, 8192, 8193, 16384, 16385, 32768, 32769, 2):
        gen = generator(T)
        ids, dout = some_ids(gen, T, V, R, hot=0.3), Gapped(T, D, torch.float32, gap=3, offset=1, values=randn(gen, T, D))
        check_backward(op.backward(ids, dout.view, num_rows=R), dout.view, ids, 0.25, V, R, "bf16")


def test_every_digit_of_a_key():
    # the most visual rows that fit beside a small table: keys of three and four digits, in turn from both ends
    for R in (1 << 18, (1 << 27) + 5):
        gen, T = generator(R), 3000
        ids = -1 - torch.randint(0, R, (T,), generator=gen, device=DEV)
        ids[0], ids[1], ids[2] = -R, -1, 0
        op = B.Embedding("bf16", 3, 1, max_tokens=T, training=True)
        dout = randn(gen, T, 1, dtype=torch.bfloat16)
        got = op.backward(ids.to(torch.int32), dout, num_rows=R)
        check_backward(got, dout, ids, 1.0, 3, R, "bf16")


@pytest.mark.parametrize("share", ["one", "two", "none", "pieces"])
def test_long_runs(share):
    T, V, D = 5000, 90, 300
    ids = {"one": torch.full((T,), 41), "two": torch.arange(T) % 2 * 89, "none": torch.full((T,), V), "pieces": torch.arange(T) // 32}[share].to(DEV).to(torch.int32)
    V = 200
    gen = generator(3)
    dout = randn(gen, T, D, dtype=torch.bfloat16)
    op = B.Embedding("bf16", V, D, max_tokens=T, training=True)
    check_backward(op.backward(ids, dout), dout, ids, 1.0, V, 0, "bf16")


def test_gradient_against_differences():
    gen, T, V, D, R = generator(8), 200, 20, 24, 6
    ids = some_ids(gen, T, V, R)
    table, rows, dout = randn(gen, V, D), randn(gen, R, D), randn(gen, T, D)
    op = B.Embedding("f32", V, D, scale=3.0, max_tokens=T, training=True)
    grads = op.backward(ids, dout, num_rows=R)
    for name, t in (("table", table), ("rows", rows)):
        v = randn(gen, *t.shape)
        # forward is linear: a difference over a step of one is the derivative, up to the roundings of both passes
        a = op.forward(table + v if name == "table" else table, ids, rows + v if name == "rows" else rows)
        b = op.forward(table - v if name == "table" else table, ids, rows - v if name == "rows" else rows)
        slope = ((a.double() - b.double()) / 2 * dout.double()).sum()
        size = ((a.double().abs() + b.double().abs()) * dout.double().abs()).sum() + 3 * (grads[name].double().abs() * v.double().abs()).sum()
        assert abs(slope - (grads[name].double() * v.double()).sum()) <= 250 * U32 * size


def test_rows_apart_and_rows_behind():
    gen, T, V, D, R = generator(2), 45, 30, 77, 9
    for dtype, out in TYPES:
        ids = some_ids(gen, T, V, R)
        table, rows = randn(gen, V, D, dtype=KINDS[dtype]), randn(gen, R, D, dtype=KINDS[dtype])
        op = B.Embedding(dtype, V, D, out=out, max_tokens=64, training=True)
        want = op.forward(table, ids, rows)
        y = Gapped(T, D, KINDS[out])
        op.forward(table, ids, rows, out=y.view)
        assert torch.equal(y.view, want) and y.untouched()
        d = Gapped(T, D, KINDS[out], gap=1, offset=1, values=want)
        a, b = op.backward(ids, d.view, num_rows=R), op.backward(ids, want, num_rows=R)
        assert all(torch.equal(a[n], b[n]) for n in b) and d.untouched()
        # a table that starts on any element
        t = Gapped(V, D, KINDS[dtype], gap=0, offset=1, values=table)
        assert torch.equal(op.forward(t.view, ids, rows), want)


def test_gradients_behind_their_ends_are_left():
    gen, T, V, D = generator(5), 50, 33, 7
    ids = some_ids(gen, T, V, 0)
    dout = randn(gen, T, D, dtype=torch.bfloat16)
    op = B.Embedding("bf16", V, D, max_tokens=T, training=True)
    want = op.backward(ids, dout)["table"]
    for offset in (1, 2, 8):
        buf = torch.full((offset + V * D + 9,), 5.0, dtype=torch.bfloat16, device=DEV)
        at = buf.data_ptr() + 2 * offset
        op._with_workspace(B.epd_embed_backward, op.cfg, ids.data_ptr(), T, dout.data_ptr(), D, 0, at, None)
        torch.cuda.synchronize()
        assert torch.equal(buf[offset:offset + V * D].view(V, D), want) and (buf[:offset] == 5).all() and (buf[offset + V * D:] == 5).all()


def test_values_of_rows_come_as_they_are():
    # infinities and NaN stay in their rows, and padding gives zeros whatever the scale
    table = torch.tensor([[1.0, float("inf")], [float("nan"), 2.0], [3.0, -0.0]], dtype=torch.bfloat16, device=DEV)
    op = B.Embedding("bf16", 3, 2, scale=2.0, max_tokens=8, training=True)
    ids = torch.tensor([0, 1, 2, 3, NONE, -1, -2 ** 31], dtype=torch.int32, device=DEV)
    out = op.forward(table, ids)
    assert torch.equal(out[0].cpu(), torch.tensor([2.0, float("inf")], dtype=torch.bfloat16)) and torch.isnan(out[1, 0]) and out[1, 1] == 4
    assert (out[3:] == 0).all()
    d = torch.ones(7, 2, dtype=torch.bfloat16, device=DEV)
    d[3:] = float("nan")                                     # gradients of padding are not looked at
    d[0, 0] = float("inf")
    g = op.backward(ids, d)["table"].cpu()
    assert torch.equal(g, torch.tensor([[float("inf"), 2.0], [2.0, 2.0], [2.0, 2.0]], dtype=torch.bfloat16))


def test_no_tokens_clear_the_gradients():
    op = B.Embedding("f32", 11, 3, max_tokens=4, training=True)
    ids = torch.empty(0, dtype=torch.int32, device=DEV)
    assert op.forward(torch.ones(11, 3, device=DEV), ids).shape == (0, 3)
    g = op.backward(ids, torch.empty(0, 3, device=DEV), num_rows=2)
    assert (g["table"] == 0).all() and (g["rows"] == 0).all()


@pytest.mark.parametrize("T", [33, 9000])
def test_captured_and_replayed(T):
    gen, V, D, R = generator(T), 500, 264, 40
    ids, dout = some_ids(gen, T, V, R), randn(gen, T, D, dtype=torch.bfloat16)
    table, rows = randn(gen, V, D, dtype=torch.bfloat16), randn(gen, R, D, dtype=torch.bfloat16)
    op = B.Embedding("bf16", V, D, max_tokens=T, training=True)

    def change(i):
        ids.copy_(some_ids(generator(100 + i), T, V, R, hot=0.1 + 0.4 * i))
        dout.copy_(randn(generator(200 + i), T, D, dtype=torch.bfloat16))

    def call():
        return op.forward(table, ids, rows), op.backward(ids, dout, num_rows=R)

    replays(call, lambda r: [r[0], r[1]["table"], r[1]["rows"]], change)


def test_two_objects_graphs_and_streams():
    gen, T, V, D = generator(4), 3000, 700, 512
    ops = [B.Embedding("bf16", V, D, max_tokens=T, training=True) for _ in range(2)]
    ids = [some_ids(gen, T, V, 0) for _ in range(2)]
    dout = [randn(gen, T, D, dtype=torch.bfloat16) for _ in range(2)]
    want = [op.backward(i, d)["table"].clone() for op, i, d in zip(ops, ids, dout)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got.append((k, ops[k].backward(ids[k], dout[k])["table"]))
    torch.cuda.synchronize()
    for k, g in got:
        assert torch.equal(g, want[k])


def test_offsets_beyond_2_31_elements():
    V, D, T = 131072, 32768, 6
    table = torch.zeros(V, D, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, V - 1, 65536, V - 1, 1, NONE], dtype=torch.int32, device=DEV)
    for i in (0, V - 1, 65536, 1):
        table[i] = torch.arange(D, device=DEV) % 251 + i % 7
    op = B.Embedding("bf16", V, D, out="f32", max_tokens=T, training=True)
    out = op.forward(table, at)
    for k, i in enumerate(at.tolist()):
        assert torch.equal(out[k], table[i].float() if i < V else torch.zeros(D, device=DEV))
    del table
    g = op.backward(at, torch.ones(T, D, device=DEV))["table"]
    assert all((g[i] == (2 if i == V - 1 else 1)).all() for i in (0, 1, 65536, V - 1))
    assert sum(int(p.sum(dtype=torch.int64)) for p in (g != 0).split(4096)) == 4 * D
