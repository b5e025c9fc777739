"""Gradients that add over tokens -- the rows of Embedding.backward, the gain of AddNorm.backward -- on whole numbers, whose sums fp32 holds exactly
in any order: a token lost, counted twice or given to another row is a whole number away, however many the sum has."""

import numpy as np
import pytest
import torch

from entry_util import DEV, KINDS, generator
from paper_2601_11590_amd import binding as B
from test_gpu_embed import keys_of, some_ids

pytestmark = pytest.mark.gpu
TYPES = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")]


def whole(gen, *shape):
    """-8 ... 8 without zero."""
    v = torch.randint(1, 9, shape, generator=gen, device=DEV)
    return torch.where(torch.randint(0, 2, shape, generator=gen, device=DEV) > 0, v, -v).float()


def check(op, ids, dout, V, R, scale):
    """Every row equals the exact sum times a power of two, rounded once to the table's type."""
    key, D = keys_of(ids, V, R), dout.shape[1]
    assert 8 * int(torch.bincount(key, minlength=V + R + 1)[:V + R].max()) < 1 << 24
    sums = torch.zeros(V + R + 1, D, dtype=torch.float64, device=DEV).index_add_(0, key, dout.double())
    got = op.backward(ids, dout, num_rows=R)
    assert torch.equal(got["table"], (sums[:V] * scale).to(op.dtype))
    if R:
        assert torch.equal(got["rows"], sums[V:V + R].to(op.dtype))


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("T,V,D,hot", [(100, 30, 40, 0.5), (128, 9, 3, 0.9), (129, 50, 9, 0.9), (1000, 40, 700, 0.3), (4096, 300, 8, 0.5), (4097, 40000, 8, 0.9), (8193, 40000, 24, 0.9),
                                       (32769, 1000, 520, 0.5), (262145, 3000, 4, 0.3), (16385, 131072, 8, 0.5), (65537, 262143, 8, 0.3), (150001, 1 << 20, 4, 0.99), (150001, 70, 65, 0.6),
                                       (300000, 20, 16, 0.2), (10007, 5000, 2601, 0.3)])
def test_rows_of_many_tokens(dtype, out, T, V, D, hot):
    gen, R = generator(T + V), 100
    ids = some_ids(gen, T, V, R, hot)
    check(B.Embedding(dtype, V, D, out=out, scale=0.5, max_tokens=T, training=True), ids, whole(gen, T, D).to(KINDS[out]), V, R, 0.5)


@pytest.mark.parametrize("T", [129, 1000, 5000, 32768, 32800, 70001])
def test_runs_of_every_length(T):
    """Runs of 1, 2, 3 ... tokens, so that their ends meet those of the pieces at every distance, in order and shuffled."""
    gen = generator(T)
    V = int((2 * T) ** 0.5) + 2
    ordered = torch.repeat_interleave(torch.arange(V, device=DEV), torch.arange(1, V + 1, device=DEV))[:T]
    op = B.Embedding("f32", V, 20, scale=2.0, max_tokens=T, training=True)
    for ids in (ordered, V - 1 - ordered, ordered[torch.randperm(T, generator=gen, device=DEV)]):
        check(op, ids.to(torch.int32), whole(gen, T, 20), V, 0, 2.0)


@pytest.mark.parametrize("pieces", [1, 2, 3, 31, 32, 33, 34, 100, 2000])
@pytest.mark.parametrize("offset", [0, 1, 31])
def test_a_run_between_others(pieces, offset):
    """One long run, with others that begin and end around it, from one piece to more than the listed runs' shorter form takes."""
    gen, V = generator(pieces * 40 + offset), 50
    T = 32 * pieces + 40000
    ids = torch.cat([torch.arange(offset, device=DEV) % 7, torch.full((32 * pieces,), 7, device=DEV), torch.arange(T - 32 * pieces - offset, device=DEV) % 42 + 8]).to(torch.int32)
    check(B.Embedding("f32", V, 72, max_tokens=T, training=True), ids, whole(gen, T, 72), V, 0, 1.0)


@pytest.mark.parametrize("dtype,residual", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("T,D", [(1, 8), (33, 64), (100, 512), (40001, 40), (70000, 64), (20011, 512), (5000, 1024), (4099, 1000), (2100, 2048), (2101, 1100), (1100, 4096), (1031, 8192), (530, 16384), (521, 16392),
                                 (600, 32768), (300, 65536)])
def test_gain(dtype, residual, T, D):
    """Sums of +1 and -1: their mean square is 1, so n is what the row holds."""
    inv = np.float32(1) / np.float32(D)
    assert np.float32(float(D) * float(inv)) == 1            # as the kernel makes it, in one rounding
    gen = generator(T + D)
    s = torch.where(torch.randint(0, 2, (T, D), generator=gen, device=DEV) > 0, 1.0, -1.0)
    dy = whole(gen, T, D)
    op = B.AddNorm(dtype, D, residual=residual, eps=0.0, max_tokens=T, training=True)
    got = op.backward(torch.ones(D, dtype=KINDS[dtype], device=DEV), s.to(KINDS[residual]), dy.to(KINDS[dtype]), want=("gain",))["gain"]
    assert torch.equal(got, (dy.double() * s.double()).sum(dim=0).to(KINDS[dtype]))
