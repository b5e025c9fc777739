"""The operators at the entry of the stage behind the encoder as they are used together: visual and text rows, a norm into 8 bits, a product,
the next norm; and the backward pass of what is trained in fp32."""

import pytest
import torch

from entry_util import DEV, generator, randn, replays
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu


def test_prompt_and_single_tokens():
    gen, V, D, N, R = generator(0), 500, 320, 320, 64
    table, visual = randn(gen, V, D, dtype=torch.bfloat16), randn(gen, R, D, dtype=torch.bfloat16)
    gain = [(1 + randn(gen, D, std=0.1)).to(torch.bfloat16) for _ in range(2)]
    wf = randn(gen, N, D, std=0.05)
    wq, ws = B.quant_rows(wf)
    ids = torch.randint(0, V, (150,), generator=gen, device=DEV)
    ids[20:20 + R] = -1 - torch.arange(R, device=DEV)
    ids = ids.to(torch.int32)
    embed, linear = B.Embedding("bf16", V, D, out="f32", scale=2.0, max_tokens=150), B.Int8Linear(D, N, max_tokens=150)
    norm = B.AddNorm("bf16", D, residual="f32", max_tokens=150)

    def stage(part):
        s = embed.forward(table, part, visual)
        o = norm.forward(gain[0], residual=s, want=("q",))
        y = linear.forward({"w": wq, "scale": ws}, o["q"], o["scale"])
        return norm.forward(gain[1], y, s, want=("sum", "y"), out={"sum": s})

    whole = stage(ids)
    # the definition in 64 bits without any rounding: 8 bits of x and w are off by half a step of m / 127 each, at random signs over D terms
    s = torch.where((ids < 0)[:, None], visual[(-1 - ids.long()).clamp(min=0)].double(), table[ids.long().clamp(min=0)].double() * 2.0)

    def normed(h, g):
        return h / (h.square().mean(dim=1, keepdim=True) + 1e-6).sqrt() * g.double()

    h = normed(s, gain[0])
    sx, sw = h.abs().amax(dim=1, keepdim=True) / 127, wf.double().abs().amax(dim=1) / 127
    y = h @ wf.double().t()
    worst = (sx / 2 * wf.double().abs().sum(dim=1) + sw / 2 * h.abs().sum(dim=1, keepdim=True)) * 1.02 + y.abs() * 2.0 ** -8
    assert ((whole["sum"].double() - s - y).abs() <= worst + 1e-5 * (s + y).abs()).all()
    # norm of the sums as they are, and one token at a time: rows do not see each other
    want = normed(whole["sum"].double(), gain[1])
    assert ((whole["y"].double() - want).abs() <= want.abs() * (2.0 ** -8 + 1e-5)).all()
    for t in (0, 19, 20, 83, 149):
        one = stage(ids[t:t + 1])
        assert torch.equal(one["sum"][0], whole["sum"][t]) and torch.equal(one["y"][0], whole["y"][t])


def test_training_step_of_embedding_and_norm():
    gen, V, D, T, R = generator(1), 60, 96, 200, 16
    table, visual, gain = randn(gen, V, D), randn(gen, R, D), 1 + randn(gen, D, std=0.1)
    ids = torch.randint(-R, V, (T,), generator=gen, device=DEV).to(torch.int32)
    x, dy, ds = randn(gen, T, D), randn(gen, T, D), randn(gen, T, D)
    embed, norm = B.Embedding("f32", V, D, scale=1.5, max_tokens=T, training=True), B.AddNorm("f32", D, max_tokens=T, training=True)
    o = norm.forward(gain, x, embed.forward(table, ids, visual))
    g = norm.backward(gain, o["sum"], dy, dsum=ds)
    e = embed.backward(ids, g["dx"], num_rows=R)
    leaves = [t.double().requires_grad_() for t in (table, visual, gain, x)]
    s = torch.where((ids < 0)[:, None], leaves[1][(-1 - ids.long()).clamp(min=0)], leaves[0][ids.long().clamp(min=0)] * 1.5) + leaves[3]
    y = s / (s.square().mean(dim=1, keepdim=True) + 1e-6).sqrt() * leaves[2]
    want = torch.autograd.grad((y * dy.double()).sum() + (s * ds.double()).sum(), leaves)
    for got, w in zip((e["table"], e["rows"], g["gain"], g["dx"]), want):
        # fp32 throughout: dx within 200 half steps of terms that are a few times its size, sums of up to 200 of them
        assert (got.double() - w).norm() <= 1e-5 * w.norm()


def test_a_row_that_is_not_finite_comes_out_as_nan_alone():
    gen, D, N, T = generator(2), 640, 264, 70
    x, gain = randn(gen, T, D, dtype=torch.bfloat16), torch.ones(D, dtype=torch.bfloat16, device=DEV)
    w = dict(zip(("w", "scale"), B.quant_rows(randn(gen, N, D))))
    norm, linear = B.AddNorm("bf16", D, max_tokens=T), B.Int8Linear(D, N, max_tokens=T)

    def stage():
        o = norm.forward(gain, x, want=("q",))
        return linear.forward(w, o["q"], o["scale"])

    want = stage()
    x[33, 600] = float("inf")
    got = stage()
    others = torch.arange(T, device=DEV) != 33
    assert torch.isnan(got[33]).all() and torch.equal(got[others], want[others])


def test_operators_captured_together():
    """A prompt's way through the operators as one graph, replayed on other prompts."""
    gen, V, D, N, R, T = generator(3), 300, 512, 512, 40, 150
    table, visual, gain = randn(gen, V, D, dtype=torch.bfloat16), randn(gen, R, D, dtype=torch.bfloat16), torch.ones(D, dtype=torch.bfloat16, device=DEV)
    w = dict(zip(("w", "scale"), B.quant_rows(randn(gen, N, D))))
    ids = torch.randint(-R, V, (T,), generator=gen, device=DEV).to(torch.int32)
    embed, norm = B.Embedding("bf16", V, D, out="f32", max_tokens=T, training=True), B.AddNorm("bf16", D, residual="f32", max_tokens=T, training=True)
    linear = B.Int8Linear(D, N, max_tokens=T)

    def call():
        s = embed.forward(table, ids, visual)
        o = norm.forward(gain, residual=s, want=("q",))
        y = linear.forward(w, o["q"], o["scale"])
        o = norm.forward(gain, y, s)
        g = norm.backward(gain, o["sum"], o["y"], dsum=o["sum"])
        return [y, *o.values(), *g.values(), *embed.backward(ids, g["dresidual"], num_rows=R).values()]

    replays(call, lambda v: v, lambda i: ids.copy_(torch.randint(-R - 3, V + 3, (T,), generator=generator(50 + i), device=DEV).to(torch.int32)))
