"""Shared by the tests of the operators at the entry of the stage behind the encoder: unit roundings, rows with gaps, and captured calls."""

import torch

DEV = "cuda:0"
U32 = 2.0 ** -24                                             # half a step of fp32, relative
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}


def unit(t: torch.dtype) -> float:
    """Half a step, relative to the value (with what numbers below the normal ones add left to `within`)."""
    return torch.finfo(t).eps / 2


def randn(gen, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(dtype)


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def within(got, exact, bound):
    """|got - exact| <= bound, element by element; shows the worst place."""
    got, exact, bound = got.double(), exact.double(), bound.double() + 2.0 ** -126
    assert got.shape == exact.shape
    assert not (torch.isnan(got) ^ torch.isnan(exact)).any()
    over = ((got - exact).abs() - bound).nan_to_num(nan=-1.0, posinf=1e300)
    if over.numel():
        i = over.flatten().argmax()
        assert over.flatten()[i] <= 0, (int(i), float(got.flatten()[i]), float(exact.flatten()[i]), float(bound.expand_as(got).flatten()[i]))


class Gapped:
    """A matrix whose rows lie `gap` elements further apart than they are long, from `offset` elements into its buffer; `untouched` says
    whether all between the rows is still what it was."""

    def __init__(self, rows, cols, dtype, gap=5, offset=3, values=None):
        self.rows, self.cols, self.ld, self.offset = rows, cols, cols + gap, offset
        n = offset + max(rows, 1) * self.ld + 7
        self.mark = 77 if dtype == torch.int8 else 1234.5
        self.buf = torch.full((n,), self.mark, dtype=torch.float32, device=DEV).to(dtype)
        self.mark = self.buf[0].item()
        self.view = self.buf[offset:offset + rows * self.ld].view(rows, self.ld)[:, :cols]
        if values is not None:
            self.view.copy_(values)

    def untouched(self):
        keep = self.buf.clone()
        keep[self.offset:self.offset + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = self.mark
        return bool((keep == self.mark).all())


def replays(call, outputs, change, times=3):
    """call() captured into a graph and replayed on other inputs each time (`change(i)` writes them), with eager work between; every
    replay's `outputs()` equal an eager call's."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = call()
    for i in range(times):
        change(i)
        eager = [t.clone() for t in outputs(call())]
        for t in outputs(kept):
            t.view(torch.uint8).fill_(0x5a)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outputs(kept), eager):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
    return graph
