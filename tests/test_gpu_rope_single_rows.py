"""Rotation of one token or one head, whose stride means nothing, and positions of one token in a column."""

import pytest
import torch

from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape,other", [((1, 6, 64), (5001, 64, 1)), ((7, 1, 64), (64, 3, 1)), ((1, 1, 64), (17, 5, 1))])
def test_in_place_through_another_view_of_the_same_rows(dtype, shape, other):
    op = B.Rope(dtype, 64, (8, 12, 12))
    x = torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(op.dtype)
    pos = torch.arange(3 * shape[0], device=DEV, dtype=torch.int32).view(3, -1) + 5
    want = op.apply([x], pos)[0]
    view = x.as_strided(shape, other)                                  # the same elements: only strides of single rows differ
    assert torch.equal(view, x)
    got = op.apply([view], pos, out=[x])[0]
    assert torch.equal(got, want) and torch.equal(x, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_of_single_rows_do_not_matter(dtype):
    op = B.Rope(dtype, 64, (8, 12, 12))
    x = torch.randn((1, 4, 64), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(op.dtype)
    pos = torch.tensor([[3], [700], [12]], device=DEV, dtype=torch.int32)
    want = op.apply([x], pos)[0]
    far = torch.zeros((1, 4, 64), dtype=op.dtype, device=DEV)
    assert torch.equal(op.apply([x.as_strided((1, 4, 64), (3, 64, 1))], pos, out=[far.as_strided((1, 4, 64), (1 << 41, 64, 1))])[0], want)


def test_positions_of_one_token_in_a_column():
    base = torch.zeros((1, 3), dtype=torch.int32, device=DEV)
    out, after = B.rope_positions([(1, 0, 0)], [0, 1], start=[41], out=base.t())
    assert base.tolist() == [[41, 41, 41]] and after.tolist() == [42] and out.data_ptr() == base.data_ptr()
