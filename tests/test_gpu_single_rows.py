"""One row, whose stride means nothing: the last token of a long sequence, a column of a wide buffer."""

import pytest
import torch

from gated_util import make
from paper_2601_11590_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def last_token(row, apart):
    """The same row as the only one of a view whose rows would be `apart` elements apart."""
    far = torch.zeros(apart + row.shape[1], dtype=row.dtype, device=DEV)
    view = far.as_strided((1, row.shape[1]), (apart, 1))
    view.copy_(row)
    return view


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("apart", [(1 << 22) + 64, 323, 1 << 23, 5])
def test_gated_mlp_of_a_strided_row(dtype, apart):
    D, F = 320, 648
    w, x, dy = make(1, D, F, DT[dtype], True, 1)
    op = B.GatedMLP(dtype, D, F, max_tokens=4, use_bias=True, training=True)
    y, saved = op.forward(w, x, save=True)
    want = op.backward(w, x, dy, saved)
    x1, dy1, out = last_token(x, apart), last_token(dy, apart), last_token(torch.zeros_like(x), apart)
    y1, saved1 = op.forward(w, x1, save=True, out=out)
    assert y1.data_ptr() == out.data_ptr() and torch.equal(y1, y)        # (the parts of `saved` have gaps between them)
    got = op.backward(w, x1, dy1, saved1)
    assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ld", [0, -7, 3, (1 << 40) + 1])
def test_gated_mlp_entries_do_not_look_at_the_stride_of_one_row(dtype, ld):
    D, F = 72, 136
    w, x, dy = make(1, D, F, DT[dtype], False, 2)
    op = B.GatedMLP(dtype, D, F, max_tokens=4, training=True)
    y, saved = op.forward(w, x, save=True)
    want = op.backward(w, x, dy, saved)
    ws = B.epd_gated_mlp_weights()
    ws.gate_up_w, ws.down_w = w["gate_up_w"].data_ptr(), w["down_w"].data_ptr()
    stream, base = torch.cuda.current_stream().cuda_stream, (op.workspace.data_ptr() + 255) // 256 * 256
    y1, dx1, saved1 = torch.empty_like(y), torch.empty_like(x), torch.empty_like(saved)
    B.epd_gated_mlp(op.cfg, ws, x.data_ptr(), ld, 1, y1.data_ptr(), ld, saved1.data_ptr(), base, op.workspace_bytes, stream)
    g = B.epd_gated_mlp_grads()
    g.dx, g.ld_dx = dx1.data_ptr(), ld
    B.epd_gated_mlp_backward(op.cfg, ws, x.data_ptr(), ld, dy.data_ptr(), ld, 1, saved1.data_ptr(), g, base, op.workspace_bytes, stream)
    assert torch.equal(y1, y) and torch.equal(dx1, want["dx"])


def test_last_token_of_a_sequence():
    D, F, S = 3200, 64, 1400
    w, x, _ = make(1, D, F, torch.bfloat16, False, 3)
    h = torch.zeros((1, S, D), dtype=torch.bfloat16, device=DEV)
    h[:, -1, :] = x
    op = B.GatedMLP("bf16", D, F, max_tokens=1)
    assert h[:, -1, :].stride(0) >= 1 << 22 and torch.equal(op.forward(w, h[:, -1, :]), op.forward(w, x))
