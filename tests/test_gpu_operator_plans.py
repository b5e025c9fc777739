"""The operators at sizes whose launches no other test has: products cut in two, turned first or in parts that the sizes elsewhere do not
reach, weights beyond the caches for one token, rows that only allow narrow accesses.  (test_operator_host_logic.py counts what is reached.)"""

import pytest
import torch

from gated_util import check, make, reference
from paper_2601_11590_amd import binding as B
from test_gpu_rope import check as check_rope

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

PLANS = [(1, 2048, 8200), (1, 16392, 1032),
         # K in parts, by tile and number: of Y (64 x 64: 2, 3, 4, 6; 256 x 128: 4, 6, 7; 256 x 256: 2, 3, 5, 6, 7, 8) and of dX (256 x 128: 4; 256 x 256: 2, 5, 8)
         (3516, 8, 1664), (2083, 8, 1280), (73, 8, 1160), (67, 8, 1712), (169, 6800, 4200), (214, 3344, 4504), (199, 3080, 5168), (518, 8816, 8672), (781, 4128, 6544),
         (362, 5536, 5944), (75, 9816, 12232), (306, 3976, 11808), (86, 6848, 16160), (2, 1192, 608), (800, 5488, 2800), (2, 11336, 824), (1, 6984, 1528),
         # gradients of the weights, each in two launches
         (701, 4632, 4608), (3273, 7584, 3736), (11593, 5688, 5768)]

ROPE_PLANS = [(37, 3, 2, 64, (1, 2, 3)), (19, 2, 1, 65, (7,))]


@pytest.mark.parametrize("T,D,F", PLANS)
def test_a_step_with_every_plan(T, D, F):
    w, x, dy = make(T, D, F, torch.bfloat16, True, T + D)
    op = B.GatedMLP("bf16", D, F, act="geglu_erf", max_tokens=T, use_bias=True, training=True)
    op.workspace.fill_(0xFF)                                           # nothing is read that was not written
    y, saved = op.forward(w, x, save=True)
    op.workspace.fill_(0xFF)
    grads = op.backward(w, x, dy, saved)
    check({"y": y, **grads}, reference("geglu_erf", w, x, dy))
    assert torch.equal(op.forward(w, x), y)
    for n in ("dx", "gate_up_w", "down_w"):
        assert torch.equal(op.backward(w, x, dy, saved, want=[n])[n], grads[n]), n


@pytest.mark.parametrize("dtype,pairing,T,hq,hk,d,pairs", [(t, p, *s) for t in ("bf16", "f32") for p in ("half", "adjacent") for s in ROPE_PLANS])
def test_rotation_in_accesses_of_every_width(dtype, pairing, T, hq, hk, d, pairs):
    op = B.Rope(dtype, d, pairs, pairing=pairing)
    g = torch.Generator(device=DEV).manual_seed(T)
    q, k = (torch.randn((T, h, d), generator=g, device=DEV).to(op.dtype) for h in (hq, hk))
    pos = torch.randint(0, 5000, (len(pairs), T), generator=g, device=DEV, dtype=torch.int32)
    for inverse in (False, True):
        for got, x in zip(op.apply([q, k], pos, inverse=inverse), (q, k)):
            check_rope(got, x, pos, pairs, "sections", "axis", pairing, inverse=inverse)
