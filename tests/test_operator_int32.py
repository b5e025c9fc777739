"""Sizes and positions beyond 32 bits are refused, not wrapped to others."""

import numpy as np
import pytest
import torch

from paper_2601_11590_amd import binding as B

FAR = 2 ** 32 + 1


@pytest.mark.parametrize("span", [np.array([[FAR, 0, 0]]), [(FAR, 0, 0)], [(2, 2 ** 31, 3)], [(-FAR, 0, 0)], np.array([[FAR, 0, 0]], dtype=np.uint64),
                                  np.array([[1.5, 0, 0]]), [(float("nan"), 0, 0)]])
def test_spans(span):
    with pytest.raises(ValueError):
        B.epd_rope_tokens(span)
    with pytest.raises(ValueError):
        B.rope_positions(span, [0, 1])
    with pytest.raises(ValueError):
        B.epd_rope_positions(span, np.array([0, 1]), None, 1, 0x1000, 64, 0)


@pytest.mark.parametrize("kw", [dict(cu=np.array([0, FAR])), dict(cu=np.array([2 ** 32, 1])), dict(cu=[0.0, 1.5]), dict(start=np.array([FAR])), dict(start=[0.5]),
                                dict(start=[2 ** 31]), dict(t_step=FAR), dict(t_step=-FAR)])
def test_positions(kw):
    a = {**dict(cu=[0, 1], start=None, t_step=1), **kw}
    with pytest.raises(ValueError):
        B.epd_rope_positions(np.array([[3, 0, 0]]), a["cu"], a["start"], a["t_step"], 0x1000, 64, 0)


def test_every_integer_type_is_taken():
    for t in (np.int8, np.uint8, np.int16, np.int32, np.int64, np.uint64):
        assert B.epd_rope_tokens(np.array([(3, 0, 0), (2, 3, 4)], dtype=t)) == 27
    assert B.epd_rope_tokens(np.array([(3.0, 0.0, 0.0)])) == 3 and B.epd_rope_tokens(np.zeros((0, 3))) == 0 and B.epd_rope_tokens([]) == 0
    assert B.epd_rope_tokens(np.array([(3, 9, 0, 0, 0, 0)], dtype=np.int32)[:, ::2]) == 3        # not contiguous


@pytest.mark.gpu
def test_tensors_of_2_32_rows():
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    T = 2 ** 32 + 5
    pos = torch.empty((1, T), dtype=torch.int32, device="cuda:0")
    x = torch.ones((1, 1, 2), dtype=torch.bfloat16, device="cuda:0").expand(T, 1, 2)
    with pytest.raises(ValueError):
        B.Rope("bf16", 2, (1,)).apply([x], pos)
    del pos
    rows = torch.empty((T, 8), dtype=torch.bfloat16, device="cuda:0")
    w = {"gate_up_w": torch.ones((16, 8), dtype=torch.bfloat16, device="cuda:0"), "down_w": torch.ones((8, 8), dtype=torch.bfloat16, device="cuda:0")}
    with pytest.raises(B.EpdError) as e:
        B.GatedMLP("bf16", 8, 8, max_tokens=16, training=True).forward(w, rows, out=rows)
    assert e.value.status == B.EPD_ERR_SHAPE
    del rows
    torch.cuda.empty_cache()
