"""What the operators beside the encoder refuse, all on the host: nothing is launched, no GPU is needed."""

import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2601_11590_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "epd_encode.h")


def test_every_declared_operator_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(epd_(?:op|rope|gated)_\w+)\s*\(", text))
    assert names == set(B.OPERATOR_EXPORTS)
    for n in names:
        assert getattr(B.lib, n) is not None


def test_structs_and_enums_match_the_header(tmp_path):
    structs = {"epd_rope_cfg": B.epd_rope_cfg, "epd_rope_tensor": B.epd_rope_tensor, "epd_gated_mlp_cfg": B.epd_gated_mlp_cfg,
               "epd_gated_mlp_weights": B.epd_gated_mlp_weights, "epd_gated_mlp_grads": B.epd_gated_mlp_grads}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "epd_encode.h"', "int main(void) {"]
    want = []
    for name, t in structs.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(C.sizeof(t))
        for f, _ in t._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, {"input": "in", "output": "out"}.get(f, f)))
            want.append(getattr(t, f).offset)
    for e in ("EPD_ROPE_SECTIONS", "EPD_ROPE_INTERLEAVED", "EPD_ROPE_LADDER_AXIS", "EPD_ROPE_LADDER_HEAD", "EPD_ROPE_HALF", "EPD_ROPE_ADJACENT",
              "EPD_SWIGLU", "EPD_GEGLU_ERF", "EPD_GEGLU_TANH"):
        lines.append('printf("%%d\\n", (int)%s);' % e)
        want.append(getattr(B, e))
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "probe")], check=True)
    out = subprocess.run([str(tmp_path / "probe")], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    assert [int(v) for v in out] == want


# ------------------------------------------------------------------ rotation

def rope(cfg=None, tensors=None, positions=0x1000, stride=64, tokens=10, inverse=0, **change):
    c = B.Rope("bf16", 64, (8, 12, 12)).cfg
    for k, v in change.items():
        if k == "pairs":
            v = (C.c_int32 * 4)(*v)
        setattr(c, k, v)
    if tensors is None:
        tensors = [dict()]
    arr = (B.epd_rope_tensor * max(1, len(tensors)))()
    for a, t in zip(arr, tensors):
        d = dict(input=0x10000, output=0x20000, in_token=256, in_head=64, out_token=256, out_head=64, heads=4)
        d.update(t)
        for k, v in d.items():
            setattr(a, k, v)
    st = B.lib.epd_rope_apply(C.byref(c) if cfg is None else cfg, arr, len(tensors), positions, stride, tokens, inverse, None)
    return st, B.epd_op_last_error()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(struct_size=4), B.EPD_ERR_INVALID_ARG, "struct_size"),
    (dict(dtype=2), B.EPD_ERR_INVALID_ARG, "dtype"),
    (dict(layout=2), B.EPD_ERR_INVALID_ARG, "layout"),
    (dict(ladder=-1), B.EPD_ERR_INVALID_ARG, "ladder"),
    (dict(pairing=5), B.EPD_ERR_INVALID_ARG, "pairing"),
    (dict(axes=0), B.EPD_ERR_INVALID_ARG, "axes"),
    (dict(axes=5), B.EPD_ERR_INVALID_ARG, "axes"),
    (dict(base=0.0), B.EPD_ERR_INVALID_ARG, "base"),
    (dict(base=float("nan")), B.EPD_ERR_INVALID_ARG, "base"),
    (dict(base=float("inf")), B.EPD_ERR_INVALID_ARG, "base"),
    (dict(head_dim=258), B.EPD_ERR_UNSUPPORTED, "head_dim"),
    (dict(head_dim=0), B.EPD_ERR_UNSUPPORTED, "head_dim"),
    (dict(pairs=(-1, 12, 12, 0)), B.EPD_ERR_INVALID_ARG, "pairs"),
    (dict(pairs=(0, 0, 0, 0)), B.EPD_ERR_UNSUPPORTED, "pairs"),
    (dict(pairs=(9, 12, 12, 0)), B.EPD_ERR_UNSUPPORTED, "33 pairs"),
    (dict(pairs=(2147483647, 2147483647, 12, 0)), B.EPD_ERR_INVALID_ARG, "pairs"),
    (dict(tokens=-1), B.EPD_ERR_SHAPE, "tokens"),
    (dict(stride=9), B.EPD_ERR_SHAPE, "position_stride"),
    (dict(positions=None), B.EPD_ERR_INVALID_ARG, "NULL"),
    (dict(inverse=2), B.EPD_ERR_INVALID_ARG, "inverse"),
    (dict(tensors=[]), B.EPD_ERR_INVALID_ARG, "num_tensors"),
    (dict(tensors=[{}] * 5), B.EPD_ERR_INVALID_ARG, "num_tensors"),
    (dict(tensors=[{}, dict(input=None)]), B.EPD_ERR_INVALID_ARG, "tensor 1"),
    (dict(tensors=[dict(output=None)]), B.EPD_ERR_INVALID_ARG, "NULL"),
    (dict(tensors=[dict(input=0x10001)]), B.EPD_ERR_INVALID_ARG, "aligned"),
    (dict(tensors=[dict(heads=257)]), B.EPD_ERR_UNSUPPORTED, "heads"),
    (dict(tensors=[dict(heads=-1)]), B.EPD_ERR_UNSUPPORTED, "heads"),
    (dict(tensors=[dict(in_token=-64)]), B.EPD_ERR_SHAPE, "stride"),
    (dict(tensors=[dict(out_head=1 << 41)]), B.EPD_ERR_SHAPE, "stride"),
    (dict(tensors=[dict(out_token=0)]), B.EPD_ERR_SHAPE, "overlap"),
    (dict(tensors=[dict(out_head=63)]), B.EPD_ERR_SHAPE, "overlap"),
    (dict(tensors=[dict(out_token=255)]), B.EPD_ERR_SHAPE, "overlap"),
    (dict(tensors=[dict(out_token=64, out_head=639)]), B.EPD_ERR_SHAPE, "overlap"),
    (dict(tensors=[dict(output=0x10000, in_token=512)]), B.EPD_ERR_SHAPE, "in place"),
])
def test_rope_refusals(kw, status, needle):
    st, msg = rope(**kw)
    assert st == status and needle in msg, msg


def test_rope_calls_without_work_launch_nothing():
    assert rope(tokens=0)[0] == B.EPD_OK
    assert rope(tokens=0, tensors=[dict(input=None, output=None)])[0] == B.EPD_OK
    assert rope(tensors=[dict(heads=0, input=None, output=None)])[0] == B.EPD_OK
    assert rope(cfg=C.POINTER(B.epd_rope_cfg)())[0] == B.EPD_ERR_INVALID_ARG


# ------------------------------------------------------------------ positions

def pos(spans, cu, start=None, t_step=1, positions=0x1000, stride=1 << 40):
    span, cu = np.array(spans, dtype=np.int32).reshape(-1, 3), np.array(cu, dtype=np.int32)
    st0 = None if start is None else np.array(start, dtype=np.int32)
    st = B.lib.epd_rope_positions(span.ctypes.data, cu.ctypes.data, len(cu) - 1, None if st0 is None else st0.ctypes.data, t_step, positions, stride, None, None)
    return st, B.epd_op_last_error()


@pytest.mark.parametrize("kw,needle", [
    (dict(spans=[(-1, 0, 0)], cu=[0, 1]), "span 0"),
    (dict(spans=[(3, 0, 0), (0, 2, 2)], cu=[0, 2]), "span 1"),
    (dict(spans=[(1, 2, 0)], cu=[0, 1]), "span 0"),
    (dict(spans=[(1, -2, -2)], cu=[0, 1]), "span 0"),
    (dict(spans=[(3, 0, 0)], cu=[1, 1]), "start at 0"),
    (dict(spans=[(3, 0, 0), (3, 0, 0)], cu=[0, 2, 1]), "decreases"),
    (dict(spans=[(3, 0, 0)], cu=[0, 1 << 30, 1]), "decreases"),        # before a span beyond the last is read
    (dict(spans=[(2, 65536, 65536)], cu=[0, 1]), "too many tokens"),
    (dict(spans=[(2 ** 31 - 1, 0, 0), (1, 0, 0)], cu=[0, 1, 2]), "more than"),
    (dict(spans=[(3, 0, 0)], cu=[0, 1], start=[2 ** 31 - 3]), "position"),
    (dict(spans=[(2 ** 16, 1, 1)], cu=[0, 1], t_step=2 ** 16), "position"),
    (dict(spans=[(3, 0, 0), (1, 2, 2)], cu=[0, 2], stride=6), "position_stride"),
])
def test_position_refusals(kw, needle):
    st, msg = pos(**kw)
    assert st == B.EPD_ERR_SHAPE and needle in msg, msg


def test_tokens_of_spans():
    assert B.epd_rope_tokens([(3, 0, 0), (2, 3, 4), (0, 0, 0)]) == 27 and B.epd_rope_tokens(np.zeros((0, 3))) == 0
    for bad in ([(-1, 0, 0)], [(1, 0, 2)], [(0, 1, 1)], [(2, 65536, 65536)], [(2 ** 31 - 1, 0, 0), (1, 0, 0)]):
        with pytest.raises(B.EpdError) as e:
            B.epd_rope_tokens(bad)
        assert e.value.status == B.EPD_ERR_SHAPE and "span" in str(e.value)
    assert B.lib.epd_rope_tokens(None, 1) == -1 and B.lib.epd_rope_tokens(0x1000, -1) == -1


def test_position_arguments():
    assert pos([(1, 0, 0)], [0, 1], positions=None)[0] == B.EPD_ERR_INVALID_ARG
    assert pos([(1, 0, 0)], [0, 1], t_step=-1)[0] == B.EPD_ERR_INVALID_ARG
    assert pos([], [0])[0] == B.EPD_OK and pos([(0, 0, 0)], [0, 0, 1])[0] == B.EPD_OK       # no tokens: nothing to launch
    with pytest.raises(ValueError):
        B.epd_rope_positions([(1, 0, 0)], [0, 2], None, 1, 0x1000, 64, 0)


# ------------------------------------------------------------------ gated MLP

def mlp_cfg(**change):
    c = B.epd_gated_mlp_cfg()
    base = dict(struct_size=C.sizeof(B.epd_gated_mlp_cfg), dtype=B.EPD_BF16, hidden=64, mlp_dim=128, act=B.EPD_SWIGLU, use_bias=1, max_tokens=100, training=1)
    base.update(change)
    for k, v in base.items():
        setattr(c, k, v)
    return c


def mlp(backward=False, cfg=None, x=0x10000, ld_x=64, tokens=10, y=0x20000, ld_y=64, saved=0x30000, workspace=0x100000, size=1 << 40, weights=None, grads=None, **change):
    c = mlp_cfg(**change) if cfg is None else cfg
    w = B.epd_gated_mlp_weights(0x40000, 0x50000, 0x60000, 0x70000)
    for k, v in (weights or {}).items():
        setattr(w, k, v)
    if backward:
        g = B.epd_gated_mlp_grads(0x80000, 64, 0x90000, 0xA0000, 0xB0000, 0xC0000)
        for k, v in (grads or {}).items():
            setattr(g, k, v)
        st = B.lib.epd_gated_mlp_backward(C.byref(c), C.byref(w), x, ld_x, y, ld_y, tokens, saved, C.byref(g), workspace, size, None)
    else:
        st = B.lib.epd_gated_mlp(C.byref(c), C.byref(w), x, ld_x, tokens, y, ld_y, saved, workspace, size, None)
    return st, B.epd_op_last_error()


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,status,needle", [
    (dict(struct_size=8), B.EPD_ERR_INVALID_ARG, "struct_size"),
    (dict(dtype=3), B.EPD_ERR_INVALID_ARG, "dtype"),
    (dict(use_bias=2), B.EPD_ERR_INVALID_ARG, "use_bias"),
    (dict(training=-1), B.EPD_ERR_INVALID_ARG, "training"),
    (dict(act=B.EPD_GELU_ERF), B.EPD_ERR_INVALID_ARG, "gated"),
    (dict(act=5), B.EPD_ERR_INVALID_ARG, "gated"),
    (dict(hidden=0), B.EPD_ERR_INVALID_ARG, "positive"),
    (dict(mlp_dim=-8), B.EPD_ERR_INVALID_ARG, "positive"),
    (dict(max_tokens=0), B.EPD_ERR_INVALID_ARG, "positive"),
    (dict(hidden=60), B.EPD_ERR_UNSUPPORTED, "multiples of 8"),
    (dict(mlp_dim=4), B.EPD_ERR_UNSUPPORTED, "multiples of 8"),
    (dict(hidden=65536, mlp_dim=16384), B.EPD_ERR_UNSUPPORTED, "2^30"),
    (dict(mlp_dim=131080), B.EPD_ERR_UNSUPPORTED, "131072"),
    (dict(max_tokens=1 << 22), B.EPD_ERR_UNSUPPORTED, "max_tokens"),
    (dict(tokens=101), B.EPD_ERR_SHAPE, "tokens"),
    (dict(tokens=-1), B.EPD_ERR_SHAPE, "tokens"),
    (dict(weights=dict(gate_up_w=None)), B.EPD_ERR_INVALID_ARG, "NULL"),
    (dict(weights=dict(down_w=None)), B.EPD_ERR_INVALID_ARG, "NULL"),
    (dict(weights=dict(gate_up_b=None)), B.EPD_ERR_INVALID_ARG, "NULL"),
    (dict(weights=dict(down_b=None)), B.EPD_ERR_INVALID_ARG, "NULL"),
    (dict(weights=dict(down_w=0x60008)), B.EPD_ERR_UNSUPPORTED, "aligned"),
    (dict(workspace=None), B.EPD_ERR_WORKSPACE, "workspace"),
    (dict(workspace=0x100010), B.EPD_ERR_WORKSPACE, "aligned"),
    (dict(size=1000), B.EPD_ERR_WORKSPACE, "required"),
    (dict(x=None), B.EPD_ERR_INVALID_ARG, "x is NULL"),
    (dict(y=None), B.EPD_ERR_INVALID_ARG, "NULL"),
    (dict(x=0x10008), B.EPD_ERR_UNSUPPORTED, "16 bytes"),
    (dict(ld_x=63), B.EPD_ERR_SHAPE, "rows of x"),
    (dict(ld_x=68), B.EPD_ERR_UNSUPPORTED, "16 bytes"),
    (dict(ld_y=1 << 22), B.EPD_ERR_SHAPE, "rows of"),
    (dict(saved=0x30004), B.EPD_ERR_UNSUPPORTED, "saved"),
    (dict(dtype=B.EPD_F32, x=0x10002), B.EPD_ERR_UNSUPPORTED, "4 (fp32)"),
])
def test_gated_mlp_refusals(backward, kw, status, needle):
    st, msg = mlp(backward, **kw)
    assert st == status and needle in msg, msg


@pytest.mark.parametrize("kw,status,needle", [
    (dict(training=0), B.EPD_ERR_INVALID_ARG, "training"),
    (dict(saved=None), B.EPD_ERR_INVALID_ARG, "saved"),
    (dict(use_bias=0), B.EPD_ERR_INVALID_ARG, "biases"),
    (dict(grads=dict(dx=0x80008)), B.EPD_ERR_UNSUPPORTED, "dx"),
    (dict(grads=dict(ld_dx=8)), B.EPD_ERR_SHAPE, "dx"),
    (dict(grads=dict(down_w=0x80004)), B.EPD_ERR_UNSUPPORTED, "gradients"),
])
def test_gated_mlp_backward_refusals(kw, status, needle):
    st, msg = mlp(True, **kw)
    assert st == status and needle in msg, msg


def test_gated_mlp_without_tokens_and_null_arguments():
    assert mlp(tokens=0, x=None, y=None, saved=None)[0] == B.EPD_OK
    st = B.lib.epd_gated_mlp(None, None, None, 0, 0, None, 0, None, None, 0, None)
    assert st == B.EPD_ERR_INVALID_ARG
    w = B.epd_gated_mlp_weights(0x40000, 0x50000, 0x60000, 0x70000)
    st = B.lib.epd_gated_mlp_backward(C.byref(mlp_cfg()), C.byref(w), 0x1000, 64, 0x1000, 64, 4, 0x1000, None, 0x100000, 1 << 40, None)
    assert st == B.EPD_ERR_INVALID_ARG and "grads" in B.epd_op_last_error()


def test_gated_mlp_workspace():
    assert B.epd_gated_mlp_workspace_bytes(mlp_cfg(hidden=60)) == 0
    small = B.epd_gated_mlp_workspace_bytes(mlp_cfg(training=0))
    assert small == 100 * 128 * 2 and small % 256 == 0
    assert B.epd_gated_mlp_workspace_bytes(mlp_cfg(training=0, max_tokens=1, mlp_dim=8)) == 256
    big = B.epd_gated_mlp_workspace_bytes(mlp_cfg(hidden=3200, mlp_dim=12800, max_tokens=32768))
    assert 32768 * 12800 * 2 < big < 32768 * (12800 * 16 + 3200 * 8) + 3200 * 12800 * 8


def test_gated_mlp_saved_bytes():
    assert B.epd_gated_mlp_saved_bytes(mlp_cfg(), 10) == 3 * 10 * 128 * 2 + 10 * 128
    assert B.epd_gated_mlp_saved_bytes(mlp_cfg(mlp_dim=8), 3) == 3 * 256 + 24
    assert B.epd_gated_mlp_saved_bytes(mlp_cfg(dtype=B.EPD_F32), 10) == 10 * 128 * 8
    assert B.epd_gated_mlp_saved_bytes(mlp_cfg(), 0) == 0
    for c, t in ((mlp_cfg(act=0), 1), (mlp_cfg(), 101), (mlp_cfg(), -1)):
        assert B.epd_gated_mlp_saved_bytes(c, t) == 0 and B.epd_op_last_error()


def test_encoder_takes_gated_activations_only_by_their_names():
    from paper_2601_11590_amd import workloads as W
    cfg = W.EncoderConfig(name="t", dtype="bf16", num_layers=1, hidden=64, num_heads=1, head_dim=64, mlp_dim=128, patch=4, temporal_patch=1, norm="rmsnorm",
                          rope="2d", rope_pairs=(0, 16, 16), out_dim=64)
    plain = B.epd_encode_workspace_bytes(B.make_cfg(cfg, 64, 4, 4))
    for act in W.GATED_ACTS:
        assert B.epd_encode_workspace_bytes(B.make_cfg(cfg.replace(act=act), 64, 4, 4)) == plain + 128 * 64 * 2 + 128 * 2     # the up rows and their biases
    c = B.make_cfg(cfg, 64, 4, 4)
    c.act = 5
    assert B.epd_encode_workspace_bytes(c) == 0
    with pytest.raises(KeyError):
        B.make_cfg(cfg.replace(act="reglu"), 64, 4, 4)
