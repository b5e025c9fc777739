"""What the operators at the entry of the stage behind the encoder refuse, all on the host: nothing is launched, no GPU is needed."""

import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2601_11590_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "epd_encode.h")
INVALID, UNSUPPORTED, SHAPE, WORKSPACE = B.EPD_ERR_INVALID_ARG, B.EPD_ERR_UNSUPPORTED, B.EPD_ERR_SHAPE, B.EPD_ERR_WORKSPACE
A = [(i + 1) << 40 for i in range(12)]                       # made-up addresses, never dereferenced
MAX = 2 ** 31 - 1


def test_every_declared_operator_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(epd_(?:embed|add_norm|quant|dequant|int8)\w*)\s*\(", text))
    assert names == set(B.ENTRY_EXPORTS)
    assert all(getattr(B.lib, n) is not None for n in names)


def test_structs_match_the_header(tmp_path):
    structs = [B.epd_embed_cfg, B.epd_add_norm_cfg, B.epd_add_norm_rows, B.epd_add_norm_grads, B.epd_int8_linear_cfg, B.epd_int8_linear_weights]
    lines, want = ['#include <stdio.h>', '#include <stddef.h>', '#include "epd_encode.h"', "int main(void) {"], []
    for t in structs:
        lines.append('printf("%%zu\\n", sizeof(%s));' % t.__name__)
        want.append(C.sizeof(t))
        for f, _ in t._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (t.__name__, f))
            want.append(getattr(t, f).offset)
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "probe")], check=True)
    out = subprocess.run([str(tmp_path / "probe")], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    assert [int(v) for v in out] == want


def said(status):
    return status, B.epd_op_last_error()


# ------------------------------------------------------------------ embeddings

def embed_cfg(**change):
    c = B.epd_embed_cfg()
    B._sizes(c, dtype=B.EPD_BF16, out_dtype=B.EPD_F32, vocab=100, hidden=24, max_tokens=50, scale=1.0)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def embed(table=A[0], rows=A[1], num_rows=3, ids=A[2], tokens=10, out=A[3], ld=24, cfg=None, **change):
    return said(B.lib.epd_embed(embed_cfg(**change) if cfg is None else cfg, table, rows, num_rows, ids, tokens, out, ld, None))


def embed_backward(ids=A[2], tokens=10, dout=A[3], ld=24, num_rows=3, dtable=A[0], drows=A[1], ws=A[4], ws_bytes=1 << 40, **change):
    return said(B.lib.epd_embed_backward(embed_cfg(**change), ids, tokens, dout, ld, num_rows, dtable, drows, ws, ws_bytes, None))


EMBED_BOTH = [
    (dict(struct_size=3), INVALID, "struct_size"), (dict(dtype=7), INVALID, "dtype"), (dict(out_dtype=-1), INVALID, "out_dtype"),
    (dict(dtype=B.EPD_F32, out_dtype=B.EPD_BF16), UNSUPPORTED, "fp32"), (dict(vocab=0), UNSUPPORTED, "vocab"), (dict(vocab=(1 << 30) + 1), UNSUPPORTED, "vocab"),
    (dict(hidden=0), UNSUPPORTED, "hidden"), (dict(hidden=65537), UNSUPPORTED, "hidden"), (dict(max_tokens=0), UNSUPPORTED, "max_tokens"),
    (dict(max_tokens=(1 << 24) + 1), UNSUPPORTED, "max_tokens"), (dict(max_tokens=1 << 24, hidden=16385), UNSUPPORTED, "2^38"), (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(tokens=-1), SHAPE, "tokens"), (dict(tokens=51), SHAPE, "max_tokens"), (dict(num_rows=-1), UNSUPPORTED, "num_rows"),
    (dict(num_rows=(1 << 30) + 1), UNSUPPORTED, "num_rows"), (dict(ids=None), INVALID, "ids"), (dict(ids=A[2] + 2), INVALID, "ids"),
    (dict(ld=23), SHAPE, "apart"), (dict(ld=-24), SHAPE, "apart"), (dict(ld=(1 << 40) + 1), SHAPE, "apart")]


@pytest.mark.parametrize("kw,status,needle", EMBED_BOTH + [
    (dict(table=None), INVALID, "NULL"), (dict(rows=None), INVALID, "NULL"), (dict(out=None), INVALID, "out"), (dict(out=A[3] + 2), INVALID, "aligned"),
    (dict(table=A[0] + 1), INVALID, "aligned"), (dict(rows=A[1] + 1), INVALID, "aligned")])
def test_embed_refusals(kw, status, needle):
    got, msg = embed(**kw)
    assert got == status and needle in msg, (got, msg)


@pytest.mark.parametrize("kw,status,needle", EMBED_BOTH + [
    (dict(dout=None), INVALID, "dout"), (dict(dtable=A[0] + 1), INVALID, "aligned"), (dict(drows=A[1] + 1), INVALID, "aligned"), (dict(ws=None), WORKSPACE, "workspace"),
    (dict(ws=A[4] + 128), WORKSPACE, "256"), (dict(ws_bytes=4 * 256 + 7 * 2 * 24 * 4 - 1), WORKSPACE, "required")])
def test_embed_backward_refusals(kw, status, needle):
    got, msg = embed_backward(**kw)
    assert got == status and needle in msg, (got, msg)


def test_embed_calls_without_work():
    assert embed(tokens=0, ids=None, out=None)[0] == B.EPD_OK
    assert embed_backward(dtable=None, drows=None)[0] == B.EPD_OK
    assert embed_backward(dtable=None, num_rows=0)[0] == B.EPD_OK            # no rows: their gradient is none
    assert embed(cfg=C.POINTER(B.epd_embed_cfg)())[0] == INVALID


def test_workspaces_grow_with_the_tokens():
    sizes = [B.epd_embed_workspace_bytes(embed_cfg(max_tokens=t)) for t in (1, 100, 8192, 8193, 16384, 16385, 40000, 1 << 24)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0 and all(s % 256 == 0 for s in sizes)
    assert B.epd_embed_workspace_bytes(embed_cfg(vocab=0)) == 0 and "vocab" in B.epd_op_last_error()


# ------------------------------------------------------------------ norm

def norm_cfg(**change):
    c = B.epd_add_norm_cfg()
    B._sizes(c, dtype=B.EPD_BF16, residual_dtype=B.EPD_F32, hidden=24, max_tokens=50, eps=1e-6)
    for k, v in change.items():
        setattr(c, k, v)
    return c


CFG = set(n for n, _ in B.epd_add_norm_cfg._fields_)


def norm(gain=A[9], tokens=10, **change):
    r = B.epd_add_norm_rows(A[0], A[1], A[2], A[3], A[4], A[5], 24, 24, 24, 24, 24)
    for k, v in change.items():
        if k not in CFG:
            setattr(r, k, v)
    return said(B.lib.epd_add_norm(norm_cfg(**{k: v for k, v in change.items() if k in CFG}), r, gain, tokens, None))


def norm_backward(gain=A[9], tokens=10, ws=A[10], ws_bytes=1 << 40, **change):
    g = B.epd_add_norm_grads(A[0], A[1], A[2], A[3], A[4], A[5], 24, 24, 24, 24, 24)
    for k, v in change.items():
        if k == "dgain":
            g.gain = v
        elif k not in CFG:
            setattr(g, k, v)
    return said(B.lib.epd_add_norm_backward(norm_cfg(**{k: v for k, v in change.items() if k in CFG}), g, gain, tokens, ws, ws_bytes, None))


NORM_BOTH = [
    (dict(struct_size=0), INVALID, "struct_size"), (dict(dtype=3), INVALID, "dtype"), (dict(residual_dtype=2), INVALID, "residual_dtype"),
    (dict(dtype=B.EPD_F32, residual_dtype=B.EPD_BF16), UNSUPPORTED, "fp32"), (dict(hidden=0), UNSUPPORTED, "hidden"), (dict(hidden=65537), UNSUPPORTED, "hidden"),
    (dict(max_tokens=0), INVALID, "max_tokens"), (dict(eps=-1e-6), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(eps=float("inf")), INVALID, "eps"),
    (dict(tokens=-1), SHAPE, "tokens"), (dict(tokens=51), SHAPE, "max_tokens"), (dict(gain=None), INVALID, "gain"), (dict(gain=A[9] + 1), INVALID, "gain")]


@pytest.mark.parametrize("kw,status,needle", NORM_BOTH + [
    (dict(x=None, residual=None), INVALID, "neither"), (dict(sum=None, y=None, q=None), INVALID, "no output"), (dict(scale=None), INVALID, "scale"),
    (dict(scale=A[5] + 2), INVALID, "scale"), (dict(x=A[0] + 1), INVALID, "aligned"), (dict(residual=A[1] + 2), INVALID, "aligned"), (dict(sum=A[2] + 2), INVALID, "aligned"),
    (dict(ld_x=23), SHAPE, "rows of x"), (dict(ld_residual=0), SHAPE, "rows of residual"), (dict(ld_sum=-1), SHAPE, "rows of sum"), (dict(ld_y=23), SHAPE, "rows of y"),
    (dict(ld_q=23), SHAPE, "rows of q"), (dict(sum=A[1], ld_sum=32), SHAPE, "in place"), (dict(y=A[0], ld_y=32), SHAPE, "in place")])
def test_norm_refusals(kw, status, needle):
    got, msg = norm(**kw)
    assert got == status and needle in msg, (got, msg)


@pytest.mark.parametrize("kw,status,needle", NORM_BOTH + [
    (dict(sum=None), INVALID, "sum"), (dict(dy=None), INVALID, "dy"), (dict(dgain=A[5] + 1), INVALID, "gain"), (dict(ws=None), WORKSPACE, "workspace"),
    (dict(ws=A[10] + 16), WORKSPACE, "256"), (dict(ws_bytes=255), WORKSPACE, "required"), (dict(ld_sum=23), SHAPE, "rows of sum"), (dict(ld_dy=1), SHAPE, "rows of dy"),
    (dict(ld_dsum=23), SHAPE, "rows of dsum"), (dict(ld_dx=23), SHAPE, "rows of dx"), (dict(ld_dresidual=23), SHAPE, "rows of dresidual"),
    (dict(dx=A[1], ld_dx=25), SHAPE, "in place"), (dict(dresidual=A[2], ld_dresidual=25), SHAPE, "in place"), (dict(dx=A[3] + 1), INVALID, "aligned")])
def test_norm_backward_refusals(kw, status, needle):
    got, msg = norm_backward(**kw)
    assert got == status and needle in msg, (got, msg)


def test_norm_calls_without_work():
    assert norm(tokens=0, x=None, residual=None)[0] == B.EPD_OK
    assert norm_backward(dx=None, dresidual=None, dgain=None, ws=None)[0] == B.EPD_OK
    assert norm_backward(tokens=0, dgain=None, sum=None, dy=None)[0] == B.EPD_OK
    sizes = [B.epd_add_norm_workspace_bytes(norm_cfg(max_tokens=t, hidden=3200)) for t in (1, 4, 5, 1000, 4096, 1 << 20)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0


# ------------------------------------------------------------------ 8 bits

@pytest.mark.parametrize("change,status,needle", [
    (dict(dtype=2), INVALID, "dtype"), (dict(rows=-1), SHAPE, "rows"), (dict(cols=0), UNSUPPORTED, "cols"), (dict(cols=65537), UNSUPPORTED, "cols"),
    (dict(m=None), INVALID, "NULL"), (dict(m=A[0] + 1), INVALID, "aligned"), (dict(ld_m=39), SHAPE, "apart"), (dict(q=None), INVALID, "q"), (dict(ld_q=39), SHAPE, "apart"),
    (dict(scale=None), INVALID, "scale"), (dict(scale=A[2] + 1), INVALID, "scale")])
def test_quant_refusals(change, status, needle):
    a = {**dict(dtype=B.EPD_F32, m=A[0], ld_m=40, rows=5, cols=40, q=A[1], ld_q=40, scale=A[2]), **change}
    for got, msg in (said(B.lib.epd_quant_rows(a["dtype"], a["m"], a["ld_m"], a["rows"], a["cols"], a["q"], a["ld_q"], a["scale"], None)),
                     said(B.lib.epd_dequant_rows(a["q"], a["ld_q"], a["scale"], a["rows"], a["cols"], a["dtype"], a["m"], a["ld_m"], None))):
        assert got == status and needle in msg, (got, msg)


def linear(x=A[0], ld_x=64, x_scale=A[1], tokens=10, y=A[2], ld_y=40, w=A[3], scale=A[4], bias=A[5], ws=A[6], ws_bytes=1 << 40, **change):
    c = B.epd_int8_linear_cfg()
    B._sizes(c, in_features=64, out_features=40, out_dtype=B.EPD_BF16, use_bias=1, max_tokens=50)
    for k, v in change.items():
        setattr(c, k, v)
    return said(B.lib.epd_int8_linear(c, B.epd_int8_linear_weights(w, scale, bias), x, ld_x, x_scale, tokens, y, ld_y, ws, ws_bytes, None))


@pytest.mark.parametrize("kw,status,needle", [
    (dict(struct_size=1), INVALID, "struct_size"), (dict(out_dtype=2), INVALID, "out_dtype"), (dict(use_bias=2), INVALID, "use_bias"), (dict(in_features=0), INVALID, "size"),
    (dict(out_features=-8), INVALID, "size"), (dict(max_tokens=0), INVALID, "size"), (dict(in_features=72), UNSUPPORTED, "multiple of 16"),
    (dict(in_features=131072), UNSUPPORTED, "131056"), (dict(out_features=44), UNSUPPORTED, "multiple of 8"), (dict(out_features=(1 << 20) + 8), UNSUPPORTED, "out_features"),
    (dict(in_features=65536, out_features=65536), UNSUPPORTED, "2^32"), (dict(max_tokens=1 << 22), UNSUPPORTED, "max_tokens"),
    (dict(max_tokens=1 << 20, out_features=65536), UNSUPPORTED, "max_tokens"),
    (dict(tokens=-1), SHAPE, "tokens"), (dict(tokens=51), SHAPE, "max_tokens"), (dict(w=None), INVALID, "weight"), (dict(scale=None), INVALID, "weight"),
    (dict(bias=None), INVALID, "weight"), (dict(w=A[3] + 8), UNSUPPORTED, "16 bytes"), (dict(scale=A[4] + 4), UNSUPPORTED, "16 bytes"), (dict(bias=A[5] + 8), UNSUPPORTED, "16 bytes"),
    (dict(ws=None), WORKSPACE, "workspace"), (dict(ws=A[6] + 1), WORKSPACE, "256"), (dict(ws_bytes=10), WORKSPACE, "required"), (dict(x=None), INVALID, "NULL"),
    (dict(x_scale=None), INVALID, "NULL"), (dict(y=None), INVALID, "NULL"), (dict(x_scale=A[1] + 2), INVALID, "aligned"), (dict(ld_x=48), SHAPE, "rows of x"),
    (dict(ld_x=72), SHAPE, "rows of x"), (dict(ld_x=1 << 22), SHAPE, "rows of x"), (dict(ld_y=32), SHAPE, "rows of y"), (dict(ld_y=44), SHAPE, "rows of y"),
    (dict(ld_y=1 << 22), SHAPE, "rows of y"), (dict(ld_y=1 << 21, out_dtype=B.EPD_F32), SHAPE, "rows of y"), (dict(x=A[0] + 8), UNSUPPORTED, "16 bytes"),
    (dict(y=A[2] + 8), UNSUPPORTED, "16 bytes")])
def test_linear_refusals(kw, status, needle):
    got, msg = linear(**kw)
    assert got == status and needle in msg, (got, msg)


def test_linear_without_tokens():
    assert linear(tokens=0, x=None, x_scale=None, y=None)[0] == B.EPD_OK


# ------------------------------------------------------------------ the binding

def test_sizes_beyond_32_bits_are_refused():
    for kw in (dict(vocab=2 ** 32 + 1), dict(hidden=2 ** 32 + 8), dict(max_tokens=2 ** 33)):
        with pytest.raises(ValueError):
            B.Embedding("bf16", **{**dict(vocab=10, hidden=8), **kw})
    with pytest.raises(ValueError):
        B.AddNorm("bf16", 2 ** 32 + 8)
    with pytest.raises(ValueError):
        B.Int8Linear(2 ** 32 + 16, 8)
    for make in (lambda: B.Embedding("bf16", 0, 8), lambda: B.AddNorm("bf16", 0), lambda: B.Int8Linear(8, 8), lambda: B.AddNorm("f32", 8, residual="bf16")):
        with pytest.raises(B.EpdError):
            make()


def test_host_tensors_are_refused():
    x = torch.zeros(4, 8)
    for call in (lambda: B.quant_rows(x), lambda: B.dequant_rows(x.to(torch.int8), x[:, 0]), lambda: B.quant_rows(x.double())):
        with pytest.raises(ValueError):
            call()
