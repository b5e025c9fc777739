"""The operators beside the encoder on the stand-in runtime:  python operators.py <stand-in .so> <libepd_encode.so> <function of this
file> [<JSON>]."""

import ctypes as C
import json
import random
import re
import sys

from driver import ERR_HIP, LAST_ERROR, LAUNCH_STATUS, OK, binding, launches, load

X, Y, DY, DX, SAVED, GRADS, WEIGHTS, WORKSPACE = ((i + 1) << 40 for i in range(8))       # made-up addresses, never dereferenced


def mlp_cfg(dtype, T, D, F, act="swiglu", bias=True, training=True):
    B = binding()
    c = B.epd_gated_mlp_cfg()
    c.struct_size, c.dtype, c.act = C.sizeof(c), {"f32": B.EPD_F32, "bf16": B.EPD_BF16}[dtype], B._GATED[act]
    c.hidden, c.mlp_dim, c.max_tokens, c.use_bias, c.training = D, F, T, int(bias), int(training)
    return c


def mlp_weights():
    return binding().epd_gated_mlp_weights(*(WEIGHTS + (i << 36) for i in range(4)))


def forward(lib, cfg, T, save=True):
    return lib.epd_gated_mlp(C.byref(cfg), C.byref(mlp_weights()), X, cfg.hidden, T, Y, cfg.hidden, SAVED if save else None, WORKSPACE, 1 << 60, None)


def backward(lib, cfg, T, want=("dx", "gate_up_w", "gate_up_b", "down_w", "down_b")):
    g = binding().epd_gated_mlp_grads()
    for i, n in enumerate(want):
        setattr(g, n, DX if n == "dx" else GRADS + (i << 36))
    g.ld_dx = cfg.hidden
    return lib.epd_gated_mlp_backward(C.byref(cfg), C.byref(mlp_weights()), X, cfg.hidden, DY, cfg.hidden, T, SAVED, C.byref(g), WORKSPACE, 1 << 60, None)


def rotate(lib, T, dtype="bf16", pairing="half", heads=(4,), d=64, pairs=(8, 12, 12)):
    B = binding()
    arr = (B.epd_rope_tensor * len(heads))(*((X + (i << 36), Y + (i << 36), h * d, d, h * d, d, h) for i, h in enumerate(heads)))
    return lib.epd_rope_apply(C.byref(B.Rope(dtype, d, pairs, pairing=pairing).cfg), arr, len(heads), 0x1000, T, T, 0, None)


def positions(lib, spans, cu):
    s, c = (C.c_int32 * (3 * len(spans)))(*(v for t in spans for v in t)), (C.c_int32 * len(cu))(*cu)
    return lib.epd_rope_positions(s, c, len(cu) - 1, None, 1, X, 1 << 40, None, None)


# ------------------------------------------------------------------ the tests

def a_failed_launch_is_reported(fake, lib):
    """Whatever error the program left uncollected before the call, and it stays where no launch fails."""
    calls = {"rope": lambda: rotate(lib, 100), "positions": lambda: positions(lib, [(40, 0, 0), (1, 4, 4)], [0, 2])}
    for dtype, T, D, F in (("bf16", 1, 1024, 4096), ("bf16", 40, 512, 2048), ("bf16", 40, 2056, 8200), ("bf16", 200, 1024, 4096), ("bf16", 257, 1152, 264),
                           ("bf16", 6272, 1024, 4096), ("bf16", 32768, 3200, 12800), ("f32", 40, 256, 1024), ("f32", 2048, 1024, 4096)):
        c = mlp_cfg(dtype, T, D, F)
        calls["forward", dtype, T, D, F] = lambda c=c, T=T: forward(lib, c, T)
        calls["backward", dtype, T, D, F] = lambda c=c, T=T: backward(lib, c, T)
    none = mlp_cfg("bf16", 8, 64, 64)
    calls["no tokens"] = lambda: backward(lib, none, 0)
    for what, call in calls.items():
        fake.fake_forget()
        fake.fake_set(LAST_ERROR, 1)
        assert call() == OK, what
        assert fake.fake_get(LAST_ERROR) == 1, what
        names = {l[0] for l in launches(fake)}
        assert names, what
        for name in names:
            for before in (0, 1, 98):
                fake.fake_set(LAST_ERROR, before)
                fake.fake_refuse(name.encode(), 98)
                assert call() == ERR_HIP, (what, name, before)
                assert b"98" in lib.epd_op_last_error() and fake.fake_get(LAST_ERROR) == 0, (what, name, before)      # reported once
                fake.fake_refuse(b"", 0)
    fake.fake_set(LAST_ERROR, 0)


def sequences_of_2_31_tokens(fake, lib):
    """Positions of as many tokens as the entry takes: a thread each."""
    most = 2 ** 31 - 1
    for tokens in (most, most - 1, most - 254, most - 255, most - 256):
        fake.fake_forget()
        assert positions(lib, [(tokens - 10, 0, 0), (10, 0, 0)], [0, 1, 2]) == OK
        ((_, grid, block),) = launches(fake)
        assert (grid, block) == ((-(-tokens // 256), 1, 1), (256, 1, 1)), (tokens, grid)
    fake.fake_forget()
    assert rotate(lib, most) == OK
    assert all(g * b < 2 ** 32 for l in launches(fake) for g, b in zip(l[1], l[2]))


def launches_stay_within_the_thread_limit(fake, lib):
    """Every call that the entries take is launched, in fewer than 2^32 threads along each axis of a grid."""
    most, threads = {"bf16": 1 << 36, "f32": 1 << 33}, 0
    for dtype in most:
        for D in (8, 64, 2040, 2047, 2048, 8184, 65536):
            for F in (8, 16, 64, 128, 2048, 8192, 131072):
                if D * F >= 1 << 30 or (dtype == "bf16" and (D % 8 or F % 8)):
                    continue
                T = min((1 << 22) - 1, (most[dtype] - 1) // max(D, F))
                c = mlp_cfg(dtype, T, D, F)
                assert lib.epd_gated_mlp_workspace_bytes(C.byref(c)) > 0, (dtype, T, D, F)
                for call in (forward, backward):
                    fake.fake_forget()
                    assert call(lib, c, T) == OK, (call, dtype, T, D, F)
                    for name, grid, block in launches(fake):
                        assert all(0 < g * b < 2 ** 32 for g, b in zip(grid, block)) and grid[1] < 65536, (dtype, T, D, F, name, grid, block)
                        threads = max(threads, grid[0] * block[0])
    assert threads > 1 << 30


# ------------------------------------------------------------------ what the sizes of the GPU tests reach

def kernels(fake):
    """The library's kernels that only the operators launch."""
    fake.fake_kernel.restype = C.c_char_p
    names = [fake.fake_kernel(i).decode() for i in range(fake.fake_kernels())]
    own = ["gemm_bf16_pair", "gemm_bf16_split", "few_tokens", "one_token", "transpose_bf16", "part_sums", "sum_parts", "join_kernel", "gemm_f32_group",
           "gemm_f32_lds_group", "rope_kernel", "rope_positions"]
    return {n for n in names if any(o in n for o in own) or tag(n) == 2}


GEMM = r"gemm_bf16_(kernel|pair_kernel|split_kernel)INS_4TileILi(\d+)ELi(\d+)E.*?EE"


def tag(name):
    m = re.search(GEMM + r"Li\d+ELi\d+ELb[01]ELb[01]ELi(\d)E", name)
    return int(m[4]) if m and m[1] == "kernel" else -1


def product(launched, M, N):
    """How a product of M x N was made: by a kernel for few tokens, in K parts (of which tile and how many), else whole or cut in two, and
    whether operands were turned first."""
    turned = [l for l in launched if "transpose" in l[0]]
    rest = [l for l in launched if "transpose" not in l[0]]
    for few in ("few_tokens", "one_token"):
        if few in rest[0][0]:
            assert len(rest) == 1
            return (few,)
    m = re.search(GEMM, rest[0][0])
    tile = (int(m[2]), int(m[3]))
    if m[1] == "split_kernel":
        assert len(rest) == 2 and "join_kernel" in rest[1][0] and not turned
        return ("parts", tile, rest[0][1][0] // (-(-M // tile[0]) * -(-N // tile[1])))
    assert len(rest) <= 2
    return ("cut" if len(rest) == 2 else "whole", "turned" if turned else "as they stand")


def plans(fake, lib, T, D, F):
    """Every product of a bf16 training step, and how it was made."""
    c, out = mlp_cfg("bf16", T, D, F), set()

    def launched(call, *args):
        fake.fake_forget()
        assert call(lib, c, T, *args) == OK, (T, D, F)
        return launches(fake)

    is_epilogue = lambda l, e: re.search(GEMM + "Li%dE" % e, l[0])
    for save in (False, True):
        l = launched(forward, save)
        up = max(1, sum(1 for x in l if is_epilogue(x, 4)))
        out |= {("up", save, *product(l[:up], T, 2 * F)), ("down", *product(l[up:], T, D))}
    l = launched(backward, ("dx",))
    first = max(i for i, x in enumerate(l) if is_epilogue(x, 5)) + 1
    out |= {("dh", *product(l[:first], T, F)), ("dx", *product(l[first:], T, D))}
    both = launched(backward, ("gate_up_w", "down_w"))[first:]
    alone = [launched(backward, ("gate_up_w",))[first:], launched(backward, ("down_w",))]
    if len(both) == 1 and "pair" in both[0][0]:
        assert all(len(a) == 1 and a[0][0] == both[0][0] for a in alone)
        out.add(("weights together", re.search(GEMM, both[0][0]).groups()[1:]))
    else:
        out |= {("gate_up_w", *product(alone[0], 2 * F, D)), ("down_w", *product(alone[1], D, F))}
    return out


def the_gpu_tests_reach_every_kernel_and_plan(fake, lib, mlp, rope):
    """mlp: [dtype, T, D, F]; rope: [dtype, pairing, T, hq, hk, d, pairs] of the GPU tests."""
    seen, reached = set(), set()
    for dtype, T, D, F in mlp:
        c = mlp_cfg(dtype, T, D, F)
        for call in (lambda: forward(lib, c, T), lambda: forward(lib, c, T, save=False), lambda: backward(lib, c, T)):
            fake.fake_forget()
            assert call() == OK, (dtype, T, D, F)
            seen |= {l[0] for l in launches(fake)}
        if dtype == "bf16":
            reached |= plans(fake, lib, T, D, F)
    fake.fake_forget()
    for dtype, pairing, T, hq, hk, d, pairs in rope:
        assert rotate(lib, T, dtype, pairing, (hq, hk), d, pairs) == OK
    assert positions(lib, [(3, 0, 0)], [0, 1]) == OK
    seen |= {l[0] for l in launches(fake)}
    own = kernels(fake)
    assert len(own) > 60 and own <= seen, sorted(own - seen)
    # ... and every plan that any of 20 000 other sizes has
    rng, missing = random.Random(1), {}
    for _ in range(20000):
        T, D, F = round(2 ** rng.uniform(0, 16)), max(1, round(2 ** rng.uniform(0, 10.5))) * 8, max(1, round(2 ** rng.uniform(0, 12))) * 8
        if D * F < 1 << 29:
            for p in plans(fake, lib, T, D, F) - reached:
                missing.setdefault(p, []).append((T * D * F, T, D, F))
    assert not missing, {p: min(s)[1:] for p, s in missing.items()}


if __name__ == "__main__":
    loaded = load(sys.argv[1], sys.argv[2])
    globals()[sys.argv[3]](*loaded, *(json.loads(a) for a in sys.argv[4:]))
    print("passed", sys.argv[3])
