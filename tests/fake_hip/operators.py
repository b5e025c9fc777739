"""The operators beside the encoder on the stand-in runtime:  python operators.py <stand-in .so> <libepd_encode.so> <function of this
file> [<JSON>]."""

import ctypes as C
import json
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


def rotate(lib, T):
    B = binding()
    arr = (B.epd_rope_tensor * 1)((X, Y, 256, 64, 256, 64, 4))
    return lib.epd_rope_apply(C.byref(B.Rope("bf16", 64, (8, 12, 12)).cfg), arr, 1, 0x1000, T, T, 0, None)


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


if __name__ == "__main__":
    loaded = load(sys.argv[1], sys.argv[2])
    globals()[sys.argv[3]](*loaded, *(json.loads(a) for a in sys.argv[4:]))
    print("passed", sys.argv[3])
