"""The operators at the entry of the stage behind the encoder on the stand-in runtime:  python entry.py <stand-in .so> <libepd_encode.so>
<function of this file> [<JSON>]."""

import ctypes as C
import json
import random
import re
import sys

from driver import ERR_HIP, LAST_ERROR, OK, binding, launches, load

A = [(i + 1) << 44 for i in range(12)]                       # made-up addresses, never dereferenced
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


def code(t):
    return {"f32": binding().EPD_F32, "bf16": binding().EPD_BF16}[t]


def embed_cfg(types, T, V, D):
    c = binding().epd_embed_cfg()
    c.struct_size, c.dtype, c.out_dtype, c.vocab, c.hidden, c.max_tokens, c.scale = C.sizeof(c), code(types[0]), code(types[1]), V, D, max(T, 1), 1.0
    return c


def embed(lib, types, T, V, D, R=0):
    return lib.epd_embed(embed_cfg(types, T, V, D), A[0], A[1], R, A[2], T, A[3], D, None)


def embed_backward(lib, types, T, V, D, R=0):
    return lib.epd_embed_backward(embed_cfg(types, T, V, D), A[2], T, A[3], D, R, A[0], A[1], A[4], 1 << 60, None)


def norm_cfg(types, T, D):
    c = binding().epd_add_norm_cfg()
    c.struct_size, c.dtype, c.residual_dtype, c.hidden, c.max_tokens, c.eps = C.sizeof(c), code(types[0]), code(types[1]), D, max(T, 1), 1e-6
    return c


def norm(lib, types, T, D):
    return lib.epd_add_norm(norm_cfg(types, T, D), binding().epd_add_norm_rows(*A[:6], *[D] * 5), A[7], T, None)


def norm_backward(lib, types, T, D):
    return lib.epd_add_norm_backward(norm_cfg(types, T, D), binding().epd_add_norm_grads(*A[:6], *[D] * 5), A[7], T, A[8], 1 << 60, None)


def quant(lib, t, T, D):
    return lib.epd_quant_rows(code(t), A[0], D, T, D, A[1], D, A[2], None)


def dequant(lib, t, T, D):
    return lib.epd_dequant_rows(A[1], D, A[2], T, D, code(t), A[0], D, None)


def linear(lib, out, T, K, N):
    c = binding().epd_int8_linear_cfg()
    c.struct_size, c.in_features, c.out_features, c.out_dtype, c.use_bias, c.max_tokens = C.sizeof(c), K, N, code(out), 1, T
    return lib.epd_int8_linear(c, binding().epd_int8_linear_weights(*A[3:6]), A[0], K, A[1], T, A[2], N, A[6], 1 << 60, None)


def launched(fake, call, *args):
    fake.fake_forget()
    assert call(*args) == OK, args
    return launches(fake)


# ------------------------------------------------------------------ the tests

def a_failed_launch_is_reported(fake, lib):
    """Whatever error the program left uncollected before the call, and it stays where no launch fails."""
    calls = {}
    for t in TYPES:
        for T in (0, 20, 9000):
            calls["embed backward", t, T] = lambda t=t, T=T: embed_backward(lib, t, T, 50, 16, 3)
            calls["norm backward", t, T] = lambda t=t, T=T: norm_backward(lib, t, T, 320)
        calls["embed", t] = lambda t=t: embed(lib, t, 20, 50, 16)
        calls["norm", t] = lambda t=t: norm(lib, t, 20, 320)
    for t in ("bf16", "f32"):
        calls["quant", t] = lambda t=t: quant(lib, t, 20, 320)
        calls["dequant", t] = lambda t=t: dequant(lib, t, 20, 320)
        for T, K, N in ((1, 64, 64), (9, 64, 64), (200, 12800, 320), (32768, 3200, 12800), (500, 64, 512)):
            calls["linear", t, T] = lambda t=t, T=T, K=K, N=N: linear(lib, t, T, K, N)
    for what, call in calls.items():
        fake.fake_forget()
        fake.fake_set(LAST_ERROR, 1)
        assert call() == OK, what
        assert fake.fake_get(LAST_ERROR) == 1, what
        names = {l[0] for l in launches(fake)}
        assert names, what
        for name in names:
            for before in (0, 98):
                fake.fake_set(LAST_ERROR, before)
                fake.fake_refuse(name.encode(), 98)
                assert call() == ERR_HIP, (what, name, before)
                assert b"98" in lib.epd_op_last_error() and fake.fake_get(LAST_ERROR) == 0, (what, name, before)      # reported once
                fake.fake_refuse(b"", 0)
    fake.fake_set(LAST_ERROR, 0)


def launches_stay_within_the_thread_limit(fake, lib):
    """The largest calls that the entries take, in fewer than 2^32 threads along each axis of a grid."""
    most = 2 ** 31 - 1
    calls = [(quant, t, T, D) for t in ("bf16", "f32") for T in (most, most - 1, 1 << 24) for D in (1, 512, 2048, 4096, 65536)]
    calls += [(dequant, *c[1:]) for c in calls]
    calls += [(f, t, T, D) for f in (norm, norm_backward) for t in TYPES for T in (most, 1 << 24) for D in (1, 2048, 65536)]
    calls += [(f, t, min(1 << 24, (1 << 38) // D), V, D, R) for f in (embed, embed_backward) for t in TYPES for V in (1, 1 << 30) for D in (1, 512, 2049, 16384, 65536) for R in (0, 1 << 30)]
    for K in (16, 1024, 131056):
        for N in (8, 64, 72, 4096, 1 << 15, 1 << 20):
            if K * N < 1 << 32:
                calls += [(linear, t, T, K, N) for t in ("bf16", "f32") for T in (1, 2, 17, 64, 65, min((1 << 22) - 1, ((1 << 36) - 1) // N))]
    for f, *args in calls:
        if f is linear and args[0] == "f32" and args[3] >= 1 << 21:
            continue
        for name, grid, block in launched(fake, f, lib, *args):
            assert all(0 < g * b < 2 ** 32 for g, b in zip(grid, block)) and grid[1] < 65536 and grid[2] == 1, (f, args, name, grid, block)


def work_grows_with_the_launch(fake, lib):
    """Every row of a call belongs to exactly one launch of the norm's kernels, however many they are."""
    for T in (1, 3, 1 << 24, (1 << 24) + 1, 2 ** 31 - 1):
        for D, per in ((100, 4), (3200, 1)):
            blocks = sum(l[1][0] for l in launched(fake, quant, lib, "bf16", T, D))
            assert blocks == -(-T // per), (T, D, blocks)


# ------------------------------------------------------------------ what the sizes of the GPU tests reach

NAMES = r"_GLOBAL__N_1\d+((?:embed|sort|merge|sums|runs|few|norm|norm_grad|gain|dequant|int8_\w+?)_kernel)"


def kernels(fake):
    fake.fake_kernel.restype = C.c_char_p
    names = [fake.fake_kernel(i).decode() for i in range(fake.fake_kernels())]
    return {n for n in names if re.search(NAMES, n)}


def plan(l):
    """How a product was made: the kernel for few tokens, one tile, a body of one tile, or parts in one tile."""
    tile = [re.search(r"TileILi(\d+)ELi(\d+)", n) for n, _, _ in l]
    if "int8_gemm" in l[0][0]:
        return ("cut" if len(l) == 2 else "whole", *map(int, tile[0].groups()))
    if "int8_split" in l[0][0]:
        return ("parts", *map(int, tile[0].groups()))
    return (l[0][0],)


def the_gpu_tests_reach_every_kernel_and_plan(fake, lib, embeds, norms, linears):
    """embeds: [types, T, V, D, R]; norms: [types, T, D]; linears: [out, T, K, N] of the GPU tests."""
    seen, plans = set(), set()
    for t, T, V, D, R in embeds:
        for f in (embed, embed_backward):
            seen |= {l[0] for l in launched(fake, f, lib, t, T, V, D, R)}
    for t, T, D in norms:
        for f in (norm, norm_backward):
            seen |= {l[0] for l in launched(fake, f, lib, t, T, D)}
        for f in (quant, dequant):
            seen |= {l[0] for l in launched(fake, f, lib, t[0], T, D)}
    for out, T, K, N in linears:
        l = launched(fake, linear, lib, out, T, K, N)
        seen |= {x[0] for x in l}
        plans.add((out, plan(l)))
    own = kernels(fake)
    rng, missing = random.Random(2), {}
    for _ in range(20000):
        out, T, K, N = rng.choice(["bf16", "f32"]), round(2 ** rng.uniform(0, 15.5)), 16 * round(2 ** rng.uniform(0, 11)), 8 * round(2 ** rng.uniform(0, 11))
        if T * K * N < 3e12:
            p = (out, plan(launched(fake, linear, lib, out, T, K, N)))
            if p not in plans:
                missing.setdefault(p, []).append((T * K * N, T, K, N))
    assert len(own) > 50 and own <= seen and not missing, (sorted(own - seen), {p: min(s)[1:] for p, s in missing.items()})


if __name__ == "__main__":
    loaded = load(sys.argv[1], sys.argv[2])
    globals()[sys.argv[3]](*loaded, *(json.loads(a) for a in sys.argv[4:]))
    print("passed", sys.argv[3])
