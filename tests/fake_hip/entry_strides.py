"""Strides of the products in 8 bits on the stand-in runtime:  python entry_strides.py <stand-in .so> <libepd_encode.so> <most of x> <most of y
in bf16> <most of y in fp32>, the largest that the header allows."""

import ctypes as C
import sys

from driver import OK, binding, launches, load
from entry import A


def call(fake, lib, T, K, N, ld_x, ld_y, kind):
    B = binding()
    c = B.epd_int8_linear_cfg()
    c.struct_size, c.in_features, c.out_features, c.out_dtype, c.use_bias, c.max_tokens = C.sizeof(c), K, N, kind, 0, T
    fake.fake_forget()
    status = lib.epd_int8_linear(c, B.epd_int8_linear_weights(*A[3:6]), A[0], ld_x, A[1], T, A[2], ld_y, A[6], 1 << 60, None)
    return status, len(launches(fake)), lib.epd_op_last_error().decode()


if __name__ == "__main__":
    fake, lib = load(sys.argv[1], sys.argv[2])
    most_x, bf16, f32 = map(int, sys.argv[3:])
    B = binding()
    for T, K, N in ((2, 64, 64), (40, 64, 64), (64, 64, 64), (200, 12800, 320), (500, 64, 512), (32768, 3200, 4304)):
        for kind, most_y in ((B.EPD_BF16, bf16), (B.EPD_F32, f32)):
            for ld_x, ld_y in ((K, N), (most_x, N), (K, most_y), (most_x, most_y)):
                assert call(fake, lib, T, K, N, ld_x, ld_y, kind)[0] == OK, (T, ld_x, ld_y, kind)
            for ld_x, ld_y, said in ((most_x + 16, N, most_x), (K, most_y + 8, most_y), (1 << 40, N, most_x), (K, 1 << 40, most_y)):
                status, n, text = call(fake, lib, T, K, N, ld_x, ld_y, kind)
                assert status == B.EPD_ERR_SHAPE and n == 0 and (str(said) in text or "2^22 - 16" in text), (T, ld_x, ld_y, kind, status, text)
    print("passed")
