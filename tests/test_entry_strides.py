"""The strides that the header allows the rows of a product in 8 bits are those that the library takes, on the stand-in runtime."""

import os
import re
import shutil
import subprocess
import sys

from paper_2601_11590_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_the_largest_strides_of_the_header(tmp_path):
    text = " ".join(open(os.path.join(os.path.dirname(HERE), "include", "epd_encode.h")).read().replace("\n *", " ").split())
    x = re.search(r"x device int8 \[tokens, K\].*?rows ld_x apart: a multiple of 16, K \.\. 2\^(\d+) - (\d+)", text)
    y = re.search(r"rows ld_y elements apart: a multiple of 8, N \.\. 2\^(\d+) - (\d+) in bf16, N \.\. 2\^(\d+) - (\d+) in fp32", text)
    assert x and y
    most = [2 ** int(a) - int(b) for a, b in (x.groups(), y.groups()[:2], y.groups()[2:])]
    fake = str(tmp_path / "libfake_hip.so")
    subprocess.run([shutil.which("g++") or "c++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "fake_hip", "fake_hip.cpp"), "-o", fake], check=True)
    r = subprocess.run([sys.executable, os.path.join(HERE, "fake_hip", "entry_strides.py"), fake, build.library_path(), *map(str, most)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "passed" in r.stdout, r.stdout[-3000:]
