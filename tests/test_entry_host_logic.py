"""Host logic of the operators at the entry of the stage behind the encoder on the stand-in runtime (fake_hip/), on the CPU: launches that
fail, launches of the largest sizes, and which kernels and plans the GPU tests reach."""

import json
import os
import shutil
import subprocess
import sys

import pytest

from paper_2601_11590_amd import build

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "fake_hip")


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    fake = str(tmp_path_factory.mktemp("fake") / "libfake_hip.so")
    subprocess.run([shutil.which("g++") or "c++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "fake_hip.cpp"), "-o", fake], check=True)

    def call(name, *args):
        r = subprocess.run([sys.executable, os.path.join(HERE, "entry.py"), fake, build.library_path(), name, *map(json.dumps, args)],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
        assert r.returncode == 0 and "passed " + name in r.stdout, r.stdout[-3000:]
    return call


@pytest.mark.parametrize("name", ["a_failed_launch_is_reported", "launches_stay_within_the_thread_limit", "work_grows_with_the_launch"])
def test_launches(run, name):
    run(name)


def test_the_gpu_tests_reach_every_kernel_and_plan(run):
    import test_gpu_add_norm as N
    import test_gpu_embed as E
    import test_gpu_int8_linear as L

    def sizes(test, names):
        return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == names)

    embeds = [(t, *s) for t in E.TYPES for s in sizes(E.test_forward_and_gradients, "T,V,D,R")]
    embeds += [(("bf16", "f32"), T, V, D, 100) for T, V, D, _ in sizes(E.test_gradients_of_many_tokens, "T,V,D,hot")]
    embeds += [(t, T, 100, D, 0) for t in E.TYPES for T, D in sizes(E.test_rows_of_many_tokens, "T,D")]
    run("the_gpu_tests_reach_every_kernel_and_plan", embeds, [(t, *s) for t in N.TYPES for s in N.SIZES], [(out, *s) for out in ("bf16", "f32") for s in L.SIZES + L.PLANS])
