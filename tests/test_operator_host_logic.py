"""Host logic of the operators beside the encoder on the stand-in runtime (fake_hip/), on the CPU: launches that fail, launches of sizes that
take all of a card, and which kernels a call takes."""

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
        r = subprocess.run([sys.executable, os.path.join(HERE, "operators.py"), fake, build.library_path(), name, *map(json.dumps, args)],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
        assert r.returncode == 0 and "passed " + name in r.stdout, r.stdout[-3000:]
    return call


def test_a_failed_launch_is_reported(run):
    run("a_failed_launch_is_reported")


def test_sequences_of_2_31_tokens(run):
    run("sequences_of_2_31_tokens")


def test_launches_stay_within_the_thread_limit(run):
    run("launches_stay_within_the_thread_limit")


def test_gated_encoders_have_the_limits_of_the_operator():
    from paper_2601_11590_amd import binding as B, workloads as W

    def size(act, hidden, mlp_dim, max_tokens=64, dtype="bf16"):
        cfg = W.EncoderConfig(name="t", dtype=dtype, num_layers=1, hidden=hidden, num_heads=hidden // 64, head_dim=64, mlp_dim=mlp_dim, patch=4,
                              temporal_patch=1, norm="layernorm", rope="2d", rope_pairs=(0, 16, 16), out_dim=64)
        return B.epd_encode_workspace_bytes(B.make_cfg(cfg.replace(act=act), max_tokens, 4, 4))

    for act in W.GATED_ACTS:
        # below 2^30 weights a half, as the operator: with 2^31 the up rows would lie 2^32 bytes from the gate rows, past the tiles' offsets
        assert size(act, 8192, 131064) > 0 and size(act, 8192, 131072) == 0 and size(act, 8192, 262144) == 0
        assert size(act, 64, 131072) > 0 and size(act, 64, 131080) == 0
        assert size(act, 64, 64, (1 << 24) - 1) > 0
        # 2^33 gates in fp32: a launch of 64 x 64 tiles has a thread for 16 of both halves
        assert size(act, 64, 1024, (1 << 23) - 1, "f32") > 0 and size(act, 64, 1024, 1 << 23, "f32") == 0
    assert size("gelu_erf", 8192, 262144) > 0 and size("gelu_erf", 64, 1024, 1 << 23, "f32") > 0      # as before


def test_the_gpu_tests_reach_every_kernel_and_plan(run):
    import test_gpu_gated_mlp as G
    import test_gpu_operator_plans as P
    import test_gpu_operators_large as L
    import test_gpu_rope as R

    def sizes(test, names):
        return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == names)

    mlp = [("bf16", *s) for s in G.SIZES + G.LARGE + P.PLANS + sizes(L.test_every_kernel_of_the_products, "T,D,F") + sizes(L.test_products_in_parts, "T,D,F")]
    mlp += [("f32", *s) for t in (G.test_f32_training_step, G.test_f32_many_tokens) for s in sizes(t, "T,D,F")]
    mlp += [("bf16", T, D, F) for T in (1, 2) for D, F in sizes(G.test_bf16_one_and_two_tokens, "D,F")]
    mlp += [("bf16", T, D, F) for T in sizes(G.test_bf16_few_tokens, "T") for D, F, _, _ in sizes(G.test_bf16_few_tokens, "D,F,act,bias")]
    rope = [(t, p, *s) for t in ("bf16", "f32") for p in ("half", "adjacent") for s in sizes(R.test_rotation_and_inverse, "T,hq,hk,d,pairs") + P.ROPE_PLANS]
    run("the_gpu_tests_reach_every_kernel_and_plan", mlp, rope)
