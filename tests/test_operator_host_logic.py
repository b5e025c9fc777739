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
