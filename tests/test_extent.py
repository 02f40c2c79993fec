"""Sizes of a call whose product leaves 64 bits (scores of strides 0), compiled for the CPU with the undefined-behaviour sanitizer."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2006_15704_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_products_that_leave_64_bits(tmp_path):
    exe = str(tmp_path / "extent")
    build = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", CSRC, "-o", exe,
                            os.path.join(ROOT, "tests", "host_sanitize", "extent.cpp")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout


def test_the_gradient_of_the_position_bias_uses_it():
    with open(os.path.join(CSRC, "position_bias.hip")) as fh:
        source = fh.read()
    assert "product_reaches(kStreamBytes, {batch, h->heads, queries, keys, elem_bytes(dtype)})" in source
