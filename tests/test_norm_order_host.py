"""The order in which a norm adds up, on the host: what the header says that it depends on, and nothing else."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_order_of_a_norms_sums(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "san_norm_order"
    subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
                    "-static-libubsan", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2302_08545_amd", "csrc"), os.path.join(ROOT, "tests", "san_norm_order.cpp"), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "0 problem(s)" in res.stdout


def test_the_header_says_that_adjoining_tensors_matter():
    """Two layouts with the same addresses modulo 128 bytes are added up in two orders (above): the promise has to leave them out."""
    with open(os.path.join(ROOT, "include", "thc.h")) as f:
        text = re.sub(r"[\s*]+", " ", f.read())
    promise = text[text.index("Global norm v over all elements"):text.index("int thc_grad_norm(")]
    assert "modulo 128 bytes" in promise and "adjoin" in promise
