"""The host layer of the optimizer step (csrc/optim_api.hip: checks, tables of tensors, launches) built with a host compiler under
-fsanitize=address,undefined against launchers that write down what they are given (CPU only, no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "host_sanitize")
CSRC = os.path.join(ROOT, "paper_2506_03077_amd", "csrc")


@pytest.fixture(scope="module")
def binary(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    out = str(tmp_path_factory.mktemp("host_sanitize_optim") / "optim")
    p = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-I", SRC, "-I", CSRC,
                        "-x", "c++", os.path.join(CSRC, "optim_api.hip"), os.path.join(SRC, "optim.cpp"), "-o", out], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-4000:]
    return out


def run(binary, *args):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)          # the sanitizer runtime must come first in the library list
    return subprocess.run([binary, *args], capture_output=True, text=True, env=env, timeout=600)


def test_tables_launches_and_workspace(binary):
    p = run(binary)
    assert p.returncode == 0 and p.stdout.strip() == "OK: 40 cases", (p.stdout[-2000:], p.stderr[-4000:])
    assert "runtime error" not in p.stderr and "AddressSanitizer" not in p.stderr


def test_a_planted_short_workspace_is_reported(binary):
    p = run(binary, "planted")
    assert p.returncode != 0 and "heap-buffer-overflow" in p.stderr
