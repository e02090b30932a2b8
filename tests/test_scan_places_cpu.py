"""Gradients of packed sequences in any order: ``csrc/scan_places.h``, which the kernels include, compiled for the host and checked over
random offsets (tests/scan_places/check_places.cpp)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_two_sequences_share_a_place(tmp_path):
    exe = tmp_path / "check_places"
    src = os.path.join(ROOT, "tests", "scan_places", "check_places.cpp")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", str(exe), src])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.startswith("ok ")
