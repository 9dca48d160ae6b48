"""Which steps of K a wave of the 4-bit products for few rows loads (csrc/k_steps.h), walked on the host."""
import ctypes
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1705_09864_amd", "csrc")
SOURCE = """
#define __host__
#define __device__
#include "k_steps.h"
extern "C" int step(int wave, int waves, int n, int full) { return bmx::k_step(wave, waves, n, full); }
"""


def test_steps_stay_inside_the_weights(tmp_path):
    """In the kernel's order: every step is in its registers when it is used, and none that is not there is asked for."""
    src, so = str(tmp_path / "steps.cpp"), str(tmp_path / "steps.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", so])
    L = ctypes.CDLL(so)
    for full in list(range(1, 40)) + [72, 131071]:
        for waves in (1, 2, 3, 4, 8):
            for depth in (2, 4):
                used = set()
                for wave in range(min(waves, full)):
                    held = [L.step(wave, waves, d, full) for d in range(depth)]
                    kt = wave
                    while kt < full and len(used) < 10000:
                        for d in range(depth):
                            if kt < full:
                                assert held[d] == kt
                                used.add(kt)
                                held[d] = L.step(kt, waves, depth, full)
                                assert 0 <= held[d] < full
                            kt += waves
                    assert all(0 <= step < full for step in held)
                assert len(used) >= min(full, 10000)
