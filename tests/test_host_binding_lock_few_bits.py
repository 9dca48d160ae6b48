"""The decoder layer's calls give Python's lock back too (see test_host_binding_lock.py): the native module on top of a stand-in for
libbmx.so whose entry points ask whether the calling thread holds the lock, and launch nothing."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_IN = """#include <stddef.h>
#include <stdint.h>
extern "C" {
int PyGILState_Check(void);
int calls, held;
static int asked() { ++calls; held += PyGILState_Check(); return 0; }
size_t bmx_workspace_bytes(int, const int64_t*, int) { return 512; }
int64_t bmx_conv_weight_row_words(int, int, int) { return 2; }
#define ENTRY(name) int name() { return asked(); }
ENTRY(bmx_binarize_pack) ENTRY(bmx_unpack_pm1) ENTRY(bmx_xnor_gemm) ENTRY(bmx_xnor_gemm_count) ENTRY(bmx_widen_words32)
ENTRY(bmx_binary_fc_static) ENTRY(bmx_binary_fc_packed) ENTRY(bmx_pack_conv_weights) ENTRY(bmx_pack_nchw)
ENTRY(bmx_binary_conv2d_packed) ENTRY(bmx_alpha_mean_abs) ENTRY(bmx_lazy_binary_fc) ENTRY(bmx_lazy_binary_conv2d)
ENTRY(bmx_lazy_xnor_gemm_w32) ENTRY(bmx_lazy_binary_conv2d_bits) ENTRY(bmx_lazy_quant_gemm)
ENTRY(bmx_w4_quantize) ENTRY(bmx_w4_dequantize) ENTRY(bmx_w4_fc) ENTRY(bmx_kv_write) ENTRY(bmx_kv_read) ENTRY(bmx_kv_attention)
ENTRY(bmx_fresh_kv_attention)
}
"""

CHILD = """
import ctypes, sys
import torch
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_1705_09864_amd import _bmx_host as h
h.set_error(RuntimeError)
z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")
n = None
tiles, scales = z(2, 1, 1024, t=torch.uint8), z(2, 2, 16, 2, t=torch.bfloat16)
cache = z(4, 2, 2, 64 * 64, t=torch.int8), z(4, 2, 2, 4), z(3, 2, t=torch.int32), z(3, t=torch.int32)
kv, q = z(3, 2, 64, t=torch.float16), z(3, 4, 64, t=torch.float16)
CALLS = [("w4_quantize", z(20, 100), 64, n), ("w4_dequantize", tiles, scales, 20, 100, n, n), ("w4_fc", z(3, 100), tiles, scales, 20, n, n, n),
         ("kv_write", kv, kv, *cache, n, 0, n), ("kv_read", *cache, 64, torch.float16, 3, n, 0, n, n, n),
         ("kv_attention", q, *cache, n, 0, n, True, 0, True, n, n, n),
         ("kv_attention", q, *cache, n, 0, 0.5, False, 7, False, n, z(1024, t=torch.uint8), n)]
calls, held = ctypes.c_int.in_dll(stand_in, "calls"), ctypes.c_int.in_dll(stand_in, "held")
for name, *args in CALLS:
    calls.value = held.value = 0
    getattr(h, name)(*args)
    print(name, calls.value, held.value, flush=True)
"""


def test_decoder_calls_run_without_pythons_lock(tmp_path):
    (tmp_path / "stand_in.cpp").write_text(STAND_IN)
    so = str(tmp_path / "stand_in.so")
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", str(tmp_path / "stand_in.cpp"), "-o", so], check=True)
    r = subprocess.run([sys.executable, "-c", CHILD, so, ROOT], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    seen = [line.split() for line in r.stdout.splitlines()]
    assert [(calls, held) for _, calls, held in seen] == [("1", "0")] * 7, r.stdout
