"""Refusals of the calls for pages on the GPU, rotary positions and the cache of 4 bits: every one on the host, before any launch."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_1705_09864_amd import binding as B

P = 0x7F0000001000  # a fake, well aligned, never dereferenced device address
OK, E_NULL, E_SHAPE, E_LD, E_ALIGN, E_UNSUP, E_WS = 0, -1, -2, -3, -4, -5, -6
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1705_09864_amd", "csrc")
TOP = 2**31 - 1


def resize(change=P, sequences=4, table=P, table_ld=8, width=8, lengths=P, pool=P, num_pages=40, starts=P, positions=P, slots=P, rows=10):
    return B.lib().bmx_kv_resize(change, sequences, table, table_ld, width, lengths, pool, num_pages, starts, positions, slots, rows, None)


@pytest.mark.parametrize("change,status", [
    (dict(sequences=-1), E_SHAPE), (dict(sequences=65536), E_SHAPE), (dict(width=-1), E_SHAPE), (dict(num_pages=-1), E_SHAPE), (dict(num_pages=TOP), E_SHAPE),
    (dict(rows=-1), E_SHAPE), (dict(rows=1 << 31), E_SHAPE), (dict(change=None), E_NULL), (dict(table=None), E_NULL), (dict(lengths=None), E_NULL),
    (dict(pool=None), E_NULL), (dict(starts=None), E_NULL), (dict(table_ld=7), E_LD), (dict(change=P + 2), E_ALIGN), (dict(table=P + 1), E_ALIGN),
    (dict(lengths=P + 2), E_ALIGN), (dict(pool=P + 2), E_ALIGN), (dict(starts=P + 2), E_ALIGN), (dict(positions=P + 2), E_ALIGN), (dict(slots=P + 4), E_ALIGN)])
def test_kv_resize_refusals(change, status):
    assert resize(**change) == status


def turn(x=P, type=2, x_row=192, x_head=96, heads=2, dim=96, rows=5, positions=P, freq=P, rot=96, out=P + 4096, out_row=192, out_head=96):
    return B.lib().bmx_rotary(x, type, x_row, x_head, heads, dim, rows, positions, freq, rot, 0, 1.0, 0, out, out_row, out_head, None)


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), OK), (dict(rows=-1), E_SHAPE), (dict(rows=(1 << 23) + 1), E_SHAPE), (dict(heads=0), E_SHAPE), (dict(heads=65536), E_SHAPE), (dict(dim=0), E_SHAPE),
    (dict(dim=257), E_SHAPE), (dict(rot=0), E_SHAPE), (dict(rot=98), E_SHAPE), (dict(rot=95), E_SHAPE), (dict(type=3), E_UNSUP), (dict(x=None), E_NULL),
    (dict(out=None), E_NULL), (dict(positions=None), E_NULL), (dict(freq=None), E_NULL), (dict(x_row=95), E_LD), (dict(x_head=95), E_LD), (dict(out_row=95), E_LD),
    (dict(out_head=95), E_LD), (dict(out=P, out_row=200), E_LD), (dict(out=P, out_head=100), E_LD), (dict(x=P + 1), E_ALIGN), (dict(type=0, out=P + 2), E_ALIGN),
    (dict(positions=P + 2), E_ALIGN), (dict(freq=P + 4), E_ALIGN)])
def test_rotary_refusals(change, status):
    assert turn(**change) == status


def cache(**change):
    c = dict(pages=P, scales=P, table=P, table_ld=8, lengths=P, starts=None, sequences=4, table_width=8, num_pages=40, heads=2, dim=96)
    c.update(change)
    return B.Kv4Cache(**c)


def calls(c, rows=8, max_new=0, type=2, p=P, row=192, head=96, q_heads=4, out=P, lse=None, window=0, ws=P, ws_bytes=1 << 30):
    c = ctypes.byref(c) if c is not None else None
    L = B.lib()
    return {"write": L.bmx_kv4_write(c, p, out, type, row, head, row, head, rows, max_new, None),
            "read": L.bmx_kv4_read(c, p, out, type, row, head, row, head, rows, max_new, None),
            "attention": L.bmx_kv4_attention(c, p, type, row * 2, head, q_heads, rows, max_new, 1.0, 1, window, out, row * 2, head, lse, ws, ws_bytes, None)}


@pytest.mark.parametrize("change,status", [
    (dict(sequences=-1), E_SHAPE), (dict(sequences=65536), E_SHAPE), (dict(table_width=-1), E_SHAPE), (dict(num_pages=-1), E_SHAPE),
    (dict(heads=0), E_SHAPE), (dict(heads=32768), E_SHAPE), (dict(dim=0), E_SHAPE), (dict(dim=257), E_SHAPE), (dict(sequences=0), E_SHAPE),
    (dict(sequences=3), E_SHAPE), (dict(pages=None), E_NULL), (dict(scales=None), E_NULL), (dict(table=None), E_NULL), (dict(lengths=None), E_NULL),
    (dict(table_ld=7), E_LD), (dict(pages=P + 8), E_ALIGN), (dict(scales=P + 8), E_ALIGN), (dict(table=P + 2), E_ALIGN), (dict(lengths=P + 1), E_ALIGN),
    (dict(starts=P + 2), E_ALIGN)])
def test_cache_refusals(change, status):
    assert set(calls(cache(**change)).values()) == {status}


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), OK), (dict(rows=-1), E_SHAPE), (dict(rows=1 << 31), E_SHAPE), (dict(rows=7), E_SHAPE), (dict(max_new=-1), E_SHAPE),
    (dict(type=3), E_UNSUP), (dict(p=None), E_NULL), (dict(out=None), E_NULL), (dict(row=95), E_LD), (dict(head=95), E_LD),
    (dict(p=P + 1), E_ALIGN), (dict(type=0, out=P + 2), E_ALIGN)])
def test_row_refusals(change, status):
    got = calls(cache(), **change)
    if "row" in change:
        got.pop("attention")  # (rows twice as far apart there)
    assert set(got.values()) == {status}
    assert set(calls(None).values()) == {E_NULL}


@pytest.mark.parametrize("change,status", [
    (dict(q_heads=3), E_SHAPE), (dict(q_heads=0), E_SHAPE), (dict(q_heads=65536), E_SHAPE), (dict(window=-1), E_SHAPE), (dict(lse=P + 2), E_ALIGN)])
def test_attention_refusals(change, status):
    assert calls(cache(), **change)["attention"] == status


def test_binding_refusals():
    """What the native module refuses before it calls the library."""
    x, n = torch.zeros((2, 3, 64)), torch.zeros((2,), dtype=torch.int32)
    for f, args in ((B.rotary, (x, n, n)), (B.kv4_write, (x, x, x, x, x, x)), (B.kv4_attention, (x, x, x, x, x)), (B.kv_resize, (n, n, n, n, 3))):
        with pytest.raises(ValueError, match="must live on the GPU"):
            f(*args)
    with pytest.raises(ValueError, match="no such frequencies"):
        B.rotary_frequencies(7)
    with pytest.raises(ValueError, match="no such frequencies"):
        B.rotary_frequencies(8, trained=100, slow=4, fast=1)
    assert B.page_pool(3, device="cpu").tolist() == [3, 0, 2, 1, 0]
    pages, scales = B.kv4_cache(3, 2, 80, device="cpu")
    assert pages.shape == (3, 2, 2, 64 * 48) and scales.shape == (3, 2, 2, 64, 2)


def test_attention_workspace():
    dims = (4, 80, 2, 4, 96, 2)
    need = B.workspace_bytes(B.OP_KV4_ATTENTION, dims)
    assert need > 4 * 16384 and need % 256 == 0
    c = cache(table_width=80, table_ld=80)
    one = B.workspace_bytes(B.OP_KV4_ATTENTION, dims + (8,))
    assert 0 < one <= need
    for ws, size, status in ((None, one, E_WS), (P, one - 1, E_WS), (P + 8, one, E_ALIGN)):
        assert calls(c, ws=ws, ws_bytes=size)["attention"] == status
    for bad in ((4, 80, 2, 3, 96, 2), (-1, 80, 2, 4, 96, 2), (4, 80, 0, 4, 96, 2), (4, 80, 2, 4, 257, 2), (4, 80, 2, 4, 96)):
        assert B.workspace_bytes(B.OP_KV4_ATTENTION, bad) == 0


@pytest.mark.parametrize("sizes", [(1, 16, 8, 32, 128), (8, 16, 8, 32, 128), (4, 80, 2, 4, 96), (1, 400, 1, 1, 64), (3, 33, 16, 256, 200), (64, 80, 8, 32, 128),
                                   (2, 64, 8, 32, 128), (1, 2000, 8, 64, 256), (7, 5, 3, 9, 40), (1, 4, 1, 8, 32), (255, 100, 1, 4, 64)])
def test_bound_covers_every_call(sizes):
    """The workspace for a bound of new rows is enough for every call below it."""
    share = sizes[3] // sizes[2]
    most = last = 0
    for n in sorted({*range(1, 70), *(n // share + k for n in range(64, 70000, 128) for k in (0, 1))} - {0}):
        most = max(most, B.workspace_bytes(B.OP_KV4_ATTENTION, sizes + (n, n * sizes[0])))
        bound = B.workspace_bytes(B.OP_KV4_ATTENTION, sizes + (n,))
        assert bound >= most and bound >= last, n
        last = bound
    unknown = B.workspace_bytes(B.OP_KV4_ATTENTION, sizes + (0,))
    assert unknown == B.workspace_bytes(B.OP_KV4_ATTENTION, sizes + (1 << 30,)) >= last


def test_changes_walked_on_the_host(tmp_path):
    """What a sequence's change of tokens comes to (csrc/kv_range.h), up to the ends of 32 bits, with traps for overflow."""
    src, so = tmp_path / "change.cpp", tmp_path / "change.so"
    src.write_text("""#define __host__
#define __device__
#include "kv_range.h"
extern "C" int change_of(int tokens, int change, int width, int* out) {
  const bmx::KvChange c = bmx::kv_change_of(tokens, change, width);
  out[0] = c.pages, out[1] = c.pages_then, out[2] = c.tokens_then, out[3] = c.more;
  return c.fits;
}
""")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-ftrapv", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)])
    f, out = ctypes.CDLL(str(so)).change_of, (ctypes.c_int * 4)()
    numbers = [-TOP - 1, -TOP, -65, -64, -1, 0, 1, 63, 64, 65, 128, 1000, TOP - 64, TOP - 63, TOP - 1, TOP]
    for tokens in numbers:
        for change in numbers:
            for width in (0, 1, 2, 16, 1 << 25, TOP):
                fits = f(tokens, change, width, out)
                then = tokens + change
                assert bool(fits) == (0 <= tokens <= 64 * width and 0 <= then <= min(64 * width, TOP))
                assert list(out) == ([-(-tokens // 64), -(-then // 64), then, max(change, 0)] if fits else [0] * 4)
