"""Refusals of the decoder layer's calls (4-bit weights, cache of 8 bits, attention): every one on the host, before any launch."""
import ctypes

import pytest
import torch

from paper_1705_09864_amd import binding as B

P = 0x7F0000001000  # a fake, well aligned, never dereferenced device address
OK, E_NULL, E_SHAPE, E_LD, E_ALIGN, E_UNSUP, E_WS = 0, -1, -2, -3, -4, -5, -6


def fc(x=P, type=0, ldx=256, tiles=P, scales=P, group=64, bias=None, M=3, N=40, K=200, out=P, ldo=40):
    return B.lib().bmx_w4_fc(x, type, ldx, tiles, scales, group, bias, M, N, K, out, ldo, None)


@pytest.mark.parametrize("change,status", [
    (dict(M=0), OK), (dict(N=0), OK), (dict(M=0, x=None), OK), (dict(M=-1), E_SHAPE), (dict(N=-1), E_SHAPE), (dict(K=0), E_SHAPE),
    (dict(K=1 << 24), E_SHAPE), (dict(M=1 << 22), E_SHAPE), (dict(N=1 << 22), E_SHAPE), (dict(type=3), E_UNSUP), (dict(type=-1), E_UNSUP),
    (dict(group=16), E_UNSUP), (dict(group=256), E_UNSUP), (dict(x=None), E_NULL), (dict(tiles=None), E_NULL), (dict(scales=None), E_NULL),
    (dict(out=None), E_NULL), (dict(ldx=199), E_LD), (dict(ldo=39), E_LD), (dict(x=P + 2), E_ALIGN), (dict(type=2, x=P + 1), E_ALIGN),
    (dict(tiles=P + 8), E_ALIGN), (dict(scales=P + 4), E_ALIGN), (dict(out=P + 1), E_ALIGN), (dict(bias=P + 2), E_ALIGN)])
def test_w4_fc_refusals(change, status):
    assert fc(**change) == status


def test_w4_quantize_refusals():
    L = B.lib()
    for f, good in ((L.bmx_w4_quantize, (P, 200, 40, 200, 64, P, P, None)), (L.bmx_w4_dequantize, (P, P, 40, 200, 64, P, 200, None))):
        at = {"N": 2, "K": 3, "group": 4, "ldw": 1 if f is L.bmx_w4_quantize else 6}
        for name, value, status in (("N", 0, OK), ("N", -1, E_SHAPE), ("K", 0, E_SHAPE), ("K", 1 << 24, E_SHAPE), ("group", 48, E_UNSUP),
                                    ("ldw", 199, E_LD)):
            a = list(good)
            a[at[name]] = value
            assert f(*a) == status, (name, value)
        for i, v in enumerate(good[:-1]):
            if v == P:
                assert f(*(good[:i] + (None,) + good[i + 1:])) == E_NULL
                assert f(*(good[:i] + (P + 2,) + good[i + 1:])) == E_ALIGN


def cache(**change):
    c = dict(pages=P, scales=P, table=P, table_ld=8, lengths=P, starts=None, sequences=4, table_width=8, num_pages=40, heads=2, dim=96,
             block=32)
    c.update(change)
    return B.KvCache(**c)


CACHE_FAULTS = [
    (dict(sequences=-1), E_SHAPE), (dict(sequences=65536), E_SHAPE), (dict(table_width=-1), E_SHAPE), (dict(num_pages=-1), E_SHAPE),
    (dict(heads=0), E_SHAPE), (dict(heads=32768), E_SHAPE), (dict(dim=0), E_SHAPE), (dict(dim=257), E_SHAPE), (dict(sequences=0), E_SHAPE),
    (dict(sequences=3), E_SHAPE), (dict(block=8), E_UNSUP), (dict(block=128), E_UNSUP), (dict(pages=None), E_NULL),
    (dict(scales=None), E_NULL), (dict(table=None), E_NULL), (dict(lengths=None), E_NULL), (dict(table_ld=7), E_LD),
    (dict(pages=P + 8), E_ALIGN), (dict(scales=P + 2), E_ALIGN), (dict(table=P + 2), E_ALIGN), (dict(lengths=P + 1), E_ALIGN),
    (dict(starts=P + 2), E_ALIGN)]


def calls(c, rows=8, max_new=0, type=2, p=P, row=192, head=96, q_heads=4, out=P, lse=None, window=0, ws=P, ws_bytes=1 << 30):
    c = ctypes.byref(c) if c is not None else None
    L = B.lib()
    return {"write": L.bmx_kv_write(c, p, out, type, row, head, row, head, rows, max_new, None),
            "read": L.bmx_kv_read(c, p, out, type, row, head, row, head, rows, max_new, None),
            "attention": L.bmx_kv_attention(c, p, type, row * 2, head, q_heads, rows, max_new, 1.0, 1, window, out, row * 2, head, lse,
                                            ws, ws_bytes, None)}


@pytest.mark.parametrize("change,status", CACHE_FAULTS)
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
    """What the native module refuses before it calls the library: kinds of tensors that the C functions would misread."""
    x = torch.zeros((2, 64))
    with pytest.raises(ValueError, match="must live on the GPU"):
        B.w4_fc(x, x, x, 3)
    with pytest.raises(ValueError, match="expected a torch tensor"):
        B.w4_fc([1.0], x, x, 3)
    with pytest.raises(ValueError, match="dtype"):
        B.w4_fc(x.double(), x, x, 3)
    with pytest.raises(ValueError, match="must live on the GPU"):
        B.kv_write(x, x, x, x, x, x)
    with pytest.raises(ValueError, match="block must be"):
        B.kv_cache(1, 1, 64, block=48, device="cpu")
    pages, scales = B.kv_cache(3, 2, 80, 32, device="cpu")
    assert pages.shape == (3, 2, 2, 64 * 96) and scales.shape == (3, 2, 2, 2)


def test_attention_workspace():
    """What one token over a long sequence needs, and what is refused: none, too little, one on an odd address; sizes that are none."""
    dims = (4, 80, 2, 4, 96, 2)
    need = B.workspace_bytes(B.OP_KV_ATTENTION, dims)
    assert need > 4 * 16384 and need % 256 == 0
    c = cache(table_width=80, table_ld=80)
    for ws, size, status in ((None, need, E_WS), (P, need - 1, E_WS), (P + 8, need, E_ALIGN)):
        assert calls(c, ws=ws, ws_bytes=size)["attention"] == status
    # rows enough to fill the chip are not split, and need none
    assert B.workspace_bytes(B.OP_KV_ATTENTION, (64, 80, 8, 32, 128, 1)) == 0
    for bad in ((4, 80, 2, 3, 96, 2), (-1, 80, 2, 4, 96, 2), (4, 80, 0, 4, 96, 2), (4, 80, 2, 4, 257, 2), (4, 80, 2, 4, 96)):
        assert B.workspace_bytes(B.OP_KV_ATTENTION, bad) == 0
