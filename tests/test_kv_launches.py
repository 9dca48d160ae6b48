"""Calls on either cache whose new rows lie in more pages than a launch has workgroups: 2^32 threads along its first dimension are 2^24 of 256.  Refused on the host."""
import ctypes

import pytest

from paper_1705_09864_amd import binding as B

P = 0x7F0000001000  # a fake, well aligned, never dereferenced device address
E_SHAPE = -2


@pytest.mark.parametrize("sequences,rows,max_new", [(65535, 1 << 27, 64 * 256), (1024, 1 << 20, 0), (1 << 13, 1 << 17, 0), (65535, 65535 * 16384, 16384),
                                                    (259, 1 << 22, 64 * 65026)])
@pytest.mark.parametrize("bits", [8, 4])
def test_more_pages_than_a_launch_has(bits, sequences, rows, max_new):
    c = (B.KvCache if bits == 8 else B.Kv4Cache)(pages=P, scales=P, table=P, table_ld=8, lengths=P, starts=P, sequences=sequences, table_width=8, num_pages=40, heads=2, dim=96)
    if bits == 8:
        c.block = 16
    most = min(max_new or rows, rows)
    assert 2**24 <= sequences * ((most + 62) // 64 + 1) < 2**31
    L = B.lib()
    for f in (L.bmx_kv_write, L.bmx_kv_read) if bits == 8 else (L.bmx_kv4_write, L.bmx_kv4_read):
        assert f(ctypes.byref(c), P, P, 2, 192, 96, 192, 96, rows, max_new, None) == E_SHAPE
