"""How much scratch memory an attention call over the cache asks for: what is said for a bound of new rows is enough for every call below it."""
import ctypes

import pytest

from paper_1705_09864_amd import binding as B

P = 0x7F0000001000  # a fake, well aligned, never dereferenced device address
E_SHAPE, E_WS = -2, -6
SIZES = [(1, 16, 8, 32, 128), (8, 16, 8, 32, 128), (4, 80, 2, 4, 96), (1, 400, 1, 1, 64), (1, 40, 16, 128, 64), (3, 33, 16, 256, 200),
         (64, 80, 8, 32, 128), (2, 64, 8, 32, 128), (1, 2000, 8, 64, 256), (7, 5, 3, 9, 40), (1, 4, 1, 8, 32), (255, 100, 1, 4, 64), (128, 70, 1, 16, 160)]


@pytest.mark.parametrize("sizes", SIZES)
def test_bound_covers_every_call(sizes):
    share = sizes[3] // sizes[2]
    calls = sorted({*range(1, 70), *(n // share + k for n in range(64, 70000, 128) for k in (0, 1))} - {0})
    most, last = 0, 0
    for n in calls:
        one = B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (n, n * sizes[0]))
        most = max(most, one)
        bound = B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (n,))
        assert bound >= most and bound >= last, n
        # (no more than rounding up the splits costs; a workgroup's part is 128 rows at most)
        line = ((sizes[4] + 31) // 32 * 32 + 4) * 4
        assert bound <= most + 512 * 128 * line, n
        last = bound
    unknown = B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (0,))
    assert unknown == B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (1 << 30,)) >= last
    # (one row a sequence asks for what it needs)
    assert B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (1,)) <= B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (1, sizes[0])) + 256 * 16 * line


def attention(sizes, rows, max_new, ws_bytes, starts=P):
    sequences, width, heads, q_heads, dim = sizes
    c = B.KvCache(pages=P, scales=P, table=P, table_ld=width, lengths=P, starts=starts, sequences=sequences, table_width=width, num_pages=40,
                  heads=heads, dim=dim, block=16)
    # (on an address that is refused behind the size, so that nothing is launched)
    return B.lib().bmx_kv_attention(ctypes.byref(c), P, 2, q_heads * dim, dim, q_heads, rows, max_new, 1.0, 1, 0, P, q_heads * dim, dim, None, P + 8,
                                    ws_bytes, None)


@pytest.mark.parametrize("sizes", SIZES)
def test_calls_take_the_workspace_of_a_bound(sizes):
    """A workspace of the stated size is never too small: fewer rows than the bound, a bound that is not known."""
    for bound in (1, 7, 64, 500, 5000, 0):
        size = B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (bound,))
        for rows in sorted({1, 2, 8, sizes[0], 3 * sizes[0], 64, 500, bound * sizes[0]} - {0}):
            if (min(bound, rows) or rows) * (sizes[3] // sizes[2]) > 65535 * 16:
                continue
            if B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (bound, rows)) == 0:
                continue  # (nothing is needed, and the call would launch)
            assert attention(sizes, rows, bound, size) == -4, (bound, rows)
            need = B.workspace_bytes(B.OP_KV_ATTENTION, sizes + (bound, rows))
            assert attention(sizes, rows, bound, need - 1) == E_WS


def test_sizes_that_are_none():
    good = (4, 80, 2, 4, 96, 2, 8)
    assert B.workspace_bytes(B.OP_KV_ATTENTION, good) > 0
    for i, v in ((0, 65536), (2, 32768), (3, 3), (4, 257), (6, -1), (6, 1 << 31)):
        bad = list(good)
        bad[i] = v
        if i == 2:
            bad[3] = v
        assert B.workspace_bytes(B.OP_KV_ATTENTION, bad) == 0
    assert B.workspace_bytes(B.OP_KV_ATTENTION, good + (1,)) == 0
    assert attention((1, 4, 1, 8, 32), 131072, 0, 1 << 30) == E_SHAPE
