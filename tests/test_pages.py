"""The decoder layer's bookkeeping, on the CPU."""
import pytest
import torch

from paper_1705_09864_amd.decoder_layer import Pages


def state(p):
    return list(p.free), list(p.count), list(p.tokens), p.table.tolist(), p.lengths.tolist()


def test_extend():
    p = Pages(6, 3, 4, device="cpu")
    assert p.extend([64, 1, 100]).tolist() == [0, 64, 65, 165]
    assert p.extend([1, 1, 1]) is None
    assert p.tokens == [65, 2, 101] == p.lengths.tolist() and p.count == [2, 1, 2] and len(p.free) == 1
    pages = [p.table[i, j].item() for i in range(3) for j in range(p.count[i])]
    assert len(set(pages)) == 5 and not set(pages) & set(p.free)


@pytest.mark.parametrize("new", [[10, 400, 0], [1, 0, 30], [200, 0, 0], [0, 0, 300], [1, 1], [1, 1, 1, 1], [1, -1, 1], [64, 64, 64]])
def test_a_refused_extend_changes_nothing(new):
    """No room in a sequence's row of the table, none in the pool, for the first sequence or one behind those that have room."""
    p = Pages(6, 3, 4, device="cpu")
    p.extend([64, 100, 110])
    before = state(p)
    with pytest.raises(ValueError, match="no room" if len(new) == 3 and min(new) >= 0 else "expected"):
        p.extend(new)
    assert state(p) == before
    p.extend([1, 0, 0])
    assert p.lengths.tolist() == [65, 100, 110] and len(p.free) == 0
