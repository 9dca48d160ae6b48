"""GPU tests of the decoder layer's calls at the ends of what they take."""
import numpy as np
import pytest
import torch

from paper_1705_09864_amd import binding as B

pytestmark = pytest.mark.gpu
TOP = 2**31 - 1


@pytest.mark.parametrize("rows", [2, 5, 70])
@pytest.mark.parametrize("below", [0, 1, 63, 64, 130])
def test_kv_lengths_at_the_end_of_32_bits(rows, below):
    """Tokens far behind the table: nothing is written for them, zeros come back, and the sequence beside them is as ever."""
    heads, dim = 2, 64
    pages, scales = B.kv_cache(5, heads, dim)
    pages.fill_(55)
    scales.fill_(0.001)
    table = torch.tensor([[1, 2], [0, 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([TOP - below, 100], dtype=torch.int32, device="cuda")
    kv = torch.randn((2 * rows, heads, dim), device="cuda")
    B.kv_write(kv, kv, pages, scales, table, lengths)
    assert bool((pages[[1, 2, 4]] == 55).all()) and bool((scales[[1, 2, 4]] == 0.001).all())
    k, v = B.kv_read(pages, scales, table, lengths, dim, torch.float32, 2 * rows)
    for x in (k, v):
        assert not bool(x[:rows].any()) and float((x[rows:] - kv[rows:]).abs().max()) < 0.03
    out = B.kv_attention(torch.randn((2 * rows, heads, dim), device="cuda"), pages, scales, table, lengths)
    assert bool(torch.isfinite(out).all())
