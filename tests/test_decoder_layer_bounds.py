"""Steps of the decoder layer that its calls would refuse, or answer with tokens left out, are refused before anything changes."""
import pytest
import torch

from paper_1705_09864_amd import binding as B
from paper_1705_09864_amd.decoder_layer import DevicePages, FewBitAttention


def make(bits, num_pages=40, **named):
    g = torch.Generator(device="cuda").manual_seed(0)
    w_qkv = torch.randn((4 * 64, 200), device="cuda", generator=g) / 14
    w_out = torch.randn((200, 2 * 64), device="cuda", generator=g) / 11
    return FewBitAttention(w_qkv, w_out, 2, 1, 64, num_pages, 64, bits=bits, **named), g


def gpu(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_more_new_tokens_than_said(bits):
    """A sequence with more new rows than `most`: the calls behind would take its first rows for its last tokens, and leave those between unwritten."""
    layer, g = make(bits)
    where = DevicePages(40, 3, 3)
    layer.step(torch.randn((76, 200), device="cuda", generator=g).bfloat16(), where, gpu([70, 1, 5]), most=70)
    x = torch.randn((5, 200), device="cuda", generator=g).bfloat16()
    before = layer.pages.clone(), layer.scales.clone(), where.lengths.clone(), where.table.clone(), where.pool[2:].clone(), where.pool[:1].clone()
    for change, most, who in (([3, 0, 0], 1, 1), ([1, -1, 2], 1, 3), ([0, 5, 0], 4, 2)):
        y = layer.step(x, where, gpu(change), most=most)
        assert where.refused() == who and not bool(y.any())
        now = layer.pages, layer.scales, where.lengths, where.table, where.pool[2:], where.pool[:1]
        assert all(torch.equal(a, b) for a, b in zip(now, before))
    y = layer.step(x, where, gpu([3, -1, 2]), most=3)
    assert where.refused() == 0 and bool(y.any(1).all()) and where.lengths.tolist() == [73, 0, 7]
