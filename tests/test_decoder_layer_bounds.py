"""Steps of the decoder layer that its calls would refuse, or answer with tokens left out, are refused before anything changes."""
import pytest
import torch

from paper_1705_09864_amd import binding as B
from paper_1705_09864_amd.decoder_layer import DevicePages, FewBitAttention, Pages


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


class Changed(Exception):
    pass


@pytest.mark.parametrize("rows,sequences,most,heads,freq", [(131071, 2, 0, 8, None), (131071, 2, 131071, 8, None), (1048561, 1, 0, 1, None), (2**20, 1024, 0, 1, None),
                                                            (5, 2, -1, 8, None), ((1 << 23) + 1, 65535, 1, 1, 1)])
@pytest.mark.parametrize("bits", [8, 4])
def test_what_later_calls_refuse(monkeypatch, bits, rows, sequences, most, heads, freq):
    """Refused on the host, while the pages are as they were."""
    def change(*args, **named):
        raise Changed
    monkeypatch.setattr(B, "w4_fc", lambda x, n: torch.zeros(()).expand(x.shape[0], n))
    monkeypatch.setattr(B, "kv_resize", change)
    layer = FewBitAttention.__new__(FewBitAttention)
    layer.__dict__.update(heads=heads, kv_heads=1, dim=8, hidden=1, n_qkv=(heads + 2) * 8, n_out=1, bits=bits, qkv=(), out=(), interleaved=False, scratch=None, kept=[],
                          freq=freq, pages=torch.zeros((4, 1), dtype=torch.uint8), scales=None)
    x = torch.zeros(()).expand(rows, 1)
    where = DevicePages(4, sequences, 3, device="cpu")
    with pytest.raises(ValueError, match="than a step takes|below 0"):
        layer.step(x, where, torch.zeros((sequences,), dtype=torch.int32), most=most)
    if most == 131071:
        where = Pages(3000, 2, 2500, device="cpu")
        layer.pages = torch.zeros((3000, 1), dtype=torch.uint8)
        with pytest.raises(ValueError, match="than a step takes"):
            layer.step(x, where, [rows, 0])
        assert where.tokens == [0, 0] and len(where.free) == 3000


@pytest.mark.parametrize("heads,kv_heads,dim,freq", [(3, 2, 8, None), (2, 0, 8, None), (1, 1, 257, None), (1, 2, 8, None), (65535, 1, 1, None),
                                                     (2, 1, 8, torch.zeros(4)), (2, 1, 8, torch.zeros((2, 2)).double()), (2, 1, 8, torch.zeros(0).double()),
                                                     (2, 1, 8, torch.zeros(8).double()[::2]), (2, 1, 8, torch.zeros(4, dtype=torch.float64, device="meta"))])
def test_layers_whose_steps_would_be_refused(heads, kv_heads, dim, freq):
    """What each step would refuse behind its first calls is refused when the layer is made."""
    with pytest.raises(ValueError, match="a step would refuse|freq: expected"):
        FewBitAttention(torch.zeros(((heads + 2 * kv_heads) * dim, 4)), torch.zeros((4, heads * dim)), heads, kv_heads, dim, 3, freq=freq)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_more_pages_than_the_cache_has(bits):
    """Tokens on pages behind the cache's end would be left out of every answer."""
    layer, g = make(bits, num_pages=2)
    x = torch.randn((130, 200), device="cuda", generator=g).bfloat16()
    host, device = Pages(3, 1, 4), DevicePages(3, 1, 4)
    for where, new in ((host, [130]), (device, gpu([130]))):
        with pytest.raises(ValueError, match="3 pages, the cache 2"):
            layer.step(x, where, new)
    assert host.tokens == [0] and device.lengths.tolist() == [0]
    assert bool(layer.step(x[:128], DevicePages(2, 1, 4), gpu([128])).any(1).all())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("heads,kv_heads,width", [(8, 2, 512), (32, 8, 2048), (1, 1, 10)])
def test_scratch_memory_of_growing_prompts(bits, heads, kv_heads, width):
    """Prompts a token longer each: every step has what it needs, and what is held in all is less than two of what any number of rows needs."""
    layer = FewBitAttention.__new__(FewBitAttention)
    layer.__dict__.update(heads=heads, kv_heads=kv_heads, dim=128, bits=bits, scratch=None, kept=[], pages=torch.zeros(0))
    op = B.OP_KV4_ATTENTION if bits == 4 else B.OP_KV_ATTENTION
    bound = B.workspace_bytes(op, (1, width, kv_heads, heads, 128, 0))
    for most in [*range(1, 2049), 0]:
        assert layer.workspace(1, width, most).numel() >= B.workspace_bytes(op, (1, width, kv_heads, heads, 128, most))
        assert sum(t.numel() for t in layer.kept) <= 2 * max(bound, 16)
    first = layer.workspace(1, width, 1)
    assert first is layer.workspace(1, width, 700) is layer.scratch and first is layer.kept[-1] and not bool(first.any())


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_captured_before_it_ran(bits):
    """New scratch memory in a capture would be zeros in the graph's replays alone; the capture is refused, and the layer goes on as before."""
    layer, g = make(bits)
    where, x, new = DevicePages(40, 2, 20), torch.randn((2, 200), device="cuda", generator=g).bfloat16(), gpu([1, 1])
    torch.cuda.synchronize()
    for _ in range(2):
        with pytest.raises(ValueError, match="has to run before"):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                layer.step(x, where, new, most=1)
    assert layer.scratch is None and where.lengths.tolist() == [0, 0]
    y = layer.step(x, where, new, most=1)
    where.resize(-new, 0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = layer.step(x, where, new, most=1)
    for _ in range(3):
        graph.replay()
        where.resize(-new, 0)
        assert torch.equal(y, z) and where.lengths.tolist() == [0, 0]
