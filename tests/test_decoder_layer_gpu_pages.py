"""The decoder layer with positions, either cache, and its pages on the GPU: prompts, tokens, tokens taken back, sequences that end and others in their
place, against the definition in 64 bits on the weights and the cache that the layer itself holds; padded, refused, captured and replayed."""
import pytest
import torch

from paper_1705_09864_amd import binding as B
from paper_1705_09864_amd.decoder_layer import DevicePages, FewBitAttention, Pages, plain

pytestmark = pytest.mark.gpu


def make(heads, kv_heads, dim, hidden, bits, seed=0, **named):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w_qkv = torch.randn(((heads + 2 * kv_heads) * dim, hidden), device="cuda", generator=g) * hidden**-0.5
    w_out = torch.randn((hidden, heads * dim), device="cuda", generator=g) * (heads * dim)**-0.5
    return FewBitAttention(w_qkv, w_out, heads, kv_heads, dim, 40, 64, bits=bits, **named), g


def gpu(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rotated(t, positions, freq, interleaved):
    n = freq.numel()
    a = torch.arange(n, device="cuda") * (2 if interleaved else 1)
    b = a + (1 if interleaved else n)
    z = torch.complex(t[..., a], t[..., b]) * torch.polar(torch.ones_like(freq), freq)[None].pow(positions.double()[:, None])[:, None]
    t = t.clone()
    t[..., a], t[..., b] = z.real, z.imag
    return t


def check(layer, where, x, y, total, new):
    """As for the layer without positions: bf16 is rounded to four times (q, q rotated, the attention's result, the layer's), 2^-8 each at most."""
    heads, kv_heads, dim = layer.heads, layer.kv_heads, layer.dim
    dq = B.w4_dequantize(*layer.qkv, layer.n_qkv, layer.hidden).double()
    do = B.w4_dequantize(*layer.out, layer.n_out, heads * dim).double()
    starts = gpu([sum(total[:i]) for i in range(len(total) + 1)])
    read = B.kv4_read if layer.bits == 4 else B.kv_read
    k, v = read(layer.pages, layer.scales, where.table, where.lengths, dim, torch.float32, sum(total), starts=starts)
    at = row = 0
    for n, m in zip(total, new):
        if m > 0:
            q = (x[row:row + m].double() @ dq[:heads * dim].t().contiguous()).view(m, heads, dim)
            if layer.freq is not None:
                q = rotated(q, torch.arange(n - m, n, device="cuda"), layer.freq, layer.interleaved)
            kk, vv = (t[at:at + n].double().repeat_interleave(heads // kv_heads, 1).transpose(0, 1).contiguous() for t in (k, v))
            z = q.transpose(0, 1).contiguous() @ kk.transpose(1, 2).contiguous() * dim**-0.5
            hide = torch.arange(n, device="cuda")[None, :] > torch.arange(n - m, n, device="cuda")[:, None]
            o = torch.softmax(z.masked_fill(hide, float("-inf")), -1) @ vv
            want = o.transpose(0, 1).reshape(m, heads * dim) @ do.t().contiguous()
            err = (y[row:row + m].double() - want).norm(dim=1)
            assert bool((err <= 4 * 2.0**-8 * want.norm(dim=1)).all()), float((err / want.norm(dim=1)).max())
            row += m
        at += n


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("heads,kv_heads,dim,hidden,rot,interleaved", [(4, 2, 64, 256, 64, False), (6, 1, 80, 200, 32, True), (2, 2, 128, 384, 0, False)])
def test_steps_on_the_gpus_pages(bits, heads, kv_heads, dim, hidden, rot, interleaved):
    layer, g = make(heads, kv_heads, dim, hidden, bits, freq=B.rotary_frequencies(rot) if rot else None, interleaved=interleaved)
    where = DevicePages(40, 3, 10)
    total = [0, 0, 0]
    for change, pad in (([70, 1, 200], 0), ([1, 1, 1], 2), ([5, -1, 2], 0), ([1, 130, 1], 7), ([-60, 1, -203], 0), ([0, 0, 64], 1), ([90, 64, 1], 0)):
        new = [max(c, 0) for c in change]
        x = torch.randn((sum(new) + pad, hidden), device="cuda", generator=g).bfloat16()
        y = layer.step(x, where, gpu(change), most=max(new) if pad else 0)
        total = [t + c for t, c in zip(total, change)]
        assert where.refused() == 0 and where.lengths.tolist() == total
        assert not bool(y[sum(new):].any())
        check(layer, where, x, y, total, new)
    held = sum(-(-t // 64) for t in total)
    assert where.pool[0].item() == 40 - held
    where.resize(gpu([-t for t in total]), 0)
    assert where.pool[0].item() == 40 and sorted(where.pool[2:].tolist()) == list(range(40))


@pytest.mark.parametrize("bits", [8, 4])
def test_the_hosts_pages_and_the_gpus_give_the_same(bits):
    freq = B.rotary_frequencies(64)
    (a, g), (b, _) = make(4, 2, 64, 256, bits, freq=freq), make(4, 2, 64, 256, bits, freq=freq)
    host, device = Pages(40, 3, 10), DevicePages(40, 3, 10)
    for new in ([70, 1, 200], [1, 1, 1], [5, 0, 2], [1, 1, 1]):
        x = torch.randn((sum(new), 256), device="cuda", generator=g).bfloat16()
        assert torch.equal(a.step(x, host, new), b.step(x, device, gpu(new), most=max(new)))
    assert torch.equal(a.pages, b.pages) and torch.equal(a.scales, b.scales) and torch.equal(host.table, device.table)


@pytest.mark.parametrize("bits", [8, 4])
def test_refused_steps(bits):
    """No room: nothing changes, and every row comes back as zeros."""
    layer, g = make(2, 1, 64, 200, bits)
    where = DevicePages(40, 2, 3)
    layer.step(torch.randn((140, 200), device="cuda", generator=g).bfloat16(), where, gpu([70, 70]))
    before = layer.pages.clone(), layer.scales.clone(), where.lengths.clone(), where.table.clone(), where.pool.clone()
    for change, rows, who in (([130, 1], 131, 1), ([1, 130], 131, 2), ([1, 1], 1, 2), ([-71, 1], 1, 1)):
        y = layer.step(torch.randn((rows, 200), device="cuda", generator=g).bfloat16(), where, gpu(change))
        assert where.refused() == who and not bool(y.any())
        now = layer.pages, layer.scales, where.lengths, where.table, where.pool
        assert all(torch.equal(a, b) for a, b in zip(now[:4], before)) and torch.equal(now[4][2:], before[4][2:]) and now[4][0] == before[4][0]
    for bad in (torch.zeros((2, 201), device="cuda").bfloat16(), torch.zeros((200,), device="cuda").bfloat16()):
        with pytest.raises(ValueError):
            layer.step(bad, where, gpu([1, 1]))
    assert where.lengths.tolist() == [70, 70]
    y = layer.step(torch.randn((2, 200), device="cuda", generator=g).bfloat16(), where, gpu([1, 1]), most=1)
    assert where.refused() == 0 and bool(y.any()) and where.lengths.tolist() == [71, 71]


@pytest.mark.parametrize("bits", [8, 4])
def test_a_captured_step(bits):
    """A graph of a step over 200 of them, across pages, with eager work between the replays; other sequences end in between."""
    layer, g = make(4, 2, 64, 256, bits, freq=B.rotary_frequencies(64))
    where = DevicePages(40, 3, 10)
    x = torch.randn((91, 256), device="cuda", generator=g).bfloat16()
    layer.step(x, where, gpu([60, 1, 30]), most=60)
    one, change = torch.zeros((3, 256), device="cuda").bfloat16(), gpu([1, 1, 1])
    layer.step(one, where, change, most=1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(one, where, change, most=1)
    total = [61, 2, 31]
    for turn in range(12):
        c = [1, 1, 1] if turn != 5 else [1, -6, 1]
        change.copy_(gpu(c))
        one.normal_(generator=g)
        graph.replay()
        total = [t + k for t, k in zip(total, c)]
        assert where.lengths.tolist() == total
        if turn != 5:
            check(layer, where, one, y, total, c)
        else:
            check(layer, where, one, y, total, [1, 0, 1])
            assert not bool(y[2].any())


def test_against_the_layer_in_fp32():
    """The plain layer, which rotates too, is as near as 4 bits of weights and of cache allow: their steps are 2.5 / 7.5 and 2.2 / 7.5 of a normal value's size,
    an error of 0.1 and 0.09 of it, 0.1 for each of two products, and scores and values that carry theirs; 0.35 in all."""
    for interleaved in (False, True):
        g = torch.Generator(device="cuda").manual_seed(4)
        w_qkv = torch.randn((8 * 64, 256), device="cuda", generator=g) / 16
        w_out = torch.randn((256, 4 * 64), device="cuda", generator=g) / 16
        freq = B.rotary_frequencies(64)
        layer = FewBitAttention(w_qkv, w_out, 4, 2, 64, 8, 32, bits=4, freq=freq, interleaved=interleaved)
        x = torch.randn((100, 256), device="cuda", generator=g).bfloat16()
        y = layer.step(x, DevicePages(8, 1, 4), gpu([100])).float()
        want = plain(x, w_qkv, w_out, 4, 2, 64, freq, interleaved)
        assert float((y - want).norm() / want.norm()) < 0.35
        # positions matter: without them it is further off than any rounding
        assert float((y - plain(x, w_qkv, w_out, 4, 2, 64)).norm() / want.norm()) > 0.35


@pytest.mark.parametrize("bits", [8, 4])
def test_steps_without_rows(bits):
    """Sequences that only lose tokens, and none that gain any."""
    layer, g = make(2, 1, 64, 200, bits, freq=B.rotary_frequencies(64))
    where, host = DevicePages(40, 2, 3), Pages(40, 2, 3)
    layer.step(torch.randn((140, 200), device="cuda", generator=g).bfloat16(), where, gpu([70, 70]))
    none = torch.zeros((0, 200), device="cuda").bfloat16()
    assert layer.step(none, where, gpu([-70, -5])).shape == (0, 200)
    assert where.refused() == 0 and where.lengths.tolist() == [0, 65] and where.pool[0].item() == 38
    assert layer.step(none, host, [0, 0]).shape == (0, 200) and host.tokens == [0, 0]


def test_what_does_not_fit():
    with pytest.raises(ValueError, match="bits"):
        make(2, 1, 64, 200, 5)
    with pytest.raises(ValueError, match="pairs"):
        make(2, 1, 64, 200, 4, freq=B.rotary_frequencies(66))
