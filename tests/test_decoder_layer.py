"""The decoder layer in few bits as a program runs it: prompts of uneven lengths, then tokens, against the definition in 64 bits on the
weights and the cache that the layer itself holds."""
import pytest
import torch

from paper_1705_09864_amd import binding as B
from paper_1705_09864_amd.decoder_layer import FewBitAttention, Pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,dim,hidden,group,block", [(4, 2, 64, 256, 64, 16), (6, 1, 80, 200, 32, 32), (2, 2, 128, 384, 128, 64)])
def test_layer_against_its_own_cache(heads, kv_heads, dim, hidden, group, block):
    """bf16 is rounded to three times (q, the attention's result, the layer's), 2^-8 each at most, in the 2-norm of a row's results:
    2^-8 for the result itself, and as much again for each of the others through a product with as many terms as results."""
    g = torch.Generator(device="cuda").manual_seed(dim)
    w_qkv = torch.randn(((heads + 2 * kv_heads) * dim, hidden), device="cuda", generator=g) * hidden**-0.5
    w_out = torch.randn((hidden, heads * dim), device="cuda", generator=g) * (heads * dim)**-0.5
    layer = FewBitAttention(w_qkv, w_out, heads, kv_heads, dim, 40, group, block)
    dq = B.w4_dequantize(*layer.qkv, w_qkv.shape[0], hidden).double()
    do = B.w4_dequantize(*layer.out, hidden, heads * dim).double()
    where = Pages(40, 3, 10)
    for new in ([70, 1, 200], [1, 1, 1], [5, 0, 2], [1, 1, 1], [90, 64, 1]):
        x = torch.randn((sum(new), hidden), device="cuda", generator=g).bfloat16()
        y = layer.step(x, where, new).double()
        total = where.tokens
        starts = torch.tensor([0] + [sum(total[:i + 1]) for i in range(3)], dtype=torch.int32, device="cuda")
        k, v = B.kv_read(layer.pages, layer.scales, where.table, where.lengths, dim, torch.float32, sum(total), starts=starts)
        q = (x.double() @ dq[:heads * dim].t().contiguous()).view(-1, heads, dim)
        at = row = 0
        for n, m in zip(total, new):
            kk, vv = (t[at:at + n].double().repeat_interleave(heads // kv_heads, 1).transpose(0, 1).contiguous() for t in (k, v))
            z = q[row:row + m].transpose(0, 1) @ kk.transpose(1, 2).contiguous() * dim**-0.5
            hide = torch.arange(n, device="cuda")[None, :] > torch.arange(n - m, n, device="cuda")[:, None]
            o = torch.softmax(z.masked_fill(hide, float("-inf")), -1) @ vv
            want = o.transpose(0, 1).reshape(m, heads * dim) @ do.t().contiguous()
            err = (y[row:row + m] - want).norm(dim=1) if m else torch.zeros(0)
            assert bool((err <= 3 * 2.0**-8 * want.norm(dim=1)).all() if m else True), float((err / want.norm(dim=1)).max())
            at, row = at + n, row + m


def test_pages_and_shapes_are_checked():
    where = Pages(4, 2, 3)
    where.extend([64, 100])
    with pytest.raises(ValueError, match="no room"):
        where.extend([70, 64])
    with pytest.raises(ValueError, match="do not fit"):
        FewBitAttention(torch.zeros((10, 64), device="cuda"), torch.zeros((64, 64), device="cuda"), 1, 1, 64, 4)
