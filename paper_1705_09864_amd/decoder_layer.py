"""Attention of a decoder layer in few bits: 4-bit projections around a paged cache of 8 bits.

    python -m paper_1705_09864_amd.decoder_layer

runs prompts of uneven lengths and then a token at a time, and prints how far the layer is from the same layer in float32 with
its own weights, and what a step takes.  It rotates nothing by position and gives no pages back, and a step copies the lengths from the host.
"""
import torch

from . import binding as B


class Pages:
    """Which pages of a cache are whose: a table of page numbers, a row for each sequence, and each one's tokens."""

    def __init__(self, num_pages, sequences, pages_each, device="cuda"):
        self.free = list(range(num_pages - 1, -1, -1))
        self.count = [0] * sequences
        self.tokens = [0] * sequences
        self.table = torch.zeros((sequences, pages_each), dtype=torch.int32, device=device)
        self.lengths = torch.zeros((sequences,), dtype=torch.int32, device=device)

    def extend(self, new):
        """Room for new[i] more tokens of sequence i; returns the rows' starts, None where each has as many.  Where there is no room for all of
        them, nothing changes."""
        if len(new) != len(self.tokens) or min(new, default=0) < 0:
            raise ValueError("expected how many tokens are new for each of %d sequences, got %r" % (len(self.tokens), new))
        needs, left = [-(-(t + n) // B.PAGE) for t, n in zip(self.tokens, new)], len(self.free)
        for i, need in enumerate(needs):
            left -= max(0, need - self.count[i])
            if need > self.table.shape[1] or left < 0:
                raise ValueError("sequence %d: no room for %d more tokens" % (i, new[i]))
        for i, (n, need) in enumerate(zip(new, needs)):
            if need > self.count[i]:
                pages = [self.free.pop() for _ in range(need - self.count[i])]
                self.table[i, self.count[i]:need] = torch.tensor(pages, dtype=torch.int32)
                self.count[i] = need
            self.tokens[i] += n
        self.lengths.copy_(torch.tensor(self.tokens, dtype=torch.int32))
        if len(set(new)) == 1:
            return None
        at = [0]
        for n in new:
            at.append(at[-1] + n)
        return torch.tensor(at, dtype=torch.int32, device=self.table.device)


class FewBitAttention:
    """x -> W_out attention(W_qkv x), causal, with the keys and values of earlier tokens in the cache.

    w_qkv [(heads + 2 * kv_heads) * dim, hidden] and w_out [hidden, heads * dim] in float32 are kept in 4 bits, a scale and an
    offset for each `group` values of a row; the cache in 8 bits, a scale for each `block` tokens and head."""

    def __init__(self, w_qkv, w_out, heads, kv_heads, dim, num_pages, group=128, block=16):
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.n_qkv, self.n_out, self.hidden = w_qkv.shape[0], w_out.shape[0], w_qkv.shape[1]
        if self.n_qkv != (heads + 2 * kv_heads) * dim or w_out.shape[1] != heads * dim:
            raise ValueError("w_qkv and w_out do not fit the heads")
        self.qkv, self.out = B.w4_quantize(w_qkv, group), B.w4_quantize(w_out, group)
        self.pages, self.scales = B.kv_cache(num_pages, kv_heads, dim, block, device=w_qkv.device)
        self.scratch = None

    def workspace(self, sequences, width, most):
        """The attention's scratch memory: zeros before its first use, kept from step to step."""
        need = B.workspace_bytes(B.OP_KV_ATTENTION, (sequences, width, self.kv_heads, self.heads, self.dim, most))
        if self.scratch is None or self.scratch.numel() < need:
            self.scratch = torch.zeros((max(need, 16),), dtype=torch.uint8, device=self.pages.device)
        return self.scratch

    def step(self, x, where, new):
        """x [sum(new), hidden], new[i] more tokens of sequence i; `where`: the sequences' Pages, unchanged where the step is refused."""
        if x.dim() != 2 or tuple(x.shape) != (sum(new), self.hidden):
            raise ValueError("x: expected the shape [%d, %d], got %r" % (sum(new), self.hidden, list(x.shape)))
        q, k, v = (B.w4_fc(x, *self.qkv, self.n_qkv).view(x.shape[0], -1, self.dim)
                   .split([self.heads, self.kv_heads, self.kv_heads], 1))
        starts = where.extend(new)
        cache = (self.pages, self.scales, where.table, where.lengths)
        B.kv_write(k, v, *cache, starts=starts, max_new=max(new))
        o = B.kv_attention(q, *cache, starts=starts, max_new=max(new),
                           workspace=self.workspace(len(new), where.table.shape[1], max(new)))
        return B.w4_fc(o.view(x.shape[0], -1), *self.out, self.n_out)


def plain(x, w_qkv, w_out, heads, kv_heads, dim):
    """One sequence x [tokens, hidden] through the same layer, all of it in float32."""
    q, k, v = (x.float() @ w_qkv.t()).view(x.shape[0], -1, dim).split([heads, kv_heads, kv_heads], 1)
    k, v = (t.repeat_interleave(heads // kv_heads, 1).transpose(0, 1) for t in (k, v))
    scores = (q.transpose(0, 1) @ k.transpose(1, 2).contiguous()) * dim**-0.5
    scores.masked_fill_(torch.ones_like(scores[0], dtype=torch.bool).triu(1), float("-inf"))
    return (torch.softmax(scores, -1) @ v).transpose(0, 1).reshape(x.shape[0], -1) @ w_out.t()


def main():
    heads, kv_heads, dim, hidden, prompts, tokens = 32, 8, 128, 4096, [700, 33, 1500, 256], 8
    g = torch.Generator(device="cuda").manual_seed(1)
    w_qkv = torch.randn(((heads + 2 * kv_heads) * dim, hidden), device="cuda", generator=g) * hidden**-0.5
    w_out = torch.randn((hidden, heads * dim), device="cuda", generator=g) * hidden**-0.5
    layer = FewBitAttention(w_qkv, w_out, heads, kv_heads, dim, num_pages=256)
    where = Pages(256, len(prompts), 64)
    xs = [torch.randn((n + tokens, hidden), device="cuda", generator=g).bfloat16() for n in prompts]
    got = [[part] for part in layer.step(torch.cat([x[:n] for x, n in zip(xs, prompts)]), where, prompts).split(prompts)]
    for t in range(tokens):
        y = layer.step(torch.stack([x[n + t] for x, n in zip(xs, prompts)]), where, [1] * len(prompts))
        for part, row in zip(got, y):
            part.append(row[None])
    for n, x, part in zip(prompts, xs, got):
        want, y = plain(x, w_qkv, w_out, heads, kv_heads, dim), torch.cat(part).float()
        print("%5d tokens, then %d: relative difference from float32 %.3f" % (n, tokens, float((y - want).norm() / want.norm())))
    one = torch.randn((len(prompts), hidden), device="cuda", generator=g).bfloat16()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(20):
        layer.step(one, where, [1] * len(prompts))
    end.record()
    end.synchronize()
    print("a token for each of %d sequences: %.0f us a step, with the host's bookkeeping" % (len(prompts), 1000 * start.elapsed_time(end) / 20))


if __name__ == "__main__":
    main()
