"""GPU tests of the decoder layer in few bits against plain implementations in 64 bits (numpy), and of the cache bit for bit.

Tolerances, from the formulas.  u(type) is half a unit in the last place: 2^-24, 2^-11, 2^-8 for float32, float16, bfloat16.
  w4_fc      products are exact and their sums fp32: u(type) |y| + n 2^-24 S, S the sum of the terms' sizes as the kernel adds them,
             |x| (s (16 + 15) + |b - 16 s|), n the longest chain of additions, K / 32 + 64.
  attention  a score's error e is at most (2^-21 + dim 2^-24) scale sum |q k|, a weight's 2 e + w with w = 2^-11 for 16-bit types (weights go to
             the products in f16) and 2^-20 for float32; with T = sum p |v| / sum p: u(type) |o| + (2 e + w + n 2^-24) T.  A weight in f16
             is p c / C 2^14 (c its block's scale, C the largest) to 2^-25 at best: for 16-bit types 2^-39 max |v| more for each token.
             And a float16 result is a multiple of 2^-24.
"""
import numpy as np
import pytest
import torch

from paper_1705_09864_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"f32": (torch.float32, 2.0**-24), "f16": (torch.float16, 2.0**-11), "bf16": (torch.bfloat16, 2.0**-8)}


def host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------ 4-bit weights
def unpack(tiles, scales, N, K):
    """Weights, scales and offsets [N, K] of tiles, by the format's formula."""
    tiles, scales = tiles.cpu().numpy(), host(scales)
    kt = tiles.shape[1]
    group = kt * 128 // scales.shape[1]
    n, k = np.arange(N)[:, None], np.arange(K)[None, :]
    step, g, j = k % 128 // 32, k % 32 // 8, k % 8
    c = j // 2 + j % 2 * 4
    byte = tiles[n // 16, k // 128, (n % 16 + 16 * g) * 16 + 4 * step + c // 2]
    q = np.where(c % 2, byte >> 4, byte & 15).astype(np.float64)
    s, b = scales[n // 16, k // group, n % 16, 0], scales[n // 16, k // group, n % 16, 1]
    return q, s, b


def random_tiles(g, N, K, group):
    nt, kt = -(-N // 16), -(-K // 128)
    tiles = torch.randint(0, 256, (nt, kt, 1024), dtype=torch.uint8, device="cuda", generator=g)
    s = torch.rand((nt, kt * 128 // group, 16), device="cuda", generator=g) * 0.01 + 0.001
    scales = torch.stack([s, -s * 7 + 0.01 * torch.randn(s.shape, device="cuda", generator=g)], -1).bfloat16()
    # what lies past the last row and the last group is anything
    if N % 16:
        scales[-1, :, N % 16:] = float("nan")
    scales[:, -(-K // group):] = float("nan")
    return tiles, scales


def check_fc(y, x, tiles, scales, N, K, kind, bias=None):
    q, s, b = unpack(tiles, scales, N, K)
    xs = host(x)
    want = xs @ (q * s + b).T
    size = np.abs(xs) @ (31 * np.abs(s) + np.abs(b - 16 * s)).T
    if bias is not None:
        want, size = want + host(bias), size + np.abs(host(bias))
    err = np.abs(host(y) - want)
    bound = TYPES[kind][1] * np.abs(want) + (K / 32 + 64) * 2.0**-24 * size + 1e-30
    assert y.dtype == x.dtype and (err <= bound).all(), (err / bound).max()


SHAPES = [(1, 1, 1, 32), (1, 256, 512, 32), (2, 17, 127, 32), (3, 16, 128, 128), (7, 1000, 2100, 64), (16, 33, 129, 64), (17, 40, 96, 128),
          (32, 64, 640, 64), (33, 100, 1000, 32), (63, 48, 260, 128), (64, 130, 1024, 128), (65, 31, 300, 32), (100, 272, 513, 64),
          (129, 128, 384, 128), (200, 300, 1100, 32), (300, 512, 1536, 128), (1, 4096, 9216, 128), (5, 64, 9216, 32)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,N,K,group", SHAPES)
def test_w4_fc(M, N, K, group, kind):
    g = torch.Generator(device="cuda").manual_seed(M * 7 + N * 3 + K)
    tiles, scales = random_tiles(g, N, K, group)
    x = torch.randn((M, K), device="cuda", generator=g).to(TYPES[kind][0])
    check_fc(B.w4_fc(x, tiles, scales, N), x, tiles, scales, N, K, kind)
    assert "w4_" in B.last_kernel()


@pytest.mark.parametrize("M,N,K,group,kind,kernel", [
    (100, 4100, 300, 64, "bf16", "1,1,64,4"), (260, 4100, 300, 32, "f16", "1,1,32,2"), (520, 4200, 700, 64, "bf16", "1,1,64,1"),
    (577, 4200, 1000, 32, "f16", "1,1,32,1"), (1050, 4250, 300, 128, "bf16", "2,2,128,1"), (2000, 2100, 1024, 128, "f16", "2,2,128,1"),
    (1050, 4250, 150, 64, "bf16", "1,1,64,1"), (20, 7001, 520, 128, "bf16", "1,1,128,4"), (300, 2500, 300, 32, "f32", "f32_kernel<32>"),
    (700, 1000, 200, 64, "f32", "f32_kernel<64>"), (260, 4097, 513, 128, "f32", "f32_kernel<128>")])
def test_w4_fc_many_results(M, N, K, group, kind, kernel):
    """Sizes that reach the kernels of many tiles, rows on odd elements too; the values in 64 bits made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(M + N)
    tiles, scales = random_tiles(g, N, K, group)
    q, s, b = (torch.from_numpy(a).cuda() for a in unpack(tiles, scales, N, K))
    for shift in (0, 3):
        x = torch.randn((M, K + 2 * shift), device="cuda", generator=g).to(TYPES[kind][0])[:, shift:shift + K]
        y = B.w4_fc(x, tiles, scales, N)
        assert kernel in B.last_kernel()
        want = x.double() @ (q * s + b).t().contiguous()
        size = x.double().abs() @ (31 * s.abs() + (b - 16 * s).abs()).t().contiguous()
        bound = TYPES[kind][1] * want.abs() + (K / 32 + 64) * 2.0**-24 * size + 1e-30
        assert bool(((y.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,pad,shift", [(3, 0, 1), (20, 3, 0), (70, 8, 2), (150, 5, 3), (150, 8, 8)])
def test_w4_fc_strides_and_bias(M, pad, shift, kind):
    """Rows further apart than their length, on any element; results into part of a matrix whose rest stays as it was."""
    N, K, group = 70, 330, 64
    g = torch.Generator(device="cuda").manual_seed(M + pad + shift)
    tiles, scales = random_tiles(g, N, K, group)
    x = torch.randn((M, shift + K + pad), device="cuda", generator=g).to(TYPES[kind][0])[:, shift:shift + K]
    bias = torch.randn((N,), device="cuda", generator=g)
    whole = torch.full((M, N + 7), -77.0, device="cuda", dtype=x.dtype)
    out = whole[:, 3:3 + N]
    assert B.w4_fc(x, tiles, scales, N, bias=bias, out=out) is out
    check_fc(out, x, tiles, scales, N, K, kind, bias)
    whole[:, 3:3 + N] = -77.0
    assert bool((whole == -77.0).all())


@pytest.mark.parametrize("M", [1, 40, 200])
@pytest.mark.parametrize("kind", list(TYPES))
def test_w4_fc_rows_do_not_touch_each_other(M, kind):
    """A row of NaN and one of infinities spoil their own results only; a large value beside small ones keeps them."""
    N, K, group = 48, 256, 32
    g = torch.Generator(device="cuda").manual_seed(M)
    tiles, scales = random_tiles(g, N, K, group)
    x = torch.randn((M + 2, K), device="cuda", generator=g).to(TYPES[kind][0])
    x[0, 5] = float("nan")
    x[M + 1, 7] = float("inf")
    x[1, 9] = 3e4
    y = B.w4_fc(x, tiles, scales, N)
    assert bool(torch.isnan(y[0]).all()) and not bool(torch.isfinite(y[M + 1]).any())
    check_fc(y[1:M + 1], x[1:M + 1], tiles, scales, N, K, kind)


def test_w4_fc_does_not_depend_on_the_stream_or_on_earlier_calls():
    g = torch.Generator(device="cuda").manual_seed(5)
    tiles, scales = random_tiles(g, 512, 1024, 64)
    for M in (1, 33, 300):
        x = torch.randn((M, 1024), device="cuda", generator=g).bfloat16()
        want = B.w4_fc(x, tiles, scales, 512)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = B.w4_fc(x, tiles, scales, 512, stream=side)
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(B.w4_fc(x, tiles, scales, 512), want)


def quantised(w, group):
    """The quantiser of the format in float32, group by group: (levels, scale, offset), each [N, K]."""
    N, K = w.shape
    q, s, b = np.zeros((N, K), np.float32), np.zeros((N, K), np.float32), np.zeros((N, K), np.float32)

    def bf16(x):
        return torch.tensor(np.clip(x, -3.38e38, 3.38e38), dtype=torch.float32).bfloat16().float().numpy()
    with np.errstate(all="ignore"):
        for k in range(0, K, group):
            x = w[:, k:k + group]
            fine = np.isfinite(x)
            lo = np.where(fine, x, np.float32(np.inf)).min(1)
            hi = np.where(fine, x, np.float32(-np.inf)).max(1)
            lo, hi = np.where(lo <= hi, lo, np.float32(0)), np.where(lo <= hi, hi, np.float32(0))
            step, off = bf16(hi / np.float32(15) - lo / np.float32(15)), bf16(lo)
            r = np.where(step >= 2.0**-126, np.float32(1) / step, np.float32(0)).astype(np.float32)
            z = np.rint((x - off[:, None]) * r[:, None])
            q[:, k:k + group] = np.clip(np.where(np.isnan(z), 0, z), 0, 15)
            s[:, k:k + group], b[:, k:k + group] = step[:, None], off[:, None]
    return q, s, b


@pytest.mark.parametrize("N,K,group", [(1, 1, 32), (16, 128, 128), (17, 100, 64), (40, 333, 32), (64, 512, 128), (5, 130, 64)])
def test_w4_quantize(N, K, group):
    rng = np.random.default_rng(N * K)
    w = rng.standard_normal((N, K)).astype(np.float32) * 0.05
    w[0, : K // 2] = 0.25  # (groups of one value)
    if N > 3:
        w[1, :3] = (np.nan, np.inf, -np.inf)
        w[2] = np.nan
        w[3] *= np.float32(1e-38)
    tiles, scales = B.w4_quantize(torch.from_numpy(w).cuda(), group)
    q, s, b = unpack(tiles, scales, N, K)
    wq, ws, wb = quantised(w, group)
    np.testing.assert_array_equal(s, ws)
    np.testing.assert_array_equal(b, wb)
    np.testing.assert_array_equal(q, wq)
    back = B.w4_dequantize(tiles, scales, N, K).cpu().numpy()
    want = q * s + b
    assert (np.abs(back - want) <= 2.0**-23 * (np.abs(q * s) + np.abs(b))).all()
    # a weight is half a step off at most, and what rounding the scale and the offset to 8 bits adds
    fine = np.isfinite(w)
    step = (0.5 + 15 * 2.0**-8) * s + 2.0**-8 * np.abs(b) + 1e-36
    assert (np.abs(want - w)[fine] <= step[fine]).all()


def test_w4_strided_weights():
    w = torch.randn((20, 150), device="cuda")
    a, b = B.w4_quantize(w[:, 10:110], 32), B.w4_quantize(w[:, 10:110].contiguous(), 32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1].view(torch.int16), b[1].view(torch.int16))
    out = torch.zeros((20, 130), device="cuda")
    B.w4_dequantize(*a, 20, 100, out=out[:, 7:107])
    assert torch.equal(out[:, 7:107], B.w4_dequantize(*a, 20, 100)) and not bool(out[:, :7].any()) and not bool(out[:, 107:].any())


# ------------------------------------------------------------------ the cache
class Cache:
    """A cache and what it holds by the definition, in float32 as the format says it: levels and scales per sequence."""

    def __init__(self, seqs, width, heads, dim, block, seed, spare=3):
        self.heads, self.dim, self.block, self.width = heads, dim, block, width
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = seqs * width + spare
        # memory as it is found: any bytes, and scales that are no numbers
        self.pages, self.scales = B.kv_cache(n, heads, dim, block)
        self.pages.random_(-128, 128, generator=g)
        self.scales.fill_(float("nan"))
        order = torch.randperm(n, device="cuda", generator=g).int()
        self.table = order[: seqs * width].view(seqs, width).contiguous()
        self.lengths = [0] * seqs
        tokens = width * 64
        self.q = np.zeros((seqs, 2, heads, tokens, dim), np.float32)
        self.s = np.zeros((seqs, 2, heads, tokens // block), np.float32)

    def lens(self):
        return torch.tensor(self.lengths, dtype=torch.int32, device="cuda")

    def write_host(self, seq, x):
        """x: [2, tokens, heads, dim] float32 goes to the sequence's end."""
        n, B_ = x.shape[1], self.block
        for i in range(2):
            t = self.lengths[seq]
            end = t + n
            at = 0
            while t < end:
                b, stop = t // B_, min(end, (t // B_ + 1) * B_)
                new = x[i, at:at + stop - t].transpose(1, 0, 2)  # [heads, tokens, dim]
                size = np.abs(new)
                top = np.where(np.isfinite(size), size, 0).max((1, 2)).astype(np.float32)
                was = self.s[seq, i, :, b] if t > b * B_ else np.zeros(self.heads, np.float32)
                s = np.maximum(was, top * np.float32(1 / 127))
                with np.errstate(all="ignore"):
                    old = self.q[seq, i, :, b * B_:t]
                    ratio = np.where(s > was, was / s, 1).astype(np.float32)
                    self.q[seq, i, :, b * B_:t] = np.rint(old * ratio[:, None, None])
                    r = np.where(s >= np.float32(2.0**-126), np.float32(1) / s, 0).astype(np.float32)
                    q = np.clip(np.rint(new * r[:, None, None]), -127, 127)
                q = np.where(np.isnan(new), 0, np.where(np.isinf(new), np.sign(new) * 127, q))
                self.q[seq, i, :, t:stop] = q
                self.s[seq, i, :, b] = s
                at += stop - t
                t = stop
        self.lengths[seq] += n

    def values(self, seq, n=None):
        """[2, heads, tokens, dim] float32."""
        n = self.lengths[seq] if n is None else n
        return (self.q[seq] * np.repeat(self.s[seq], self.block, -1)[..., None])[:, :, :n]

    def check_memory(self):
        """Every byte and scale that tokens have reached, by the format's formulas."""
        row = self.pages.shape[3] // 64
        pages, scales, table = self.pages.cpu().numpy(), self.scales.cpu().numpy(), self.table.cpu().numpy()
        for seq, n in enumerate(self.lengths):
            t, d = np.arange(n)[:, None], np.arange(self.dim)[None, :]
            p = t % 64
            key = p // 16 * 16 * row + d // 64 * 1024
            key = key + np.where(d // 64 * 64 + 64 <= row, d % 64 // 16 * 256 + p % 16 * 16 + d % 16, d % 32 // 8 * 128 + p % 16 * 8 + d % 8)
            value = d // 16 * 1024 + p % 16 // 4 * 256 + d % 16 * 16 + p // 16 * 4 + p % 4
            for i, at in enumerate((key, value)):
                for h in range(self.heads):
                    np.testing.assert_array_equal(pages[table[seq, t // 64], h, i, at], self.q[seq, i, h, :n])
                    b = np.arange(-(-n // self.block))
                    np.testing.assert_array_equal(scales[table[seq, b * self.block // 64], h, i, b % (64 // self.block)], self.s[seq, i, h, b])

    def write(self, new, kind, gen, change=None):
        """new[i] more tokens for sequence i, in one call: on the GPU and on the host."""
        rows = sum(new)
        kv = torch.randn((2, rows, self.heads, self.dim), device="cuda", generator=gen)
        kv = kv * (0.2 + 2 * torch.rand((2, rows, 1, 1), device="cuda", generator=gen))
        kv = kv.to(TYPES[kind][0])
        if change:
            change(kv)
        x = kv.float().cpu().numpy()
        at = 0
        for i, n in enumerate(new):
            self.write_host(i, x[:, at:at + n])
            at += n
        starts = None if len(set(new)) == 1 else torch.tensor(np.cumsum([0] + list(new)), dtype=torch.int32, device="cuda")
        B.kv_write(kv[0], kv[1], self.pages, self.scales, self.table, self.lens(), starts=starts, max_new=max(new) if starts is not None else 0)
        return starts


SETS = [(1, 1, 1, 16, "f32"), (2, 3, 64, 16, "bf16"), (3, 2, 128, 32, "f16"), (2, 1, 96, 64, "bf16"), (2, 2, 80, 16, "f32"),
        (1, 2, 256, 64, "f16"), (4, 1, 33, 32, "f32"), (2, 8, 128, 16, "bf16")]
PLANS = [[[1], [1], [1], [1]], [[5], [1], [1], [64], [17]], [[100], [1], [1], [29], [62]], [[63], [2], [60], [3]], [[16], [16], [32], [130]]]


@pytest.mark.parametrize("seqs,heads,dim,block,kind", SETS)
@pytest.mark.parametrize("plan", range(len(PLANS)))
def test_kv_write_and_read(seqs, heads, dim, block, kind, plan):
    """Writes of one token and many, into fresh blocks and blocks in use, evenly and ragged; every byte, every scale; read back."""
    c = Cache(seqs, 5, heads, dim, block, plan)
    g = torch.Generator(device="cuda").manual_seed(plan * 10 + seqs)
    for k, (n,) in enumerate(PLANS[plan]):
        # (every other call ragged, with sequences that get nothing)
        new = [n] * seqs if k % 2 == 0 else [max(0, n - 2 * i) for i in range(seqs)]
        if sum(new):
            c.write(new, kind, g)
    c.check_memory()
    for count in (1, 7, 10**6):
        back = [min(count, n) for n in c.lengths]
        starts = torch.tensor(np.cumsum([0] + back), dtype=torch.int32, device="cuda")
        for name, (dtype, _) in TYPES.items():
            k, v = B.kv_read(c.pages, c.scales, c.table, c.lens(), dim, dtype, sum(back), starts=starts, max_new=max(back))
            at = 0
            for i, n in enumerate(back):
                want = torch.from_numpy(c.values(i)[:, :, c.lengths[i] - n:].transpose(0, 2, 1, 3).copy()).to(dtype)
                assert torch.equal(torch.stack([k, v])[:, at:at + n].cpu(), want)
                at += n


def test_kv_write_special_values():
    """NaN is level 0, an infinity the last level, and neither has a say in the scale; blocks of zeros and of denormals hold zeros."""
    c = Cache(1, 2, 2, 64, 16, 3)
    g = torch.Generator(device="cuda").manual_seed(8)

    def change(kv):
        kv[0, 3, 0, 5], kv[0, 4, 0, 6], kv[1, 5, 1, 7] = float("nan"), float("inf"), -float("inf")
        kv[:, 16:32] = 0.0
        kv[:, 32:48] = 1e-40
        kv[:, 48:64] *= 1e30
        kv[1, 64:80] = float("nan")
    c.write([90], "f32", g, change)
    c.check_memory()


def test_kv_strided_rows():
    """Keys, values and what is read back as parts of larger rows; what lies beside them stays."""
    c = Cache(2, 2, 3, 72, 32, 4)
    buf = torch.randn((40, 2 * 3 * 72 + 11), device="cuda")
    k, v = buf[:, 5:5 + 216].unflatten(1, (3, 72)), buf[:, 221:437].unflatten(1, (3, 72))
    x = torch.stack([k, v]).cpu().numpy()
    for i in range(2):
        c.write_host(i, x[:, 20 * i:20 * i + 20])
    B.kv_write(k, v, c.pages, c.scales, c.table, c.lens())
    c.check_memory()
    out = torch.full((3, 40, 2, 72), 9.0, device="cuda", dtype=torch.float16)  # (heads before rows)
    spare = torch.full((40, 3, 80), 9.0, device="cuda", dtype=torch.float16)
    B.kv_read(c.pages, c.scales, c.table, c.lens(), 72, torch.float16, 40, out_k=out[:, :, 0].transpose(0, 1), out_v=spare[:, :, :72])
    for i in range(2):
        want = torch.from_numpy(c.values(i).copy()).half()
        assert torch.equal(out[:, 20 * i:20 * i + 20, 0].cpu(), want[0]) and torch.equal(spare[20 * i:20 * i + 20, :, :72].cpu(), want[1].transpose(0, 1))
    assert bool((out[:, :, 1] == 9.0).all()) and bool((spare[:, :, 72:] == 9.0).all())


def test_kv_numbers_from_device_memory_stay_inside():
    """Lengths past the table, page numbers that are none, rows of positions below 0: nothing is written for them, zeros come back."""
    heads, dim = 2, 64
    pages, scales = B.kv_cache(4, heads, dim)
    pages.fill_(55)
    scales.fill_(0.001)
    table = torch.tensor([[1, 2], [7, -3], [0, 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([200, 100, 2], dtype=torch.int32, device="cuda")  # (more than 128; on no page; fewer than its rows)
    kv = torch.randn((3 * 80, heads, dim), device="cuda")
    B.kv_write(kv, kv, pages, scales, table, lengths)
    k, v = B.kv_read(pages, scales, table, lengths, dim, torch.float32, 240)
    x = kv.view(3, 80, heads, dim)
    k = k.view(3, 80, heads, dim)
    # sequence 0: positions 120 .. 199, of which 120 .. 127 are there; sequence 2: positions -78 .. 1
    assert float((k[0, :8] - x[0, :8]).abs().max()) < 0.03 and not bool(k[0, 8:].any()) and not bool(k[1].any())
    assert not bool(k[2, :78].any()) and float((k[2, 78:] - x[2, 78:]).abs().max()) < 0.03
    assert bool((pages[1] == 55).all()) and bool((pages[3] == 55).all()) and bool((scales[1] == 0.001).all()) and bool((scales[3] == 0.001).all())
    q = torch.randn((240, heads, dim), device="cuda")
    o = B.kv_attention(q, pages, scales, table, lengths).view(3, 80, heads, dim)
    assert not bool(o[1].any()) and not bool(o[2, :78].any()) and bool(torch.isfinite(o).all())
    bad = torch.tensor([-5, 300, 20, 400], dtype=torch.int32, device="cuda")  # (starts that are no starts)
    B.kv_write(kv, kv, pages, scales, table, lengths, starts=bad)
    B.kv_read(pages, scales, table, lengths, dim, torch.float32, 240, starts=bad)
    B.kv_attention(q, pages, scales, table, lengths, starts=bad)
    torch.cuda.synchronize()


def test_kv_pages_past_32_bits():
    """A cache of more than 4 GiB: its last pages are its last pages."""
    heads, dim = 32, 128
    n = (1 << 32) // (heads * 2 * 64 * dim) + 40
    pages = torch.empty((n, heads, 2, 64 * dim), dtype=torch.int8, device="cuda")
    scales = torch.empty((n, heads, 2, 4), dtype=torch.float32, device="cuda")
    table = torch.tensor([[n - 1, n - 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([100], dtype=torch.int32, device="cuda")
    kv = torch.randn((2, 100, heads, dim), device="cuda")
    small, few = B.kv_cache(2, heads, dim)
    at = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    q = torch.randn((1, heads, dim), device="cuda")
    got = []
    for p, s, t in ((pages, scales, table), (small, few, at)):
        B.kv_write(kv[0], kv[1], p, s, t, lengths)
        got.append((*B.kv_read(p, s, t, lengths, dim, torch.float32, 100), B.kv_attention(q, p, s, t, lengths)))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    del pages
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ attention
def check_attention(out, q, c, new, kind, causal=True, window=0, scale=None, lse=None):
    dtype, u = TYPES[kind]
    w = 2.0**-20 if kind == "f32" else 2.0**-11
    xs, got = host(q), host(out)
    assert out.dtype == dtype
    scale = c.dim**-0.5 if scale is None else scale
    share = q.shape[1] // c.heads
    at = 0
    for seq, m in enumerate(new):
        n = c.lengths[seq]
        kv = c.values(seq).astype(np.float64)
        pos = np.arange(n - m, n)
        for h in range(q.shape[1]):
            k, v = kv[0, h // share], kv[1, h // share]
            z = xs[at:at + m, h] @ k.T * scale
            e = (2.0**-21 + c.dim * 2.0**-24) * abs(scale) * (np.abs(xs[at:at + m, h]) @ np.abs(k).T)
            t = np.arange(n)[None, :]
            see = np.ones((m, n), bool)
            if causal:
                see &= t <= pos[:, None]
            if window:
                see &= t > pos[:, None] - window
            z = np.where(see, z, -np.inf)
            top = z.max(1, initial=-np.inf)
            p = np.exp(z - np.where(np.isfinite(top), top, 0)[:, None])
            total = p.sum(1)
            some = total > 0
            p = p / np.where(some, total, 1)[:, None]
            want, size = p @ v, p @ np.abs(v)
            worst = np.where(see, e, 0).max(1, initial=0)[:, None]
            bound = u * np.abs(want) + (2 * worst + w + (n + 100) * 2.0**-24) * size + 1e-30
            if kind != "f32":
                bound = bound + n * 2.0**-39 * np.abs(v).max(initial=0) + (2.0**-25 if kind == "f16" else 0)
            err = np.abs(got[at:at + m, h] - want)
            assert (err <= bound).all(), (seq, h, (err / bound).max())
            if lse is not None:
                wl = np.where(some, np.log(np.where(some, total, 1)) + np.where(some, top, 0), -np.inf)
                gl = host(lse[at:at + m, h])
                with np.errstate(invalid="ignore"):
                    assert ((gl == wl) | (np.abs(gl - wl) <= worst[:, 0] + (n + 100) * 2.0**-24 + 2.0**-22 * np.abs(wl))).all()
        at += m


def fill(c, totals, kind, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c.write([int(n) for n in totals], kind, g) if sum(totals) else None
    return g


# sequences' lengths, their new rows, heads of queries, heads of the cache, dim, block
ATTEND = [([1], [1], 1, 1, 64, 16), ([0, 3], [1, 1], 4, 2, 128, 32), ([64, 65, 63, 1], [1, 1, 1, 1], 8, 8, 64, 64),
          ([200, 7, 0, 129], [1, 1, 0, 1], 32, 4, 128, 16), ([700], [1], 8, 1, 96, 32), ([333, 100], [1, 1], 6, 2, 80, 16),
          ([150, 60], [5, 3], 12, 2, 96, 64), ([130], [130], 2, 1, 64, 16), ([300, 90, 5], [70, 90, 5], 6, 3, 128, 32),
          ([250], [33], 4, 4, 256, 16), ([90], [20], 2, 2, 1, 16), ([70, 190], [17, 1], 20, 1, 32, 32), ([1300, 20], [1, 1], 4, 4, 40, 64),
          ([400], [200], 8, 2, 128, 64), ([320, 500], [256, 100], 4, 1, 160, 32), ([190], [64], 2, 2, 224, 16), ([260, 40], [40, 40], 3, 3, 192, 64)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("totals,new,q_heads,heads,dim,block", ATTEND)
def test_kv_attention(totals, new, q_heads, heads, dim, block, kind):
    c = Cache(len(totals), -(-max(totals) // 64) + 1, heads, dim, block, sum(totals))
    g = fill(c, totals, kind, dim)
    q = torch.randn((sum(new), q_heads, dim), device="cuda", generator=g).to(TYPES[kind][0])
    starts = torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device="cuda")
    for causal, window in ((True, 0), (False, 0), (True, 50), (False, 64), (True, 1)):
        out, lse = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), starts=starts, max_new=max(new), causal=causal, window=window, lse=True)
        check_attention(out, q, c, new, kind, causal, window, lse=lse)
    assert torch.equal(out, B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), starts=starts, causal=causal, window=window))
    if len(set(new)) == 1:
        assert torch.equal(out, B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), causal=causal, window=window))


@pytest.mark.parametrize("seqs,heads,share,dim,block,kind", [
    (64, 2, 4, 64, 16, "bf16"), (43, 3, 5, 96, 32, "f16"), (128, 1, 7, 128, 64, "bf16"), (16, 8, 3, 40, 16, "f16"), (64, 2, 8, 160, 16, "bf16"),
    (128, 1, 6, 256, 32, "f16"), (32, 4, 4, 20, 64, "bf16"), (64, 2, 4, 192, 16, "f16"), (128, 1, 9, 224, 16, "bf16")])
def test_kv_attention_many_rows(seqs, heads, share, dim, block, kind):
    """Batches of prompts that fill the chip: evenly, and ragged with sequences of few rows, none, and rows of positions below 0."""
    totals = [(37 * i + 11) % 230 for i in range(seqs)]
    c = Cache(seqs, 4, heads, dim, block, seqs + dim)
    g = fill(c, totals, kind, dim)
    for ragged in (False, True):
        new = [min(n, (13 * i) % 90) for i, n in enumerate(totals)] if ragged else [30] * seqs
        q = torch.randn((sum(new), heads * share, dim), device="cuda", generator=g).to(TYPES[kind][0])
        starts = torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device="cuda") if ragged else None
        for causal, window in ((True, 0), (False, 0), (True, 40)):
            out, lse = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), starts=starts, max_new=max(new) if ragged else 0,
                                      causal=causal, window=window, lse=True)
            assert "kv_prompt_kernel" in B.last_kernel()
            check_attention(out, q, c, new, kind, causal, window, lse=lse)


def test_kv_attention_many_rows_large_and_small_values():
    """As the test below, where many rows share a page: negative and large factors, blocks whose scales differ by 2^20, zeros, NaN in a query."""
    c = Cache(8, 5, 4, 64, 16, 9)
    g = torch.Generator(device="cuda").manual_seed(1)

    def change(kv):
        kv[0] *= 8
        kv[1, 30:60] *= 2.0**-10
        kv[1, 100:130] *= 2.0**10
        kv[1, 160:176] = 0
        kv[1, 700:900] = 0
    c.write([300] * 8, "f32", g, change)
    q = torch.randn((8 * 250, 8, 64), device="cuda", generator=g)
    q[:, 1] *= 30
    q[:, 2] = 0
    q[:, 3] *= 2.0**-13
    for kind in ("f16", "bf16"):
        for scale in (0.3, -0.2):
            x = q.to(TYPES[kind][0])
            out = B.kv_attention(x, c.pages, c.scales, c.table, c.lens(), scale=scale)
            assert "kv_prompt_kernel" in B.last_kernel()
            check_attention(out, x, c, [250] * 8, kind, scale=scale)
        x[17, 5, 3] = float("nan")
        got = B.kv_attention(x, c.pages, c.scales, c.table, c.lens(), scale=scale)
        assert bool(torch.isnan(got[17, 5]).all())
        got[17, 5] = out[17, 5]
        assert torch.equal(got, out)


@pytest.mark.parametrize("rows", [1, 40, 200])
@pytest.mark.parametrize("kind", list(TYPES))
def test_kv_attention_large_and_small_values(kind, rows):
    """Scores in the hundreds, values whose blocks differ by 2^20, a block of zeros, queries of zeros and of small values."""
    c = Cache(1, 5, 2, 64, 16, 9)
    g = torch.Generator(device="cuda").manual_seed(1)

    def change(kv):
        kv[0] *= 8
        kv[1, 30:60] *= 2.0**-10
        kv[1, 100:130] *= 2.0**10
        kv[1, 160:176] = 0
    c.write([300], "f32", g, change)
    q = torch.randn((rows, 4, 64), device="cuda", generator=g)
    q[:, 1] *= 30
    q[:, 2] = 0
    q[:, 3] *= 2.0**-13
    q = q.to(TYPES[kind][0])
    out = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), scale=0.3)
    check_attention(out, q, c, [rows], kind, scale=0.3)


@pytest.mark.parametrize("rows", [1, 100])
def test_kv_attention_masked_places_may_hold_anything(rows):
    """Levels and scales that no row sees do not reach the result, whatever they are (scales of unwritten blocks are NaN in every test
    here): the same bits with other garbage."""
    c = Cache(2, 4, 2, 128, 16, 11)
    g = fill(c, [130, 200], "bf16", 4)
    q = torch.randn((2 * rows, 8, 128), device="cuda", generator=g).bfloat16()
    for window in (0, 30):
        want = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), window=window)
        assert bool(torch.isfinite(want).all())
        pages, scales = c.pages.clone(), c.scales.clone()
        used = torch.zeros_like(scales, dtype=torch.bool)
        low = [0, 0] if not window else [max(0, n - rows - window + 1) for n in c.lengths]
        for i, n in enumerate(c.lengths):
            for b in range(low[i] // 16, -(-n // 16)):
                used[c.table[i, b * 16 // 64].item(), :, :, b % 4] = True
        for fill_with in (float("inf"), float("nan"), -3e38):
            scales[~used] = fill_with
            got = B.kv_attention(q, pages, scales, c.table, c.lens(), window=window)
            assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [1, 60])
def test_kv_attention_nan_in_a_query(rows):
    c = Cache(1, 3, 1, 64, 16, 12)
    g = fill(c, [150], "f16", 4)
    q = torch.randn((rows, 4, 64), device="cuda", generator=g).half()
    q[0, 2, 7] = float("nan")
    out = B.kv_attention(q, c.pages, c.scales, c.table, c.lens())
    assert bool(torch.isnan(out[0, 2]).all())
    out[0, 2] = 0
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("rows", [1, 3, 50])
def test_kv_attention_strides(rows):
    c = Cache(2, 4, 2, 96, 32, 13)
    g = fill(c, [140, 230], "bf16", 5)
    buf = torch.randn((2 * rows, 6 * 96 + 9), device="cuda", generator=g).bfloat16()
    q = buf[:, 7:7 + 576].unflatten(1, (6, 96))
    whole = torch.full((6, 2 * rows, 100), 5.0, device="cuda", dtype=torch.bfloat16)
    out = whole[:, :, 1:97].transpose(0, 1)  # (heads before rows)
    assert B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), out=out) is out
    check_attention(out, q, c, [rows, rows], "bf16")
    assert torch.equal(out, B.kv_attention(q.contiguous(), c.pages, c.scales, c.table, c.lens()))
    whole[:, :, 1:97] = 5.0
    assert bool((whole == 5.0).all())


def test_kv_attention_long():
    """A long sequence, one row and few: as the plain form, and the same in several calls and workspaces."""
    heads, dim, n = 2, 128, 30011
    width = -(-n // 64)
    c = Cache(1, width, heads, dim, 64, 14)
    g = fill(c, [n], "bf16", 6)
    for rows in (1, 4):
        q = torch.randn((rows, 8, dim), device="cuda", generator=g).bfloat16()
        out = B.kv_attention(q, c.pages, c.scales, c.table, c.lens())
        check_attention(out, q, c, [rows], "bf16")
        need = B.workspace_bytes(B.OP_KV_ATTENTION, (1, width, heads, 8, dim, rows))
        ws = torch.zeros((max(need, 16),), dtype=torch.uint8, device="cuda")
        for _ in range(3):
            assert torch.equal(out, B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), workspace=ws))


def test_kv_attention_one_workspace_for_calls_of_all_sizes():
    """A program's scratch memory goes from call to call, whatever their sizes."""
    caches = [Cache(s, w, h, d, 16, 20 + s) for s, w, h, d in ((1, 80, 2, 64), (3, 9, 1, 128), (16, 2, 4, 96))]
    gens = [fill(c, [c.width * 64 - 5 - 3 * i for i in range(c.table.shape[0])], "bf16", 7) for c in caches]
    qs = [torch.randn((c.table.shape[0] * r, c.heads * 2, c.dim), device="cuda", generator=g).bfloat16() for c, g, r in zip(caches, gens, (1, 3, 1))]
    dims = [(c.table.shape[0], c.width, c.heads, c.heads * 2, c.dim, q.shape[0] // c.table.shape[0]) for c, q in zip(caches, qs)]
    ws = torch.zeros((max([B.workspace_bytes(B.OP_KV_ATTENTION, d) for d in dims] + [16]),), dtype=torch.uint8, device="cuda")
    want = [B.kv_attention(q, c.pages, c.scales, c.table, c.lens()) for c, q in zip(caches, qs)]
    for _ in range(3):
        for c, q, o in zip(caches, qs, want):
            assert torch.equal(o, B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), workspace=ws))


@pytest.mark.parametrize("lengths,rows,heads,share,dim,block,kind,splits", [
    ([4400], [130], 16, 8, 64, 16, "bf16", 3), ([2500], [300], 8, 7, 128, 32, "f16", 2), ([2100], [70], 16, 16, 200, 16, "bf16", 1),
    ([2100], [60], 16, 16, 200, 16, "bf16", 2), ([4400, 2100, 300, 0], [100, 12, 5, 3], 8, 8, 96, 64, "f16", 2),
    ([1, 2600], [40, 90], 12, 8, 20, 16, "bf16", 2)])
def test_kv_attention_many_rows_long(lengths, rows, heads, share, dim, block, kind, splits):
    """Many rows over sequences so long that workgroups share their pages: with sequences of few rows and none beside them, rows of positions
    below 0, windows; and the same bits in several calls and on a workspace that goes from one to the next."""
    width = -(-max(lengths) // 64) + 2
    c = Cache(len(lengths), width, heads, dim, block, 40 + dim)
    g = fill(c, lengths, kind, dim)
    q = torch.randn((sum(rows), heads * share, dim), device="cuda", generator=g).to(TYPES[kind][0])
    starts = torch.tensor(np.cumsum([0] + rows), dtype=torch.int32, device="cuda")
    need = B.workspace_bytes(B.OP_KV_ATTENTION, (len(lengths), width, heads, heads * share, dim, max(rows)))
    ws = torch.zeros((max(need, 16),), dtype=torch.uint8, device="cuda")
    for causal, window in ((True, 0), (False, 0), (True, 1500), (False, 1100)):
        out, lse = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), starts=starts, max_new=max(rows), causal=causal, window=window, lse=True)
        name = B.last_kernel()
        assert "kv_prompt_kernel" in name and int(name.split("grid ")[1].split("x")[0]) == splits * heads
        check_attention(out, q, c, rows, kind, causal, window, lse=lse)
        for _ in range(3):
            assert torch.equal(out, B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), starts=starts, max_new=max(rows), causal=causal,
                                                   window=window, workspace=ws))


def test_decoder_calls_in_a_graph():
    """A step of a layer captured once and replayed on new inputs, with eager work between the replays."""
    heads, dim, seqs = 2, 64, 3
    c = Cache(seqs, 30, heads, dim, 16, 30)
    g = fill(c, [1500, 3, 700], "bf16", 8)
    tiles, scales = random_tiles(g, 8 * dim, 256, 32)
    x = torch.randn((seqs, 256), device="cuda", generator=g).bfloat16()
    lengths = c.lens() + 1
    keep = c.pages.clone(), c.scales.clone()
    need = B.workspace_bytes(B.OP_KV_ATTENTION, (seqs, 30, heads, 4, dim, 1))
    ws = torch.zeros((max(need, 16),), dtype=torch.uint8, device="cuda")
    qkv = torch.empty((seqs, 8 * dim), device="cuda", dtype=torch.bfloat16)
    out = torch.empty((seqs, 4, dim), device="cuda", dtype=torch.bfloat16)

    def step():
        B.w4_fc(x, tiles, scales, 8 * dim, out=qkv)
        parts = qkv.view(seqs, 8, dim)
        B.kv_write(parts[:, 4:6], parts[:, 6:], c.pages, c.scales, c.table, lengths)
        B.kv_attention(parts[:, :4], c.pages, c.scales, c.table, lengths, out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.copy_(torch.randn((seqs, 256), device="cuda", generator=g))
        c.pages.copy_(keep[0]), c.scales.copy_(keep[1])
        step()
        want, held = out.clone(), c.scales.clone()
        out.zero_()
        c.pages.copy_(keep[0]), c.scales.copy_(keep[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(held.nan_to_num(), c.scales.nan_to_num()), k
