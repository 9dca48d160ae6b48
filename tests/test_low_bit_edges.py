"""GPU tests of the decoder layer's calls at the ends of what they take."""
import numpy as np
import pytest
import torch

from paper_1705_09864_amd import binding as B
from test_low_bit import TYPES, Cache, check_fc, fill, host, random_tiles, unpack

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


def test_kv_attention_positions_at_the_end_of_32_bits():
    """A table as wide as positions have room for, of which the last pages are there: what a short table of the same pages gives."""
    heads, dim, width, there = 1, 32, 1 << 25, 40
    pages, scales = B.kv_cache(there, heads, dim)
    pages.random_(-127, 128)
    scales.uniform_(0.001, 0.01)
    scales[-1, :, :, -1] = 0.004
    short = torch.arange(there, dtype=torch.int32, device="cuda")[None]
    wide = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    wide[:, -there:] = short
    lengths = [torch.tensor([n], dtype=torch.int32, device="cuda") for n in (there * 64 - 1, TOP)]
    for rows, share, window, causal in ((1, 1, 100, True), (3, 4, 700, True), (5, 2, 100, False), (2048, 8, 100, True)):
        for kind in (torch.float32, torch.bfloat16):
            if rows * share > 64 and kind == torch.float32:
                continue
            q = torch.randn((rows, share, dim), device="cuda").to(kind)
            want, got = (B.kv_attention(q, pages, scales, t, n, causal=causal, window=window) for t, n in zip((short, wide), lengths))
            assert float(want.float().abs().min()) > 0 or rows > 64
            assert float((got.float() - want.float()).abs().max()) <= 2.0**-7 * float(want.float().abs().max()), (rows, kind)


def test_kv_read_rounds_the_product():
    """Levels and scales whose fp32 product lies halfway between two 16-bit values, and the exact product beside it: the product is rounded to
    fp32, then to the type, whatever the type, for keys as for values."""
    rng = np.random.default_rng(0)
    found = []
    while len(found) < 64:
        s = rng.uniform(0.001, 0.1, 400000).astype(np.float32)
        q = rng.integers(1, 128, s.size)
        exact = s.astype(np.float64) * q
        other = np.flatnonzero(exact.astype(np.float16) != exact.astype(np.float32).astype(np.float16))
        found += [(s[i], q[i]) for i in other]
    dim, n = 64, 64  # a block of 16 tokens for each pair, four to a page
    pages, scales = B.kv_cache(n // 4, 1, dim)
    s = torch.tensor([a for a, _ in found[:n]]).view(n // 4, 1, 1, 4)
    q = torch.tensor([b for _, b in found[:n]]).view(n // 4, 4)
    scales.copy_(s.expand(-1, -1, 2, -1))
    t, d = np.arange(64)[:, None], np.arange(dim)[None, :]
    key = t // 16 * 16 * dim + d % 64 // 16 * 256 + t % 16 * 16 + d % 16
    value = d // 16 * 1024 + t % 16 // 4 * 256 + d % 16 * 16 + t // 16 * 4 + t % 4
    body = torch.zeros((n // 4, 1, 2, 64 * dim), dtype=torch.int8)
    levels = q.repeat_interleave(16, 1)[:, :, None].expand(-1, -1, dim) * torch.where(torch.arange(dim) % 2 == 0, 1, -1)
    for i, at in enumerate((key, value)):
        body[:, 0, i, torch.from_numpy(at).reshape(-1)] = levels.reshape(n // 4, -1).to(torch.int8)
    pages.copy_(body)
    table = torch.arange(n // 4, dtype=torch.int32, device="cuda")[None]
    lengths = torch.tensor([16 * n], dtype=torch.int32, device="cuda")
    want = (levels.float() * s.view(-1, 4).repeat_interleave(16, 1)[:, :, None]).reshape(16 * n, 1, dim)
    for kind in (torch.float32, torch.float16, torch.bfloat16):
        for x in B.kv_read(pages, scales, table, lengths, dim, kind, 16 * n):
            assert torch.equal(x.cpu(), want.to(kind)), kind


# ------------------------------------------------------------------ what a row does not see or weigh leaves it as it is
def check_rows(out, q, c, rows, kind, scale=None, first=0, last=None):
    """Rows `first` to `last` of each sequence's `rows` new ones, causal.  As in test_low_bit.py, but what a weight in f16 loses is bounded by the
    row itself: a weight times its block's scale is held to 2^-25 of 2^14, which stands for the row's largest, for each token."""
    u, w = TYPES[kind][1], 2.0**-20 if kind == "f32" else 2.0**-11
    scale = c.dim**-0.5 if scale is None else scale
    share, last = q.shape[1] // c.heads, rows if last is None else last
    x, got = host(q), host(out)
    for seq, n in enumerate(c.lengths):
        mine = slice(seq * rows + first, seq * rows + last)
        pos, t = np.arange(n - rows + first, n - rows + last)[:, None], np.arange(n)[None, :]
        kv = c.values(seq).astype(np.float64)
        for h in range(q.shape[1]):
            k, v = kv[0, h // share], kv[1, h // share]
            z = np.where(t <= pos, x[mine, h] @ k.T * scale, -np.inf)
            e = np.where(t <= pos, (2.0**-21 + c.dim * 2.0**-24) * abs(scale) * (np.abs(x[mine, h]) @ np.abs(k).T), 0).max(1, keepdims=True)
            p = np.exp(z - z.max(1, keepdims=True))
            p = p / p.sum(1, keepdims=True)
            want, size = p @ v, p @ np.abs(v)
            bound = u * np.abs(want) + (2 * e + w + (n + 100) * 2.0**-24) * size + 1e-30
            if kind != "f32":
                steps = np.repeat(np.abs(c.s[seq, 1, h // share].astype(np.float64)), c.block)[:n]
                bound = bound + n * 2.0**-39 * 127 * (p * steps).max(1, keepdims=True) + (2.0**-25 if kind == "f16" else 0)
            err = np.abs(got[mine, h] - want)
            assert (err <= bound).all(), (seq, h, (err / bound).max())


# the kernel of 16 rows and, for 16-bit types, the one of many
@pytest.mark.parametrize("seqs", [1, 64])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("kind", list(TYPES))
def test_kv_attention_values_behind_a_row(kind, block, seqs):
    """Tokens behind a row's position, of its page and beside rows of its tile that see them, hold values 2^60 times as large."""
    rows, c = 40, Cache(seqs, 3, 2, 64, block, 50)
    g = torch.Generator(device="cuda").manual_seed(3)
    c.write([88] * seqs, "f32", g)
    large = (112 if block == 16 else 96) - 88  # from a block's first token on

    def change(kv):
        kv.unflatten(1, (seqs, rows))[1, :, large:] *= 2.0**60
    c.write([rows] * seqs, "f32", g, change)
    q = torch.randn((seqs * rows, 6, 64), device="cuda", generator=g).to(TYPES[kind][0])
    out = B.kv_attention(q, c.pages, c.scales, c.table, c.lens())
    assert ("kv_prompt" in B.last_kernel()) == (seqs > 1 and kind != "f32")
    check_rows(out, q, c, rows, kind, last=large)
    if kind != "f16":  # (there these are infinities)
        check_rows(out, q, c, rows, kind, first=large)


@pytest.mark.parametrize("seqs", [1, 64])
@pytest.mark.parametrize("kind", list(TYPES))
def test_kv_attention_values_without_weight(kind, seqs):
    """A block of large values whose weights are nothing, and one whose weights are 2^-40 and bring as much as all others."""
    rows, c = 40, Cache(seqs, 3, 2, 64, 16, 51)
    g = torch.Generator(device="cuda").manual_seed(4)

    def change(kv):
        x = kv.unflatten(1, (seqs, 130))
        x[0, :, :, :, 0] = 0
        x[0, :, 16:32] = 0
        x[0, :, 16:32, :, 0] = -100
        x[1, :, 16:32] *= 2.0**60
        x[0, :, 48:64] = 0
        x[0, :, 48:64, :, 0] = -2.2
        x[1, :, 48:64] *= 2.0**36
    c.write([130] * seqs, "f32", g, change)
    q = torch.randn((seqs * rows, 6, 64), device="cuda", generator=g)
    q[:, :, 0] = 100
    q = q.to(TYPES[kind][0])
    out = B.kv_attention(q, c.pages, c.scales, c.table, c.lens())
    assert ("kv_prompt" in B.last_kernel()) == (seqs > 1 and kind != "f32")
    check_rows(out, q, c, rows, kind)


# ------------------------------------------------------------------ scores beyond what 32 bits tell apart
@pytest.mark.parametrize("seqs", [1, 64])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("log_scale", [14, 18, 22, 26, 40, 80])
def test_kv_attention_large_scores(kind, seqs, log_scale):
    """Scores of 2^17 to 2^83: results stay inside what values there are, and where the largest score stands out it is its token's value."""
    rows, c, scale = 40, Cache(seqs, 5, 2, 64, 16, 52), 2.0**log_scale
    g = fill(c, [260] * seqs, "f32", 9)
    q = torch.randn((seqs * rows, 6, 64), device="cuda", generator=g).to(TYPES[kind][0])
    out, lse = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), scale=scale, lse=True)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    x, got = host(q), host(out)
    for seq in range(seqs):
        kv = c.values(seq).astype(np.float64)
        pos, t = np.arange(260 - rows, 260)[:, None], np.arange(260)[None, :]
        for h in range(6):
            k, v = kv[0, h // 3], kv[1, h // 3]
            mine = slice(seq * rows, seq * rows + rows)
            z = np.where(t <= pos, x[mine, h] @ k.T * scale, -np.inf)
            e = (2.0**-21 + 64 * 2.0**-24) * scale * (np.abs(x[mine, h]) @ np.abs(k).T).max(1)
            order = np.argsort(z, 1)
            gap = np.take_along_axis(z, order[:, -1:], 1)[:, 0] - np.take_along_axis(z, order[:, -2:-1], 1)[:, 0]
            assert (np.abs(got[mine, h]) <= np.abs(v).max() * (1 + 2.0**-7)).all()
            clear = gap > 4 * e + 100
            assert clear.sum() > rows // 4
            want = v[order[:, -1]]
            assert (np.abs(got[mine, h] - want) <= (TYPES[kind][1] + 2.0**-11) * np.abs(want) + 2.0**-25 + 260 * 2.0**-39 * np.abs(v).max())[clear].all()


# ------------------------------------------------------------------ scales of either sign
@pytest.mark.parametrize("seqs", [1, 64])
@pytest.mark.parametrize("kind", list(TYPES))
def test_kv_attention_negative_scales(kind, seqs):
    """A value is its level times its block's scale, whatever the scale's sign."""
    rows, c = 40, Cache(seqs, 4, 2, 64, 16, 53)
    g = fill(c, [230] * seqs, "f32", 10)
    rng = np.random.default_rng(1)
    c.s *= rng.choice([-1.0, 1.0], c.s.shape).astype(np.float32)
    c.s[:, :, :, :6] = -np.abs(c.s[:, :, :, :6])
    table = c.table.cpu().numpy()
    scales = c.scales.cpu().numpy()
    for seq in range(seqs):
        for b in range(-(-230 // 16)):
            scales[table[seq, b // 4], :, :, b % 4] = c.s[seq, :, :, b].T
    c.scales.copy_(torch.from_numpy(scales))
    q = torch.randn((seqs * rows, 6, 64), device="cuda", generator=g).to(TYPES[kind][0])
    for scale in (0.125, -0.3):
        out = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), scale=scale)
        assert ("kv_prompt" in B.last_kernel()) == (seqs > 1 and kind != "f32")
        check_rows(out, q, c, rows, kind, scale=scale)
    k, v = B.kv_read(c.pages, c.scales, c.table, c.lens(), 64, torch.float32, 230 * seqs)
    want = np.concatenate([c.values(i).transpose(0, 2, 1, 3) for i in range(seqs)], 1)
    np.testing.assert_array_equal(torch.stack([k, v]).cpu().numpy(), want)


# ------------------------------------------------------------------ 4-bit products of values that are not finite, or nearly so
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,N,K,group", [(6, 70, 300, 32), (6, 100, 1100, 128), (20, 40, 330, 64), (33, 60, 300, 32), (50, 70, 520, 128), (64, 6200, 200, 64),
                                         (100, 130, 300, 64), (260, 4100, 200, 32), (520, 4200, 200, 64), (1050, 4250, 150, 128), (330, 2100, 300, 64)])
def test_w4_fc_not_finite(M, N, K, group, kind):
    """Infinities of one sign, of both, on weights that are 0, beside a NaN; values whose 31-fold is beyond fp32: what the definition gives, and the
    rows beside them as ever."""
    g = torch.Generator(device="cuda").manual_seed(M)
    tiles = random_tiles(g, N, K, group)[0]
    s = (torch.rand((tiles.shape[0], tiles.shape[1] * 128 // group, 16), device="cuda", generator=g) * 0.01 + 0.001).bfloat16()
    scales = torch.stack([s, -8 * s], -1)  # (level 8 is a weight of 0)
    x = torch.randn((M, K), device="cuda", generator=g).to(TYPES[kind][0])
    top = 65504.0 if kind == "f16" else 2.9e38
    x[0, 3] = float("inf")
    x[1, K - 1] = -float("inf")
    x[2, 5], x[2, K - 2] = float("inf"), -float("inf")
    x[3, 7], x[3, 40] = float("inf"), float("nan")
    x[4, :6] = torch.tensor([top, -top, top, top, -top, top], device="cuda")
    special = list(range(5)) + ([M - 1] if M > 6 else [])
    x[special[-1] if M > 6 else 0, 9] = float("inf")
    bias = torch.randn((N,), device="cuda", generator=g)
    out = B.w4_fc(x, tiles, scales, N, bias=bias)
    q, sc, b = unpack(tiles, scales, N, K)
    w, xs, add = q * sc + b, host(x), host(bias)
    got = host(out)
    u = TYPES[kind][1]
    for r in special:
        with np.errstate(invalid="ignore"):
            terms = xs[r][None] * w
            want = terms.sum(1) + add
            size = np.abs(terms).sum(1) + np.abs(add)
        fine = np.isfinite(want)
        assert (np.isnan(got[r]) == np.isnan(want)).all(), r
        assert (got[r][np.isinf(want)] == want[np.isinf(want)]).all(), r
        if fine.any():
            assert r == 4
            # (results beyond the type's largest value are infinite)
            limit = {"f16": 65504.0, "bf16": 3.3895e38, "f32": 3.4028e38}[kind]
            bound = u * np.abs(want) + K * 2.0**-24 * size + 2.0**-25
            inside = fine & (np.abs(want) + bound < limit)
            assert (np.abs(got[r] - want) <= bound)[inside].all(), r
            assert (np.abs(got[r]) >= limit * (1 - 2.0**-7))[fine & (np.abs(want) - bound > limit)].all()
    rest = [r for r in range(M) if r not in special]
    if rest:
        check_fc(out[rest[:50]], x[rest[:50]], tiles, scales, N, K, kind, bias)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("K", [1, 2, 7, 8, 9, 15, 63, 120, 127, 129, 134, 200, 255, 257, 383])
@pytest.mark.parametrize("M,N", [(10, 40), (30, 50), (40, 70), (64, 33), (100, 64), (9, 6200), (200, 1100)])
def test_w4_fc_rows_that_end_in_a_step(M, N, K, kind):
    """Row lengths that end anywhere in a step of 128 and in eight values, rows on whole dwords and on odd elements, the last of them at the end of
    its memory; what lies behind a row is NaN."""
    g = torch.Generator(device="cuda").manual_seed(K)
    tiles, scales = random_tiles(g, N, K, 64)
    q, s, b = (torch.from_numpy(a).cuda() for a in unpack(tiles, scales, N, K))
    for ld, shift in ((K, 0), (K + 1, 0), (K + 3, 1), (K + (K % 2) + 2, 0), (K + 8, 2)):
        memory = torch.full((M * ld,), float("nan"), device="cuda", dtype=TYPES[kind][0])
        x = memory.as_strided((M, K), (ld, 1), shift if shift + (M - 1) * ld + K <= M * ld else 0)
        x.copy_(torch.randn((M, K), device="cuda", generator=g))
        y = B.w4_fc(x, tiles, scales, N)
        want = x.double() @ (q * s + b).t().contiguous()
        size = x.double().abs() @ (31 * s.abs() + (b - 16 * s).abs()).t().contiguous()
        least = 2.0**-25 if kind == "f16" else 1e-30  # (a float16 is a multiple of 2^-24)
        assert bool(((y.double() - want).abs() <= TYPES[kind][1] * want.abs() + (K / 32 + 64) * 2.0**-24 * size + least).all()), (ld, shift)


@pytest.mark.parametrize("M,N,K,group,kind,pad,kernel", [
    (2, 700, 8192, 128, "bf16", 0, "block 512"), (3, 700, 8192, 128, "bf16", 0, "block 256"), (1, 4113, 8192, 128, "f16", 0, "block 256"),
    (8, 300, 4096, 32, "f32", 0, "block 512"), (9, 300, 4096, 32, "f32", 0, "block 256"), (8, 300, 4000, 32, "f32", 0, "block 256"),
    (9, 12288, 256, 64, "bf16", 0, "few_kernel<2,2"), (32, 12289, 256, 64, "bf16", 0, "deep_kernel"), (16, 12289, 256, 64, "bf16", 0, "rows_kernel"),
    (16, 6145, 260, 64, "f16", 0, "rows_kernel"), (16, 6145, 256, 64, "f16", 1, "deep_kernel"), (16, 6144, 255, 64, "f16", 0, "few_kernel<1,2"),
    (33, 4096, 300, 128, "f16", 0, "few_kernel<1,4"), (33, 4097, 300, 128, "f16", 0, "deep_kernel"), (64, 500, 300, 128, "f16", 1, "deep_kernel"),
    (96, 4096, 512, 64, "f32", 0, "rows_kernel"), (160, 4096, 512, 64, "f32", 0, "f32_kernel"), (160, 2048, 2048, 64, "f32", 0, "rows_kernel")])
def test_w4_fc_on_both_sides_of_each_line(M, N, K, group, kind, pad, kernel):
    """Which kernel takes a call: sizes, types and alignment beside each line, and the kernels' results there."""
    g = torch.Generator(device="cuda").manual_seed(M + K)
    tiles, scales = random_tiles(g, N, K, group)
    x = torch.randn((M, K + pad), device="cuda", generator=g).to(TYPES[kind][0])[:, :K]
    y = B.w4_fc(x, tiles, scales, N)
    assert kernel in B.last_kernel(), B.last_kernel()
    q, s, b = (torch.from_numpy(a).cuda() for a in unpack(tiles, scales, N, K))
    want = x.double() @ (q * s + b).t().contiguous()
    size = x.double().abs() @ (31 * s.abs() + (b - 16 * s).abs()).t().contiguous()
    bound = TYPES[kind][1] * want.abs() + (K / 32 + 64) * 2.0**-24 * size + (2.0**-25 if kind == "f16" else 1e-30)
    assert bool(((y.double() - want).abs() <= bound).all())


def test_kv_rows_of_no_sequence_are_left_alone():
    """Rows before, between and behind those that starts gives out, and rows beyond max_new."""
    c = Cache(3, 2, 2, 64, 16, 60)
    g = fill(c, [70, 5, 30], "bf16", 11)
    starts = torch.tensor([2, 6, 6, 11], dtype=torch.int32, device="cuda")  # (rows 2 to 5, none, 6 to 10)
    q = torch.randn((13, 4, 64), device="cuda", generator=g).bfloat16()
    taken = [2, 3, 4, 6, 7, 8]
    out, k, v = (torch.full((13, h, 64), 7.0, device="cuda", dtype=torch.bfloat16) for h in (4, 2, 2))
    B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), starts=starts, max_new=3, out=out)
    B.kv_read(c.pages, c.scales, c.table, c.lens(), 64, torch.bfloat16, 13, starts=starts, max_new=3, out_k=k, out_v=v)
    for x in (out, k, v):
        rest = [r for r in range(13) if r not in taken]
        assert bool((x[rest] == 7.0).all()) and not bool((x[taken] == 7.0).any())
    q[rest] = float("nan")
    again = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), starts=starts, max_new=3, out=torch.empty_like(out))
    assert torch.equal(again[taken], out[taken])


@pytest.mark.parametrize("seqs", [1, 64])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 20), (False, 0)])
def test_kv_attention_scales_that_are_no_numbers(kind, seqs, causal, window):
    """A block whose scale is NaN or infinite spoils the rows that see it, of keys as of values, and no row beside them in their tile."""
    rows, c = 40, Cache(seqs, 3, 2, 64, 16, 70)
    g = fill(c, [128] * seqs, "f32", 12)
    q = torch.randn((seqs * rows, 6, 64), device="cuda", generator=g).to(TYPES[kind][0])
    args = dict(causal=causal, window=window)
    want = B.kv_attention(q, c.pages, c.scales, c.table, c.lens(), **args)
    assert ("kv_prompt" in B.last_kernel()) == (seqs > 1 and kind != "f32")
    pos = torch.arange(88, 128, device="cuda")
    for which in (0, 1):
        for bad in (float("nan"), float("inf")):
            for block in (7, 6, 5):  # (positions 112 to 127, 96 to 111, 80 to 95)
                scales = c.scales.clone()
                scales[c.table[:, block // 4].long(), 1, which, block % 4] = bad  # (of the second head of the cache)
                out = B.kv_attention(q, c.pages, scales, c.table, c.lens(), **args).unflatten(0, (seqs, rows))
                sees = torch.ones(rows, dtype=torch.bool, device="cuda")
                if causal:
                    sees &= pos >= 16 * block
                if window:
                    sees &= pos - window < 16 * block + 15
                clean = want.unflatten(0, (seqs, rows))
                assert torch.equal(out[:, :, :3], clean[:, :, :3]) and torch.equal(out[:, ~sees], clean[:, ~sees])
                if which == 0 and bad == float("inf"):  # (a score of -infinity is no weight)
                    continue
                assert not bool(torch.isfinite(out[:, sees][:, :, 3:]).all(-1).any())
