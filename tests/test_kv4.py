"""The cache of 4 bits, written, read and attended to, against the definitions in 64 bits on the host."""
import numpy as np
import pytest
import torch

from paper_1705_09864_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
TOP = 2**31 - 1


def row_of(dim):
    return (dim + 31) // 32 * 16


def places(dim):
    """Nibbles of token t, value d: keys and values, [64, dim] each."""
    t, d = np.arange(64)[:, None], np.arange(dim)[None, :]
    k = t * row_of(dim) + d // 2
    v = d // 32 * 1024 + t % 16 // 4 * 256 + d % 32 // 2 * 16 + t // 16 * 4 + t % 4
    return 2 * k + d % 2, 2 * v + d % 2


def unpack(pages, dim):
    """The levels [num_pages, heads, 2, 64, dim] of a cache's pages."""
    b = pages.cpu().numpy()
    nib = np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:3], 2 * b.shape[3])
    return np.stack([nib[:, :, i][..., p] for i, p in enumerate(places(dim))], 2)


class Cache:
    def __init__(self, heads, dim, lengths, seed=0, extra=3, fill=True, num_pages=None, table_pad=0):
        rng = np.random.default_rng(seed)
        self.heads, self.dim, self.lengths = heads, dim, list(lengths)
        each = [max(0, -(-n // 64)) for n in lengths]
        self.num_pages = num_pages or sum(each) + extra
        order = rng.permutation(self.num_pages)
        self.table = np.full((len(lengths), max(each + [1]) + table_pad), 10**6, np.int32)  # (places not in use: no page)
        at = 0
        for i, n in enumerate(each):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.pages, self.scales = B.kv4_cache(self.num_pages, heads, dim)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.pages.random_(0, 256, generator=g)
        if fill:
            s = torch.rand((self.num_pages, heads, 2, 64), device="cuda", generator=g) * 0.2 + 0.2
            self.scales.copy_(torch.stack([s, -s * (7.5 + torch.randn(s.shape, device="cuda", generator=g))], -1))
            # what no sequence holds is no number
            held = torch.zeros((self.num_pages, 64), dtype=torch.bool)
            for i, n in enumerate(lengths):
                for t0 in range(0, max(n, 0), 64):
                    held[self.table[i, t0 // 64], :n - t0] = True
            self.scales.permute(0, 3, 1, 2, 4)[~held.cuda()] = float("nan")
        else:
            self.scales.fill_(float("nan"))
        self.args = (self.pages, self.scales, torch.from_numpy(self.table).cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"))

    def values(self, i, n=None):
        """Sequence i's keys and values [2, heads, tokens, dim] in 64 bits."""
        n = self.lengths[i] if n is None else n
        p = self.table[i, :-(-n // 64)]
        x = unpack(self.pages[torch.from_numpy(p).long().cuda()], self.dim).astype(np.float64)
        s = self.scales[torch.from_numpy(p).long().cuda()].double().cpu().numpy()
        x = x * s[..., :1] + s[..., 1:]
        return x.transpose(2, 1, 0, 3, 4).reshape(2, self.heads, 64 * len(p), self.dim)[:, :, :n]


def starts_of(new):
    return torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).float().numpy()


def quantised(x):
    """Levels, scales and offsets of x [..., dim] by the definition, whose scales are fp32 results rounded to bf16."""
    x = x.float().cpu().numpy()
    low = bf16(x.min(-1))
    step = bf16(np.maximum(x.max(-1) - low, 0).astype(np.float32) / np.float32(15))
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.clip(np.rint((x.astype(np.float64) - low[..., None]) / step[..., None].astype(np.float64)), 0, 15)
    return np.where(step[..., None] > 0, q, 0), step, low


def check_written(cache, before, k, v, new):
    levels, pages, scales = unpack(cache.pages, cache.dim), unpack(before[0], cache.dim), cache.scales.float().cpu().numpy()
    old = before[1].float().cpu().numpy()
    touched = np.zeros(levels.shape[:1] + (64,), bool)
    at = 0
    for i, (n, m) in enumerate(zip(cache.lengths, new)):
        for j in range(m):
            pos = n - m + j
            if pos >= 0:
                page, t = cache.table[i, pos // 64], pos % 64
                touched[page, t] = True
                for which, x in ((0, k), (1, v)):
                    q, step, low = quantised(x[at + j])
                    assert (scales[page, :, which, t, 0] == step).all() and (scales[page, :, which, t, 1] == low).all()
                    got = levels[page, :, which, t].astype(np.float64)
                    # fp32 quotients: (x - low) and its quotient are off by 2^-24 each of at most 15.06 levels
                    exact = np.divide(x[at + j].double().cpu().numpy() - low[:, None], step[:, None], where=step[:, None] > 0, out=np.zeros_like(got))
                    off = np.abs(got - np.clip(exact, 0, 15))
                    assert (off <= 0.5 + 16 * 2.0**-23).all() and (got[off < 0.5 - 16 * 2.0**-23] == q[off < 0.5 - 16 * 2.0**-23]).all()
        at += m
    keep = ~touched
    assert (levels.transpose(0, 3, 1, 2, 4)[keep] == pages.transpose(0, 3, 1, 2, 4)[keep]).all()
    a, b = scales.transpose(0, 3, 1, 2, 4)[keep], old.transpose(0, 3, 1, 2, 4)[keep]
    assert ((a == b) | (np.isnan(a) & np.isnan(b))).all()


DIMS = [1, 2, 15, 31, 32, 33, 64, 80, 96, 100, 127, 128, 160, 200, 224, 255, 256]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("kind", TYPES)
def test_write_and_read(kind, dim):
    heads = 3 if dim < 128 else 2
    for case, (lengths, new) in enumerate([([1], [1]), ([64, 70, 3], [1, 1, 1]), ([200, 9, 64, 0, 130], [200, 9, 10, 0, 66]), ([40, 128], [8, 8]), ([100, 65], [9, 9]),
                                           ([3, 70], [5, 5]), ([2, 20, 90], [20, 20, 20])]):
        cache = Cache(heads, dim, lengths, seed=dim + case)
        rows = sum(new)
        g = torch.Generator(device="cuda").manual_seed(dim)
        gap = case % 3
        whole = torch.randn((rows, 2 * heads * (dim + gap) + case % 2), device="cuda", generator=g).to(kind)
        k, v = (whole[:, o:o + heads * (dim + gap)].unflatten(1, (heads, dim + gap))[..., :dim] for o in (0, heads * (dim + gap)))
        before = cache.pages.clone(), cache.scales.clone()
        ragged = len(set(new)) > 1
        starts = starts_of(new) if ragged or case % 2 else None
        B.kv4_write(k, v, *cache.args, starts=starts, max_new=max(new) if case % 2 else 0)
        check_written(cache, before, k, v, new)
        got = B.kv4_read(*cache.args, dim, kind, rows, starts=starts)
        at = 0
        for i, (n, m) in enumerate(zip(lengths, new)):
            there = min(n, m)
            for x, want in zip(got, cache.values(i)):
                want = np.concatenate([np.zeros((m - there, heads, dim)), want[:, n - there:].transpose(1, 0, 2)])
                x = x[at:at + m].double().cpu().numpy()
                # one fp32 rounding, then the type's
                near = np.abs(want) * (2.0**-24 + (torch.finfo(kind).eps / 2 if kind != torch.float32 else 0)) * 1.01 + torch.finfo(kind).smallest_normal * torch.finfo(kind).eps
                assert (np.abs(x - want) <= near).all()
            at += m


@pytest.mark.parametrize("kind,bits", [(torch.float32, 8), (torch.float16, 6), (torch.bfloat16, 3)])
@pytest.mark.parametrize("new", [1, 70])
def test_halfway_between_two_levels(kind, bits, new):
    """Values that lie exactly between two levels go to the even one, whatever the scale (of so many bits that its multiples by a half are values of the type)."""
    rng = np.random.default_rng(bits)
    cache = Cache(2, 64, [new] * 40, seed=1)
    step = np.ldexp(rng.integers(2**(bits - 1), 2**bits, (40 * new, 2)).astype(np.float64), rng.integers(-8, 3, (40 * new, 2)))
    half = rng.integers(0, 31, (40 * new, 2, 64)) / 2
    half[..., 5], half[..., 60] = 0, 15  # (the least and the largest)
    x = torch.from_numpy(half * step[..., None]).cuda().to(kind)
    assert bool((x.double().cpu() == torch.from_numpy(half * step[..., None])).all())
    B.kv4_write(x, -x, *cache.args)
    levels, scales = unpack(cache.pages, 64), cache.scales.float().cpu().numpy()
    for i in range(40):
        for t in range(new):
            page, r = cache.table[i, t // 64], i * new + t
            assert (scales[page, :, 0, t % 64, 0] == step[r]).all() and not scales[page, :, 0, t % 64, 1].any()
            assert (levels[page, :, 0, t % 64] == np.rint(half[r])).all()
            # (the least is -15 steps, rounded to bf16: exact where it has 8 bits)
            if (bf16(-15 * step[r].astype(np.float32)) == -15 * step[r]).all():
                assert (levels[page, :, 1, t % 64] == np.rint(15 - half[r])).all()


def test_rows_that_are_not_finite():
    """Scales go by what is finite; infinity is the highest level, what is below or no number the lowest; a row of one value, and one without any."""
    for kind in TYPES:
        for rows in (1, 16):
            cache = Cache(1, 64, [rows])
            x = torch.randn((rows, 1, 64), device="cuda").to(kind)
            x[0, 0, 3], x[0, 0, 5], x[0, 0, 60] = float("inf"), float("-inf"), float("nan")
            y = torch.full((rows, 1, 64), 2.5, device="cuda").to(kind)
            if rows > 1:
                x[4], x[5], y[6], y[7] = float("nan"), float("inf"), 0, float("-inf")
            B.kv4_write(x, y, *cache.args)
            levels, scales = unpack(cache.pages, 64)[cache.table[0, 0], 0], cache.scales[cache.table[0, 0], 0].float().cpu().numpy()
            assert np.isfinite(scales[:, :rows]).all()
            f = x[0, 0][torch.isfinite(x[0, 0])]
            q, step, low = quantised(f)
            assert scales[0, 0].tolist() == [step, low] and levels[0, 0][[3, 5, 60]].tolist() == [15, 0, 0]
            assert scales[1, 0].tolist() == [0, 2.5] and not levels[1, 0].any()
            if rows > 1:
                assert not scales[0, 4:6].any() and not scales[1, 6:8].any()
    cache = Cache(1, 32, [2])
    x = torch.zeros((2, 1, 32), device="cuda")
    x[0, 0, 0], x[0, 0, 1], x[1, 0, 2] = 3.4e38, -3.4e38, 1e-45
    B.kv4_write(x, x, *cache.args)
    assert bool(torch.isfinite(cache.scales[cache.table[0, 0], 0, :, :2].float()).all())


@pytest.mark.parametrize("rows", [2, 5, 70])
@pytest.mark.parametrize("below", [0, 1, 63, 64, 130])
def test_lengths_at_the_end_of_32_bits(rows, below):
    """Tokens far behind the table: nothing is written for them, zeros come back, and the sequence beside them is as ever."""
    heads, dim = 2, 64
    pages, scales = B.kv4_cache(5, heads, dim)
    pages.fill_(55)
    scales.fill_(0.5)
    table = torch.tensor([[1, 2], [0, 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([TOP - below, 100], dtype=torch.int32, device="cuda")
    kv = torch.randn((2 * rows, heads, dim), device="cuda")
    B.kv4_write(kv, kv, pages, scales, table, lengths)
    assert bool((pages[[1, 2, 4]] == 55).all()) and bool((scales[[1, 2, 4]] == 0.5).all())
    k, v = B.kv4_read(pages, scales, table, lengths, dim, torch.float32, 2 * rows)
    for x in (k, v):
        # (half a step of at most 10 / 15, and the offset's rounding)
        assert not bool(x[:rows].any()) and float((x[rows:] - kv[rows:]).abs().max()) < 0.4
    out = B.kv4_attention(torch.randn((2 * rows, heads, dim), device="cuda"), pages, scales, table, lengths)
    assert bool(torch.isfinite(out).all())


def check_attention(cache, q, new, got, scale=None, causal=True, window=0, lse=None, there=None):
    """A score is off by (dim + 8) 2^-24 of the sum of its terms' sizes, 24 at most a level as an operand, and its offset; its exponential by that twice, and by 2^-22 of
    log2 e times the score's size; weights by 2^-17 (16-bit types; 2^-24 fp32) of what they multiply, at most 31 scales of the value and its offset; sums over n tokens by
    (n / 32 + 16) 2^-24 of that.  Then the type's rounding."""
    scale = cache.dim**-0.5 if scale is None else scale
    share, at = q.shape[1] // cache.heads, 0
    x, out = q.double().cpu().numpy(), got.double().cpu().numpy()
    eps = torch.finfo(q.dtype).eps / 2
    fine = q.dtype == torch.float32
    worst = 0.0
    for i, (n, m) in enumerate(zip(cache.lengths, new)):
        k, v = cache.values(i)
        pos, t = np.arange(n - m, n)[:, None], np.arange(n)[None]
        see = (t <= pos) if causal else (t < n) & (pos > -TOP)
        if window:
            see = see & (t > pos - window)
        if there is not None:
            see = see & there[i][None, :n]
        p = cache.table[i, :-(-n // 64)].clip(0, cache.num_pages - 1)
        sc = np.nan_to_num(np.abs(cache.scales[torch.from_numpy(p).long().cuda()].double().cpu().numpy())).transpose(2, 1, 0, 3, 4).reshape(2, cache.heads, 64 * len(p), 2)[:, :, :n]
        for h in range(q.shape[1]):
            z = x[at:at + m, h] @ np.nan_to_num(k[h // share]).T * scale
            terms = np.abs(x[at:at + m, h]).sum(1)[:, None] * (31 * sc[0, h // share, :, 0] + sc[0, h // share, :, 1])[None] * abs(scale)
            off_z = (cache.dim + 8) * 2.0**-24 * terms + 2.0**-22 * np.abs(z)
            z = np.where(see, z, -np.inf)
            top = z.max(1, initial=-np.inf, keepdims=True)
            e = np.exp(z - np.where(np.isfinite(top), top, 0))
            total = e.sum(1, keepdims=True)
            w = e / np.where(total > 0, total, 1)
            vh = np.nan_to_num(v[h // share])
            want = w @ vh
            amp = w @ (31 * sc[1, h // share, :, 0] + sc[1, h // share, :, 1])
            off_w = 2 * np.where(see, off_z, 0).max(1, initial=0)
            off = (off_w[:, None] + 2.0**-21) * (w @ np.abs(vh)) + (((2.0**-24 if fine else 2.0**-17) + (n / 32 + 16) * 2.0**-24) * amp)[:, None]
            off = off + eps * (np.abs(want) + off) + torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps
            err = np.abs(out[at:at + m, h] - want)
            assert (err <= off).all(), (i, h, float(err.max()), float(off[err > off].min()), np.argwhere(err > off)[:3].tolist())
            worst = max(worst, float((err / off).max(initial=0)))
            if lse is not None:
                with np.errstate(divide="ignore"):
                    l = np.log(total[:, 0]) + np.where(np.isfinite(top[:, 0]), top[:, 0], 0)
                g = lse[at:at + m, h].double().cpu().numpy()
                none = ~see.any(1)
                assert (g[none] == -np.inf).all()
                assert (np.abs(g[~none] - l[~none]) <= off_w[~none] + 2.0**-20 + 2.0**-22 * np.abs(l[~none])).all()
        at += m
    return worst


def attend(cache, share, new, kind, seed=0, gap=0, **named):
    g = torch.Generator(device="cuda").manual_seed(seed)
    whole = torch.randn((sum(new), cache.heads * share * (cache.dim + gap) + gap % 2), device="cuda", generator=g).to(kind)
    q = whole[:, :cache.heads * share * (cache.dim + gap)].unflatten(1, (cache.heads * share, cache.dim + gap))[..., :cache.dim]
    starts = starts_of(new) if len(set(new)) > 1 or seed % 2 else None
    out, lse = B.kv4_attention(q, *cache.args, starts=starts, max_new=max(new) if seed % 2 else 0, lse=True, **named)
    named.pop("workspace", None)
    return check_attention(cache, q, new, out, lse=lse, **named)


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("kind", TYPES)
def test_attention_dims(kind, dim):
    cache = Cache(2, dim, [100, 1, 64, 333], seed=dim)
    attend(cache, 2, [1, 1, 1, 1], kind, seed=dim)
    attend(cache, 3, [10, 1, 0, 70], kind, seed=dim + 1, gap=dim % 4)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lengths,new", [([1], [1]), ([63], [1]), ([64], [1]), ([65], [1]), ([0, 5], [1, 1]), ([3, 200], [7, 7]), ([1000, 999], [33, 33]), ([129, 0, 64, 500], [129, 0, 1, 3]),
                                         ([4000], [1]), ([2500], [17]), ([700, 40], [40, 40])])
def test_attention_lengths(kind, lengths, new):
    for share in (1, 4, 8):
        cache = Cache(2, 64, lengths, seed=len(lengths) + share)
        attend(cache, share, new, kind, seed=1)
    attend(cache, 8, new, kind, seed=3, causal=False)
    for window in (1, 16, 65, 300):
        attend(cache, 1, new, kind, seed=4, window=window)
        attend(cache, 8, new, kind, seed=5, window=window, causal=False)


@pytest.mark.parametrize("kind", TYPES)
def test_attention_of_many_rows(kind):
    """Prompts, in tiles of rows of one head or of several."""
    for heads, share, dim, lengths, new in ((8, 4, 64, [600, 90], [513, 90]), (2, 8, 128, [300] * 4, [300] * 4), (16, 1, 96, [700], [700]), (4, 6, 32, [1100, 800], [400, 800])):
        cache = Cache(heads, dim, lengths, seed=dim)
        attend(cache, share, new, kind, seed=1)
        attend(cache, share, new, kind, seed=2, window=100)
        attend(cache, share, new, kind, seed=3, causal=False)


@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [20, 32, 64, 80, 96, 128, 150, 192, 224, 255, 256])
def test_prompts_split_and_not(kind, dim):
    """Rows enough for the kernel of 128 rows: with pages split over workgroups (a long table and few tiles), and not; with few rows beside them."""
    cache = Cache(4, dim, [2100], seed=dim)
    for named in (dict(), dict(window=700), dict(causal=False)):
        attend(cache, 8, [520], kind, seed=1, gap=dim % 3, **named)
        assert "prompt" in B.last_kernel()
    cache = Cache(4, dim, [900, 70, 500], seed=dim)
    attend(cache, 8, [400, 3, 500], kind, seed=2, window=90)
    attend(cache, 8, [400, 3, 9], kind, seed=3)


@pytest.mark.parametrize("kind,dim,named", [(torch.bfloat16, 128, {}), (torch.float16, 128, {}), (torch.float16, 96, {}), (torch.bfloat16, 64, dict(causal=False)),
                                            (torch.bfloat16, 20, {}), (torch.float16, 64, dict(window=1000)), (torch.bfloat16, 100, dict(scale=-0.05))])
def test_prompts_in_two_groups(kind, dim, named):
    """Prompts alike and long enough for workgroups whose halves take turns."""
    cache = Cache(8, dim, [1536, 1500], seed=dim)
    attend(cache, 4, [1000, 1000], kind, seed=2, gap=dim % 3, **named)
    assert "prompt_kernel" in B.last_kernel() and "block 512" in B.last_kernel()


@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
def test_two_groups_and_pages_that_are_not_there(kind):
    """More than 64 pages, some of them none, the first and the last among them."""
    cache = Cache(16, 32, [4400], seed=6)
    there = [np.ones(4400, bool)]
    for place, none in ((0, -1), (2, cache.num_pages), (30, TOP), (31, -7), (63, -1), (64, -1), (67, 10**6), (68, -1)):
        cache.table[0, place] = none
        there[0][place * 64:place * 64 + 64] = False
    q = torch.randn((1000, 64, 32), device="cuda").to(kind)
    out = B.kv4_attention(q, *cache.args[:2], torch.from_numpy(cache.table).cuda(), cache.args[3])
    assert "block 512" in B.last_kernel()
    cache.table = np.where((cache.table >= 0) & (cache.table < cache.num_pages), cache.table, 0)
    check_attention(cache, q, [1000], out, there=there)
    # none at all, and no tokens
    for table, lengths in ((torch.full_like(cache.args[2], -1), cache.args[3]), (cache.args[2], torch.zeros_like(cache.args[3]))):
        out, lse = B.kv4_attention(q, *cache.args[:2], table, lengths, lse=True)
        assert not bool(out.any()) and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("which", [0, 1])
def test_scales_that_are_no_numbers_in_two_groups(which):
    """A row that does not see the token is as ever, also where its wave's rows see nothing of the token's page."""
    cache, q = Cache(8, 64, [1536, 1500], seed=4), torch.randn((2000, 32, 64), device="cuda").bfloat16()
    want = B.kv4_attention(q, *cache.args)
    for value in (float("nan"), float("inf")):
        for part in (0, 1):
            kept = cache.scales.clone()
            cache.scales[int(cache.table[0, 1300 // 64]), :, which, 1300 % 64, part] = value
            out = B.kv4_attention(q, *cache.args)
            assert "block 512" in B.last_kernel()
            assert torch.equal(out[:1300 - 536], want[:1300 - 536]) and torch.equal(out[1000:], want[1000:])
            if which or value != value:
                assert not bool(torch.isfinite(out[1300 - 536:1000]).all(-1).any())
            cache.scales.copy_(kept)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.3, 5.0, 1e-6])
def test_attention_scales(kind, scale):
    cache = Cache(2, 64, [300, 70], seed=1)
    attend(cache, 2, [1, 1], kind, seed=1, scale=scale)
    attend(cache, 2, [150, 70], kind, seed=1, scale=scale)
    attend(Cache(4, 64, [600], seed=1), 8, [600], kind, seed=2, scale=scale)


@pytest.mark.parametrize("kind", TYPES)
def test_values_of_uneven_sizes(kind):
    """Tokens whose values are 2^40 as large as others', seen or not, cost these nothing: weights have fp32's range."""
    cache = Cache(1, 64, [400], seed=2)
    n = cache.lengths[0]
    page = torch.from_numpy(cache.table[0].astype(np.int64)).cuda()
    for t in (5, 100, 399):
        cache.scales[page[t // 64], :, 1, t % 64] *= 2.0**(30 if kind != torch.float16 else 10)
    # (rows whose window leaves the large ones out)
    new = [250]
    q = torch.randn((250, 2, 64), device="cuda").to(kind)
    out = B.kv4_attention(q, *cache.args, window=60)
    check_attention(cache, q, new, out, window=60)
    # (their scale alone may be 2^-40 of the others')
    cache = Cache(1, 64, [400], seed=2)
    cache.scales[page, :, 1] *= 2.0**-30
    if kind != torch.float16:
        out = B.kv4_attention(q, *cache.args)
        check_attention(cache, q, new, out)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("new", [[1] * 5, [4] * 5, [30, 0, 1, 300, 2]])
def test_scales_that_are_no_numbers(kind, new):
    """A token's scale or offset that is infinite or no number spoils the rows that see the token (an infinite one of a key may make a score of -infinity), and no others."""
    lengths = [70, 300, 130, 400, 200]
    clean = Cache(4, 64, lengths, seed=9)
    q = torch.randn((sum(new), 32, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(kind)
    want = B.kv4_attention(q, *clean.args, starts=starts_of(new), window=50)
    for which in (0, 1):
        for part, value in ((0, float("nan")), (1, float("nan")), (0, float("inf")), (1, float("-inf"))):
            cache = Cache(4, 64, lengths, seed=9)
            spoilt = [(0, 5), (1, 260), (2, 129), (3, 120), (4, 100)]
            for i, t in spoilt:
                cache.scales[int(cache.table[i, t // 64]), :, which, t % 64, part] = value
            out = B.kv4_attention(q, *cache.args, starts=starts_of(new), window=50)
            at = 0
            for (i, t), n, m in zip(spoilt, lengths, new):
                pos = torch.arange(n - m, n, device="cuda")
                sees = (t <= pos) & (t > pos - 50)
                rows, same = out[at:at + m], want[at:at + m]
                assert (which == 0 and value != value) <= (not bool(torch.isfinite(rows[sees]).any()))
                assert which == 0 or not bool(torch.isfinite(rows[sees]).all(-1).any())
                assert torch.equal(rows[~sees], same[~sees])
                at += m


def test_many_sequences_of_unknown_rows():
    """More tiles of rows, of all sequences together, than 32 bits have room for their numbers: starts alone say how few there are."""
    sequences, rows = 40000, 60000
    pages, scales = B.kv4_cache(3, 1, 32)
    pages.random_(0, 256)
    scales.copy_(torch.tensor([0.2, -1.5], device="cuda"))
    table = torch.ones((sequences, 1), dtype=torch.int32, device="cuda")
    lengths = torch.full((sequences,), 64, dtype=torch.int32, device="cuda")
    starts = torch.zeros((sequences + 1,), dtype=torch.int32, device="cuda")
    starts[sequences:] = 3
    q = torch.randn((rows, 16, 32), device="cuda")
    out = torch.full_like(q, 7)
    B.kv4_attention(q, pages, scales, table, lengths, starts=starts, max_new=900, out=out)
    alone = B.kv4_attention(q[:3], pages, scales, table[:1], lengths[:1])
    assert torch.equal(out[:3], alone) and bool((out[3:] == 7).all())


def test_tokens_that_are_not_there():
    """Places of the table outside the pages: their tokens count for nothing."""
    for kind in TYPES:
        cache = Cache(2, 64, [400, 200], seed=5)
        cache.table[0, 2], cache.table[0, 5], cache.table[1, 0] = -1, cache.num_pages, TOP
        args = cache.args[:2] + (torch.from_numpy(cache.table).cuda(),) + cache.args[3:]
        there = [np.ones(400, bool), np.ones(200, bool)]
        there[0][128:192], there[0][320:384], there[1][:64] = False, False, False
        kept = cache.table.copy()
        cache.table = np.where((kept >= 0) & (kept < cache.num_pages), kept, 0)
        for new in ([1, 1], [90, 90], [300, 200]):
            q = torch.randn((sum(new), 4, 64), device="cuda").to(kind)
            out = B.kv4_attention(q, *args, starts=starts_of(new))
            check_attention(cache, q, new, out, there=there)
        cache.table = kept


def test_far_pages_of_a_large_cache():
    """Pages behind 4 GiB."""
    heads, dim = 8, 128
    cache = Cache(heads, dim, [500, 65], num_pages=70000, seed=7)
    cache.table[0, :8], cache.table[1, :2] = np.arange(69990, 69998), [69999, 65540]
    args = cache.args[:2] + (torch.from_numpy(cache.table).cuda(),) + cache.args[3:]
    cache.args = args
    k, v = (torch.randn((565, heads, dim), device="cuda").bfloat16() for _ in range(2))
    B.kv4_write(k, v, *args, starts=starts_of([500, 65]))
    got = B.kv4_read(*args, dim, torch.float32, 565, starts=starts_of([500, 65]))
    for x, y in zip(got, (k, v)):
        assert float((x - y.float()).abs().max()) < 0.4
    attend(cache, 4, [1, 1], torch.bfloat16)


@pytest.mark.parametrize("kind", TYPES)
def test_a_prefix_shared_by_sequences(kind):
    """Three sequences that begin with the same pages, read on a stream of their own behind the one that made them, one step and one prompt."""
    for lengths, new in (([400, 130, 900], [1, 1, 1]), ([400, 300, 900], [200, 100, 150])):
        cache = Cache(4, 64, lengths, seed=len(new))
        cache.table[1:, :2] = cache.table[0, :2]
        cache.args[2].copy_(torch.from_numpy(cache.table))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            attend(cache, 4, new, kind, seed=7)
        torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("kind", TYPES)
def test_workspace_kept_and_given(kind):
    """Calls of several sizes one after the other on one workspace give what each gives alone, and leave its counters at zero."""
    ws = torch.zeros((B.workspace_bytes(B.OP_KV4_ATTENTION, (4, 100, 2, 8, 64, 0)),), dtype=torch.uint8, device="cuda")
    for seed, (lengths, new) in enumerate([([5000], [1]), ([6000, 10, 3000, 64], [1, 1, 1, 1]), ([4000, 100], [9, 3]), ([6400], [2])]):
        cache = Cache(2, 64, lengths, seed=seed, table_pad=100 - max(-(-n // 64) for n in lengths))
        g = torch.Generator(device="cuda").manual_seed(seed)
        q = torch.randn((sum(new), 8, 64), device="cuda", generator=g).to(kind)
        outs = [B.kv4_attention(q, *cache.args, starts=starts_of(new), workspace=w) for w in (ws, None, ws)]
        check_attention(cache, q, new, outs[0])
        assert all(torch.equal(outs[0], o) for o in outs[1:])
        assert not bool(ws[:65536].any())


def test_rows_of_no_sequence_are_left():
    """Rows behind the last sequence's and beyond max_new: out and cache stay."""
    cache = Cache(2, 64, [100, 50], seed=1)
    starts = starts_of([3, 2])
    for kind in TYPES:
        q = torch.randn((9, 4, 64), device="cuda").to(kind)
        out = torch.full_like(q, 7)
        B.kv4_attention(q, *cache.args, starts=starts, max_new=2, out=out)
        assert bool((out[[2, 5, 6, 7, 8]] == 7).all()) and not bool((out[[0, 1, 3, 4]] == 7).all(-1).any())
        k = torch.full((9, 2, 64), 7.0, device="cuda").to(kind)
        v = k.clone()
        B.kv4_read(*cache.args, 64, kind, 9, starts=starts, max_new=2, out_k=k, out_v=v)
        assert bool((k[[2, 5, 6, 7, 8]] == 7).all()) and bool((v[[2, 5, 6, 7, 8]] == 7).all())


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_captured_and_replayed(kind):
    """A step's write and attention in a graph: lengths and table are those of the time, eager work between the replays."""
    cache = Cache(2, 64, [3000, 70], seed=3)
    k, v = (torch.randn((2, 2, 64), device="cuda").to(kind) for _ in range(2))
    q = torch.randn((2, 8, 64), device="cuda").to(kind)
    out = torch.empty_like(q)
    ws = torch.zeros((B.workspace_bytes(B.OP_KV4_ATTENTION, (2, cache.table.shape[1], 2, 8, 64, 1)),), dtype=torch.uint8, device="cuda")

    def step():
        B.kv4_write(k, v, *cache.args)
        B.kv4_attention(q, *cache.args, out=out, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in ([2999, 1], [2001, 65], [128, 64], [1, 70]):
        cache.lengths = n
        cache.args[3].copy_(torch.tensor(n, dtype=torch.int32))
        for x in (k, v, q):
            x.normal_()
        torch.zeros(5000, device="cuda").sum().item()
        graph.replay()
        check_attention(cache, q, [1, 1], out)
        eager = B.kv4_attention(q, *cache.args)
        assert torch.equal(eager, out)
