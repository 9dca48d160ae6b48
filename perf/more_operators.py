"""More operators of a decoder layer in few bits, as cases that can be measured.

A case is a dict of plain values with an "op":
  pages   sequences grow, end and are taken back: lengths, the table of pages, the pool of free ones and the new rows' places (kv_resize)
  rotary  heads rotated by their tokens' positions (rotary)
  cache   new tokens' keys and values into a paged cache of 4 bits, the last of them read back (kv4_write, kv4_read)
  attend  attention of new tokens over such a cache (kv4_attention)

`own` chooses between the operators' plain form, written with elementary torch operations, and the calls of this framework.  Both
read and leave a cache, a table and a pool in the framework's layouts (include/bmx.h).
"""
import math

import torch

own = False

PAGE = 64  # tokens of a page of the cache
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # a step of 64 sequences, a token each, which the next pass takes back: as a proposal that is refused
        {"name": "pages_step", "op": "pages", "seqs": 64, "lo": 1, "hi": 4096, "width": 80, "grow": 1, "ended": 0},
        # a server's turn: of 300 sequences every other one is put aside and the others come back with prompts of uneven lengths
        {"name": "pages_turn", "op": "pages", "seqs": 300, "lo": 0, "hi": 4000, "width": 130, "grow": 4000, "ended": 2},
        # queries and keys of a step of 64 sequences, out of a projection's rows
        {"name": "rotary_step", "op": "rotary", "rows": 64, "heads": 40, "others": 8, "dim": 128, "rot": 128, "interleaved": False, "type": "bf16",
         "far": 4096, "factor": 1.0, "inverse": False},
        # those of prompts: bound by memory
        {"name": "rotary_prompt", "op": "rotary", "rows": 8192, "heads": 40, "others": 8, "dim": 128, "rot": 128, "interleaved": False, "type": "bf16",
         "far": 8192, "factor": 1.0, "inverse": False},
        # far positions with a factor on the result, neighbours as pairs, part of a head, the gradient's way
        {"name": "rotary_far", "op": "rotary", "rows": 1501, "heads": 12, "others": 0, "dim": 80, "rot": 32, "interleaved": True, "type": "f32",
         "far": 1000000, "factor": 1.2, "inverse": True},
        # a step of 64 sequences: a token each goes in, and the last page's worth comes back
        {"name": "cache4_step", "op": "cache", "seqs": 64, "lo": 1, "hi": 2048, "new": 1, "ragged": False, "read": 64, "heads": 8, "dim": 128,
         "type": "bf16"},
        # prompts of uneven lengths go in and come back whole
        {"name": "cache4_prompt", "op": "cache", "seqs": 5, "lo": 500, "hi": 4096, "new": 4096, "ragged": True, "read": 4096, "heads": 8, "dim": 128,
         "type": "f16"},
        # one token of one short sequence, every head with a cache of its own, the framework's own type
        {"name": "attend4_short", "op": "attend", "seqs": 1, "lo": 100, "hi": 100, "new": 1, "ragged": False, "heads": 8, "share": 1, "dim": 64,
         "window": 0, "type": "f32"},
        # a step of 64 sequences of uneven lengths, four heads to a head of the cache
        {"name": "attend4_batch", "op": "attend", "seqs": 64, "lo": 0, "hi": 4096, "new": 1, "ragged": False, "heads": 32, "share": 4, "dim": 128,
         "window": 0, "type": "bf16"},
        # one token over a long document: the cache's bytes, split over the chip
        {"name": "attend4_long", "op": "attend", "seqs": 1, "lo": 131072, "hi": 131072, "new": 1, "ragged": False, "heads": 32, "share": 4, "dim": 128,
         "window": 0, "type": "bf16"},
        # some proposed tokens for each of a few sequences, a window, a row length that is no power of two
        {"name": "attend4_few", "op": "attend", "seqs": 6, "lo": 3, "hi": 5000, "new": 5, "ragged": True, "heads": 12, "share": 6, "dim": 96,
         "window": 1000, "type": "f16"},
        # the second half of two prompts over the whole of them: bound by the matrix cores
        {"name": "attend4_prompt", "op": "attend", "seqs": 2, "lo": 4096, "hi": 4096, "new": 2048, "ragged": False, "heads": 32, "share": 4, "dim": 128,
         "window": 0, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, its logarithm spread evenly."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pages", "rotary", "rotary", "cache", "attend", "attend", "attend"])
    kind = rng.choice(["f32", "f16", "bf16", "bf16"])
    if op == "pages":
        while True:
            hi = _log(rng, 1, 20000)
            c = {"op": op, "seqs": _log(rng, 1, 3000), "lo": rng.randint(0, hi), "hi": hi, "width": 0,
                 "grow": rng.choice([1, _log(rng, 1, 16), _log(rng, 1, 8192)]), "ended": rng.choice([0, 2, 3, 16])}
            c["width"] = (hi + c["grow"] + PAGE - 1) // PAGE + rng.randint(0, 20)
            if c["seqs"] * c["grow"] <= 1 << 20 and c["seqs"] * c["width"] <= 1 << 18 and (not c["ended"] or c["seqs"] // c["ended"] * hi <= 1 << 20):
                return c
    if op == "rotary":
        while True:
            dim = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256, 2 * rng.randint(1, 128)])
            c = {"op": op, "rows": _log(rng, 1, 16384), "heads": rng.choice([1, 2, 5, 10, 20, 40, 72]), "others": rng.choice([0, 0, 1, 8]), "dim": dim,
                 "rot": rng.choice([dim, dim, dim // 4 * 2 or 2, 2 * rng.randint(1, dim // 2)]), "interleaved": rng.random() < 0.4, "type": kind,
                 "far": _log(rng, 1, 1 << 24), "factor": rng.choice([1.0, 1.0, round(rng.uniform(0.5, 1.5), 3)]), "inverse": rng.random() < 0.3}
            if c["rows"] * c["heads"] * dim <= 1 << 25:
                return c
    dim, share = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 256]), rng.choice([1, 2, 4, 6, 8])
    if op == "cache":
        while True:
            hi = _log(rng, 16, 4096)
            c = {"op": op, "seqs": _log(rng, 1, 128), "lo": rng.randint(0, hi), "hi": hi, "new": rng.choice([1, 1, _log(rng, 2, 16), hi]),
                 "ragged": rng.random() < 0.5, "read": _log(rng, 1, hi), "heads": rng.choice([1, 2, 4, 8, 8, 16]), "dim": dim, "type": kind}
            if c["seqs"] * (c["new"] + c["read"]) * c["heads"] * dim <= 1 << 25 and c["seqs"] * hi * c["heads"] * dim <= 1 << 28:
                return c
    while True:
        hi = _log(rng, 16, 131072)
        lo = rng.choice([hi, rng.randint(0, hi)])
        c = {"op": op, "seqs": _log(rng, 1, 128), "lo": lo, "hi": hi, "new": rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 17, 2048)]),
             "ragged": rng.random() < 0.4, "heads": rng.choice([1, 2, 4, 8]) * share, "share": share, "dim": dim,
             "window": rng.choice([0, 0, 0, _log(rng, 16, 4096)]), "type": kind}
        if (c["seqs"] * hi * c["heads"] // share * dim <= 1 << 27 and c["seqs"] * c["new"] * hi * c["heads"] * dim <= 1 << 36 and
                c["seqs"] * c["new"] * hi * c["heads"] <= 1 << 29 and c["seqs"] * c["new"] * c["heads"] * dim <= 1 << 25):
            return c


def _lengths(case):
    """Each sequence's tokens in the cache, the new ones among them, and how many are new.  They follow from the case alone."""
    seqs, lo, hi = case["seqs"], case["lo"], case["hi"]
    total = [lo + int(((i + 1) * 0.6180339887 + 0.35) % 1.0 * (hi - lo + 1)) for i in range(seqs)]
    # (a ragged batch: the whole length or a share of it; otherwise as many for each, be the sequence shorter or not)
    new = [min(n, max(1, int(case["new"] * (0.25 + ((i + 1) * 0.754877666) % 0.75)))) if case["ragged"] else case["new"]
           for i, n in enumerate(total)]
    if case["op"] == "cache" and case["ragged"] and case["new"] >= hi:
        new = list(total)
    if not sum(new):
        new[0] = 1
    return total, new


def _changes(case):
    """Each sequence's tokens at first, and by how many tokens they change in the first pass (in the next one by as many the other way)."""
    seqs, lo, hi = case["seqs"], case["lo"], case["hi"]
    held = [lo + int(((i + 1) * 0.6180339887 + 0.35) % 1.0 * (hi - lo + 1)) for i in range(seqs)]
    out = []
    for i, n in enumerate(held):
        if case["ended"] and i % case["ended"] == 0:
            out.append(-n)
        else:
            out.append(case["grow"] if case["grow"] < 16 else 1 + int(((i + 1) * 0.754877666) % 1.0 * (case["grow"] - 1)))
    return held, out


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _read(case):
    """How many of each sequence's last tokens are read back."""
    return [min(n, case["read"]) for n in _lengths(case)[0]]


def _row(dim):
    """Bytes that a token's head takes in a page."""
    return (dim + 31) // 32 * 16


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _prepare_pages(case, g, s):
    held, change = _changes(case)
    used = sum(_pages(n) for n in held)
    # as many pages as either state needs
    count = max(used, sum(_pages(n + c) for n, c in zip(held, change))) + 5
    order = torch.randperm(count, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros((case["seqs"], case["width"]), dtype=torch.int32)
    where = torch.full((case["seqs"], case["width"]), -1, dtype=torch.int64)
    at = 0
    for i, n in enumerate(held):
        where[i, :_pages(n)] = torch.arange(at, at + _pages(n))
        at += _pages(n)
    where = where.cuda()
    s["table"] = torch.where(where >= 0, order[where.clamp(min=0)], torch.zeros_like(table.cuda())).contiguous()
    s["lengths"] = torch.tensor(held, dtype=torch.int32, device="cuda")
    s["pool"] = torch.zeros((count + 2,), dtype=torch.int32, device="cuda")
    s["pool"][0] = count - used
    s["pool"][2:2 + count - used] = order[used:]
    s["change"] = [torch.tensor([k * c for c in change], dtype=torch.int32, device="cuda") for k in (1, -1)]
    s["rows"] = max(1, sum(max(c, 0) for c in change), sum(max(-c, 0) for c in change))
    s["turn"] = 0
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["op"] == "pages":
        return _prepare_pages(case, g, s)
    kind = TYPES[case["type"]]
    if case["op"] == "rotary":
        rows, heads, dim, rot = case["rows"], case["heads"], case["dim"], case["rot"]
        whole = torch.randn((rows, (heads + case["others"]) * dim), device="cuda", generator=g).to(kind)
        s["x"] = whole[:, :heads * dim].unflatten(1, (heads, dim))
        s["positions"] = torch.randint(0, case["far"], (rows,), device="cuda", generator=g, dtype=torch.int32)
        s["freq"] = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        return s
    total, new = _lengths(case)
    heads = case["heads"] // case.get("share", 1)
    dim, row = case["dim"], _row(case["dim"])
    rows = sum(new)
    most = max(1, max(_pages(n) for n in total))
    used = sum(_pages(n) for n in total)
    count = used + 3
    # a page goes to one sequence, in no order
    order = torch.randperm(count, device="cuda", generator=g).to(torch.int32)
    where = torch.full((len(total), most), -1, dtype=torch.int64)
    at = 0
    for i, n in enumerate(total):
        where[i, :_pages(n)] = torch.arange(at, at + _pages(n))
        at += _pages(n)
    where = where.cuda()
    s["table"] = torch.where(where >= 0, order[where.clamp(min=0)], torch.zeros_like(where, dtype=torch.int32)).contiguous()
    s["lengths"] = torch.tensor(total, dtype=torch.int32, device="cuda")
    s["starts"] = _starts(new) if case["ragged"] else None
    s["rows"], s["most_new"] = rows, max(new)
    # levels of normal values between the least and the largest of a token
    shape = (count, heads, 2, PAGE * row)
    lo = (torch.randn(shape, device="cuda", generator=g) * 3 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
    s["pages"] = lo + (torch.randn(shape, device="cuda", generator=g) * 3 + 7.5).round_().clamp_(0, 15).to(torch.uint8) * 16
    step = torch.rand((count, heads, 2, PAGE), device="cuda", generator=g) * 0.2 + 0.25
    s["scales"] = torch.stack([step, -step * (7.5 + 0.5 * torch.randn(step.shape, device="cuda", generator=g))], -1).to(torch.bfloat16)
    # queries, keys and values are parts of one projection's rows
    mine = case["heads"]
    if case["op"] == "cache":
        both = torch.randn((rows, 2 * heads * dim), device="cuda", generator=g).to(kind)
        s["k"] = both[:, : heads * dim].unflatten(1, (heads, dim))
        s["v"] = both[:, heads * dim :].unflatten(1, (heads, dim))
        count_read = _read(case)
        s["read_rows"], s["most_read"] = sum(count_read), max(count_read)
        s["read_starts"] = _starts(count_read)
    else:
        both = torch.randn((rows, (mine + 2 * heads) * dim), device="cuda", generator=g).to(kind)
        s["q"] = both[:, : mine * dim].unflatten(1, (mine, dim))
        # scratch memory that a program keeps from call to call
        s["scratch"] = torch.zeros((64 << 20,), dtype=torch.uint8, device="cuda")
    return s


def work(case):
    if case["op"] == "pages":
        held, change = _changes(case)
        moved = sum(abs(_pages(n + c) - _pages(n)) for n, c in zip(held, change))
        rows = (sum(max(c, 0) for c in change) + sum(max(-c, 0) for c in change)) / 2
        return {"bytes": 16 * case["seqs"] + 8 * moved + 12 * rows, "flops": 0.0}
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "rotary":
        values = case["rows"] * case["heads"] * case["dim"]
        return {"bytes": 2 * values * size + 4 * case["rows"] + 4 * case["rot"], "flops": 3.0 * case["rows"] * case["heads"] * case["rot"]}
    total, new = _lengths(case)
    heads, dim = case["heads"] // case.get("share", 1), case["dim"]
    if case["op"] == "cache":
        into, back = sum(min(a, b) for a, b in zip(total, new)), sum(_read(case))
        return {"bytes": (into + back) * 2 * heads * (dim * (size + 0.5) + 4), "flops": 4.0 * heads * dim * (into + back)}
    seen = pairs = 0
    for n, m in zip(total, new):
        w = case["window"] or n
        q = min(n, m)  # the rows that see anything
        first = max(0, n - q - w + 1)
        seen += n - first if q else 0
        full = max(0, min(q, n - max(n - q, w - 1)))  # rows that see a whole window
        pairs += full * w + sum(range(n - q + 1, n - full + 1))
    rows = sum(new)
    return {"bytes": seen * heads * 2 * (dim / 2 + 4) + 2 * rows * case["heads"] * dim * size, "flops": 4.0 * pairs * case["heads"] * dim}


# ------------------------------------------------------------------ plain forms
def _resize(s, change):
    table, lengths, pool = s["table"], s["lengths"], s["pool"]
    seqs, width = table.shape
    old = lengths.long()
    new = old + change.long()
    p_old, p_new = (old + PAGE - 1) // PAGE, (new + PAGE - 1) // PAGE
    back, take, more = (p_old - p_new).clamp(min=0), (p_new - p_old).clamp(min=0), change.long().clamp(min=0)
    free = pool[0].long()
    bad = (new < 0) | (new > PAGE * width) | (take.cumsum(0) > free + back.sum()) | (more.cumsum(0) > s["rows"])
    ok = ~bad.any()
    status = torch.where(ok, 0, bad.int().argmax() + 1)
    stack = torch.cat([pool[2:], pool.new_zeros(1)])  # (one place more for what goes nowhere)
    place, nowhere = torch.arange(width, device="cuda")[None, :], stack.numel() - 1
    gone = (place >= p_new[:, None]) & (place < p_old[:, None])
    at = free + (back.cumsum(0) - back)[:, None] + p_old[:, None] - 1 - place
    pushed = stack.scatter(0, torch.where(gone & ok, at, nowhere).flatten(), table.flatten())
    got = (place >= p_old[:, None]) & (place < p_new[:, None]) & ok
    at = free + back.sum() - 1 - ((take.cumsum(0) - take)[:, None] + place - p_old[:, None])
    s["table"].copy_(torch.where(got, pushed[torch.where(got, at, nowhere)], table))
    pool[2:] = pushed[:-1]
    pool[0] = torch.where(ok, free + back.sum() - take.sum(), free)
    pool[1] = status
    more = torch.where(ok, more, 0)
    starts = torch.cat([more.new_zeros(1), more.cumsum(0)])
    s["lengths"].copy_(torch.where(ok, new, old))
    r = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(starts[1:], r, right=True)
    there = seq < seqs
    seq = seq.clamp(max=seqs - 1)
    pos = torch.where(there, old[seq] + r - starts[seq], -1)
    page = s["table"][seq, (pos // PAGE).clamp(min=0)].long()
    return starts.int(), pos.int(), torch.where(there, page * PAGE + pos % PAGE, -1)


def _rotary(s):
    x, rot = s["x"], s["rot"]
    angle = s["positions"].double()[:, None] * s["freq"]
    c, d = (angle.cos() * s["factor"]).float()[:, None], (angle.sin() * (-s["factor"] if s["inverse"] else s["factor"])).float()[:, None]
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if s["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * c - b * d, b * c + a * d
    turned = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _places(dim):
    """Where a page holds token t, value d, as nibbles: for keys and for values, [64, dim] each."""
    row = _row(dim)
    t, d = torch.arange(PAGE, device="cuda")[:, None], torch.arange(dim, device="cuda")[None, :]
    k = t * row + d // 2
    v = d // 32 * 1024 + t % 16 // 4 * 256 + d % 32 // 2 * 16 + t // 16 * 4 + t % 4
    return 2 * k + d % 2, 2 * v + d % 2


def _rows(starts, rows, lengths):
    """For each row: its sequence, its position, and the position of the sequence's first new row."""
    seqs = lengths.numel()
    r = torch.arange(rows, device="cuda")
    if starts is None:
        each = rows // seqs
        seq = r // each
        first = lengths.long() - each
        return seq, first[seq] + r - seq * each, first[seq]
    seq = torch.bucketize(r, starts[1:].long(), right=True)
    first = lengths.long() - (starts[1:] - starts[:-1]).long()
    return seq, first[seq] + r - starts.long()[seq], first[seq]


def _write(s):
    pages, scales, table, dim = s["pages"], s["scales"], s["table"].long(), s["dim"]
    seq, pos, _ = _rows(s["starts"], s["rows"], s["lengths"])
    live = pos >= 0
    page, t = table[seq[live], pos[live] // PAGE], pos[live] % PAGE
    heads = torch.arange(scales.shape[1], device="cuda")
    for which, x in ((0, s["k"]), (1, s["v"])):
        x = x[live].float()
        low = x.amin(2).to(torch.bfloat16)
        step = ((x.amax(2) - low.float()) / 15).to(torch.bfloat16)
        scales[page[:, None], heads, which, t[:, None]] = torch.stack([step, low], -1)
        wide = step.float()[..., None]
        q = torch.where(wide > 0, (x - low.float()[..., None]) / wide, torch.zeros_like(x)).round().clamp(0, 15).to(torch.uint8)
        if dim % 2:
            q = torch.cat([q, torch.zeros_like(q[..., :1])], -1)
        at = _places(dim)[which][:, ::2] // 2
        pages[page[:, None, None], heads[:, None], which, at[t][:, None]] = q[..., ::2] + 16 * q[..., 1::2]
    return scales


def _nibbles(body, at):
    """The levels at these places of the last axis."""
    return body[..., at // 2] >> (at % 2 * 4).to(torch.uint8) & 15


def _read_back(s):
    seq, pos, _ = _rows(s["read_starts"], s["read_rows"], s["lengths"])
    page, t = s["table"].long()[seq, pos // PAGE], pos % PAGE
    got = []
    for which in (0, 1):
        at = _places(s["dim"])[which][t]
        q = s["pages"][:, :, which][page[:, None], :, at // 2] >> (at % 2 * 4).to(torch.uint8)[..., None] & 15
        sc = s["scales"][page, :, which, t].float()
        got.append((q.transpose(1, 2).float() * sc[..., :1] + sc[..., 1:]).to(s["k"].dtype))
    return got


def _attend(s):
    q, lengths, dim, share = s["q"], s["lengths"].long(), s["dim"], s["share"]
    seqs, most = s["table"].shape
    heads = s["heads"] // share
    mine = s["pages"][s["table"].long()]  # [sequences, pages, heads, 2, bytes]
    sc = s["scales"][s["table"].long()].float()
    kv = []
    for which in (0, 1):
        x = _nibbles(mine[:, :, :, which], _places(dim)[which].reshape(-1)).unflatten(-1, (PAGE, dim)).float()
        x = x * sc[:, :, :, which, :, :1] + sc[:, :, :, which, :, 1:]
        kv.append(x.transpose(1, 2).reshape(seqs, heads, most * PAGE, dim))
    rows, (seq, pos, first) = s["rows"], _rows(s["starts"], s["rows"], s["lengths"])
    each = s["most_new"]
    j = pos - first
    wide = torch.zeros((seqs, each, s["heads"], dim), device="cuda")
    wide[seq, j] = q.float()
    wide = wide.view(seqs, each, heads, share, dim).permute(0, 2, 1, 3, 4).reshape(seqs, heads, each * share, dim)
    new = torch.bincount(seq, minlength=seqs)
    scores = (wide @ kv[0].transpose(2, 3).contiguous()) * dim**-0.5
    at = torch.arange(most * PAGE, device="cuda")
    here = (lengths - new)[:, None] + torch.arange(each, device="cuda")  # positions of the rows
    see = (at <= here[..., None]) & (at < lengths[:, None, None])
    if s["window"]:
        see = see & (at > here[..., None] - s["window"])
    see = see.repeat_interleave(share, 1)[:, None]
    scores = torch.where(see, scores, torch.full_like(scores, -math.inf))
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    out = (e @ kv[1]) / torch.where(total > 0, total, torch.ones_like(total))
    out = out.view(seqs, heads, each, share, dim).permute(0, 2, 1, 3, 4).reshape(seqs, each, s["heads"], dim)
    return out[seq, j].to(q.dtype).view(rows, s["heads"], dim)


def run(s):
    if s["op"] == "pages":  # (every other pass goes back)
        change = s["change"][s["turn"]]
        s["turn"] = 1 - s["turn"]
        if own:
            from paper_1705_09864_amd import binding as B
            starts, positions, slots = B.kv_resize(change, s["table"], s["lengths"], s["pool"], rows=s["rows"])
        else:
            starts, positions, slots = _resize(s, change)
        return {"table": s["table"], "lengths": s["lengths"], "pool": s["pool"], "starts": starts, "positions": positions, "slots": slots}
    if not own:
        if s["op"] == "rotary":
            return _rotary(s)
        if s["op"] == "cache":
            scales = _write(s)
            k, v = _read_back(s)
            return {"scales": scales, "k": k, "v": v}
        return _attend(s)
    from paper_1705_09864_amd import binding as B
    if s["op"] == "rotary":
        return B.rotary(s["x"], s["positions"], s["freq"], interleaved=s["interleaved"], factor=s["factor"], inverse=s["inverse"])
    if s["op"] == "cache":
        B.kv4_write(s["k"], s["v"], s["pages"], s["scales"], s["table"], s["lengths"], starts=s["starts"], max_new=s["most_new"])
        k, v = B.kv4_read(s["pages"], s["scales"], s["table"], s["lengths"], s["dim"], s["k"].dtype, rows=s["read_rows"],
                          starts=s["read_starts"], max_new=s["most_read"])
        return {"scales": s["scales"], "k": k, "v": v}
    return B.kv4_attention(s["q"], s["pages"], s["scales"], s["table"], s["lengths"], starts=s["starts"], max_new=s["most_new"],
                           window=s["window"], workspace=s["scratch"])


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_pages(s):
    """The pool as a list: pages go onto its end and come from there."""
    change, table, n = s["change"][0].tolist(), s["table"].cpu(), s["lengths"].tolist()
    pool = s["pool"].tolist()
    free, stack = pool[0], pool[2:]
    need = [_pages(a + c) - _pages(a) for a, c in zip(n, change)]
    for i, k in enumerate(need):
        for place in range(_pages(n[i]) - 1, _pages(n[i]) - 1 + min(k, 0), -1):
            stack[free] = int(table[i, place])
            free += 1
    starts, positions, slots = [0], [], []
    for i, k in enumerate(need):
        for place in range(_pages(n[i]), _pages(n[i]) + max(k, 0)):
            free -= 1
            table[i, place] = stack[free]
        pos = torch.arange(n[i], n[i] + max(change[i], 0))
        starts.append(starts[-1] + pos.numel())
        positions.append(pos)
        slots.append(table[i].long()[pos // PAGE] * PAGE + pos % PAGE)
    rest = [torch.full((s["rows"] - starts[-1],), -1)]
    out = {"table": table, "lengths": torch.tensor([a + c for a, c in zip(n, change)]), "pool": torch.tensor([free, 0] + stack),
           "starts": torch.tensor(starts), "positions": torch.cat(positions + rest), "slots": torch.cat(slots + rest)}
    return {name: t.to(torch.int64 if name == "slots" else torch.int32).cuda() for name, t in out.items()}


def _exact_rotary(s):
    """Each pair as a complex number times that of its angle."""
    x, rot = s["x"].double(), s["rot"]
    turn = torch.polar(torch.full((1, 1), s["factor"], dtype=torch.float64, device="cuda"),
                       (-1 if s["inverse"] else 1) * s["positions"].double()[:, None] * s["freq"][None])
    first = torch.arange(0, rot, 2, device="cuda") if s["interleaved"] else torch.arange(rot // 2, device="cuda")
    second = first + (1 if s["interleaved"] else rot // 2)
    z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_cache(s, i, tokens):
    """The first `tokens` keys and values of sequence i [heads, tokens, dim], by taking a page's axes apart."""
    row, dim, got = _row(s["dim"]), s["dim"], []
    p = s["table"][i, :_pages(tokens)].long()
    for which in (0, 1):
        body = s["pages"][p, :, which]  # [pages, heads, bytes]
        n, heads = body.shape[:2]
        two = torch.stack([body % 16, body // 16], -1)
        if which == 0:
            x = two.reshape(n, heads, PAGE, 2 * row)
        else:  # 32 values, four tokens, a pair of values, 16 tokens, token, value
            x = two.reshape(n, heads, row // 16, 4, 16, 4, 4, 2).permute(0, 1, 5, 3, 6, 2, 4, 7).reshape(n, heads, PAGE, 2 * row)
        sc = s["scales"][p, :, which].double()
        x = x[..., :dim].double() * sc[..., :1] + sc[..., 1:]
        got.append(x.transpose(0, 1).reshape(heads, n * PAGE, dim)[:, :tokens])
    return got


def _exact_write_read(s):
    total, new = _lengths(s)
    back, at, scales = {"k": [], "v": []}, 0, s["scales"].double()
    for i, (n, m) in enumerate(zip(total, new)):
        lost, m = max(0, m - n), min(n, m)
        x = [s[name][at + lost : at + lost + m].double().transpose(0, 1) for name in ("k", "v")]
        at += lost + m
        keep = min(n, s["read"])
        if not n:
            continue
        pos = torch.arange(n - m, n, device="cuda")
        page = s["table"][i].long()[pos // PAGE]
        for which, value in enumerate(_exact_cache(s, i, n)):
            y = x[which]
            if m:
                low = y.amin(2, keepdim=True).to(torch.bfloat16).double()
                step = ((y.amax(2, keepdim=True) - low) / 15).to(torch.bfloat16).double()
                level = torch.where(step > 0, (y - low) / step, torch.zeros_like(y)).round().clamp(0, 15)
                value[:, n - m :] = level * step + low
                scales[page, :, which, pos % PAGE] = torch.cat([step, low], -1).transpose(0, 1)
            back["kv"[which]].append(value[:, n - keep :].transpose(0, 1))
    none = [torch.zeros((0, s["pages"].shape[1], s["dim"]), dtype=torch.float64, device="cuda")]
    return {"scales": scales, "k": torch.cat(back["k"] or none), "v": torch.cat(back["v"] or none)}


def _exact_attend(s):
    total, new = _lengths(s)
    share, out, at = s["share"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    for i, (n, m) in enumerate(zip(total, new)):
        if n:
            k, v = _exact_cache(s, i, n)
            pos = torch.arange(n - m, n, device="cuda")
            key = torch.arange(n, device="cuda")
            hide = key[None, :] > pos[:, None]
            if s["window"]:
                hide = hide | (key[None, :] <= pos[:, None] - s["window"])
            some = ~hide.all(1)
            for h in range(s["heads"]):
                z = s["q"][at : at + m, h].double() @ k[h // share].t().contiguous() / math.sqrt(s["dim"])
                z = z.masked_fill(hide, -math.inf)[some]
                out[at : at + m, h][some] = torch.softmax(z, -1) @ v[h // share]
        at += m
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "pages":
        return _exact_pages(s)
    if case["op"] == "rotary":
        return _exact_rotary(s)
    return _exact_write_read(s) if case["op"] == "cache" else _exact_attend(s)
