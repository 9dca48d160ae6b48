"""Pages on the GPU (kv_resize) against lists: sequences that grow, end, go back, and calls that are refused."""
import numpy as np
import pytest
import torch

from paper_1705_09864_amd import binding as B

pytestmark = pytest.mark.gpu
TOP = 2**31 - 1


def pages(n):
    return -(-n // 64)


class Lists:
    """The definition, on the host."""

    def __init__(self, sequences, width, num_pages, rng=None):
        self.table = np.full((sequences, width), -7, np.int64)
        self.lengths = [0] * sequences
        order = list(range(num_pages - 1, -1, -1))
        if rng is not None:
            rng.shuffle(order)
        self.free, self.stack, self.num_pages = num_pages, order, num_pages

    def resize(self, change, rows):
        sequences, width = self.table.shape
        need = [pages(max(n + c, 0)) - pages(n) for n, c in zip(self.lengths, change)]
        room, taken, new, status = self.free - sum(min(k, 0) for k in need), 0, 0, 0
        for i, (n, c, k) in enumerate(zip(self.lengths, change, need)):
            taken, new = taken + max(k, 0), new + max(c, 0)
            if not 0 <= n + c <= 64 * width or taken > room or new > rows:
                status = i + 1
                break
        starts, positions, slots = [0] * (sequences + 1), [-1] * rows, [-1] * rows
        self.status = status
        if not status:
            for i, k in enumerate(need):
                for place in range(pages(self.lengths[i]) - 1, pages(self.lengths[i]) - 1 + min(k, 0), -1):
                    self.stack[self.free] = int(self.table[i, place])
                    self.free += 1
            r = 0
            for i, (c, k) in enumerate(zip(change, need)):
                n = self.lengths[i]
                for place in range(pages(n), pages(n) + max(k, 0)):
                    self.free -= 1
                    self.table[i, place] = self.stack[self.free]
                for pos in range(n, n + max(c, 0)):
                    positions[r], slots[r] = pos, int(self.table[i, pos // 64]) * 64 + pos % 64
                    r += 1
                self.lengths[i] = n + c
                starts[i + 1] = r
        return starts, positions, slots

    def on_gpu(self, pad=0):
        wide = torch.full((self.table.shape[0], self.table.shape[1] + pad), 99, dtype=torch.int32, device="cuda")
        table = wide[:, :self.table.shape[1]]
        table.copy_(torch.from_numpy(self.table))
        return (table, torch.tensor(self.lengths, dtype=torch.int32, device="cuda"),
                torch.tensor([self.free, 55] + self.stack, dtype=torch.int32, device="cuda"))

    def check(self, want, got, state):
        for name, w, g in zip(("starts", "positions", "slots"), want, got):
            assert g.tolist() == w, name
        table, lengths, pool = state
        assert lengths.tolist() == self.lengths and table.tolist() == self.table.tolist()
        assert pool.tolist() == [self.free, self.status] + self.stack


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("sequences", [1, 2, 63, 64, 65, 256, 257, 700, 1024, 1025, 2500])
def test_against_lists(sequences):
    rng = np.random.default_rng(sequences)
    want = Lists(sequences, 9, sequences * 5 + 3, rng)
    state = want.on_gpu(pad=sequences % 3)
    refused = 0
    for step in range(8):
        kind = step % 4
        change = []
        for n in want.lengths:
            if kind == 0:
                c = int(rng.integers(0, 300))
            elif kind == 1:
                c = 1
            elif kind == 2:
                c = int(rng.integers(-n, 65)) if rng.random() < 0.5 else 0
            else:
                c = -n if rng.random() < 0.4 else int(rng.integers(0, 200))
            change.append(c)
        total = sum(max(c, 0) for c in change)
        rows = total + (7 if step % 2 else 0) - (1 if step == 5 and total else 0)
        if sequences > 300 and kind == 0 and step:  # (mostly refused: the pool runs out)
            rows = total
        expect = want.resize(change, rows)
        refused += want.status > 0
        want.check(expect, B.kv_resize(ints(change), *state, rows), state)
    assert refused >= 1 or sequences < 3


@pytest.mark.parametrize("sequences", [4095, 4096, 4097, 6000])
def test_thousands_of_sequences(sequences):
    test_against_lists(sequences)


@pytest.mark.parametrize("place", [0, 3, 1500, 4095])
@pytest.mark.parametrize("rows", [3000, 9000])
def test_one_of_many_refused(place, rows):
    """Sequences that share a thread: the first that finds no room is named, and nothing changes; without it all have room."""
    rng = np.random.default_rng(place)
    want = Lists(4096, 3, 9000)
    want.resize([int(n) for n in rng.integers(0, 100, 4096)], 1 << 20)
    state = want.on_gpu()
    change = [int(rng.integers(-n, 2)) for n in want.lengths]
    change[place] = 64 * 3 + 1 - want.lengths[place]
    expect = want.resize(change, rows)
    assert want.status == place + 1
    want.check(expect, B.kv_resize(ints(change), *state, rows), state)
    change[place] = 0
    expect = want.resize(change, rows)
    assert want.status == 0
    want.check(expect, B.kv_resize(ints(change), *state, rows), state)


@pytest.mark.parametrize("rows", [0, 1, 1023, 1025, 4096, 4097, 70000])
def test_maps_of_many_rows(rows):
    """The maps are made by the first launch, or by one of their own."""
    want = Lists(3, 1200, 1200)
    state = want.on_gpu()
    change = [rows // 3, 0, rows - rows // 3]
    want.check(want.resize(change, rows + 5), B.kv_resize(ints(change), *state, rows + 5), state)


@pytest.mark.parametrize("change,rows", [([100, 0, 0], 99), ([0, -71, 5], 50), ([0, 0, 64 * 4 + 1], 300), ([150, 150, 100], 400), ([TOP, TOP, TOP], 100),
                                         ([-TOP - 1, 0, 0], 100), ([0, 0, -1], 100), ([250, 1, 256], 507)])
@pytest.mark.parametrize("pad", [0, 2])
def test_refused_changes(change, rows, pad):
    """No rows, fewer than no tokens, no room in the table or in the pool: nothing changes."""
    want = Lists(3, 4, 6)
    want.resize([70, 70, 0], 140)
    state = want.on_gpu(pad)
    before = [t.clone() for t in state]
    expect = want.resize(change, rows)
    assert want.status > 0
    want.check(expect, B.kv_resize(ints(change), *state, rows), state)
    assert all(torch.equal(a, b) for a, b in zip(state[:2], before[:2]))


def test_more_sequences_than_a_workgroup_refused():
    """One of 3000 sequences, behind those of the first step, finds no room."""
    want = Lists(3000, 2, 5000)
    want.resize([64] * 3000, 192000)
    state = want.on_gpu()
    change = [1] * 1900 + [0] * 500 + [-64] * 599 + [65]
    expect = want.resize(change, 5000)
    assert want.status == 3000
    want.check(expect, B.kv_resize(ints(change), *state, 5000), state)
    change[-1] = 64
    expect = want.resize(change, 5000)
    assert want.status == 0
    want.check(expect, B.kv_resize(ints(change), *state, 5000), state)


@pytest.mark.parametrize("free", [-1, 7, TOP, -TOP - 1, 6])
def test_a_pool_that_is_none(free):
    """A count of free pages that cannot be, or that the pages given back would take past the pool's end (6 of 6 free, and one held)."""
    table, lengths, pool = ints([[0, 1], [2, 3]]), ints([100, 5]), ints([free, 55, 5, 4, 3, 2, 1, 0])
    starts, positions, slots = B.kv_resize(ints([-100, 1]), table, lengths, pool, 4)
    assert pool.tolist() == [free, -1, 5, 4, 3, 2, 1, 0] and lengths.tolist() == [100, 5] and table.tolist() == [[0, 1], [2, 3]]
    assert starts.tolist() == [0, 0, 0] and positions.tolist() == [-1] * 4 == slots.tolist()


@pytest.mark.parametrize("length", [-1, -TOP - 1, 129, TOP])
def test_lengths_that_are_none(length):
    table, lengths, pool = ints([[0, 1], [2, 3]]), ints([5, length]), ints([2, 55, 5, 4, 3, 2])
    starts, positions, _ = B.kv_resize(ints([1, 0]), table, lengths, pool, 4)
    assert pool[:2].tolist() == [2, 2] and lengths.tolist() == [5, length] and starts.tolist() == [0, 0, 0] and positions.tolist() == [-1] * 4


def test_no_sequences_and_no_table():
    none = torch.zeros((0,), dtype=torch.int32, device="cuda")
    pool = B.page_pool(3)
    starts, positions, slots = B.kv_resize(none, none.view(0, 0), none.clone(), pool, 2)
    assert starts.tolist() == [0] and positions.tolist() == [-1, -1] and slots.tolist() == [-1, -1] and pool.tolist() == [3, 0, 2, 1, 0]
    starts, _, _ = B.kv_resize(ints([0, 0]), torch.zeros((2, 0), dtype=torch.int32, device="cuda"), ints([0, 0]), pool, 0)
    assert starts.tolist() == [0, 0, 0] and pool.tolist() == [3, 0, 2, 1, 0]


def test_as_the_hosts_pages():
    """The same pages as the host's bookkeeping gives."""
    from paper_1705_09864_amd.decoder_layer import Pages
    host = Pages(60, 4, 20)
    table, lengths, pool = torch.zeros_like(host.table), torch.zeros_like(host.lengths), B.page_pool(60)
    for new in ([100, 1, 0, 64], [1, 1, 1, 1], [0, 500, 28, 63], [64, 64, 64, 64]):
        starts = host.extend(new)
        got, _, _ = B.kv_resize(ints(new), table, lengths, pool, sum(new))
        assert torch.equal(table, host.table) and torch.equal(lengths, host.lengths)
        assert starts is None or torch.equal(got, starts)
        assert pool[0].item() == len(host.free) and pool[2:2 + len(host.free)].tolist() == host.free


def test_captured_and_replayed():
    """A graph of a step: the change it reads is the tensor's at the time, other work between the replays."""
    want = Lists(5, 6, 40)
    state = want.on_gpu()
    change = ints([0] * 5)
    outs = torch.zeros(6, dtype=torch.int32, device="cuda"), ints([0] * 300), torch.zeros(300, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.kv_resize(change, *state, 300, *outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_resize(change, *state, 300, *outs)
    for c in ([70, 0, 3, 64, 1], [1, 1, 1, 1, 1], [-71, 100, -4, 0, 64], [300, 1, 0, 0, 0], [0, 0, 0, 0, 0], [100, -50, 64, -65, 0]):
        change.copy_(ints(c))
        torch.zeros(1000, device="cuda").sum().item()
        graph.replay()
        want.check(want.resize(c, 300), outs, state)
