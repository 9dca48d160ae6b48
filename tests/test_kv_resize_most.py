"""kv_resize with a bound of one sequence's new tokens: a sequence past it finds no room, everything else is as ever."""
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_1705_09864_amd import binding as B
from test_host_binding_lock_more import CHILD, ROOT, STAND_IN
from test_kv_resize import Lists, ints
from test_more_refusals import E_SHAPE, P


@pytest.mark.parametrize("max_new,rows,status", [(-1, 10, E_SHAPE), (-2**31, 10, E_SHAPE), (1, -1, E_SHAPE), (0, 1 << 31, E_SHAPE)])
def test_refusals(max_new, rows, status):
    assert B.lib().bmx_kv_resize_most(P, 4, P, 8, 8, P, P, 40, P, P, P, rows, max_new, None) == status


@pytest.mark.gpu
@pytest.mark.parametrize("sequences", [1, 3, 64, 257, 1025, 4096, 4097])
@pytest.mark.parametrize("rows", [400, 20000])
def test_one_sequence_past_the_bound(sequences, rows):
    rng = np.random.default_rng(sequences + rows)
    want = Lists(sequences, 9, sequences * 5 + 3, rng)
    want.resize([int(n) for n in rng.integers(0, 100, sequences)], 1 << 20)
    state = want.on_gpu()
    change = [int(rng.integers(-n, 2)) if i % max(1, sequences // 200) == 0 else min(0, 3 - n) for i, n in enumerate(want.lengths)]
    for place in sorted({0, sequences // 2, sequences - 1}):
        past = list(change)
        past[place] = 8
        before = [t.clone() for t in state]
        starts, positions, slots = B.kv_resize(ints(past), *state, rows, max_new=7)
        assert state[2][:2].tolist() == [want.free, place + 1]
        assert all(torch.equal(a, b) for a, b in zip(state[:2], before[:2])) and torch.equal(state[2][2:], before[2][2:])
        assert not bool(starts.any()) and bool((positions == -1).all()) and bool((slots == -1).all())
    for max_new in (8, rows + 5, 2**31 - 1):
        expect = want.resize(past, rows)
        assert want.status == 0
        want.check(expect, B.kv_resize(ints(past), *state, rows, max_new=max_new), state)
        past = [0] * sequences
        past[-1] = 8


@pytest.mark.gpu
def test_without_pythons_lock(tmp_path):
    """As the calls of test_host_binding_lock_more.py, with an entry point more."""
    entry = "ENTRY(bmx_kv_resize)"
    (tmp_path / "stand_in.cpp").write_text(STAND_IN.replace(entry, entry + " ENTRY(bmx_kv_resize_most)"))
    so = str(tmp_path / "stand_in.so")
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", str(tmp_path / "stand_in.cpp"), "-o", so], check=True)
    start = CHILD.index("CALLS = ")
    calls = 'CALLS = [("kv_resize_most", z(3, t=i), z(3, 2, t=i), z(3, t=i), z(6, t=i), 5, n, n, n, n, 3)]\n'
    r = subprocess.run([sys.executable, "-c", CHILD[:start] + calls + CHILD[CHILD.index("calls, held = "):], so, ROOT], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["kv_resize_most", "1", "0"]
