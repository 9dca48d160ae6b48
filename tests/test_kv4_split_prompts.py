"""Prompts over the cache of 4 bits whose pages are split over workgroups: every width of a head, beside few rows, and between other calls on one workspace."""
import re

import pytest
import torch

from paper_1705_09864_amd import binding as B
from test_kv4 import Cache, attend, check_attention, starts_of

pytestmark = pytest.mark.gpu


def split():
    """Whether the last call's kernel was the one of prompts with split pages."""
    m = re.match(r"kv4_prompt_kernel<\d+,\d+,(\d),(\d)>", B.last_kernel())
    return m is not None and m.groups() == ("1", "1")


@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [32, 96, 128, 150, 160, 192, 224, 255, 256])
def test_heads_of_every_width(kind, dim):
    """32 tiles of 128 rows for each of 4 heads: 128 workgroups of tiles, which beyond 128 values are the most that are split."""
    cache = Cache(4, dim, [2100], seed=dim)
    for named in (dict(), dict(window=700), dict(causal=False)):
        attend(cache, 8, [512], kind, seed=1, gap=dim % 3, **named)
        assert split(), B.last_kernel()


@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,lengths,new", [(64, [2500, 70, 2300], [260, 3, 256]), (128, [2500, 2100, 90], [260, 3, 90]), (100, [40, 2600, 0, 2200], [1, 129, 0, 7]),
                                             (256, [2100, 2200], [256, 3]), (160, [2300, 2100], [8, 250])])
def test_beside_few_rows(kind, dim, lengths, new):
    """Sequences of up to 64 rows are another kernel's, which has counters and parts at the same places."""
    cache = Cache(4, dim, lengths, seed=dim)
    attend(cache, 8, new, kind, seed=3, gap=1)
    assert split(), B.last_kernel()


@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 256])
def test_between_steps_on_one_workspace(kind, dim):
    """Steps of few rows and prompts, split and not, one after the other on one workspace: each gives what it gives alone, and leaves the counters at zero."""
    width, turns = 40, []
    ws = torch.zeros((B.workspace_bytes(B.OP_KV4_ATTENTION, (2, width, 4, 32, dim, 0)),), dtype=torch.uint8, device="cuda")
    for seed, (lengths, new) in enumerate([([2500, 9], [1, 1]), ([2500, 2400], [256, 3]), ([2000, 2100], [1, 2]), ([2300, 2200], [256, 256]), ([100, 2500], [3, 4])]):
        cache = Cache(4, dim, lengths, seed=seed, table_pad=width - max(-(-n // 64) for n in lengths))
        q = torch.randn((sum(new), 32, dim), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(kind)
        outs = []
        for w in (ws, None, ws):
            outs.append(B.kv4_attention(q, *cache.args, starts=starts_of(new), max_new=max(new), workspace=w))
            assert not bool(ws[:65536].any())
        turns.append(split())
        check_attention(cache, q, new, outs[0])
        assert all(torch.equal(outs[0], o) for o in outs[1:])
    assert turns == [False, True, False, True, False]
