"""Attention behind shared prefixes where its work is cut finer, through the C ABI against the definition in 64 bits: own tokens in several parts.
(Bounds as in test_gpu_shared.)"""
import numpy as np
import pytest
import torch

import paper_2505_02380_amd as E
from test_gpu_cache import TYPES, cache_of, check_attend, dev, ints, rounded, starts
from test_gpu_shared import first_of, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def parts_of(cache, table, query, groups):
    tokens, q_heads = query.q.shape[:2]
    return E.entro_cache_attend_shared_workspace_bytes(cache, table, query, groups) // (tokens * q_heads * (cache.width + 1) * 4)


#  groups (tokens shared, lengths)                                   lone           new                          q, kv  dim  page  max_own
OWN_PARTS = [
    # pieces of new tokens, by row tiles; sequences with few tokens of their own leave later parts empty
    ([(256, [1990, 300, 1000]), (130, [190])],                       [],            [40, 40, 9, 12],             8, 2,   64,  64, 2000),
    ([(128, [1900, 160])],                                           [2100, 50],    [33, 20, 90, 50],            6, 1,   96,  16, 2100),
    # a token each of more than 32 rows a key head: own tokens by single wavefronts
    ([(512, [2300] + [540 + 20 * i for i in range(11)])],            [2600, 3],     [1] * 14,                    8, 2,  128,  64, 2600),
    ([(400, [420] * 9 + [2200])],                                    [1700],        [1] * 11,                    4, 1,   80,  32, 1900),
    # few rows
    ([(64, [70, 1800])],                                             [2000],        [1, 2, 1],                   4, 2,   64,  16, 2000),
]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1700, 5)])
@pytest.mark.parametrize("case", range(len(OWN_PARTS)))
def test_own_tokens_in_several_parts(case, window, sinks, kind):
    groups, lone, new, q_heads, heads, dim, page, max_own = OWN_PARTS[case]
    rng = np.random.default_rng(case)
    pool, table, lengths, shared = make(rng, groups, lone, heads, page, dim)
    first, start = first_of(groups), starts(new)
    q = rounded(rng.standard_normal((start[-1], q_heads, dim)), kind)
    cache, t, qd = cache_of(pool), E.CacheTable(dev(table), ints(lengths)), dev(q).to(TYPES[kind])
    out, lse = torch.zeros_like(qd), torch.zeros(qd.shape[:2], device=DEV)
    query = E.CacheQuery(qd, out, ints(start), max(new), max(lengths), lse=lse, window=window, sinks=sinks)
    said = [ints(first), ints(shared), int(np.diff(first).max()), int(max(shared))]
    one = parts_of(cache, t, query, E.CacheGroups(*said, max_own=1))
    for hint in (max_own, 2 ** 32 - 1, 1600):
        g = E.CacheGroups(*said, max_own=hint)
        assert parts_of(cache, t, query, g) > one
        ws = torch.full((E.entro_cache_attend_shared_workspace_bytes(cache, t, query, g),), 0xFF, dtype=torch.uint8, device=DEV)
        out.fill_(7), lse.fill_(7)
        E.entro_cache_attend_shared(cache, t, query, g, ws)
        check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5, window, sinks)
