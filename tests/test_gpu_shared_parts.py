"""Attention behind shared prefixes where its work is cut finer, through the C ABI against the definition in 64 bits: own tokens in several parts, row tiles
of many rows over pages of 64 tokens and more, what is shared after tokens were taken back, and long sums. (Bounds as in test_gpu_shared.)"""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2505_02380_amd as E
from test_gpu_cache import TYPES, cache_of, check_attend, dev, ints, rounded, starts
from test_gpu_shared import first_of, make, run

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


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page", [(128, 64), (64, 128), (80, 256), (192, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 70), (90, 0)])
def test_row_tiles_whose_tiles_lie_in_one_page(window, sinks, dim, page, kind):
    """Pages of 64 tokens and more, more than 32 rows a key head: windows within and over the shared tokens, pages that none of the group has and such
    that are none, in the first, a middle and the last shared page; then without those."""
    rng = np.random.default_rng(dim + page)
    pool, table, lengths, shared = make(rng, [(1024, [1030 + 23 * i for i in range(13)]), (512, [520 + i for i in range(10)])], [100], 2, page, dim)
    first, start = [0, 13, 23], starts([1] * 24)
    q = rounded(rng.standard_normal((24, 8, dim)), kind)
    out, lse = run(pool, table, lengths, first, shared, q, start, kind, window, sinks)
    check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5, window, sinks)
    last = 1024 // page - 1
    table[:13, 0], table[:13, last // 2], table[13:23, 512 // page - 1] = -1, pool.pages, -7
    out, lse = run(pool, table, lengths, first, shared, q, start, kind, window, sinks)
    check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5, window, sinks)
    table[:13, last] = pool.pages + 9
    out, lse = run(pool, table, lengths, first, shared, q, start, kind, window, sinks)
    check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5, window, sinks)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_what_is_shared_written_anew_after_tokens_were_taken_back(kind):
    """Three beams behind 96 tokens; one gives up 70 of them and goes on with others. What they share is then 16 tokens, and attention by it is the definition's."""
    rng = np.random.default_rng(13)
    heads, dim, page, beams = 2, 64, 16, 3
    cache = E.Cache.empty(1, 60, heads, page, dim, DEV)
    for x in (cache.k_scale, cache.v_scale):
        x.fill_(1.0)
    tables = [E.CacheTable.empty(beams, 12, DEV) for _ in range(2)]
    status = torch.zeros(4, dtype=torch.int32, device=DEV)
    room = torch.empty(E.entro_cache_pages_workspace_bytes(cache, *tables), dtype=torch.uint8, device=DEV)
    groups = E.CacheGroups(ints([0, beams]), torch.zeros(1, dtype=torch.int32, device=DEV), beams, 96)

    def go_on(parent, grow, rows):
        E.entro_cache_regroup(cache, tables[0], tables[1], status, room, parent=ints(parent), grow=ints(grow))
        tables.reverse()
        if sum(rows):
            k, v = (dev(rng.standard_normal((sum(rows), heads, dim)).astype(np.float32)).to(TYPES[kind]) for _ in "kv")
            E.entro_cache_append(cache, tables[0], E.CacheRows(k, v, ints(starts(rows)), max(rows)))
        E.entro_cache_shared(cache, tables[0], groups)
        assert status[0].item() == 0
        return groups.shared.item()
    go_on([0, -1, -1], [100, 0, 0], [100, 0, 0])
    assert go_on([0, 0, 0], [1, 1, 1], [1, 1, 1]) == 96
    assert go_on([0, 1, 2], [-71, 5, 5], [0, 5, 5]) == 16
    assert go_on([0, 1, 2], [90, 5, 5], [90, 5, 5]) == 16
    table, lengths = tables[0].slots.cpu().numpy(), tables[0].lengths.tolist()
    assert lengths == [120, 111, 111]
    pool = ref.Pool(rng, 1, cache.pages, heads, page, dim)
    pool.k, pool.v, pool.k_scale, pool.v_scale = (x.cpu().numpy() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale))
    q = rounded(rng.standard_normal((3, 4, dim)), kind)
    out, lse = run(pool, table, lengths, [0, beams], groups.shared.tolist(), q, starts([1] * 3), kind)
    check_attend(pool, table, lengths, q, starts([1] * 3), kind, out, lse, dim ** -0.5)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,group,shared,adds", [(2, 2, True, 256), (12, 4, True, 1024), (2, 2, False, 1024), (12, 4, False, 1024)])
def test_small_weights_behind_a_large_one_are_not_lost(seqs, group, shared, adds, kind):
    """65536 tokens, the first with a score of 16.875 and all others with 0: each of these has 0.39 of the first one's last place, and all together 0.3 %. In one
    part, by tiles of 16 rows and of 128, as shared tokens and as own ones. `adds`: tiles that one lane adds up. With u = 2^-24: the score goes
    through 8 roundings, the logarithms (up to 25, base 2) of part and join through 16, a lane's sum through one a tile and 40 within tiles and between lanes."""
    tokens, heads, dim, page = 65536, 1, 64, 64
    pool, table, lengths, _ = make(np.random.default_rng(14), [(tokens, [tokens] * seqs)], [], heads, page, dim)
    pool.k[...], pool.v[...], pool.k_scale[...], pool.v_scale[...] = 128, 128, 2.0 ** -7, 1.0
    pool.k[0, table[0, 0], 0, 0, 0] = 128 + 64
    q = np.zeros((seqs, group, dim), np.float32)
    q[..., 0] = 33.75
    out, lse = run(pool, table, lengths, [0, seqs], [tokens - 64 if shared else 0], q, starts([1] * seqs), kind, max_shared=64 if shared else tokens, scale=1.0)
    want = 16.875 + np.log1p((tokens - 1) * np.exp(-16.875))
    assert np.abs(lse.cpu().numpy().astype(np.float64) - want).max() <= (8 * 16.875 + 16 * 25 + adds + 40) * 2.0 ** -24
