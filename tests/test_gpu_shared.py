"""Attention for groups of sequences behind a shared prefix, and what they share, through the C ABI against the definitions in 64 bits.

Bounds are those of the attention over all tokens at once (test_gpu_cache), whose joins over parts these calls have too."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2505_02380_amd as E
from paper_2505_02380_amd import binding as B
from test_gpu_cache import TYPES, cache_of, check_attend, dev, ints, rounded, scales, starts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(rng, groups, lone, heads, page, dim, slots=None):
    """groups: (tokens shared, lengths of the sequences); lone: lengths of sequences in no group, behind them. The pool, the table and the pages
    that each group shares, as numbers of tokens."""
    rows = [(p, n) for p, lengths in groups for n in lengths] + [(0, n) for n in lone]
    need = sum(p // page for p, _ in groups) + sum(-(-n // page) - p // page for p, n in rows)
    pool = ref.Pool(rng, 1, need + 3, heads, page, dim)
    order = iter(rng.permutation(need + 3))
    table = np.full((len(rows), slots or max(1, max(-(-n // page) for _, n in rows))), -1, np.int32)
    b = 0
    for p, lengths in groups + [(0, [n]) for n in lone]:
        common = [next(order) for _ in range(p // page)]
        for n in lengths:
            own = [next(order) for _ in range(-(-n // page) - p // page)]
            table[b, : len(common) + len(own)] = common + own
            b += 1
    scales(rng, pool, table)
    return pool, table, [n for _, n in rows], [p // page * page for p, _ in groups]


def first_of(groups):
    return starts([len(lengths) for _, lengths in groups])


def run(pool, table, lengths, first, shared, q, start, kind, window=0, sinks=0, max_new=None, max_len=None, max_seqs=None, max_shared=None, lse=True,
        scale=None, q_dev=None, out_dev=None):
    cache, t = cache_of(pool), E.CacheTable(dev(table), ints(lengths))
    g = E.CacheGroups(ints(first), ints(shared), int(np.diff(first).max()) if max_seqs is None else max_seqs,
                      int(max(shared)) if max_shared is None else max_shared)
    qd = dev(q).to(TYPES[kind]) if q_dev is None else q_dev
    out = torch.full_like(qd, 7.0) if out_dev is None else out_dev
    ld = torch.full(qd.shape[:2], 7.0, device=DEV) if lse else None
    query = E.CacheQuery(qd, out, ints(start), int(np.diff(start).max()) if max_new is None else max_new, int(max(lengths)) if max_len is None else max_len,
                         lse=ld, scale=scale, window=window, sinks=sinks)
    ws = torch.full((E.entro_cache_attend_shared_workspace_bytes(cache, t, query, g),), 0xFF, dtype=torch.uint8, device=DEV)
    E.entro_cache_attend_shared(cache, t, query, g, ws)
    torch.cuda.synchronize()
    return out, ld


#  groups (tokens shared, lengths)                                             lone        new tokens                q, kv  dim  page  type  window sinks
SHARED = [
    ([(64, [65, 70, 100, 64 + 64])],                                           [],         [1] * 4,                  4, 4,   64,  16, "bf16", 0, 0),
    ([(200, [201, 230, 333])],                                                 [5, 100],   [1] * 5,                  8, 2,  128,  64, "f32", 0, 0),
    ([(130, [131] * 9), (500, [501, 600]), (33, [40, 34, 50])],                [1],        [1] * 15,                 4, 1,   96,  16, "bf16", 0, 0),
    ([(1000, [1001 + i for i in range(40)])],                                  [],         [1] * 40,                 4, 1,  128,  64, "bf16", 0, 0),
    ([(700, [720 + 3 * i for i in range(11)]), (90, [130] * 4)],               [64],       [1] * 16,                 10, 2,  80,  32, "f32", 0, 0),
    ([(300, [300 + 5 * i for i in range(1, 30)])],                             [],         [1] * 29,                 3, 3,  256, 128, "bf16", 0, 0),
    ([(260, [270 + i for i in range(20)])],                                    [],         [1] * 20,                 4, 2,  192,  64, "f32", 0, 0),
    ([(260, [270 + i for i in range(20)])],                                    [],         [1] * 20,                 4, 2,  256,  16, "f32", 0, 0),
    # several new tokens, none, all of what is not shared; queries among the shared tokens
    ([(150, [160, 190, 151])],                                                 [30],       [3, 40, 0, 30],           4, 2,  128,  16, "bf16", 0, 0),
    ([(400, [480, 500, 420])],                                                 [],         [80, 9, 20],              8, 2,   96,  64, "bf16", 0, 0),
    ([(400, [480, 500, 420])],                                                 [70],       [80, 100, 20, 70],        6, 2,   64,  32, "f32", 0, 0),
    ([(512, [520, 600])],                                                      [],         [100, 300],               4, 1,  128,  64, "bf16", 0, 0),
    ([(512, [520, 600])],                                                      [],         [520, 1],                 2, 1,   64,  64, "f32", 0, 0),
    # windows: within the own tokens, within the shared ones, over both; first tokens kept
    ([(320, [330, 400, 500])],                                                 [90],       [1] * 4,                  8, 2,  128,  16, "bf16", 50, 0),
    ([(320, [330, 400, 500])],                                                 [90],       [1] * 4,                  8, 2,   64,  64, "bf16", 200, 5),
    ([(1000, [1010 + 7 * i for i in range(24)])],                              [],         [1] * 24,                 4, 2,   96,  32, "bf16", 300, 70),
    ([(600, [660, 640, 700])],                                                 [],         [60, 1, 40],              4, 1,   80,  16, "f32", 128, 3),
    # groups of one sequence, of none, and nothing shared
    ([(100, [130]), (0, []), (0, [20, 50]), (10, [30, 31])],                   [],         [1] * 5,                  4, 2,   64,  16, "bf16", 0, 0),
]


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_attend_shared_against_the_definition(case):
    groups, lone, new, q_heads, heads, dim, page, kind, window, sinks = SHARED[case]
    rng = np.random.default_rng(case)
    pool, table, lengths, shared = make(rng, groups, lone, heads, page, dim)
    start = starts(new)
    q = rounded(rng.standard_normal((start[-1], q_heads, dim)) * 1.5, kind)
    out, lse = run(pool, table, lengths, first_of(groups), shared, q, start, kind, window, sinks)
    check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5, window, sinks)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 12])
def test_groups_in_the_middle_pages_missing_and_shared_tokens_that_are_fewer(kind, new):
    """Sequences before and behind the groups; pages that none has, among the shared ones too; less said to be shared than is."""
    rng = np.random.default_rng(new)
    heads, page, dim = 2, 16, 64
    pool, table, lengths, shared = make(rng, [(0, [40]), (300, [330, 350, 310, 400]), (200, [260, 230])], [77, 90], heads, page, dim)
    table[1:5, 3], table[2, -5], table[5:7, 0] = -1, pool.pages, -7
    first, start = [1, 5, 7], starts([new] * 9)
    q = rounded(rng.standard_normal((start[-1], 8, dim)), kind)
    for said in (shared[1:], [100, 64], [63, 0], [299, 130], [-5, 192]):
        out, lse = run(pool, table, lengths, first, said if said[1] != 192 else [-5, 10], q, start, kind)
        check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_hints_change_nothing_but_the_order_of_sums(kind):
    rng = np.random.default_rng(3)
    heads, page, dim = 2, 32, 128
    pool, table, lengths, shared = make(rng, [(900, [910 + 9 * i for i in range(12)]), (200, [2000, 230])], [500], heads, page, dim)
    first, start = [0, 12, 14], starts([1] * 12 + [3, 1, 40])
    q = rounded(rng.standard_normal((start[-1], 8, dim)), kind)
    for hints in [(1, 1, 1, 1), (40, 2000, 12, 896), (2 ** 32 - 1,) * 4, (0, 0, 0, 0), (5, 10 ** 6, 3, 10 ** 6), (40, 100, 14, 3000)]:
        out, lse = run(pool, table, lengths, first, shared, q, start, kind, max_new=hints[0], max_len=hints[1], max_seqs=hints[2], max_shared=hints[3])
        check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5)


def test_strides_starts_that_lie_and_rows_of_no_sequence():
    rng = np.random.default_rng(4)
    heads, page, dim, q_heads = 2, 16, 40, 4
    pool, table, lengths, shared = make(rng, [(100, [120, 130, 111])], [60], heads, page, dim)
    start = np.array([2, 3, 5, 6, 9])
    q = rng.standard_normal((11, q_heads, dim)).astype(np.float32)
    wide = torch.zeros(11, q_heads + 2, dim + 3, device=DEV)
    wide[:, 1:-1, 2:-1] = dev(q)
    wide = torch.nn.functional.pad(wide, (0, 0))[:, 1:-1, 2:-1]
    out = torch.full((11, q_heads, dim + 8), 7.0, device=DEV)[..., :dim]
    storage = torch.empty(wide.numel() * 3 + 64, device=DEV)
    shifted = storage[4:].as_strided(wide.shape, wide.stride()).copy_(wide)
    got, lse = run(pool, table, lengths, [0, 3], shared, q, start, "f32", q_dev=shifted, out_dev=out)
    check_attend(pool, table, lengths, q, start, "f32", got, lse, dim ** -0.5)
    assert torch.all(got[:2] == 7) and torch.all(got[9:] == 7) and torch.all(lse[:2] == 7) and torch.all(lse[9:] == 7)
    # starts and groups beyond what there is: rows and sequences that exist are taken, nothing else
    for first in ([-4, 2 ** 31 - 1], [3, 90], [2, 1], [9, 11]):
        got, lse = run(pool, table, lengths, first, [0], q, start, "f32", max_seqs=2)
        if first[0] <= first[1]:
            check_attend(pool, table, lengths, q, start, "f32", got, lse, dim ** -0.5)
    run(pool, table, lengths, [0, 3], shared, q, [-5, 8, 3, 40, 2 ** 31 - 1], "f32", max_new=5)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rows_without_a_token_and_scales_of_pages_that_nobody_sees(kind):
    """A sequence all of whose pages are missing, and tokens before position 0: zeros and minus infinity. Pages without a seen token hold anything."""
    rng = np.random.default_rng(5)
    heads, page, dim = 1, 16, 64
    pool, table, lengths, shared = make(rng, [(128, [140, 150, 129])], [0, 20], heads, page, dim)
    table[1] = table[0]
    table[1, 8:] = -1
    lengths[1] = 150
    table[4] = -1
    start = starts([1, 2, 1, 3, 2])
    pool.k_scale[0, table[2, 8]] = pool.v_scale[0, table[2, 8]] = np.float32(0.03)
    q = rounded(rng.standard_normal((start[-1], 2, dim)), kind)
    out, lse = run(pool, table, lengths, [0, 3], shared, q, start, kind)
    check_attend(pool, table, lengths, q, start, kind, out, lse, dim ** -0.5)
    assert torch.isneginf(lse[start[3]:]).all() and torch.all(out[start[3]:] == 0)
    # a window that leaves out the middle pages: their scales are no numbers
    pool, table, lengths, shared = make(rng, [(512, [600, 640])], [], heads, page, dim)
    pool.k_scale[0, table[0, 4:20]] = pool.v_scale[0, table[0, 4:20]] = np.nan
    q = rounded(rng.standard_normal((2, 2, dim)), kind)
    out, lse = run(pool, table, lengths, [0, 2], shared, q, starts([1, 1]), kind, window=200, sinks=10)
    check_attend(pool, table, lengths, q, starts([1, 1]), kind, out, lse, dim ** -0.5, 200, 10)


@pytest.mark.parametrize("kind,factor", [("bf16", 1e18), ("f32", 1e18), ("bf16", 300.0), ("f32", 1e-20)])
@pytest.mark.parametrize("seqs", [3, 40])
def test_extreme_queries(kind, factor, seqs):
    """Scores far apart, and such that lie far above or below what exp takes."""
    rng = np.random.default_rng(6)
    heads, page, dim = 1, 16, 64
    pool, table, lengths, shared = make(rng, [(256, [270 + i for i in range(seqs)])], [], heads, page, dim)
    q = rounded(rng.standard_normal((seqs, 2, dim)) * factor, kind)
    scale = 1e-3 / factor if factor > 1e3 else 0.1
    out, lse = run(pool, table, lengths, [0, seqs], shared, q, starts([1] * seqs), kind, scale=scale)
    check_attend(pool, table, lengths, q, starts([1] * seqs), kind, out, lse, scale)


def test_the_same_call_again_gives_the_same_bits_and_near_those_of_attend():
    rng = np.random.default_rng(7)
    pool, table, lengths, shared = make(rng, [(3000, [3010 + 17 * i for i in range(48)])], [], 2, 64, 128)
    q = rounded(rng.standard_normal((48, 8, 128)), "bf16")
    one = run(pool, table, lengths, [0, 48], shared, q, starts([1] * 48), "bf16")
    for _ in range(3):
        two = run(pool, table, lengths, [0, 48], shared, q, starts([1] * 48), "bf16")
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    cache, t = cache_of(pool), E.CacheTable(dev(table), ints(lengths))
    qd = dev(q).to(torch.bfloat16)
    out, lse = torch.zeros_like(qd), torch.zeros(48, 8, device=DEV)
    query = E.CacheQuery(qd, out, ints(starts([1] * 48)), 1, max(lengths), lse=lse)
    E.entro_cache_attend(cache, t, query, torch.empty(max(16, E.entro_cache_attend_workspace_bytes(cache, t, query)), dtype=torch.uint8, device=DEV))
    assert float((lse - one[1]).abs().max()) < 1e-4 and float((out.float() - one[0].float()).norm() / out.float().norm()) < 2.0 ** -8


def plain_shared(table, lengths, first, page, pages):
    out = []
    for a, b in zip(first[:-1], first[1:]):
        a, b = min(max(a, 0), len(lengths)), min(max(b, 0), len(lengths))
        n = 0
        while a < b and n < table.shape[1] and all((n + 1) * page <= lengths[i] and table[i, n] == table[a, n] and 0 <= table[a, n] < pages for i in range(a, b)):
            n += 1
        out.append(n * page)
    return out


@pytest.mark.parametrize("groups,lone,page", [
    ([(64, [65, 70, 100])], [], 16), ([(64, [64, 70, 100])], [3], 64), ([(0, [9, 9]), (100, [100] * 5), (31, [31, 32])], [], 16), ([(5000, [5100, 6000, 5000])], [], 16),
    ([(4096 * 5, [4096 * 5 + i for i in range(70)]), (0, []), (17, [90])], [1], 16), ([(16 * 255, [5000, 5000]), (16 * 256, [5000, 5000]), (16 * 257, [5000, 5000])], [], 16),
    ([(128, [200 + i for i in range(600)])], [], 32)])
def test_what_is_shared(groups, lone, page):
    rng = np.random.default_rng(len(groups))
    pool, table, lengths, shared = make(rng, groups, lone, 1, page, 1)
    first = [int(i) for i in first_of(groups)]
    cache, t = cache_of(pool), E.CacheTable(dev(table), ints(lengths))

    def ask(first, table=t):
        out = torch.full((len(first) - 1 + 2,), 77, dtype=torch.int32, device=DEV)
        E.entro_cache_shared(cache, table, E.CacheGroups(ints(first), out[: len(first) - 1], 1, 1))
        assert out[-2:].tolist() == [77, 77]
        return out[:-2].tolist()
    assert ask(first) == plain_shared(table, lengths, first, page, pool.pages)
    assert ask([f + 1 for f in first]) == plain_shared(table, lengths, [f + 1 for f in first], page, pool.pages)      # across the groups
    assert ask([-3, 1, 1, 10 ** 9]) == plain_shared(table, lengths, [0, 1, 1, len(lengths)], page, pool.pages)
    # pages that are none, in all rows
    cut = table.copy()
    cut[:, min(2, table.shape[1] - 1)] = pool.pages
    assert ask(first, E.CacheTable(dev(cut), ints(lengths))) == plain_shared(cut, lengths, first, page, pool.pages)


def test_many_groups():
    rng = np.random.default_rng(9)
    groups = [(16 * int(rng.integers(0, 6)), [100 + int(x) for x in rng.integers(0, 60, rng.integers(1, 4))]) for _ in range(300)]
    pool, table, lengths, shared = make(rng, groups, [50], 1, 16, 8)
    first = first_of(groups)
    cache, t = cache_of(pool), E.CacheTable(dev(table), ints(lengths))
    said = torch.zeros(300, dtype=torch.int32, device=DEV)
    E.entro_cache_shared(cache, t, E.CacheGroups(ints(first), said, 3, 80))
    assert said.tolist() == plain_shared(table, lengths, [int(i) for i in first], 16, pool.pages)
    n = len(lengths)
    q = rounded(rng.standard_normal((n, 2, 8)), "f32")
    out, lse = run(pool, table, lengths, first, shared, q, starts([1] * n), "f32")
    check_attend(pool, table, lengths, q, starts([1] * n), "f32", out, lse, 8 ** -0.5)


def test_steps_of_beams_in_a_graph():
    """Forks by entro_cache_regroup, keys rotated on their way into the cache, what is shared, and attention, captured once and replayed as beams part and
    meet: every replay against the definition."""
    rng = np.random.default_rng(10)
    beams, heads, q_heads, dim, page, prompt = 6, 2, 4, 64, 16, 100
    cache = E.Cache.empty(1, 80, heads, page, dim, DEV)
    tables = [E.CacheTable.empty(beams, 12, DEV) for _ in range(2)]
    status = torch.zeros(4, dtype=torch.int32, device=DEV)
    room = torch.empty(E.entro_cache_pages_workspace_bytes(cache, *tables), dtype=torch.uint8, device=DEV)
    rotary = E.Rotary(dev(E.entro_rotary_turns(dim).view(np.int64)), dim)
    k, v = (torch.randn(prompt, heads, dim, device=DEV) for _ in "kv")
    E.entro_cache_regroup(cache, tables[0], tables[1], status, room, grow=ints([prompt] + [0] * (beams - 1)))
    E.entro_cache_append_rotated(cache, tables[1], E.CacheRows(k, v, ints([0] + [prompt] * beams), prompt), rotary)
    k, v, q, q_turned, out = (torch.zeros(beams, n, dim, dtype=torch.bfloat16, device=DEV) for n in (heads, heads, q_heads, q_heads, q_heads))
    start, parent, one = ints(range(beams + 1)), torch.zeros(beams, dtype=torch.int32, device=DEV), ints([1] * beams)
    groups = E.CacheGroups(ints([0, beams]), torch.zeros(1, dtype=torch.int32, device=DEV), beams, prompt)
    query = E.CacheQuery(q_turned, out, start, 1, 180)
    ws = torch.empty(E.entro_cache_attend_shared_workspace_bytes(cache, tables[0], query, groups), dtype=torch.uint8, device=DEV)
    back = tables[1].slots.clone(), tables[1].lengths.clone()

    def step():
        E.entro_cache_regroup(cache, tables[1], tables[0], status, room, parent=parent, grow=one)
        E.entro_cache_append_rotated(cache, tables[0], E.CacheRows(k, v, start, 1), rotary, E.RotaryRows(q, q_turned))
        E.entro_cache_shared(cache, tables[0], groups)
        E.entro_cache_attend_shared(cache, tables[0], query, groups, ws)
        tables[1].slots.copy_(tables[0].slots)
        tables[1].lengths.copy_(tables[0].lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    tables[1].slots.copy_(back[0]), tables[1].lengths.copy_(back[1])
    seen = set()
    for i in range(5):
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, device=DEV))
        parent.copy_(ints(rng.integers(0, beams, beams) if i else [0] * beams) if i != 3 else ints([2] * beams))
        graph.replay()
        torch.cuda.synchronize()
        assert status[0].item() == 0
        table, lengths = tables[0].slots.cpu().numpy(), tables[0].lengths.tolist()
        pool = ref.Pool(rng, 1, cache.pages, heads, page, dim)
        pool.k, pool.v, pool.k_scale, pool.v_scale = (x.cpu().numpy() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale))
        assert groups.shared.tolist() == plain_shared(table, lengths, [0, beams], page, cache.pages)
        seen.add(groups.shared.item())
        check_attend(pool, table, lengths, q_turned.float().cpu().numpy(), np.arange(beams + 1), "bf16", out, None, dim ** -0.5)
    assert max(seen) >= 96


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("f32", 96), ("bf16", 192)])
def test_more_than_64_sequences_and_more_than_64_parts(kind, dim):
    """A group of 150 sequences (more than a wavefront has lanes); rows in parts of both kinds beyond 64, by hints that ask for them."""
    rng = np.random.default_rng(12)
    pool, table, lengths, shared = make(rng, [(128, [129 + i % 40 for i in range(150)]), (64, [70] * 3)], [], 1, 16, dim)
    n = len(lengths)
    q = rounded(rng.standard_normal((n, 2, dim)), kind)
    out, lse = run(pool, table, lengths, [0, 150, n], shared, q, starts([1] * n), kind)
    check_attend(pool, table, lengths, q, starts([1] * n), kind, out, lse, dim ** -0.5)
    pool, table, lengths, shared = make(rng, [(6400, [6500, 6410])], [5000], 1, 16, dim)
    q = rounded(rng.standard_normal((3, 2, dim)), kind)
    out, lse = run(pool, table, lengths, [0, 2], shared, q, starts([1] * 3), kind, max_len=200000, max_shared=100000)
    check_attend(pool, table, lengths, q, starts([1] * 3), kind, out, lse, dim ** -0.5)
    out, lse = run(pool, table, lengths, [0, 2], shared, q, starts([1] * 3), kind, max_len=120000, max_shared=6400)
    check_attend(pool, table, lengths, q, starts([1] * 3), kind, out, lse, dim ** -0.5)


def test_refusals_on_the_gpu():
    rng = np.random.default_rng(11)
    pool, table, lengths, shared = make(rng, [(64, [70, 80])], [], 1, 16, 64)
    cache, t, g = cache_of(pool), E.CacheTable(dev(table), ints(lengths)), E.CacheGroups(ints([0, 2]), ints(shared), 2, 64)
    q = torch.zeros(2, 1, 64, device=DEV)
    query = E.CacheQuery(q, torch.zeros_like(q), ints([0, 1, 2]), 1, 80)
    need = E.entro_cache_attend_shared_workspace_bytes(cache, t, query, g)
    for ws, status in ((None, B.ENTRO_ERR_NULL), (torch.zeros(need - 1, dtype=torch.uint8, device=DEV), B.ENTRO_ERR_CAPACITY)):
        with pytest.raises(E.EntroError) as err:
            E.entro_cache_attend_shared(cache, t, query, g, ws)
        assert err.value.status == status


def test_the_example_s_steps_with_positions_and_a_shared_prefix():
    """The example's last step of a few, beams forking, with norms, rotations and what the beams share: rotated queries, cache and attention against
    the definitions."""
    import rotary_reference as rot
    from examples import token_step as ex
    cfg, heads, kv_heads, dim = ex.LAYERS["smol"]
    beams, tokens = 3, 205
    layer = ex.Layer(cfg, beams)
    g = ex.Generation(layer, heads, kv_heads, dim, beams, 220, page=16, rotary=True, shared=True)
    torch.manual_seed(6)
    g.prompt(*(torch.randn(200, kv_heads, dim, device=DEV).to(torch.bfloat16) for _ in "kv"))
    for parent in ([0, 0, 0], [2, 0, 2], [0, 1, 1], [1, 1, 0], [0, 1, 2]):
        layer.x.copy_(torch.randn(layer.x.shape, device=DEV))
        g.step(ints(parent))
    torch.cuda.synchronize()
    assert g.status.tolist()[0] == 0 and g.table.lengths.tolist() == [tokens] * beams and g.groups.shared.tolist() == [192]
    pool = ref.Pool(np.random.default_rng(0), 1, 1, kv_heads, 16, dim)
    pool.pages = g.cache.pages
    pool.k, pool.v, pool.k_scale, pool.v_scale = (x.cpu().numpy() for x in (g.cache.k, g.cache.v, g.cache.k_scale, g.cache.v_scale))
    table, start = g.table.slots.cpu().numpy(), np.arange(beams + 1)
    q = layer.q.view(beams, heads, dim).float().cpu().numpy()
    check_attend(pool, table, [tokens] * beams, q, start, "bf16", layer.attended.view(beams, heads, dim), None, dim ** -0.5)
    E.entro_plan_run(layer.plans[0][0])                         # the rows before they were rotated
    turns, at = E.entro_rotary_turns(dim), np.full(beams, tokens - 1)
    want, bound = rot.rotate(layer.q.view(beams, heads, dim).float().cpu().numpy(), at, turns, "halves", "rms")
    assert np.all(np.abs(q - want) <= rot.tolerance(want, bound, "bf16"))
    want, bound = rot.rotate(layer.k.view(beams, kv_heads, dim).float().cpu().numpy(), at, turns, "halves", "rms")
    k, _ = ref.read(pool, table, [tokens] * beams, start, beams)
    step = pool.k_scale[0, table[:, (tokens - 1) // 16]][..., None]
    assert np.all(np.abs(k - want) <= step * 0.5 * (1 + 2.0 ** -16) + bound)
