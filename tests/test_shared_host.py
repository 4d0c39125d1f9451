"""Host side of attention behind shared prefixes: refusals before anything reaches a GPU, launches, and what is shared as host code (CPU only)."""
import ctypes as C

import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2505_02380_amd as E
from paper_2505_02380_amd import binding as B
from test_cache_host import Placed, calls_made  # noqa: F401
from test_cache_on_cpu import HINTS, Memory, compiled, own_memory, page_call, source

PTR = 0x10000          # an address that is aligned; no call below gets as far as using it


def good():
    return (B.CCache(PTR, PTR, PTR, PTR, 2, 100, 64, 8, 128, 0), B.CCacheTable(PTR, PTR, 4, 16),
            B.CCacheQuery(PTR, PTR, PTR, 4096, 128, 4096, 128, PTR, 5, 2, 1000, 32, E.ENTRO_BF16, 1, 0, 0, 0.1, 0), B.CCacheGroups(PTR, PTR, 2, 3, 500, 0))


def both(cache, table, query, groups):
    by = lambda x: None if x is None else C.byref(x)  # noqa: E731
    L = B.lib()
    return (L.entro_cache_shared(by(cache), by(table), by(groups), None),
            L.entro_cache_attend_shared(by(cache), by(table), by(query), by(groups), PTR, 1 << 50, None))


def test_struct_layout_matches_header():
    assert C.sizeof(B.CCacheGroups) == 32


@pytest.mark.parametrize("of,field,value,status", [
    (3, "first", None, B.ENTRO_ERR_NULL), (3, "shared", None, B.ENTRO_ERR_NULL), (3, "first", PTR + 4, B.ENTRO_ERR_ALIGN), (3, "shared", PTR + 8, B.ENTRO_ERR_ALIGN),
    (3, "groups", 0, B.ENTRO_ERR_SIZE), (3, "groups", (1 << 32) - 1, B.ENTRO_ERR_SIZE), (0, "page_tokens", 48, B.ENTRO_ERR_SIZE), (0, "k", None, B.ENTRO_ERR_NULL),
    (1, "slots", None, B.ENTRO_ERR_NULL), (1, "lengths", PTR + 4, B.ENTRO_ERR_ALIGN), (1, "seqs", 0, B.ENTRO_ERR_SIZE)])
def test_both_calls_refuse(of, field, value, status):
    given = good()
    setattr(given[of], field, value)
    assert both(*given) == (status, status)


@pytest.mark.parametrize("field,value,status", [
    ("q", None, B.ENTRO_ERR_NULL), ("out", None, B.ENTRO_ERR_NULL), ("start", None, B.ENTRO_ERR_NULL), ("q", PTR + 2, B.ENTRO_ERR_ALIGN), ("lse", PTR + 4, B.ENTRO_ERR_ALIGN),
    ("type", E.ENTRO_U8, B.ENTRO_ERR_SCHEME), ("layer", 2, B.ENTRO_ERR_SIZE), ("q_heads", 12, B.ENTRO_ERR_SIZE), ("scale", float("nan"), B.ENTRO_ERR_RANGE),
    ("out_token_stride", 1 << 50, B.ENTRO_ERR_SIZE)])
def test_attend_shared_refuses_queries_that_are_none(field, value, status):
    given = good()
    setattr(given[2], field, value)
    assert both(*given)[1] == status


def test_nothing_given_sizes_of_no_launch_and_calls_without_rows():
    for i in (0, 1, 3):
        given = list(good())
        given[i] = None
        assert both(*given) == (B.ENTRO_ERR_NULL, B.ENTRO_ERR_NULL)
    L, (cache, table, query, groups) = B.lib(), good()
    refs = [C.byref(x) for x in (cache, table, query, groups)]
    need = L.entro_cache_attend_shared_workspace_bytes(*refs)
    assert need > 0 and need % 4 == 0
    assert L.entro_cache_attend_shared(*refs, PTR, need - 1, None) == B.ENTRO_ERR_CAPACITY
    assert L.entro_cache_attend_shared(*refs, None, need, None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_attend_shared(*refs, PTR + 4, need, None) == B.ENTRO_ERR_ALIGN
    groups.groups = 1 << 21                                    # times 8 heads: no launch
    assert L.entro_cache_attend_shared(*refs, PTR, 1 << 60, None) == B.ENTRO_ERR_SIZE and L.entro_cache_attend_shared_workspace_bytes(*refs) == 0
    groups.groups, table.seqs = 2, 1 << 21
    assert L.entro_cache_attend_shared(*refs, PTR, 1 << 60, None) == B.ENTRO_ERR_SIZE
    table.seqs, query.tokens, query.q, query.out = 4, 0, None, None
    assert L.entro_cache_attend_shared(*refs, None, 0, None) == B.ENTRO_OK


def test_own_tokens_are_split_by_their_own_hint():
    """Parts of a row for tokens that a sequence has alone: by max_own where it is given, whatever max_shared says; no more than for all of max_len."""
    L, (cache, table, query, groups) = B.lib(), good()
    refs = [C.byref(x) for x in (cache, table, query, groups)]
    query.max_len, groups.max_shared = 32868, 32768

    def parts(max_own):
        groups.max_own = max_own
        need = L.entro_cache_attend_shared_workspace_bytes(*refs)
        assert need % (query.tokens * query.q_heads * (128 + 1) * 4) == 0
        return need // (query.tokens * query.q_heads * (128 + 1) * 4)
    assert parts(0) == parts(100) < parts(20000) <= parts(32868) == parts((1 << 32) - 1) <= 256
    groups.max_shared = (1 << 32) - 1
    assert parts(0) == parts(1) < parts(32868) == parts((1 << 32) - 1) <= 256


@pytest.mark.parametrize("call,tensor", [(call, tensor) for call, more in [("shared", []), ("attend_shared", ["q", "out", "lse", "start", "workspace"])]
                                         for tensor in [None, "pool.k", "pool.v", "pool.k_scale", "pool.v_scale", "slots", "lengths", "first", "shared"] + more])
def test_calls_refuse_any_one_tensor_in_host_memory(calls_made, monkeypatch, call, tensor):  # noqa: F811
    monkeypatch.setattr(B, "_run_on", lambda device, run: run())

    def at(name, *shape, dtype=torch.float32):
        x = torch.zeros(*shape, dtype=dtype)
        return x if name == tensor else x.as_subclass(Placed)
    cache = E.Cache(at("pool.k", 1, 4, 2, 16, 64, dtype=torch.uint8), at("pool.v", 1, 4, 2, 64, 16, dtype=torch.uint8), at("pool.k_scale", 1, 4, 2),
                    at("pool.v_scale", 1, 4, 2), 16, 40)
    ints = lambda name, *shape: at(name, *shape, dtype=torch.int32)  # noqa: E731
    table, groups = E.CacheTable(ints("slots", 3, 5), ints("lengths", 3)), E.CacheGroups(ints("first", 3), ints("shared", 2), 2, 64)
    query = E.CacheQuery(at("q", 7, 4, 40), at("out", 7, 4, 40), ints("start", 4), 1, 9, lse=at("lse", 7, 4))

    def run():
        if call == "shared":
            E.entro_cache_shared(cache, table, groups)
        else:
            E.entro_cache_attend_shared(cache, table, query, groups, at("workspace", 1 << 16, dtype=torch.uint8))
    if tensor is None:
        run()
        assert calls_made == ["entro_cache_" + call]
    else:
        with pytest.raises(ValueError, match="one GPU"):
            run()
        assert calls_made == []


def test_the_binding_looks_at_groups():
    ints = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    for bad in (lambda: E.CacheGroups(ints(1), ints(0), 1, 1), lambda: E.CacheGroups(ints(4), ints(2), 1, 1), lambda: E.CacheGroups(ints(4).long(), ints(3), 1, 1),
                lambda: E.CacheGroups(ints(8)[::2], ints(3), 1, 1)):
        with pytest.raises(ValueError):
            bad()


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    include, attend = '#include "entro_cache.h"', source("entro_attend.hip")

    def part(begin, end=None):
        at = attend.index(begin)
        return attend[at: attend.index(end, at) if end else None]
    stubs = """#define __builtin_amdgcn_readfirstlane(x) (x)
namespace {
template <int W, typename T, bool MANY, typename... A> void k_attend_shared(const A &...) {}
template <int W, typename T, typename... A> void k_shared_join(const A &...) {}
}
"""
    L = compiled(tmp_path_factory.mktemp("host_shared"), "host_cache.cpp", "\n".join([
        stubs, source("entro_cache.h"), source("entro_cache.hip").replace(include, ""), "namespace {", part("struct Query {", "typedef"),
        part("constexpr uint32_t kMostSplits", "constexpr float"), part("struct Groups {", "// The group of sequence b"), part("// Tokens in leading pages")]))
    for name in ("entro_cache_shared", "entro_cache_attend_shared", "entro_cache_attend_shared_workspace_bytes"):
        twin = getattr(B.lib(), name)
        getattr(L, name).argtypes, getattr(L, name).restype = twin.argtypes, twin.restype
    return L


@pytest.mark.parametrize("first_wave", [0, 2])
@pytest.mark.parametrize("first,long", [([0, 3, 3, 5], False), ([0, 5], True), ([-2, 2, 9], True), ([-2, 2, 9], False), ([4, 2, 1], True)])
def test_what_is_shared_as_host_code(host, first_wave, first, long):
    host.host_first_wave(first_wave)
    rng, mem = np.random.default_rng(len(first)), Memory()
    page, pages, stride = 16, 900, 250
    table = np.tile(rng.permutation(pages)[:stride], (5, 1))
    lengths = np.array([4000, 3990, 4000, 3700, 4200])
    table[3:, 220:] = 0
    table[2, 240], table[1, 208] = 5, 7
    if long:
        table = np.concatenate([np.full((5, 1), 3), table, table], 1)
        stride = table.shape[1]
        lengths = stride * page - np.array([0, 10, 0, 300, -100])
    slots, at = mem(table, np.int32), mem(lengths, np.int32)
    begin, out = mem(first, np.int32), mem(np.full(len(first) + 1, 77), np.int32)
    cache, t, g = B.CCache(PTR, PTR, PTR, PTR, 1, pages, page, 1, 64, 0), B.CCacheTable(slots.ctypes.data, at.ctypes.data, 5, stride), B.CCacheGroups(
        begin.ctypes.data, out.ctypes.data, len(first) - 1, 1, 1, 0)
    assert host.entro_cache_shared(C.byref(cache), C.byref(t), C.byref(g), None) == B.ENTRO_OK
    for i, (a, b) in enumerate(zip(first[:-1], first[1:])):
        a, b, n = max(a, 0), min(b, 5), 0
        while a < b and n < stride and all((n + 1) * page <= lengths[r] and table[r, n] == table[a, n] for r in range(a, b)):
            n += 1
        assert out[i] == n * page
    assert list(out[-2:]) == [77, 77]


@pytest.mark.parametrize("what", ["fork", "take back", "window", "end"])
def test_what_a_group_shares_shrinks_where_tokens_or_pages_go(host, what):
    """Three rows behind 64 tokens of a prompt, forked among themselves and grown: they share no less than before. With tokens of one taken back and others in
    their place, pages dropped by a window or a row that ends and begins anew they share less, though every row goes on from one of the group."""
    host.host_first_wave(0)
    host.entro_cache_regroup.argtypes = B.lib().entro_cache_regroup.argtypes
    host.entro_cache_pages_workspace_bytes.restype = C.c_uint64
    mem, page, pages, rows, stride = Memory(), 16, 60, 3, 20
    pool = ref.Pool(np.random.default_rng(1), 1, pages, 1, page, 1)
    own_memory(mem, pool)
    table, lengths = np.full((rows, stride), -1, np.int32), np.array([64, 64, 64], np.int32)
    table[:, :4] = [7, 3, 11, 20]

    def shared():
        slots, at, first, out = mem(table, np.int32), mem(lengths, np.int32), mem([0, rows], np.int32), mem([77], np.int32)
        cache, t, g = B.CCache(PTR, PTR, PTR, PTR, 1, pages, page, 1, 1, 0), B.CCacheTable(slots.ctypes.data, at.ctypes.data, rows, stride), B.CCacheGroups(
            first.ctypes.data, out.ctypes.data, 1, rows, 64, 0)
        assert host.entro_cache_shared(C.byref(cache), C.byref(t), C.byref(g), None) == B.ENTRO_OK
        n = 0
        while all((n + 1) * page <= lengths[r] and table[r, n] == table[0, n] and table[r, n] >= 0 for r in range(rows)):
            n += 1
        assert out[0] == n * page
        return n * page

    def regroup(parent, grow, window=0):
        parent, grow = mem(parent, np.int32), mem(grow, np.int32)
        to, then, status = page_call(host, mem, pool, table, lengths, rows, stride, lambda c, t, n, st, ws, size: host.entro_cache_regroup(
            c, t, parent.ctypes.data, grow.ctypes.data, window, 0, n, st, ws, size, None))
        assert status[0] == 0
        return to, then
    before = shared()
    assert before == 64
    steps = {"fork": [([0, 1, 2], [40, 7, 20]), ([0, 0, 2], [1, 1, 1])], "take back": [([0, 1, 2], [-30, 5, 5]), ([0, 1, 2], [60, 60, 60])],
             "window": [([0, 1, 2], [200, 1, 2], 0), ([0, 1, 2], [1, 1, 1], 50)], "end": [([-1, 1, 2], [0, 5, 5]), ([0, 1, 2], [100, 5, 5])]}[what]
    for step in steps:
        table, lengths = regroup(*step)
    assert shared() >= before if what == "fork" else shared() < before


@pytest.mark.parametrize("seqs,stride,kv_heads,group,tokens,groups", [(64, 128, 8, 4, 64, 1), (64, 128, 8, 4, 3000, 16), (1, 8, 1, 1, 1, 1), (1, 1 << 20, 8, 8, 1 << 20, 5),
                                                                      (4096, 4096, 32, 1, 4096, 4096), (60000, 30000, 64, 1, 60000, 2), (7, 100, 2, 16, 40, 100000)])
def test_hints_of_any_size_make_launches_that_a_gpu_takes(host, seqs, stride, kv_heads, group, tokens, groups):
    """Whatever hints say: less than 2^32 lanes along x, less than 2^16 workgroups along y, a workspace of 256 parts a row at most, and the call succeeds."""
    at, out = 1 << 16, (C.c_uint64 * 3000)()
    cache, table = B.CCache(at, at, at, at, 1, 1 << 20, 64, kv_heads, 64, 0), B.CCacheTable(at, at, seqs, stride)
    row = kv_heads * 64
    host.host_only_note(1)
    host.host_launches(out, 3000)
    for max_new in HINTS:
        for max_len in HINTS:
            for max_seqs in (0, 3, (1 << 32) - 1):
                for max_shared in (0, 5000, (1 << 32) - 1):
                    for window in (0, 1 << 20):
                        query = B.CCacheQuery(at, at, at, row * group, 64, row * group, 64, at, tokens, max_new, max_len, kv_heads * group, E.ENTRO_BF16, 0, window, 4, 0.1, 0)
                        g = B.CCacheGroups(at, at, groups, max_seqs, max_shared, 0)
                        refs = [C.byref(x) for x in (cache, table, query, g)]
                        need = host.entro_cache_attend_shared_workspace_bytes(*refs)
                        assert 0 < need <= tokens * kv_heads * group * 256 * 65 * 4
                        assert host.entro_cache_attend_shared(*refs, at, need, None) == B.ENTRO_OK
        n = host.host_launches(out, 3000)
        assert n == 3 * 2 * 6 * 18
        for i in range(0, n, 3):
            assert 0 < out[i] < 1 << 32 and 0 < out[i + 1] and 0 < out[i + 2] < 1 << 16
    host.host_only_note(0)
