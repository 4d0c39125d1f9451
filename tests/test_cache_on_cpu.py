"""The token cache's device sources as host code (host_cache.cpp), against the definitions in 64 bits: orders of wavefronts that a GPU
takes only now and then are taken every time here (CPU only)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import cache_reference as ref
import paper_2505_02380_amd as E
from paper_2505_02380_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_02380_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"


def source(name):
    return open(os.path.join(CSRC, name)).read().replace("#include <hip/hip_runtime.h>", "")


def compiled(build, main, text):
    """main, a file of this folder, with the text as its cache.inc."""
    (build / "cache.inc").write_text(text)
    lib = build / (os.path.splitext(main)[0] + ".so")
    subprocess.run([CLANG, "-std=c++20", "-O1", "-ffp-contract=off", "-shared", "-fPIC", "-pthread", "-Wl,-Bsymbolic", "-Wno-everything", "-I", str(build),
                    "-I", os.path.join(ROOT, "include"), os.path.join(os.path.dirname(__file__), main), "-o", str(lib)], check=True, capture_output=True)
    return C.CDLL(str(lib))


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    include, attend = '#include "entro_cache.h"', source("entro_attend.hip")

    def part(begin, end=None):
        at = attend.index(begin)
        return attend[at: attend.index(end, at) if end else None]

    L = compiled(tmp_path_factory.mktemp("host_cache"), "host_cache.cpp", "\n".join([
        source("entro_cache.h"), source("entro_cache.hip").replace(include, ""), "namespace {", part("struct Query {", "typedef"),
        part("constexpr uint32_t kMostSplits", "constexpr float"), part("entro_status check_query_sizes")]))
    for name in ("append", "read", "attend", "regroup", "compact"):
        call, twin = getattr(L, "entro_cache_" + name), getattr(B.lib(), "entro_cache_" + name)
        call.argtypes = twin.argtypes
    L.entro_cache_attend_workspace_bytes.restype = L.entro_cache_pages_workspace_bytes.restype = C.c_uint64
    return L


class Memory:
    """Arrays of a call in memory of the alignment that the calls ask for, kept as long as their addresses."""

    def __init__(self):
        self.kept = []

    def __call__(self, x, dtype=None):
        x = np.ascontiguousarray(x, dtype)
        raw = np.zeros(x.nbytes + 16, np.uint8)
        at = -raw.ctypes.data % 16
        own = raw[at: at + x.nbytes].view(x.dtype).reshape(x.shape)
        own[...] = x
        self.kept.append(own)
        return own


def append(host, mem, pool, table, lengths, k, v, start, max_new):
    """pool's arrays are the call's: they are changed in place."""
    cache = B.CCache(pool.k.ctypes.data, pool.v.ctypes.data, pool.k_scale.ctypes.data, pool.v_scale.ctypes.data, 1, pool.pages, pool.page, pool.heads, pool.dim, 0)
    slots, at, first, k, v = mem(table, np.int32), mem(lengths, np.int32), mem(start, np.int32), mem(k, np.float32), mem(v, np.float32)
    t = B.CCacheTable(slots.ctypes.data, at.ctypes.data, *slots.shape)
    r = B.CCacheRows(k.ctypes.data, v.ctypes.data, pool.heads * pool.dim, pool.dim, pool.heads * pool.dim, pool.dim, first.ctypes.data, len(k), max_new,
                     E.ENTRO_F32, 0)
    assert host.entro_cache_append(C.byref(cache), C.byref(t), C.byref(r), None) == B.ENTRO_OK


def own_memory(mem, pool):
    pool.k, pool.v, pool.k_scale, pool.v_scale = (mem(x) for x in (pool.k, pool.v, pool.k_scale, pool.v_scale))


@pytest.mark.parametrize("first_wave", [0, 1, 3])
@pytest.mark.parametrize("page,dim", [(64, 128), (16, 24)])
def test_append_moves_older_codes_whichever_wavefront_comes_first(host, first_wave, page, dim):
    """A block written token by token, every token raising its scale: all older codes move to the new grid, also those of a wavefront
    that has only begun when another one has written the new scale."""
    host.host_first_wave(first_wave)
    rng = np.random.default_rng(first_wave)
    mem, tokens = Memory(), 9
    pool = ref.Pool(rng, 1, 1, 1, page, dim)
    own_memory(mem, pool)
    twin = pool.copy()
    table = np.zeros((1, 1), int)
    for n in range(1, tokens + 1):
        k, v = (rng.standard_normal((1, 1, dim)).astype(np.float32) * np.float32(1.3 ** n) for _ in "kv")
        k[0, 0, 0], v[0, 0, 1] = 4 * 1.3 ** n, -5 * 1.3 ** n
        append(host, mem, pool, table, [n], k, v, [0, 1], 1)
        near = ref.append(twin, table, [n], k, v, [0, 1])
        assert np.array_equal(pool.k_scale, twin.k_scale) and np.array_equal(pool.v_scale, twin.v_scale)
        for name in "kv":
            away = getattr(pool, name) != getattr(twin, name)
            assert not np.any(away & ~near[name]), (n, np.argwhere(away & ~near[name])[:4])
        twin.k[...], twin.v[...] = pool.k, pool.v


def launched(host):
    out = (C.c_uint64 * 3000)()
    n = host.host_launches(out, 3000)
    return [tuple(out[i: i + 3]) for i in range(0, n, 3)]


HINTS = [1, 5, 1000, 1 << 20, (1 << 31) - 1, (1 << 32) - 1]


@pytest.mark.parametrize("seqs,stride,kv_heads,group,tokens", [
    (64, 128, 8, 4, 64), (64, 128, 8, 4, 3000), (1, 8, 1, 1, 1), (1, 1 << 20, 8, 8, 1 << 20), (4096, 4096, 32, 1, 4096), (60000, 30000, 64, 1, 60000), (7, 100, 2, 16, 40)])
def test_hints_of_any_size_make_launches_that_a_gpu_takes(host, seqs, stride, kv_heads, group, tokens):
    """Hints bound the work and nothing else: whatever they say, a launch has less than 2^32 lanes along x and less than 2^16 workgroups along
    y, and the call succeeds."""
    at = 1 << 16
    cache, table = B.CCache(at, at, at, at, 1, 1 << 20, 64, kv_heads, 64, 0), B.CCacheTable(at, at, seqs, stride)
    row = kv_heads * 64
    host.host_only_note(1)
    launched(host)
    for max_new in HINTS:
        rows = B.CCacheRows(at, at, row, 64, row, 64, at, tokens, max_new, E.ENTRO_BF16, 0)
        for call in (host.entro_cache_append, host.entro_cache_read):
            assert call(C.byref(cache), C.byref(table), C.byref(rows), None) == B.ENTRO_OK
        for max_len in HINTS:
            for window in (0, 1, 1 << 20):
                query = B.CCacheQuery(at, at, at, row * group, 64, row * group, 64, at, tokens, max_new, max_len, kv_heads * group, E.ENTRO_BF16, 0, window, 4, 0.1, 0)
                need = host.entro_cache_attend_workspace_bytes(C.byref(cache), C.byref(table), C.byref(query))
                assert host.entro_cache_attend(C.byref(cache), C.byref(table), C.byref(query), at, need, None) == B.ENTRO_OK
        for lanes, x, y in launched(host):
            assert 0 < lanes < 1 << 32 and 0 < x and 0 < y < 1 << 16, (max_new, lanes, x, y)
    host.host_only_note(0)


def test_attend_refuses_more_sequences_and_heads_than_a_launch_takes(host):
    at = 1 << 16
    cache, table = B.CCache(at, at, at, at, 1, 100, 16, 64, 64, 0), B.CCacheTable(at, at, 1 << 18, 1)
    query = B.CCacheQuery(at, at, None, 64, 64, 64, 64, at, 5, 1, 16, 64, E.ENTRO_BF16, 0, 0, 0, 0.1, 0)
    host.host_only_note(1)
    launched(host)
    assert host.entro_cache_attend(C.byref(cache), C.byref(table), C.byref(query), None, 0, None) == B.ENTRO_ERR_SIZE and not launched(host)
    table.seqs = (1 << 18) - 8
    assert host.entro_cache_attend(C.byref(cache), C.byref(table), C.byref(query), None, 0, None) == B.ENTRO_OK and len(launched(host)) == 1
    host.host_only_note(0)


def page_call(host, mem, pool, table, lengths, seqs, stride, call):
    """(next table, lengths, status) of regroup or compact; pool's pages move in place."""
    layers = pool.k.shape[0]
    cache = B.CCache(pool.k.ctypes.data, pool.v.ctypes.data, pool.k_scale.ctypes.data, pool.v_scale.ctypes.data, layers, pool.pages, pool.page, pool.heads, pool.dim, 0)
    slots, at = mem(table, np.int32), mem(lengths, np.int32)
    to, then, status = mem(np.full((seqs, stride), 77), np.int32), mem(np.full(seqs, 77), np.int32), mem(np.full(4, 77), np.int32)
    t, n = B.CCacheTable(slots.ctypes.data, at.ctypes.data, *slots.shape), B.CCacheTable(to.ctypes.data, then.ctypes.data, seqs, stride)
    need = host.entro_cache_pages_workspace_bytes(C.byref(cache), C.byref(t), C.byref(n))
    room = mem(np.full(need, 0xAB), np.uint8)
    assert call(C.byref(cache), C.byref(t), C.byref(n), status.ctypes.data, room.ctypes.data, need) == B.ENTRO_OK
    return to, then, status


@pytest.mark.parametrize("first_wave,seqs,stride,page,most", [(0, 12, 20, 16, 150), (15, 12, 20, 16, 150), (2, 40, 9, 32, 60), (1, 20, 850, 16, 120)])
def test_page_tables_whichever_wavefront_comes_first(host, first_wave, seqs, stride, page, most):
    """Regroup and compact, by one workgroup and (the last sizes) by several launches, with forks, drops, growth, windows and pages that are none."""
    host.host_first_wave(first_wave)
    rng = np.random.default_rng(first_wave + seqs)
    lengths = rng.integers(0, most, seqs)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 2 * seqs + 10
    pool, mem = ref.Pool(rng, 1, pages, 1, page, 1), Memory()
    pool.k_scale[...], pool.v_scale[...] = rng.random(pool.k_scale.shape), rng.random(pool.v_scale.shape)
    own_memory(mem, pool)
    order, table, at = rng.permutation(pages), np.full((seqs, stride), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at: at + n]
        at += n
    table[3, 0] = pages + 5
    parent = mem(np.where(rng.random(seqs) < 0.2, np.arange(seqs), rng.integers(-1, seqs + 1, seqs)), np.int32)
    grow = mem(rng.integers(-20, 12, seqs), np.int32)
    window, sinks = 50, 20
    twin = pool.copy()
    want = ref.regroup(pages, page, table, lengths, seqs, stride, parent, grow, window, sinks)
    assert want is not None and len(want[2]) > 0
    to, then, status = page_call(host, mem, pool, table, lengths, seqs, stride, lambda c, t, n, st, ws, size: host.entro_cache_regroup(
        c, t, parent.ctypes.data, grow.ctypes.data, window, sinks, n, st, ws, size, None))
    assert np.array_equal(to, want[0]) and np.array_equal(then, want[1]) and list(status) == [0, want[3], pages - want[3], len(want[2])]
    ref.copy_pages(twin, want[2])
    for name in ("k", "v", "k_scale", "v_scale"):
        assert np.array_equal(getattr(pool, name), getattr(twin, name)), name
    want = ref.compact(pages, to, then)
    to, then, status = page_call(host, mem, pool, to, then, seqs, stride, lambda c, t, n, st, ws, size: host.entro_cache_compact(c, t, n, st, ws, size, None))
    assert np.array_equal(to, want[0]) and np.array_equal(then, want[1]) and list(status) == [0, want[3], pages - want[3], len(want[2])]
    ref.copy_pages(twin, want[2])
    for name in ("k", "v", "k_scale", "v_scale"):
        assert np.array_equal(getattr(pool, name), getattr(twin, name)), name
