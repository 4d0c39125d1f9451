"""Host side of positions: angles, refusals before anything reaches a GPU, the binding's own checks, and the kernels as host code (CPU only)."""
import ctypes as C
import decimal

import numpy as np
import pytest
import torch

import cache_reference as ref
import large_rows as large
import paper_2505_02380_amd as E
import rotary_reference as rot
from paper_2505_02380_amd import binding as B
from test_cache_host import Placed, calls_made  # noqa: F401
from test_cache_on_cpu import Memory, compiled, own_memory, source

PTR = 0x10000          # an address that is aligned; no call below gets as far as using it


def test_struct_layouts_match_header():
    assert [C.sizeof(x) for x in (B.CRotary, B.CRotaryRows)] == [56, 56]


@pytest.mark.parametrize("dims,base", [(2, 1.0), (64, 10000.0), (128, 500000.0), (256, 1e6), (10, 123.5)])
def test_turns_are_the_definition_s(dims, base):
    """A pair's turns are off by no more than a rounding and the 64 bits of its frequency."""
    decimal.getcontext().prec = 60
    pi = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582")
    turns = E.entro_rotary_turns(dims, base)
    for i, t in enumerate(turns):
        f = decimal.Decimal(base) ** (decimal.Decimal(-2 * i) / dims)
        want = f / (2 * pi) * 2 ** 64
        assert abs(decimal.Decimal(int(t)) - want) <= 1 + want * decimal.Decimal(2) ** -61
    assert len(E.entro_rotary_turns(0)) == 0


def test_turns_of_longer_contexts():
    dims, base, factor, trained = 64, 10000.0, 4.0, 2048.0
    f = base ** (-np.arange(0, dims, 2) / dims)
    as_is = E.entro_rotary_turns(dims, base).astype(np.float64)
    linear = E.entro_rotary_turns(dims, base, E.ENTRO_CONTEXT_LINEAR, factor).astype(np.float64)
    assert np.allclose(linear * factor, as_is, rtol=1e-12, atol=factor)
    parts = E.entro_rotary_turns(dims, base, E.ENTRO_CONTEXT_BY_PARTS, factor, trained, 1.0, 32.0).astype(np.float64)
    r = trained * f / (2 * np.pi)
    g = np.clip((r - 1) / 31, 0, 1)
    assert np.allclose(parts, as_is * (g + (1 - g) / factor), rtol=1e-12, atol=1)
    assert (g == 1).any() and (g == 0).any() and ((g > 0) & (g < 1)).any()
    assert np.array_equal(parts[g == 1], as_is[g == 1])


@pytest.mark.parametrize("args,status", [
    ((7, 1e4, 0, 1, 1, 1, 32), B.ENTRO_ERR_SIZE), ((258, 1e4, 0, 1, 1, 1, 32), B.ENTRO_ERR_SIZE), ((64, 1e4, 3, 1, 1, 1, 32), B.ENTRO_ERR_SCHEME),
    ((64, 0.5, 0, 1, 1, 1, 32), B.ENTRO_ERR_RANGE), ((64, float("nan"), 0, 1, 1, 1, 32), B.ENTRO_ERR_RANGE), ((64, float("inf"), 0, 1, 1, 1, 32), B.ENTRO_ERR_RANGE),
    ((64, 1e4, 1, 0.5, 1, 1, 32), B.ENTRO_ERR_RANGE), ((64, 1e4, 2, 2, 0, 1, 32), B.ENTRO_ERR_RANGE), ((64, 1e4, 2, 2, 10, 32, 32), B.ENTRO_ERR_RANGE),
    ((64, 1e4, 2, 2, 10, -1, 32), B.ENTRO_ERR_RANGE), ((64, 1e4, 2, float("nan"), 10, 1, 32), B.ENTRO_ERR_RANGE)])
def test_turns_refuse_what_defines_none(args, status):
    out = (C.c_uint64 * 128)()
    assert B.lib().entro_rotary_turns(*args, out) == status
    assert B.lib().entro_rotary_turns(64, 1e4, 0, 1, 1, 1, 32, None) == B.ENTRO_ERR_NULL


def good():
    rotary = B.CRotary(PTR, PTR, PTR, 0, 128, 64, 1, 1, 1e-6, 1.0, 0)
    q, k = (B.CRotaryRows(PTR, PTR * 2, h * 128, 128, h * 128, 128, h, 0) for h in (32, 8))
    return rotary, q, k


def rotate(rotary, q, k, positions=PTR, tokens=5, head_dim=128, kind=E.ENTRO_BF16):
    by = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return B.lib().entro_rotate(by(rotary), by(q), by(k), positions, tokens, head_dim, kind, None)


def append(rotary, q, rows=None, cache=None, table=None):
    by = lambda x: None if x is None else C.byref(x)  # noqa: E731
    cache = cache or B.CCache(PTR, PTR, PTR, PTR, 2, 100, 64, 8, 128, 0)
    table = table or B.CCacheTable(PTR, PTR, 4, 16)
    rows = rows or B.CCacheRows(PTR, PTR, 1024, 128, 1024, 128, PTR, 5, 2, E.ENTRO_BF16, 1)
    return B.lib().entro_cache_append_rotated(C.byref(cache), C.byref(table), C.byref(rows), by(rotary), by(q), None)


@pytest.mark.parametrize("field,value,status", [
    ("turns", None, B.ENTRO_ERR_NULL), ("turns", PTR + 8, B.ENTRO_ERR_ALIGN), ("q_gain", PTR + 2, B.ENTRO_ERR_ALIGN), ("k_gain", PTR + 1, B.ENTRO_ERR_ALIGN),
    ("dims", 63, B.ENTRO_ERR_SIZE), ("dims", 130, B.ENTRO_ERR_SIZE), ("layout", 2, B.ENTRO_ERR_SCHEME), ("norm", 3, B.ENTRO_ERR_SCHEME), ("eps", 0.0, B.ENTRO_ERR_RANGE),
    ("eps", float("nan"), B.ENTRO_ERR_RANGE), ("amplitude", float("inf"), B.ENTRO_ERR_RANGE), ("amplitude", float("nan"), B.ENTRO_ERR_RANGE)])
def test_both_calls_refuse_rotations_that_are_none(field, value, status):
    rotary, q, k = good()
    setattr(rotary, field, value)
    assert rotate(rotary, q, k) == status and append(rotary, q) == status


@pytest.mark.parametrize("field,value,status", [
    ("x", None, B.ENTRO_ERR_NULL), ("y", None, B.ENTRO_ERR_NULL), ("x", PTR + 1, B.ENTRO_ERR_ALIGN), ("y", PTR + 1, B.ENTRO_ERR_ALIGN), ("heads", 0, B.ENTRO_ERR_SIZE),
    ("heads", 65537, B.ENTRO_ERR_SIZE), ("x_token_stride", 1 << 50, B.ENTRO_ERR_SIZE), ("y_head_stride", 1 << 50, B.ENTRO_ERR_SIZE)])
def test_both_calls_refuse_rows_that_are_none(field, value, status):
    rotary, q, k = good()
    setattr(q, field, value)
    assert rotate(rotary, q, k) == status and rotate(rotary, k, q) == status and append(rotary, q) == status
    in_place = B.CRotaryRows(PTR, PTR, 4096, 128, 8192, 128, 32, 0)
    assert rotate(rotary, in_place, None) == B.ENTRO_ERR_SIZE and append(rotary, in_place) == B.ENTRO_ERR_SIZE


def test_refusals_of_calls():
    rotary, q, k = good()
    assert rotate(None, q, k) == B.ENTRO_ERR_NULL and rotate(rotary, None, None) == B.ENTRO_ERR_NULL and rotate(rotary, q, k, None) == B.ENTRO_ERR_NULL
    assert rotate(rotary, q, k, PTR + 2) == B.ENTRO_ERR_ALIGN
    assert rotate(rotary, q, k, kind=E.ENTRO_U8) == B.ENTRO_ERR_SCHEME and rotate(rotary, q, k, head_dim=0) == B.ENTRO_ERR_SIZE
    assert rotate(rotary, q, k, head_dim=257) == B.ENTRO_ERR_SIZE and rotate(rotary, q, k, head_dim=63) == B.ENTRO_ERR_SIZE
    assert rotate(rotary, q, k, tokens=1 << 26) == B.ENTRO_ERR_SIZE and rotate(rotary, q, k, tokens=60000000) == B.ENTRO_ERR_SIZE
    assert rotate(rotary, q, k, None, 0) == B.ENTRO_OK
    assert append(None, q) == B.ENTRO_ERR_NULL
    for field, value, status in [("k", None, B.ENTRO_ERR_NULL), ("start", None, B.ENTRO_ERR_NULL), ("k", PTR + 1, B.ENTRO_ERR_ALIGN), ("start", PTR + 4, B.ENTRO_ERR_ALIGN),
                                 ("type", E.ENTRO_U8, B.ENTRO_ERR_SCHEME), ("layer", 2, B.ENTRO_ERR_SIZE), ("v_token_stride", 1 << 50, B.ENTRO_ERR_SIZE),
                                 ("tokens", 1 << 31, B.ENTRO_ERR_SIZE)]:
        rows = B.CCacheRows(PTR, PTR, 1024, 128, 1024, 128, PTR, 5, 2, E.ENTRO_BF16, 1)
        setattr(rows, field, value)
        assert append(rotary, None, rows) == status
    assert append(rotary, None, cache=B.CCache(PTR, PTR, PTR, PTR, 2, 100, 48, 8, 128, 0)) == B.ENTRO_ERR_SIZE
    assert append(rotary, None, table=B.CCacheTable(PTR, None, 4, 16)) == B.ENTRO_ERR_NULL
    assert append(rotary, None, rows=B.CCacheRows(None, None, 1024, 128, 1024, 128, PTR, 0, 2, E.ENTRO_BF16, 1)) == B.ENTRO_OK


def test_the_binding_looks_at_shapes_and_types(calls_made):  # noqa: F811
    placed = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype).as_subclass(Placed)  # noqa: E731
    turns = placed(8, dtype=torch.int64)
    for bad in (lambda: E.Rotary(turns, 18), lambda: E.Rotary(None, 16), lambda: E.Rotary(placed(8), 16), lambda: E.Rotary(turns, 16, q_gain=placed(4, dtype=torch.float64)),
                lambda: E.RotaryRows(placed(4, 2, 16), placed(4, 2, 17)), lambda: E.RotaryRows(placed(4, 2, 16).transpose(1, 2)),
                lambda: E.RotaryRows(placed(4, 2, 16), placed(1, 2, 16).expand(4, 2, 16))):
        with pytest.raises(ValueError):
            bad()
    r, q, k, at = E.Rotary(turns, 16, q_gain=placed(16)), E.RotaryRows(placed(4, 2, 16)), E.RotaryRows(placed(4, 1, 16)), placed(4, dtype=torch.int32)
    for bad in (lambda: E.entro_rotate(r, None, None, at), lambda: E.entro_rotate(r, q, E.RotaryRows(placed(5, 1, 16)), at),
                lambda: E.entro_rotate(r, q, E.RotaryRows(placed(4, 1, 16).to(torch.bfloat16).as_subclass(Placed)), at), lambda: E.entro_rotate(r, q, k, at[:3]),
                lambda: E.entro_rotate(r, E.RotaryRows(placed(4, 2, 24)), None, at), lambda: E.entro_rotate(r, q, k, placed(4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            bad()
    assert calls_made == []


@pytest.mark.parametrize("call,tensor", [(call, tensor) for call, more in [
    ("rotate", ["q", "q.y", "k", "k.y", "positions", "turns", "q_gain", "k_gain"]),
    ("append", ["pool.k", "pool.v", "pool.k_scale", "pool.v_scale", "slots", "lengths", "k", "v", "start", "q", "q.y", "turns", "q_gain", "k_gain"])] for tensor in [None] + more])
def test_calls_refuse_any_one_tensor_in_host_memory(calls_made, monkeypatch, call, tensor):  # noqa: F811
    monkeypatch.setattr(B, "_run_on", lambda device, run: run())

    def at(name, *shape, dtype=torch.float32):
        x = torch.zeros(*shape, dtype=dtype)
        return x if name == tensor else x.as_subclass(Placed)
    r = E.Rotary(at("turns", 16, dtype=torch.int64), 32, q_gain=at("q_gain", 40), k_gain=at("k_gain", 2, 40))
    q = E.RotaryRows(at("q", 7, 4, 40), at("q.y", 7, 4, 40))
    if call == "rotate":
        run = lambda: E.entro_rotate(r, q, E.RotaryRows(at("k", 7, 2, 40), at("k.y", 7, 2, 40)), at("positions", 7, dtype=torch.int32))  # noqa: E731
    else:
        cache = E.Cache(at("pool.k", 1, 4, 2, 16, 64, dtype=torch.uint8), at("pool.v", 1, 4, 2, 64, 16, dtype=torch.uint8), at("pool.k_scale", 1, 4, 2),
                        at("pool.v_scale", 1, 4, 2), 16, 40)
        table = E.CacheTable(at("slots", 3, 5, dtype=torch.int32), at("lengths", 3, dtype=torch.int32))
        run = lambda: E.entro_cache_append_rotated(cache, table, E.CacheRows(at("k", 7, 2, 40), at("v", 7, 2, 40), at("start", 4, dtype=torch.int32), 1), r, q)  # noqa: E731
    if tensor is None:
        run()
        assert len(calls_made) == 1
    else:
        with pytest.raises(ValueError, match="one GPU"):
            run()
        assert calls_made == []


# ----------------------------------------------------------------------------------------------------- kernels as host code
@pytest.fixture(scope="module")
def host(tmp_path_factory):
    include = '#include "entro_cache.h"'
    prelude = """#define __builtin_amdgcn_readfirstlane(x) (x)
namespace {
// lane moves: neighbours, pairs of neighbours, mirrored eights and sixteens
int moved(int v, int how) {
    const uint32_t l = threadIdx.x & 63u;
    return shuffle(v, how == 0xb1 ? l ^ 1 : how == 0x4e ? l ^ 2 : how == 0x141 ? l ^ 7 : l ^ 15);
}
#define __builtin_amdgcn_mov_dpp(v, how, rows, banks, bound) moved(v, how)
int __any(int x) {
    for (uint32_t o = 1; o < 64; o <<= 1) x |= shuffle(x, (threadIdx.x & 63u) ^ o);
    return x;
}
float __shfl_xor(float v, int o) { return __builtin_bit_cast(float, __shfl_xor(__builtin_bit_cast(int, v), o)); }
uint32_t __umulhi(uint32_t a, uint32_t b) { return static_cast<uint32_t>(uint64_t{a} * b >> 32); }
float rsqrtf(float x) { return 1.0f / sqrtf(x); }
}
"""
    L = compiled(tmp_path_factory.mktemp("host_rotate"), "host_cache.cpp", "\n".join([
        prelude, source("entro_cache.h"), source("entro_cache.hip").replace(include, ""), source("entro_rotate.hip").replace(include, "").replace("kWG", "kRotateWG")]))
    for name in ("entro_rotate", "entro_cache_append_rotated", "entro_cache_append"):
        getattr(L, name).argtypes = getattr(B.lib(), name).argtypes
    return L


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dim,dims,norm", [(24, 16, "rms"), (17, 10, "centred"), (128, 128, "none"), (5, 0, "rms")])
def test_rotate_as_host_code(host, dim, dims, norm, layout):
    """Rows with guards all round, in memory that ends where they do."""
    rng = np.random.default_rng(dim)
    mem, tokens, heads = Memory(), 3, (3, 1)
    turns = mem(E.entro_rotary_turns(dims))
    gain = mem(rng.standard_normal(dim), np.float32)
    rotary = B.CRotary(turns.ctypes.data if dims else None, gain.ctypes.data, None, 0, 0, dims, layout == "pairs", ["none", "rms", "centred"].index(norm), 1e-5, 1.0, 0)
    x = [mem(rng.standard_normal((tokens, h, dim)), np.float32) for h in heads]
    y = [mem(np.full((tokens + 2, h, dim), 7), np.float32) for h in heads]
    sides = [B.CRotaryRows(a.ctypes.data, b[1:].ctypes.data, h * dim, dim, h * dim, dim, h, 0) for a, b, h in zip(x, y, heads)]
    positions = mem([0, 77, -2 ** 31], np.int32)
    host.host_first_wave(1)
    assert host.entro_rotate(C.byref(rotary), C.byref(sides[0]), C.byref(sides[1]), positions.ctypes.data, tokens, dim, E.ENTRO_F32, None) == B.ENTRO_OK
    for a, b, g in zip(x, y, (gain, None)):
        want, bound = rot.rotate(a, positions, turns, layout, norm, g, 1e-5)
        assert np.all(np.abs(b[1:-1] - want) <= rot.tolerance(want, bound, "f32")) and np.all(b[[0, -1]] == 7)


@pytest.mark.parametrize("dim", [17, 80, 96, 112, 128, 192])
def test_centred_norm_of_heads_far_from_zero(host, dim):
    """Heads whose elements are equal, or nearly so, give what is left after their mean and not the mean's own rounding."""
    rng = np.random.default_rng(dim)
    mem, eps = Memory(), 1e-6
    heads = rot.far_heads(rng, dim)
    x = mem(heads[None], np.float32)
    y, at = mem(np.zeros_like(x)), mem([5], np.int32)
    rotary = B.CRotary(None, None, None, 0, 0, 0, 0, 2, eps, 1.0, 0)
    side = B.CRotaryRows(x.ctypes.data, y.ctypes.data, x[0].size, dim, x[0].size, dim, len(heads), 0)
    host.host_first_wave(0)
    assert host.entro_rotate(C.byref(rotary), C.byref(side), None, at.ctypes.data, 1, dim, E.ENTRO_F32, None) == B.ENTRO_OK
    want, bound = rot.centred(x, eps)
    assert np.all(np.abs(y - want) <= bound), np.argwhere(~(np.abs(y - want) <= bound))[:4]


def test_the_rows_of_large_calls_take_the_kernels_they_are_meant_for(host):
    """The cases that the GPU tests of large calls have, by their launches: one head a lane group or several, queries with the cache's workgroups or apart."""
    at, out = 1 << 16, (C.c_uint64 * 12)()
    host.host_only_note(1)
    host.host_launches(out, 12)
    for kind, tokens, q_heads, kv_heads, dim, dims, each in large.ROTATE:
        rotary = B.CRotary(at, None, None, 0, 0, dims, 0, 1, 1e-5, 1.0, 0)
        q, k = (B.CRotaryRows(at, 2 * at, h * dim, dim, h * dim, dim, h, 0) if h else None for h in (q_heads, kv_heads))
        assert host.entro_rotate(C.byref(rotary), C.byref(q), k and C.byref(k), at, tokens, dim, E.ENTRO_BF16 if kind == "bf16" else E.ENTRO_F32, None) == B.ENTRO_OK
        assert host.host_launches(out, 12) == 3
        assert out[1] == large.workgroups(tokens, q_heads + kv_heads, each, dim, dims), (kind, tokens)
        assert large.workgroups(tokens, q_heads + kv_heads, 1, dim, dims) != large.workgroups(tokens, q_heads + kv_heads, 8, dim, dims)
    for kind, q_heads, heads, dim, dims, page, new, apart in large.APPEND:
        rotary, tokens = B.CRotary(at, None, None, 0, 0, dims, 0, 1, 1e-5, 1.0, 0), sum(new) + 1
        cache, table = B.CCache(at, at, at, at, 1, 100, page, heads, dim, 0), B.CCacheTable(at, at, len(new), 5000)
        q = B.CRotaryRows(at, 2 * at, q_heads * dim, dim, q_heads * dim, dim, q_heads, 0)
        rows = B.CCacheRows(at, at, heads * dim, dim, heads * dim, dim, at, tokens, max(new), E.ENTRO_BF16 if kind == "bf16" else E.ENTRO_F32, 0)
        assert host.entro_cache_append_rotated(C.byref(cache), C.byref(table), C.byref(rows), C.byref(rotary), C.byref(q), None) == B.ENTRO_OK
        assert host.host_launches(out, 12) == (6 if apart else 3), (kind, new)
    host.host_only_note(0)


@pytest.mark.parametrize("first_wave", [0, 1, 3])
@pytest.mark.parametrize("page,dim,dims", [(64, 128, 128), (16, 24, 16)])
def test_append_rotated_moves_older_codes_whichever_wavefront_comes_first(host, first_wave, page, dim, dims):
    """A block written token by token, every token raising its scale, as rotate and entro_cache_append would; then pages that are none."""
    host.host_first_wave(first_wave)
    rng = np.random.default_rng(first_wave)
    mem, tokens = Memory(), 6
    pool = ref.Pool(rng, 1, 1, 1, page, dim)
    twin = pool.copy()
    own_memory(mem, pool), own_memory(mem, twin)
    turns = mem(E.entro_rotary_turns(dims))
    rotary = B.CRotary(turns.ctypes.data, None, None, 0, 0, dims, 0, 1, 1e-5, 1.0, 0)
    caches = [B.CCache(p.k.ctypes.data, p.v.ctypes.data, p.k_scale.ctypes.data, p.v_scale.ctypes.data, 1, 1, page, 1, dim, 0) for p in (pool, twin)]
    for n in range(1, tokens + 2):
        slots, lengths, start, at = mem([[0 if n <= tokens else 5]], np.int32), mem([n], np.int32), mem([0, 1], np.int32), mem([n - 1], np.int32)
        gain = mem(np.full(dim, 1.3 ** n), np.float32)
        rotary.q_gain = rotary.k_gain = gain.ctypes.data
        k, v, q = (mem(rng.standard_normal((1, h, dim)) * 1.3 ** n, np.float32) for h in (1, 1, 2))
        turned, q_out, q_want = mem(np.zeros_like(k)), mem(np.zeros_like(q)), mem(np.zeros_like(q))
        table = B.CCacheTable(slots.ctypes.data, lengths.ctypes.data, 1, 1)
        rows = [B.CCacheRows(x.ctypes.data, v.ctypes.data, dim, dim, dim, dim, start.ctypes.data, 1, 1, E.ENTRO_F32, 0) for x in (k, turned)]
        sides = [B.CRotaryRows(a.ctypes.data, b.ctypes.data, h * dim, dim, h * dim, dim, h, 0) for a, b, h in ((q, q_out, 2), (q, q_want, 2), (k, turned, 1))]
        assert host.entro_rotate(C.byref(rotary), C.byref(sides[1]), C.byref(sides[2]), at.ctypes.data, 1, dim, E.ENTRO_F32, None) == B.ENTRO_OK
        assert host.entro_cache_append(C.byref(caches[1]), C.byref(table), C.byref(rows[1]), None) == B.ENTRO_OK
        assert host.entro_cache_append_rotated(C.byref(caches[0]), C.byref(table), C.byref(rows[0]), C.byref(rotary), C.byref(sides[0]), None) == B.ENTRO_OK
        assert np.array_equal(q_out, q_want) and np.any(q_out)
        for name in ("k", "v", "k_scale", "v_scale"):
            assert np.array_equal(getattr(pool, name), getattr(twin, name)), (n, name)


@pytest.mark.parametrize("seqs,stride,kv_heads,q_heads,tokens", [(64, 128, 8, 32, 3000), (1, 8, 1, 1, 1), (4096, 4096, 32, 32, 4096), (60000, 30000, 64, 64, 60000), (1 << 23, 8, 1, 2, 9)])
def test_hints_of_any_size_make_launches_that_a_gpu_takes(host, seqs, stride, kv_heads, q_heads, tokens):
    at = 1 << 16
    cache, table = B.CCache(at, at, at, at, 1, 1 << 20, 64, kv_heads, 64, 0), B.CCacheTable(at, at, seqs, stride)
    rotary = B.CRotary(at, None, None, 0, 0, 64, 0, 1, 1e-5, 1.0, 0)
    q = B.CRotaryRows(at, at * 2, q_heads * 64, 64, q_heads * 64, 64, q_heads, 0)
    out = (C.c_uint64 * 300)()
    host.host_only_note(1)
    host.host_launches(out, 300)
    for max_new in (0, 1, 5, 1000, 1 << 20, (1 << 32) - 1):
        rows = B.CCacheRows(at, at, kv_heads * 64, 64, kv_heads * 64, 64, at, tokens, max_new, E.ENTRO_BF16, 0)
        assert host.entro_cache_append_rotated(C.byref(cache), C.byref(table), C.byref(rows), C.byref(rotary), C.byref(q), None) == B.ENTRO_OK
    assert host.entro_rotate(C.byref(rotary), C.byref(q), None, at, (1 << 31) // q_heads - 1, 64, E.ENTRO_BF16, None) == B.ENTRO_OK
    n = host.host_launches(out, 300)
    assert 3 * 7 <= n <= 3 * 13
    for i in range(0, n, 3):
        assert 0 < out[i] < 1 << 32 and 0 < out[i + 1] and 0 < out[i + 2] < 1 << 16
    host.host_only_note(0)
