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
    L = compiled(tmp_path_factory.mktemp("host_cache"), "host_cache.cpp", source("entro_cache.h") + source("entro_cache.hip").replace('#include "entro_cache.h"', ""))
    for call in (L.entro_cache_append, L.entro_cache_read):
        call.argtypes = [C.POINTER(B.CCache), C.POINTER(B.CCacheTable), C.POINTER(B.CCacheRows), C.c_void_p]
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
