"""Host side of the token cache: sizes, refusals before anything reaches a GPU, and the binding's own checks (CPU only)."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2505_02380_amd as E
from paper_2505_02380_amd import binding as B

PTR = 0x10000          # an address that is aligned; no call below gets as far as using it


def good():
    cache = B.CCache(PTR, PTR, PTR, PTR, 2, 100, 64, 8, 128, 0)
    table = B.CCacheTable(PTR, PTR, 4, 16)
    rows = B.CCacheRows(PTR, PTR, 1024, 128, 1024, 128, PTR, 5, 2, E.ENTRO_BF16, 1)
    query = B.CCacheQuery(PTR, PTR, PTR, 4096, 128, 4096, 128, PTR, 5, 2, 1000, 32, E.ENTRO_BF16, 1, 0, 0, 0.1, 0)
    return cache, table, rows, query


def test_struct_layouts_match_header():
    assert [C.sizeof(x) for x in (B.CCache, B.CCacheTable, B.CCacheRows, B.CCacheQuery)] == [56, 24, 72, 104]


def test_widths_and_sizes():
    assert [E.entro_cache_width(d) for d in (0, 1, 64, 65, 96, 97, 128, 129, 192, 193, 256, 257)] == [0, 64, 64, 96, 96, 128, 128, 192, 192, 256, 256, 0]
    for d in range(1, 257):
        assert E.entro_cache_width(d) == ref.width(d)
    cache = good()[0]
    assert B.lib().entro_cache_codes_bytes(C.byref(cache)) == 2 * 100 * 64 * 8 * 128
    cache.page_tokens = 48
    assert B.lib().entro_cache_codes_bytes(C.byref(cache)) == 0


def statuses(call, edits):
    return {name: call(edit) for name, edit in edits}


@pytest.mark.parametrize("field,value,status", [
    ("k", None, B.ENTRO_ERR_NULL), ("v", None, B.ENTRO_ERR_NULL), ("k_scale", None, B.ENTRO_ERR_NULL), ("v_scale", None, B.ENTRO_ERR_NULL),
    ("k", PTR + 8, B.ENTRO_ERR_ALIGN), ("v_scale", PTR + 4, B.ENTRO_ERR_ALIGN), ("layers", 0, B.ENTRO_ERR_SIZE), ("pages", 0, B.ENTRO_ERR_SIZE),
    ("pages", 1 << 31, B.ENTRO_ERR_SIZE), ("page_tokens", 8, B.ENTRO_ERR_SIZE), ("page_tokens", 48, B.ENTRO_ERR_SIZE),
    ("page_tokens", 512, B.ENTRO_ERR_SIZE), ("kv_heads", 0, B.ENTRO_ERR_SIZE), ("head_dim", 0, B.ENTRO_ERR_SIZE), ("head_dim", 257, B.ENTRO_ERR_SIZE)])
def test_every_call_refuses_a_pool_that_is_none(field, value, status):
    L = B.lib()
    cache, table, rows, query = good()
    setattr(cache, field, value)
    c, t = C.byref(cache), C.byref(table)
    following = B.CCacheTable(PTR * 2, PTR * 2, 4, 16)
    assert L.entro_cache_append(c, t, C.byref(rows), None) == status
    assert L.entro_cache_read(c, t, C.byref(rows), None) == status
    assert L.entro_cache_attend(c, t, C.byref(query), PTR, 1 << 40, None) == status
    assert L.entro_cache_regroup(c, t, None, None, 0, 0, C.byref(following), PTR, PTR, 1 << 40, None) == status
    assert L.entro_cache_compact(c, t, C.byref(following), PTR, PTR, 1 << 40, None) == status


@pytest.mark.parametrize("field,value,status", [("slots", None, B.ENTRO_ERR_NULL), ("lengths", None, B.ENTRO_ERR_NULL), ("slots", PTR + 4, B.ENTRO_ERR_ALIGN),
                                                ("seqs", 0, B.ENTRO_ERR_SIZE), ("stride", 0, B.ENTRO_ERR_SIZE), ("stride", 1 << 30, B.ENTRO_ERR_SIZE)])
def test_every_call_refuses_a_table_that_is_none(field, value, status):
    L = B.lib()
    cache, table, rows, query = good()
    other = B.CCacheTable(PTR * 2, PTR * 2, 4, 16)
    setattr(table, field, value)
    c, t = C.byref(cache), C.byref(table)
    assert L.entro_cache_append(c, t, C.byref(rows), None) == status
    assert L.entro_cache_read(c, t, C.byref(rows), None) == status
    assert L.entro_cache_attend(c, t, C.byref(query), PTR, 1 << 40, None) == status
    assert L.entro_cache_regroup(c, t, None, None, 0, 0, C.byref(other), PTR, PTR, 1 << 40, None) == status
    assert L.entro_cache_regroup(c, C.byref(other), None, None, 0, 0, t, PTR, PTR, 1 << 40, None) == status
    assert L.entro_cache_compact(c, t, C.byref(other), PTR, PTR, 1 << 40, None) == status


@pytest.mark.parametrize("field,value,status", [
    ("k", None, B.ENTRO_ERR_NULL), ("v", None, B.ENTRO_ERR_NULL), ("start", None, B.ENTRO_ERR_NULL), ("k", PTR + 2, B.ENTRO_ERR_ALIGN),
    ("start", PTR + 4, B.ENTRO_ERR_ALIGN), ("type", E.ENTRO_U8, B.ENTRO_ERR_SCHEME), ("type", 9, B.ENTRO_ERR_SCHEME), ("layer", 2, B.ENTRO_ERR_SIZE),
    ("k_token_stride", 1 << 50, B.ENTRO_ERR_SIZE), ("tokens", 1 << 31, B.ENTRO_ERR_SIZE)])
def test_append_and_read_refuse_rows_that_are_none(field, value, status):
    cache, table, rows, _ = good()
    setattr(rows, field, value)
    for call in (B.lib().entro_cache_append, B.lib().entro_cache_read):
        assert call(C.byref(cache), C.byref(table), C.byref(rows), None) == status


@pytest.mark.parametrize("field,value,status", [
    ("q", None, B.ENTRO_ERR_NULL), ("out", None, B.ENTRO_ERR_NULL), ("start", None, B.ENTRO_ERR_NULL), ("q", PTR + 2, B.ENTRO_ERR_ALIGN),
    ("lse", PTR + 4, B.ENTRO_ERR_ALIGN), ("type", E.ENTRO_U8, B.ENTRO_ERR_SCHEME), ("layer", 2, B.ENTRO_ERR_SIZE), ("q_heads", 0, B.ENTRO_ERR_SIZE),
    ("q_heads", 12, B.ENTRO_ERR_SIZE), ("scale", float("nan"), B.ENTRO_ERR_RANGE), ("scale", float("inf"), B.ENTRO_ERR_RANGE),
    ("out_token_stride", 1 << 50, B.ENTRO_ERR_SIZE)])
def test_attend_refuses_queries_that_are_none(field, value, status):
    cache, table, _, query = good()
    setattr(query, field, value)
    assert B.lib().entro_cache_attend(C.byref(cache), C.byref(table), C.byref(query), PTR, 1 << 40, None) == status


def test_null_descriptors_workspaces_and_calls_without_rows():
    L = B.lib()
    cache, table, rows, query = good()
    c, t = C.byref(cache), C.byref(table)
    following = B.CCacheTable(PTR * 2, PTR * 2, 4, 16)
    assert L.entro_cache_append(None, t, C.byref(rows), None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_append(c, None, C.byref(rows), None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_append(c, t, None, None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_attend(c, t, None, PTR, 1 << 40, None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_regroup(c, t, None, None, 0, 0, None, PTR, PTR, 1 << 40, None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_regroup(c, t, None, None, 0, 0, C.byref(following), None, PTR, 1 << 40, None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_regroup(c, t, None, None, 0, 0, C.byref(following), PTR, None, 0, None) == B.ENTRO_ERR_NULL
    need = L.entro_cache_pages_workspace_bytes(c, t, C.byref(following))
    assert need > 0 and L.entro_cache_regroup(c, t, None, None, 0, 0, C.byref(following), PTR, PTR, need - 1, None) == B.ENTRO_ERR_CAPACITY
    assert L.entro_cache_regroup(c, t, PTR + 4, None, 0, 0, C.byref(following), PTR, PTR, need, None) == B.ENTRO_ERR_ALIGN
    assert L.entro_cache_compact(c, t, C.byref(following), PTR, PTR, need - 1, None) == B.ENTRO_ERR_CAPACITY
    # in place, and tables of another shape
    assert L.entro_cache_regroup(c, t, None, None, 0, 0, t, PTR, PTR, 1 << 40, None) == B.ENTRO_ERR_SIZE
    following.stride = 15
    assert L.entro_cache_compact(c, t, C.byref(following), PTR, PTR, 1 << 40, None) == B.ENTRO_ERR_SIZE
    rows.tokens = query.tokens = 0
    rows.k = rows.v = query.q = query.out = None
    assert L.entro_cache_append(c, t, C.byref(rows), None) == B.ENTRO_OK
    assert L.entro_cache_read(c, t, C.byref(rows), None) == B.ENTRO_OK
    assert L.entro_cache_attend(c, t, C.byref(query), None, 0, None) == B.ENTRO_OK
    assert E.entro_cache_status(0) == B.ENTRO_OK and E.entro_cache_status(1) == B.ENTRO_ERR_CAPACITY


def test_the_binding_looks_at_shapes_and_types():
    k, v = torch.zeros(1, 4, 2, 16, 64, dtype=torch.uint8), torch.zeros(1, 4, 2, 64, 16, dtype=torch.uint8)
    s = torch.zeros(1, 4, 2)
    cache = E.Cache(k, v, s, s, 16, 40)
    for bad in (lambda: E.Cache(k, k, s, s, 16, 40), lambda: E.Cache(k, v, s, s[:, :3], 16, 40), lambda: E.Cache(k, v, s, s.double(), 16, 40),
                lambda: E.Cache(k, v, s, s, 16, 70), lambda: E.Cache(k, v, s, s, 32, 40), lambda: E.Cache(k.float(), v, s, s, 16, 40),
                lambda: E.Cache.empty(1, 4, 2, 16, 300, device="cpu")):
        with pytest.raises(ValueError):
            bad()
    table = E.CacheTable.empty(3, 5, device="cpu")
    assert table.slots.shape == (3, 5) and bool((table.slots == -1).all()) and not table.lengths.any()
    for bad in (lambda: E.CacheTable(table.slots.long(), table.lengths), lambda: E.CacheTable(table.slots, table.lengths[:2]),
                lambda: E.CacheTable(table.slots[:, ::2], table.lengths)):
        with pytest.raises(ValueError):
            bad()
    start = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(7, 2, 40, dtype=torch.bfloat16)
    for bad in (lambda: E.CacheRows(x, x.float(), start, 1), lambda: E.CacheRows(x.half(), x.half(), start, 1),
                lambda: E.CacheRows(x.transpose(1, 2), x.transpose(1, 2), start, 1), lambda: E.CacheRows(x, x, start.long(), 1),
                lambda: E.CacheQuery(x, x[:6], start, 1, 1), lambda: E.CacheQuery(x, x, start, 1, 1, lse=torch.zeros(7, 3)),
                lambda: E.CacheQuery(x, x[:1].expand(7, 2, 40), start, 1, 1),
                lambda: E.entro_cache_append(cache, table, E.CacheRows(x[..., :39], x[..., :39], start, 1)),
                lambda: E.entro_cache_append(cache, table, E.CacheRows(x[:, :1], x[:, :1], start, 1)),
                lambda: E.entro_cache_read(cache, table, E.CacheRows(x, x, start[:3], 1)),
                lambda: E.entro_cache_attend(cache, table, E.CacheQuery(x, x, start[:3], 1, 1))):
        with pytest.raises(ValueError):
            bad()


def test_calls_refuse_tensors_that_lie_in_host_memory():
    k, v, s = torch.zeros(1, 4, 2, 16, 64, dtype=torch.uint8), torch.zeros(1, 4, 2, 64, 16, dtype=torch.uint8), torch.zeros(1, 4, 2)
    cache, table, other = E.Cache(k, v, s, s, 16, 40), E.CacheTable.empty(3, 5, device="cpu"), E.CacheTable.empty(3, 5, device="cpu")
    start, x = torch.zeros(4, dtype=torch.int32), torch.zeros(7, 2, 40)
    status, ws = torch.zeros(4, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: E.entro_cache_append(cache, table, E.CacheRows(x, x, start, 1)), lambda: E.entro_cache_read(cache, table, E.CacheRows(x, x, start, 1)),
                 lambda: E.entro_cache_attend(cache, table, E.CacheQuery(x, x, start, 1, 1), ws),
                 lambda: E.entro_cache_regroup(cache, table, other, status, ws), lambda: E.entro_cache_compact(cache, table, other, status, ws)):
        with pytest.raises(ValueError):
            call()


def test_attend_refuses_a_workspace_that_is_none_or_too_small():
    L = B.lib()
    cache, table, _, query = good()
    table.seqs, query.max_new, query.max_len = 1, 1, 1 << 17
    c, t, q = C.byref(cache), C.byref(table), C.byref(query)
    need = L.entro_cache_attend_workspace_bytes(c, t, q)
    assert need > 0
    assert L.entro_cache_attend(c, t, q, None, need, None) == B.ENTRO_ERR_NULL
    assert L.entro_cache_attend(c, t, q, PTR + 8, need, None) == B.ENTRO_ERR_ALIGN
    assert L.entro_cache_attend(c, t, q, PTR, need - 1, None) == B.ENTRO_ERR_CAPACITY
    query.max_len = 100
    assert L.entro_cache_attend_workspace_bytes(c, t, q) == 0


def test_the_reference_s_regroup_by_hand():
    """Three rows of one sequence of 20 tokens in blocks of 16: they share the full block; the lowest keeps the open one."""
    table = np.array([[5, 2]], np.int32)
    got, lengths, copies, used = ref.regroup(8, 16, table, [20], 3, 3, [0, 0, 0], [1, 1, 13])
    assert got.tolist() == [[5, 2, -1], [5, 0, -1], [5, 1, 3]] and list(lengths) == [21, 21, 33]
    assert copies == [(2, 0), (2, 1)] and used == 5
    # a row that is taken back into a block that another row holds full gets a copy of it
    got, _, copies, _ = ref.regroup(8, 16, np.array([[5, 2]], np.int32), [32], 2, 2, [0, 0], [-20, 0])
    assert got.tolist() == [[0, -1], [5, 2]] and copies == [(5, 0)]
    # the block of positions 16..31 has left a window of 4 before position 40, that of the sink has not
    got, _, _, _ = ref.regroup(9, 16, np.array([[5, 2, 7]], np.int32), [40], 1, 3, None, None, window=4, sinks=1)
    assert got.tolist() == [[5, -1, 7]]


def test_the_reference_s_grid_by_hand():
    rng = np.random.default_rng(0)
    pool = ref.Pool(rng, 1, 1, 1, 16, 2)
    k = np.array([[[1.27, -0.5]], [[2.54, 0.02]]], np.float32)
    ref.append(pool, np.zeros((1, 1), int), [1], k[:1], k[:1], [0, 1])
    assert pool.k[0, 0, 0, 0, :2].tolist() == [255, 78]
    ref.append(pool, np.zeros((1, 1), int), [2], k[1:], k[1:], [0, 1])
    assert pool.k[0, 0, 0, :2, :2].tolist() == [[192, 103], [255, 129]]         # 63.5 is even at 64; -25; 127; 1
    assert np.isclose(pool.k_scale[0, 0, 0], 0.02)


class Placed(torch.Tensor):
    """A tensor in host memory that says it lies on a GPU."""
    device = property(lambda self: torch.device("cuda:0"))


@pytest.fixture
def calls_made(monkeypatch):
    """Names of the C calls that the binding makes; none of them runs."""
    made = []

    class Library:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith(("_bytes", "_width")) else lambda *args: made.append(name) or 0
    real = B.lib()
    monkeypatch.setattr(B, "lib", lambda: Library())
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: None)
    return made


OF_EVERY_CALL = ["pool.k", "pool.v", "pool.k_scale", "pool.v_scale", "slots", "lengths"]


@pytest.mark.parametrize("call,tensor", [
    (call, tensor) for call, more in [("append", ["k", "v", "start"]), ("read", ["k", "v", "start"]), ("attend", ["q", "out", "lse", "start", "workspace"]),
                                      ("regroup", ["next.slots", "next.lengths", "status", "workspace", "parent", "grow"]),
                                      ("compact", ["next.slots", "next.lengths", "status", "workspace"])]
    for tensor in [None] + OF_EVERY_CALL + more])
def test_calls_refuse_any_one_tensor_in_host_memory(calls_made, call, tensor):
    """Everything on the GPU but one tensor: the call is not made. (With all of them there it is.)"""
    def at(name, *shape, dtype=torch.int32):
        x = torch.zeros(*shape, dtype=dtype)
        return x if name == tensor else x.as_subclass(Placed)
    pool = [at("pool.k", 1, 4, 2, 16, 64, dtype=torch.uint8), at("pool.v", 1, 4, 2, 64, 16, dtype=torch.uint8)]
    cache = E.Cache(*pool, *(at(name, 1, 4, 2, dtype=torch.float32) for name in ("pool.k_scale", "pool.v_scale")), 16, 40)
    table = E.CacheTable(at("slots", 3, 5), at("lengths", 3))
    following, status = E.CacheTable(at("next.slots", 3, 5), at("next.lengths", 3)), at("status", 4)
    start, room = at("start", 4), at("workspace", 1 << 16, dtype=torch.uint8)
    rows = [at(name, 7, 2, 40, dtype=torch.float32) for name in "kv"]
    run = {"append": lambda: E.entro_cache_append(cache, table, E.CacheRows(*rows, start, 1)),
           "read": lambda: E.entro_cache_read(cache, table, E.CacheRows(*rows, start, 1)),
           "attend": lambda: E.entro_cache_attend(cache, table, E.CacheQuery(*(at(n, 7, 4, 40, dtype=torch.float32) for n in ("q", "out")), start, 1, 9,
                                                                             lse=at("lse", 7, 4, dtype=torch.float32)), room),
           "regroup": lambda: E.entro_cache_regroup(cache, table, following, status, room, parent=at("parent", 3), grow=at("grow", 3)),
           "compact": lambda: E.entro_cache_compact(cache, table, following, status, room)}[call]
    if tensor is None:
        run()
        assert calls_made == ["entro_cache_" + call]
    else:
        with pytest.raises(ValueError, match="one GPU"):
            run()
        assert calls_made == []


def test_read_refuses_rows_that_share_their_places(calls_made):
    placed = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype).as_subclass(Placed)  # noqa: E731
    s = placed(1, 4, 2, dtype=torch.float32)
    cache = E.Cache(placed(1, 4, 2, 16, 64, dtype=torch.uint8), placed(1, 4, 2, 64, 16, dtype=torch.uint8), s, s, 16, 40)
    table, start, x = E.CacheTable(placed(3, 5), placed(3)), placed(4), placed(7, 2, 40, dtype=torch.float32)
    for shared in (x[:1].expand(7, 2, 40), x[:, :1].expand(7, 2, 40)):
        for k, v in ((x, shared), (shared, x)):
            with pytest.raises(ValueError, match="places of their own"):
                E.entro_cache_read(cache, table, E.CacheRows(k, v, start, 1))
            E.entro_cache_append(cache, table, E.CacheRows(k, v, start, 1))         # rows that are only read may
    assert calls_made == ["entro_cache_append"] * 4


def test_the_header_says_which_calls_the_paper_does_not_define():
    """The paper defines the grid that keys and values are put on (Eq. 1), and nothing else of the cache."""
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "entro.h")).read()
    comments = dict((name, re.sub(r"[\s*]+", " ", text)) for text, name in re.findall(r"/\*((?:(?!\*/).)*)\*/\s*\w+ (entro_cache_\w+)\(", header, re.S))
    assert set(comments) == {n for n in B.EXPORTED if n.startswith("entro_cache_")}
    for name, text in comments.items():
        defined = name in ("entro_cache_append", "entro_cache_read")
        assert ("Eq. 1" in text) if defined else ("no passage of the paper defines it" in text.lower()), name
        assert "Fig. 3" not in text, name
