"""Norms and rotations of heads, alone and on the way into the token cache, through the C ABI against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2505_02380_amd as E
import rotary_reference as rot

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LAYOUTS = {"halves": E.ENTRO_ROTARY_HALVES, "pairs": E.ENTRO_ROTARY_PAIRS}
NORMS = {"none": E.ENTRO_NORM_NONE, "rms": E.ENTRO_NORM_RMS, "centred": E.ENTRO_NORM_CENTRED}


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def ints(x):
    return torch.tensor([int(i) for i in x], dtype=torch.int32, device=DEV)


def rows(rng, tokens, heads, dim, kind):
    """(numpy values, device tensor)."""
    x = dev(rng.standard_normal((tokens, heads, dim)).astype(np.float32)).to(TYPES[kind])
    return x.float().cpu().numpy(), x


def rotary(dims, layout, norm, turns=None, **kw):
    t = E.entro_rotary_turns(dims) if turns is None else turns
    return t, E.Rotary(dev(t.view(np.int64)) if dims else None, dims, LAYOUTS[layout], norm=NORMS[norm], **kw)


def check(got, want, bound, kind):
    got = got.float().cpu().numpy().astype(np.float64)
    away = np.abs(got - want) - rot.tolerance(want, bound, kind)
    assert np.all(away <= 0), (np.argwhere(~(away <= 0))[:4], np.nanmax(away))


#         tokens, q_heads, kv_heads, dim, dims
ROTATE = [(1, 32, 8, 128, 128), (3, 1, 1, 1, 0), (2, 2, 1, 2, 2), (7, 5, 1, 17, 10), (4, 20, 4, 80, 32), (9, 3, 3, 96, 96), (5, 4, 2, 64, 64),
          (6, 2, 1, 112, 56), (5, 2, 2, 192, 96), (3, 4, 1, 256, 256), (4, 2, 1, 256, 130), (11, 1, 1, 24, 24), (2, 3, 1, 72, 8), (1, 7, 7, 40, 0),
          (2500, 12, 2, 80, 80), (1100, 32, 8, 128, 128)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("layout,norm", [("halves", "none"), ("pairs", "rms"), ("halves", "centred"), ("pairs", "centred"), ("halves", "rms")])
@pytest.mark.parametrize("case", range(len(ROTATE)))
def test_rotate_against_the_definition(case, layout, norm, kind):
    tokens, q_heads, kv_heads, dim, dims = ROTATE[case]
    rng = np.random.default_rng(case)
    positions = rng.integers(-2 ** 31, 2 ** 31, tokens) if case % 3 else rng.integers(0, 5000, tokens)
    positions[: 4] = [0, 2 ** 31 - 1, -2 ** 31, -1][: tokens]
    q_gain, k_gain = (rng.standard_normal(dim).astype(np.float32) for _ in "qk")
    amplitude = [1.0, 1.25, -0.5][case % 3]
    turns, r = rotary(dims, layout, norm, q_gain=dev(q_gain), k_gain=None if case % 2 else dev(k_gain), eps=1e-5, amplitude=amplitude)
    (q, qd), (k, kd) = rows(rng, tokens, q_heads, dim, kind), rows(rng, tokens, kv_heads, dim, kind)
    qy, ky = torch.full_like(qd, 7), torch.full_like(kd, 7)
    E.entro_rotate(r, E.RotaryRows(qd, qy), E.RotaryRows(kd, ky), ints(positions))
    for x, y, gain in ((q, qy, q_gain), (k, ky, None if case % 2 else k_gain)):
        check(y, *rot.rotate(x, positions, turns, layout, norm, gain, 1e-5, amplitude), kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim,dims,layout", [(128, 128, "halves"), (80, 40, "pairs"), (33, 20, "halves"), (9, 8, "pairs")])
def test_rotate_in_place_of_rows_side_by_side_with_gains_for_each_head(dim, dims, layout, kind):
    """q, k and v in one tensor, at any alignment; q and k rotated where they lie, v and what surrounds it left alone."""
    rng = np.random.default_rng(dim)
    tokens, heads = 13, (4, 2, 2)
    x, xd = rows(rng, tokens + 2, sum(heads), dim, kind)
    q, k = xd[1: tokens + 1, :4], xd[1: tokens + 1, 4:6]
    gains = [rng.standard_normal((n, dim)).astype(np.float32) for n in (4, 2)]
    turns, r = rotary(dims, layout, "rms", q_gain=dev(gains[0]), k_gain=dev(gains[1]))
    positions = rng.integers(0, 100000, tokens)
    E.entro_rotate(r, E.RotaryRows(q), E.RotaryRows(k), ints([9, 9, 9, *positions])[3:])
    for got, part, gain in ((q, slice(0, 4), gains[0]), (k, slice(4, 6), gains[1])):
        check(got, *rot.rotate(x[1: tokens + 1, part], positions, turns, layout, "rms", gain), kind)
    after = xd.float().cpu().numpy()
    assert np.array_equal(after[:, 6:], x[:, 6:]) and np.array_equal(after[[0, -1]], x[[0, -1]])


def test_rotate_takes_queries_or_keys_alone_and_no_tokens():
    rng = np.random.default_rng(1)
    turns, r = rotary(32, "halves", "none")
    x, xd = rows(rng, 6, 3, 48, "f32")
    want, bound = rot.rotate(x, range(6), turns, "halves")
    for q, k in ((True, False), (False, True)):
        y = torch.zeros_like(xd)
        side = E.RotaryRows(xd, y)
        E.entro_rotate(r, side if q else None, side if k else None, ints(range(6)))
        check(y, want, bound, "f32")
    E.entro_rotate(r, E.RotaryRows(xd[:0]), None, ints([]))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rotating_back_gives_the_rows_again(kind):
    rng = np.random.default_rng(2)
    turns, r = rotary(128, "halves", "none")
    x, xd = rows(rng, 50, 4, 128, "f32")
    positions = ints(rng.integers(-2 ** 31 + 1, 2 ** 31, 50))
    E.entro_rotate(r, E.RotaryRows(xd), None, positions)
    E.entro_rotate(r, E.RotaryRows(xd), None, -positions)
    away = np.abs(xd.cpu().numpy() - x)
    pair = np.abs(x[..., :64]) + np.abs(x[..., 64:])
    assert np.all(away <= 2 * 12 * rot.U * 2 * np.concatenate([pair, pair], -1))


@pytest.mark.parametrize("norm", ["rms", "centred"])
def test_norms_of_extreme_heads(norm):
    """Squares beyond fp32, below it, zeros, and heads that are no numbers (which touch no other head)."""
    rng = np.random.default_rng(3)
    dim = 64
    x = rng.standard_normal((9, 2, dim)).astype(np.float32)
    for i, f in enumerate([1e18, 1e30, 2e37, 1e-12, 1e-25, 0.0]):
        x[i] *= np.float32(f)
    x[5, 1] = 1e25                                              # a head of equal elements: centred, zeros
    x[6, 0, 3], x[6, 1, 5], x[7, 0, 0] = np.nan, -np.inf, np.inf
    turns, r = rotary(dim, "halves", norm, eps=1e-20)
    y = torch.zeros(x.shape, device=DEV)
    E.entro_rotate(r, E.RotaryRows(dev(x), y), None, ints(range(9)))
    good = np.ones(9, bool)
    good[[6, 7]] = False
    want, bound = rot.rotate(x[good], np.arange(9)[good], turns, "halves", norm, None, 1e-20)
    got = y.cpu().numpy()
    away = np.abs(got[good] - want) - rot.tolerance(want, bound, "f32")
    if norm == "centred":
        away[5, 1] = np.abs(got[5, 1]) - 1e-3                   # 1e25 less a mean of it that is one rounding off at most, against nothing
        away[5, 1][got[5, 1] == 0] = 0
    assert np.all(away <= 0), np.argwhere(~(away <= 0))[:5]
    assert np.isnan(got[6, 0]).all() and np.isfinite(got[7, 1]).all()
    assert np.isnan(got[6, 1, 5]) and np.isnan(got[7, 0, 0])


@pytest.mark.parametrize("norm", ["rms", "centred"])
def test_a_head_s_bits_do_not_depend_on_the_heads_beside_it(norm):
    rng = np.random.default_rng(4)
    turns, r = rotary(24, "halves", norm)
    x = rng.standard_normal((7, 8, 24)).astype(np.float32)
    x[:, ::3] *= np.float32(3e17)                               # squares within the range
    rows_of = [x.copy(), x.copy()]
    rows_of[1][:, 1::3], rows_of[1][0, 2] = np.nan, 1e30
    got = []
    for y in rows_of:
        d = dev(y)
        E.entro_rotate(r, E.RotaryRows(d), None, ints(range(7)))
        got.append(d)
    assert torch.equal(got[0][:, ::3], got[1][:, ::3]) and torch.equal(got[0][1:, 2::3], got[1][1:, 2::3])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [3, 13000])
@pytest.mark.parametrize("dim", [17, 80, 96, 112, 128])
def test_centred_norm_of_heads_far_from_zero(dim, tokens, kind):
    """Equal elements give nothing, whatever their mean's rounding, in small calls and large ones."""
    rng = np.random.default_rng(dim)
    x = dev(np.tile(rot.far_heads(rng, dim)[None], (tokens, 1, 1))).to(TYPES[kind])
    _, r = rotary(0, "halves", "centred", eps=1e-6)
    y = torch.full_like(x, 7)
    E.entro_rotate(r, E.RotaryRows(x, y), None, ints(range(tokens)))
    want, bound = rot.centred(x[:1].float().cpu().numpy(), 1e-6)
    check(y[:1], want, bound, kind)
    assert torch.equal(y, y[:1].expand_as(y))


# ------------------------------------------------------------------------------------------------------- into the cache
#          kind, heads, kv_heads, page, dim, dims, lengths, new
APPEND = [("bf16", 32, 8, 64, 128, 128, [70, 1, 64, 128], [1, 1, 1, 1]), ("f32", 4, 2, 16, 24, 24, [40, 5, 0, 33], [40, 5, 0, 7]),
          ("bf16", 4, 4, 128, 96, 48, [300, 257], [200, 130]), ("f32", 2, 1, 256, 256, 130, [520, 40], [300, 40]), ("bf16", 6, 2, 32, 80, 32, [100, 31, 65], [9, 31, 1]),
          ("f32", 3, 3, 16, 17, 6, [20, 50], [3, 50]), ("bf16", 2, 2, 16, 1, 0, [20], [18]), ("bf16", 8, 8, 16, 64, 64, [16, 17, 15, 1], [16, 2, 15, 1]),
          ("f32", 8, 2, 64, 128, 128, [2000, 100], [1500, 1])]


def pool_and_table(rng, lengths, heads, page, dim, layers=2):
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 3
    pool = ref.Pool(rng, layers, pages, heads, page, dim)
    pool.k_scale[...], pool.v_scale[...] = (0.02 * np.exp(rng.standard_normal(pool.k_scale.shape)) for _ in "kv")
    table = np.full((len(lengths), max(max(need), 1)), -1, np.int32)
    order, at = rng.permutation(pages), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at: at + n]
        at += n
    return pool, table


def cache_of(pool):
    return E.Cache(dev(pool.k), dev(pool.v), dev(pool.k_scale), dev(pool.v_scale), pool.page, pool.dim)


def same_pool(a, b):
    for name in ("k", "v", "k_scale", "v_scale"):
        x, y = getattr(a, name), getattr(b, name)
        assert torch.equal(x, y), (name, torch.nonzero(x != y)[:4].tolist())


@pytest.mark.parametrize("layout,norm", [("halves", "none"), ("pairs", "none"), ("halves", "rms"), ("pairs", "centred")])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append_rotated_is_rotate_then_append(case, layout, norm):
    """The same codes and scales as keys rotated to fp32 rows and appended, whatever the blocks held before; the same queries as rotate's."""
    kind, q_heads, heads, page, dim, dims, lengths, new = APPEND[case]
    rng = np.random.default_rng(case)
    pool, table = pool_and_table(rng, lengths, heads, page, dim)
    if case % 2:
        table[0, 0] = -1
    start = np.concatenate([[0], np.cumsum(new)]) + 1            # a row before the first sequence's and two behind the last one's
    tokens = int(start[-1]) + 2
    gains = [rng.standard_normal((n, dim)).astype(np.float32) for n in (q_heads, heads)]
    _, r = rotary(dims, layout, norm, q_gain=dev(gains[0]), k_gain=dev(gains[1]), amplitude=1.1)
    packed = rows(rng, tokens, q_heads + 2 * heads, dim, kind)[1]
    q, k, v = packed[:, :q_heads], packed[:, q_heads: q_heads + heads], packed[:, q_heads + heads:]
    t = E.CacheTable(dev(table), ints(lengths))
    positions = np.zeros(tokens, int)
    for b, n in enumerate(new):
        positions[start[b]: start[b + 1]] = np.arange(lengths[b] - n, lengths[b])
    want, got = cache_of(pool), cache_of(pool)
    turned = k.float().contiguous()
    E.entro_rotate(r, None, E.RotaryRows(turned), ints(positions))
    E.entro_cache_append(want, t, E.CacheRows(turned, v.float().contiguous(), ints(start), max(new), layer=1))
    qy = torch.full((tokens, q_heads, dim), 7.0, dtype=TYPES[kind], device=DEV)
    hint = [max(new), 1, 10 ** 6][case % 3]
    kr = E.CacheRows(k, v, ints(start), hint, layer=1)
    for _ in range(2):                                          # again: nothing changes
        E.entro_cache_append_rotated(got, t, kr, r, E.RotaryRows(q, qy))
        same_pool(got, want)
    q_want = torch.full_like(qy, 7.0)
    E.entro_rotate(r, E.RotaryRows(q[1:-2].contiguous(), q_want[1:-2]), None, ints(positions[1:-2]))
    assert torch.equal(qy, q_want)
    got = cache_of(pool)
    E.entro_cache_append_rotated(got, t, kr, r)                  # without queries
    same_pool(got, want)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("layout,norm", [("halves", "rms"), ("pairs", "centred")])
def test_append_rotated_against_the_definition(layout, norm, kind):
    rng = np.random.default_rng(5)
    heads, page, dim, dims, lengths, new = 2, 16, 80, 48, [50, 7, 30], [50, 7, 1]
    pool, table = pool_and_table(rng, lengths, heads, page, dim, 1)
    pool.k_scale[...] = pool.v_scale[...] = 1e-6                # what blocks held before counts for nothing
    start = np.concatenate([[0], np.cumsum(new)])
    (k, kd), (v, vd) = rows(rng, start[-1], heads, dim, kind), rows(rng, start[-1], heads, dim, kind)
    gain = rng.standard_normal(dim).astype(np.float32)
    turns, r = rotary(dims, layout, norm, k_gain=dev(gain))
    cache, t = cache_of(pool), E.CacheTable(dev(table), ints(lengths))
    E.entro_cache_append_rotated(cache, t, E.CacheRows(kd, vd, ints(start), max(new)), r)
    back = torch.zeros(start[-1], heads, dim, device=DEV)
    E.entro_cache_read(cache, t, E.CacheRows(back, torch.zeros_like(back), ints(start), max(new)))
    for b, n in enumerate(new):
        at = slice(start[b], start[b + 1])
        positions = np.arange(lengths[b] - n, lengths[b])
        want, bound = rot.rotate(k[at], positions, turns, layout, norm, gain)
        got = back[at].cpu().numpy().astype(np.float64)
        for block in np.unique(positions // page):
            rows_of = positions // page == block
            scale = np.maximum(np.abs(want[rows_of]).max((0, 2)) / 127, 1e-6)[None, :, None]
            off = bound[rows_of].max((0, 2))[None, :, None]
            assert np.all(np.abs(got[rows_of] - want[rows_of]) <= scale * (0.5 + 2e-6 * 127) + 3 * off)


def test_append_rotated_takes_keys_that_are_no_numbers():
    rng = np.random.default_rng(6)
    pool, table = pool_and_table(rng, [20], 2, 16, 32, 1)
    _, r = rotary(32, "halves", "none")
    k, v = (rows(rng, 20, 2, 32, "f32")[1] for _ in "kv")
    k[3, 0, 5], k[7, 1, 30], k[9, 1, 2], v[4, 0, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    t, start = E.CacheTable(dev(table), ints([20])), ints([0, 20])
    turned = k.clone()
    E.entro_rotate(r, None, E.RotaryRows(turned), ints(range(20)))
    assert int((~torch.isfinite(turned)).sum()) >= 6            # both elements of a pair
    want, got = cache_of(pool), cache_of(pool)
    E.entro_cache_append(want, t, E.CacheRows(turned, v, start, 20))
    E.entro_cache_append_rotated(got, t, E.CacheRows(k, v, start, 20), r)
    same_pool(got, want)


def test_positions_and_lengths_that_lie():
    """Starts beyond the rows, lengths below the rows' number (rows before position 0), tokens past the table: nothing outside is touched, and what
    the two calls do is alike."""
    rng = np.random.default_rng(7)
    pool, table = pool_and_table(rng, [40, 40, 40], 2, 16, 32, 1)
    _, r = rotary(32, "halves", "none")
    k, v = (rows(rng, 30, 2, 32, "f32")[1] for _ in "kv")
    q = rows(rng, 30, 4, 32, "f32")[1]
    t, start = E.CacheTable(dev(table), ints([5, 100, 40])), ints([-3, 12, 25, 99])
    positions = np.concatenate([np.arange(5 - 12, 5), np.arange(100 - 13, 100), np.arange(40 - 5, 40)])
    turned = k.clone()
    E.entro_rotate(r, None, E.RotaryRows(turned), ints(positions))
    want, got = cache_of(pool), cache_of(pool)
    E.entro_cache_append(want, t, E.CacheRows(turned, v, start, 30))
    qy = torch.zeros_like(q)
    E.entro_cache_append_rotated(got, t, E.CacheRows(k, v, start, 30), r, E.RotaryRows(q, qy))
    same_pool(got, want)
    q_want = torch.zeros_like(q)
    E.entro_rotate(r, E.RotaryRows(q, q_want), None, ints(positions))
    assert torch.equal(qy, q_want)


def test_a_captured_step_follows_its_positions():
    """Rotation and append in a graph: replayed as lengths, positions and rows change, eager work between."""
    rng = np.random.default_rng(8)
    pool, table = pool_and_table(rng, [60, 60], 2, 16, 64, 1)
    _, r = rotary(64, "pairs", "rms")
    k, v = (rows(rng, 2, 2, 64, "bf16")[1] for _ in "kv")
    q = rows(rng, 2, 4, 64, "bf16")[1]
    qy, alone = torch.zeros_like(q), torch.zeros_like(q)
    t, start, positions = E.CacheTable(dev(table), ints([10, 20])), ints([0, 1, 2]), ints([9, 19])
    cache, twin = cache_of(pool), cache_of(pool)
    kr, qr, ar = E.CacheRows(k, v, start, 1), E.RotaryRows(q, qy), E.RotaryRows(q, alone)

    def step():
        E.entro_cache_append_rotated(cache, t, kr, r, qr)
        E.entro_rotate(r, ar, None, positions)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(cache, name).copy_(getattr(twin, name))
    for i in range(4):
        k.copy_(torch.randn_like(k)), v.copy_(torch.randn_like(v)), q.copy_(torch.randn_like(q))
        t.lengths.add_(1), positions.add_(1)
        qy.zero_(), alone.zero_()
        graph.replay()
        q_want = torch.zeros_like(q)
        E.entro_cache_append_rotated(twin, t, kr, r, E.RotaryRows(q, q_want))
        torch.cuda.synchronize()
        same_pool(cache, twin)
        assert torch.equal(qy, q_want) and torch.equal(alone, q_want) and float(q_want.abs().sum()) > 0
