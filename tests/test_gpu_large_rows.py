"""Norms and rotations of calls with many rows, through the C ABI: below and above the sizes from which other kernels take them (which kernel takes which
case is tested on the CPU, test_positions_host)."""
import numpy as np
import pytest
import torch

import large_rows as large
import paper_2505_02380_amd as E
import rotary_reference as rot
from test_gpu_positions import DEV, TYPES, cache_of, check, dev, ints, pool_and_table, rotary, rows, same_pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout,norm", [("halves", "none"), ("pairs", "rms"), ("halves", "centred")])
@pytest.mark.parametrize("case", range(len(large.ROTATE)))
def test_rotate_of_many_rows(case, layout, norm):
    """Rows side by side in one tensor, rotated where they lie, gains for each head; the rows before and behind them, and other heads, left alone."""
    kind, tokens, q_heads, kv_heads, dim, dims, _ = large.ROTATE[case]
    rng = np.random.default_rng(case)
    x, xd = rows(rng, tokens + 2, q_heads + kv_heads + 1, dim, kind)
    q, k = xd[1:-1, :q_heads], xd[1:-1, q_heads: q_heads + kv_heads]
    gains = [rng.standard_normal((h, dim)).astype(np.float32) for h in (q_heads, max(kv_heads, 1))]
    turns, r = rotary(dims, layout, norm, q_gain=dev(gains[0]), k_gain=dev(gains[1]), amplitude=1.1)
    positions = rng.integers(-2 ** 31, 2 ** 31, tokens)
    E.entro_rotate(r, E.RotaryRows(q), E.RotaryRows(k) if kv_heads else None, ints(positions))
    for got, part, gain in ((q, slice(0, q_heads), gains[0]), (k, slice(q_heads, q_heads + kv_heads), gains[1]))[: 2 if kv_heads else 1]:
        check(got, *rot.rotate(x[1:-1, part], positions, turns, layout, norm, gain, amplitude=1.1), kind)
    after = xd.float().cpu().numpy()
    assert np.array_equal(after[:, -1], x[:, -1]) and np.array_equal(after[[0, -1]], x[[0, -1]])


@pytest.mark.parametrize("layout,norm", [("halves", "rms"), ("pairs", "none")])
@pytest.mark.parametrize("case", range(len(large.APPEND)))
def test_append_rotated_of_many_rows_is_rotate_then_append(case, layout, norm):
    """The same codes, scales and queries, bit for bit, whatever the hint says; a query row that no sequence has is left alone."""
    kind, q_heads, heads, dim, dims, page, new, _ = large.APPEND[case]
    rng = np.random.default_rng(case)
    lengths = [n + 3 * i for i, n in enumerate(new)]
    pool, table = pool_and_table(rng, lengths, heads, page, dim, 1)
    start = np.concatenate([[0], np.cumsum(new)])
    tokens = int(start[-1]) + 1
    gains = [rng.standard_normal((n, dim)).astype(np.float32) for n in (q_heads, heads)]
    _, r = rotary(dims, layout, norm, q_gain=dev(gains[0]), k_gain=dev(gains[1]))
    packed = torch.randn(tokens, q_heads + 2 * heads, dim, device=DEV).to(TYPES[kind])
    q, k, v = packed[:, :q_heads], packed[:, q_heads: q_heads + heads], packed[:, q_heads + heads:]
    t, positions = E.CacheTable(dev(table), ints(lengths)), np.concatenate([np.arange(a - n, a) for a, n in zip(lengths, new)] + [[7]])
    want, turned, q_want = cache_of(pool), k.float().contiguous(), torch.full((tokens, q_heads, dim), 7.0, dtype=TYPES[kind], device=DEV)
    E.entro_rotate(r, None, E.RotaryRows(turned), ints(positions))
    E.entro_cache_append(want, t, E.CacheRows(turned, v.float().contiguous(), ints(start), max(new)))
    E.entro_rotate(r, E.RotaryRows(q[:-1], q_want[:-1]), None, ints(positions[:-1]))
    for hint in (max(new), 1, 10 ** 6):
        got, qy = cache_of(pool), torch.full_like(q_want, 7.0)
        E.entro_cache_append_rotated(got, t, E.CacheRows(k, v, ints(start), hint), r, E.RotaryRows(q, qy))
        same_pool(got, want)
        assert torch.equal(qy, q_want)
