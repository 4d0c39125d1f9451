"""Norms and rotations of heads in 64 bits, on the CPU (test infrastructure). Nothing of the library is used here.

Bounds, with u = 2^-24, fixed before the first run. A norm's sums add at most 32 elements in a lane and 6 times between lanes, so they are off by
38 u of their terms' sizes, and its factor, a square root of a mean and two products, by 24 u; a mean that is taken off by 40 u of the mean
size. A cosine or sine: the angle is off by 2^-32 turns and 3 u of an eighth of a turn, the series by 2^-28 and 4 roundings: 8 u. An element of a turned
pair adds two products and a rounding. The last rounding is half a step of the rows' type."""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def angles(positions, turns):
    """[tokens][pairs] of 2 pi * position * turns / 2^64, reduced exactly."""
    with np.errstate(over="ignore"):
        product = np.asarray(positions).astype(np.int64).astype(np.uint64)[:, None] * np.asarray(turns, np.uint64)[None]
    return (product.view(np.int64).astype(np.longdouble) * (2 * np.pi * np.longdouble(2) ** -64)).astype(np.float64)


def rotate(x, positions, turns, layout, norm="none", gain=None, eps=1e-6, amplitude=1.0):
    """(rows [tokens][heads][dim], how far each element may be off before the last rounding)."""
    x = x.astype(np.float64)
    dim, dims = x.shape[-1], 2 * len(turns)
    off = np.zeros_like(x)
    if norm != "none":
        g = np.ones(dim) if gain is None else gain.astype(np.float64)
        if norm == "centred":
            off += 40 * U * np.abs(x).mean(-1, keepdims=True)
            x = x - x.mean(-1, keepdims=True)
        by = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        # an error of all elements moves their sum of squares as well
        off = (off * (1 + by * by * (x * x)) + 45 * U * np.abs(x)) * by * np.abs(g)
        x = x * by * g
    a = angles(positions, turns)[:, None]
    at = np.arange(dims).reshape(2, -1) if layout == "halves" else np.arange(dims).reshape(-1, 2).T
    z = (x[..., at[0]] + 1j * x[..., at[1]]) * amplitude * np.exp(1j * a)
    y, bound = x.copy(), off.copy()
    y[..., at[0]], y[..., at[1]] = z.real, z.imag
    pair = np.abs(x[..., at[0]]) + np.abs(x[..., at[1]])
    pair_off = off[..., at[0]] + off[..., at[1]]
    for i in (0, 1):
        bound[..., at[i]] = abs(amplitude) * (pair * 11 * U + pair_off)
    return y, bound


def tolerance(y, bound, kind):
    return bound + (np.abs(y) + bound) * HALF_STEP[kind] + 1e-37


def far_heads(rng, dim):
    """Heads of equal elements, of nearly equal ones, and an ordinary one."""
    heads = [np.full(dim, f) for f in (1000.0, 10000.0, -777.7, 3e4)]
    return np.stack(heads + [1000 + 1e-2 * rng.standard_normal(dim), -20000 + rng.standard_normal(dim), rng.standard_normal(dim)]).astype(np.float32)


def centred(x, eps):
    """(the centred norm alone, how far fp32 results may be off), also where the mean is far from zero. With D the mean |x - mean| and A the mean |x|: sum and
    product leave a mean that is off by 40 u A; the same again of what is left takes that away, off by 40 u (D + 40 u A) and three roundings
    of elements of at most |x - mean| + 40 u A. An error of all elements moves their sum of squares as well; the factor is off by 24 u of what it is taken
    of, the squares before that mean is taken away among them, and the last product by one."""
    x = x.astype(np.float64)
    off = x - x.mean(-1, keepdims=True)
    first = 40 * U * np.abs(x).mean(-1, keepdims=True)
    away = 40 * U * (np.abs(off).mean(-1, keepdims=True) + first) + 3 * U * (np.abs(off) + first)
    by = 1 / np.sqrt((off * off).mean(-1, keepdims=True) + eps)
    return off * by, (away + np.abs(off) * (by * by * (np.abs(off) * away).mean(-1, keepdims=True) + 25 * U + 24 * U * (first * by) ** 2)) * by + 1e-37
