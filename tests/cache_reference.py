"""The token cache's definitions in 64 bits, one element or one row at a time, on the CPU (test infrastructure).

Pools are numpy arrays in the layouts of include/entro.h. Nothing of the library is used here."""
import numpy as np


def width(dim):
    return next(w for w in (64, 96, 128, 192, 256) if w >= dim)


class Pool:
    def __init__(self, rng, layers, pages, heads, page, dim):
        self.page, self.dim, self.pages, self.heads = page, dim, pages, heads
        w = width(dim)
        # what no sequence has written yet may be anything
        self.k = rng.integers(0, 256, (layers, pages, heads, page, w), dtype=np.uint8)
        self.v = rng.integers(0, 256, (layers, pages, heads, w, page), dtype=np.uint8)
        self.k_scale = np.full((layers, pages, heads), np.nan, np.float32)
        self.v_scale = np.full((layers, pages, heads), np.nan, np.float32)

    def copy(self):
        c = object.__new__(Pool)
        c.__dict__ = {n: (x.copy() if isinstance(x, np.ndarray) else x) for n, x in self.__dict__.items()}
        return c

    def at(self, which, layer, page, head):
        """(codes [token][dim] as a view, array of scales, index of the scale)."""
        if which == "k":
            return self.k[layer, page, head][:, :self.dim], self.k_scale, (layer, page, head)
        return self.v[layer, page, head][:self.dim].T, self.v_scale, (layer, page, head)

    def value(self, which, layer, table, b, pos, head):
        """The values at a position in 64 bits, or None where it has no page."""
        slot = pos // self.page
        if pos < 0 or slot >= table.shape[1] or not 0 <= table[b, slot] < self.pages:
            return None
        codes, scales, i = self.at(which, layer, table[b, slot], head)
        return (codes[pos % self.page].astype(np.float64) - 128) * np.float64(scales[i])


def append(pool, table, lengths, k, v, start, layer=0):
    """Writes into pool. Returns the share of codes whose quotient lies so near a tie that 32 bits may round it either way, as masks like
    pool.k and pool.v."""
    near = {"k": np.zeros(pool.k.shape, bool), "v": np.zeros(pool.v.shape, bool)}
    for b in range(len(lengths)):
        n = start[b + 1] - start[b]
        first = lengths[b] - n
        blocks = sorted({p // pool.page for p in range(max(first, 0), lengths[b])}) if n else []
        for block in blocks:
            if block >= table.shape[1] or not 0 <= table[b, block] < pool.pages:
                continue
            lo, hi = block * pool.page, (block + 1) * pool.page
            new = [p for p in range(lo, hi) if max(first, 0) <= p < lengths[b]]
            old = [p for p in range(lo, hi) if p < first]
            for which, x in (("k", k), ("v", v)):
                for h in range(pool.heads):
                    codes, scales, i = pool.at(which, layer, table[b, block], h)
                    mask = near[which][i] if which == "k" else near[which][i].T
                    rows = np.stack([x[start[b] + p - first, h] for p in new]).astype(np.float32)
                    finite = np.abs(rows[np.isfinite(rows)])
                    before = np.float32(scales[i]) if old else np.float32(0)
                    scale = max(before, (finite.max() if finite.size else np.float32(0)) / np.float32(127))
                    s = np.float64(scale)

                    def put(p, quotient):
                        q = np.nan_to_num(quotient, nan=0.0, posinf=127, neginf=-127)
                        codes[p - lo] = (np.clip(np.rint(q), -127, 127) + 128).astype(np.uint8)
                        mask[p - lo, :pool.dim] |= np.abs(q - np.floor(q) - 0.5) < 2.0 ** -15     # 127 * 2^-22, and more
                    if scale > before:
                        for p in old:
                            put(p, (codes[p - lo].astype(np.float64) - 128) * np.float64(before) / s)
                    for p, r in zip(new, rows):
                        with np.errstate(invalid="ignore", over="ignore"):
                            put(p, r.astype(np.float64) / s if scale > 0 else np.zeros(pool.dim))
                    scales[i] = scale
    return near


def read(pool, table, lengths, start, tokens, layer=0):
    k = np.zeros((tokens, pool.heads, pool.dim))
    v = np.zeros_like(k)
    for b in range(len(lengths)):
        for r in range(start[b], start[b + 1]):
            pos = lengths[b] - (start[b + 1] - r)
            for h in range(pool.heads):
                for which, x in (("k", k), ("v", v)):
                    value = pool.value(which, layer, table, b, pos, h)
                    if value is not None:
                        x[r, h] = value
    return k, v


def attend(pool, table, lengths, q, start, scale, window=0, sinks=0, layer=0):
    """(out, lse, the sums of p |v|, the largest sum of scale |q| |k|) of every row: the last two for bounds of rounding errors."""
    tokens, q_heads, dim = q.shape
    per = q_heads // pool.heads
    out, weight = np.zeros(q.shape), np.zeros(q.shape)
    lse, size = np.full((tokens, q_heads), -np.inf), np.zeros((tokens, q_heads))
    for b in range(len(lengths)):
        if start[b + 1] == start[b]:
            continue
        there = [p for p in range(lengths[b]) if pool.value("k", layer, table, b, p, 0) is not None]
        values = {(w, h): np.array([pool.value(w, layer, table, b, p, h) for p in there]).reshape(-1, dim)
                  for w in "kv" for h in range(pool.heads)}
        there = np.array(there, int)
        for r in range(start[b], start[b + 1]):
            pos = lengths[b] - (start[b + 1] - r)
            seen = there <= pos
            if window:
                seen &= (pos - there < window) | (there < sinks)
            if not seen.any():
                continue
            for h in range(q_heads):
                k, v = values["k", h // per][seen], values["v", h // per][seen]
                z = k @ q[r, h].astype(np.float64) * scale
                e = np.exp(z - z.max())
                out[r, h] = e @ v / e.sum()
                weight[r, h] = e @ np.abs(v) / e.sum()
                lse[r, h] = z.max() + np.log(e.sum())
                size[r, h] = (np.abs(k) @ np.abs(q[r, h].astype(np.float64))).max() * abs(scale)
    return out, lse, weight, size


def regroup(pages, page, table, lengths, seqs, stride, parent=None, grow=None, window=0, sinks=0):
    """(table, lengths, copies as (from, to), pages in use), or None where pages or slots do not suffice."""
    rows, kept_of, length_of = [], [], []
    for b in range(seqs):
        p = b if parent is None else parent[b]
        if not 0 <= p < len(lengths):
            rows.append({})
            kept_of.append(0)
            length_of.append(0)
            continue
        old = lengths[p]
        length = max(0, old + (0 if grow is None else grow[b]))
        kept = min(old, length)
        row = {}
        for s in range(min(-(-kept // page), table.shape[1])):
            if not 0 <= table[p, s] < pages:
                continue
            last = (s + 1) * page - 1
            # the next query stands at position kept or later
            if window and not any(kept - j < window or j < sinks for j in (s * page, last)):
                continue
            row[s] = table[p, s]
        rows.append(row)
        kept_of.append(kept)
        length_of.append(length)
    held = {}
    for b, row in enumerate(rows):
        for s, id_ in row.items():
            held.setdefault(id_, []).append((b, kept_of[b] % page > 0 and s == kept_of[b] // page))
    free = [i for i in range(pages) if i not in held]
    copies, taken = [], 0
    need = 0
    for b, row in enumerate(rows):
        s = kept_of[b] // page
        plan = []
        if kept_of[b] % page and s in row:
            holders = held[row[s]]
            owner = None if any(not is_open for _, is_open in holders) else min(x for x, _ in holders)
            if owner != b:
                plan.append(("copy", s))
        plan += [("new", i) for i in range(-(-kept_of[b] // page), -(-length_of[b] // page))]
        if -(-length_of[b] // page) > stride:
            return None
        need += len(plan)
        if need > len(free):
            return None
        for what, i in plan:
            if what == "copy":
                copies.append((row[i], free[taken]))
            row[i] = free[taken]
            taken += 1
    out = np.full((seqs, stride), -1, np.int32)
    for b, row in enumerate(rows):
        for s, id_ in row.items():
            out[b, s] = id_
    return out, np.array(length_of, np.int32), copies, len(held) + taken


def compact(pages, table, lengths):
    used = sorted({int(i) for i in table.ravel() if 0 <= i < pages})
    n = len(used)
    free = [i for i in range(n) if i not in set(used)]
    moves = list(zip([i for i in used if i >= n], free))
    to = {**{i: i for i in used}, **dict(moves)}
    return np.array([[to.get(int(i), -1) for i in row] for row in table], np.int32), lengths.copy(), moves, n


def copy_pages(pool, copies):
    for a, z in copies:
        for x in (pool.k, pool.v, pool.k_scale, pool.v_scale):
            x[:, z] = x[:, a]
