"""Timed cases of the 8-bit token cache: writing keys and values, attending over them, and moving its pages.

A case is a dict of plain values. Its "op" says what one pass does:

  attend   entro_cache_attend: queries against the keys and values of their sequences, causal, with or without a sliding
           window whose first tokens stay visible
  append   entro_cache_append and, so that what was written comes back as values, entro_cache_read of every block it touched
  regroup  entro_cache_regroup: the page table of the next step (forks, drops, reorders, new tokens, pages that left the window)
  compact  entro_cache_compact: pages in use move to the front of the pool

The cache holds codes c in 0..255 with one 32-bit scale s for each block of tokens (a page) and head: a value is (c - 128) * s.
Pool layouts, "width" being the head's dimensions rounded up to 64, 96, 128, 192 or 256:

  k [layers][pages][kv_heads][page_tokens][width]      v [layers][pages][kv_heads][width][page_tokens]
  k_scale, v_scale [layers][pages][kv_heads]           table [sequences][slots], lengths [sequences]

Lengths follow from the case alone (a spread over (0, len] where "ragged" is set), everything else from the seed.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attend(name, **kw):
    c = {"name": name, "op": "attend", "seqs": 1, "new": 1, "len": 1024, "ragged": False, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "window": 0, "sinks": 0, "type": "bf16"}
    c.update(kw)
    return c


def _append(name, **kw):
    c = {"name": name, "op": "append", "seqs": 1, "new": 1, "len": 1024, "ragged": False, "kv_heads": 8, "dim": 128, "page": 64,
         "type": "bf16"}
    c.update(kw)
    return c


def _pages(name, op, **kw):
    c = {"name": name, "op": op, "seqs": 16, "len": 1024, "ragged": True, "layers": 32, "kv_heads": 8, "dim": 128, "page": 64}
    if op == "regroup":
        c.update({"parents": 16, "grow": 1, "window": 0, "sinks": 0})
    else:
        c["used"] = 0.5
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: one user's next token over a short context, heads of the 1.7B set
        _attend("token_short_32x64", len=517, kv_heads=32, dim=64, page=16),
        # a serving step: a next token for each of many users with contexts of all lengths, heads of the 7B set
        _attend("token_64_users_8k", seqs=64, len=8192, ragged=True),
        # one user deep in a very long context: the work has to be split along it
        _attend("token_one_128k", len=131072),
        # next tokens under a sliding window with a few first tokens kept, as many heads of keys as of queries (the 3.8B set)
        _attend("token_window_32x96", seqs=32, len=32768, ragged=True, kv_heads=32, dim=96, page=32, window=4096, sinks=4),
        # a long prompt's second half over the first one
        _attend("prompt_4096_of_8192", new=4096, len=8192),
        # prompts' pieces and single tokens in one call, odd sizes, 32-bit in and out, under a window
        _attend("mixed_f32_20x80", seqs=12, new=333, len=5000, ragged=True, q_heads=20, kv_heads=4, dim=80, page=16, window=1000,
                sinks=16, type="f32"),
        # a serving step's keys and values
        _append("append_64_users", seqs=64, len=8192, ragged=True),
        # prompts of several users written at once
        _append("append_prompts", seqs=6, new=8192, len=9000, ragged=True),
        # a step of beam search: 16 requests with 4 beams each, every one from the beam it grew out of
        _pages("regroup_beams", "regroup", seqs=64, len=2048, layers=16, parents=32),
        # one prompt answered 48 times over: all rows share its pages, each with an open page of its own
        _pages("fork_prompt_48", "regroup", seqs=48, len=4001, ragged=False, parents=1, grow=1),
        # a small pool of small pages after its users left
        _pages("compact_small", "compact", seqs=24, len=300, layers=24, kv_heads=4, dim=64, page=16, used=0.4),
        # a large pool, half of it in use and scattered, brought together before its upper half is given back
        _pages("compact_pool", "compact", seqs=32, len=4096, layers=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "regroup", "compact"])
    heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    dim = rng.choice([64, 96, 128, 128, 72, 80, 112, 192, 256, rng.randint(16, 256)])
    page = rng.choice([16, 32, 64, 64, 128])
    if op == "attend":
        c = _attend("", kv_heads=heads, dim=dim, page=page, ragged=rng.random() < 0.7, type=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        c["q_heads"] = heads * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if heads * g <= 64])
        c["seqs"] = _log_int(rng, 1, 64)
        c["len"] = _log_int(rng, 16, 65536)
        c["new"] = min(c["len"], rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 16, 2048)]))
        if rng.random() < 0.3:
            c["window"], c["sinks"] = _log_int(rng, 16, 8192), rng.choice([0, 1, 4, 16, 100])
        # no more keys, scores or multiplications than the largest listed cases take
        while c["seqs"] * c["len"] * heads * max(dim, 64) > 1 << 28 or c["seqs"] * c["new"] * c["len"] * c["q_heads"] > 1 << 29:
            if c["seqs"] > 1:
                c["seqs"] = c["seqs"] // 2
            else:
                c["len"] = max(16, c["len"] // 2)
                c["new"] = min(c["new"], c["len"])
    elif op == "append":
        c = _append("", kv_heads=heads, dim=dim, page=page, ragged=rng.random() < 0.7, type=rng.choice(["bf16", "bf16", "f32"]))
        c["seqs"] = _log_int(rng, 1, 128)
        c["len"] = _log_int(rng, 1, 16384)
        c["new"] = min(c["len"], rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 16, 8192)]))
        while c["seqs"] * max(c["new"], page) * heads * max(dim, 64) > 1 << 25 or c["seqs"] * c["len"] * heads * max(dim, 64) > 1 << 29:
            if c["seqs"] > 1:
                c["seqs"] = c["seqs"] // 2
            else:
                c["len"] = max(1, c["len"] // 2)
                c["new"] = min(c["new"], c["len"])
    else:
        c = _pages("", op, kv_heads=rng.choice([1, 2, 4, 8]), dim=dim, page=page, layers=rng.choice([1, 2, 4, 16, 24, 32]))
        c["seqs"] = _log_int(rng, 1, 96)
        c["len"] = _log_int(rng, 8, 8192)
        c["ragged"] = rng.random() < 0.7
        if op == "regroup":
            c["parents"], c["grow"] = rng.randint(1, c["seqs"]), rng.choice([0, 1, 1, 3, 40])
            if rng.random() < 0.3:
                c["window"], c["sinks"] = _log_int(rng, 16, 4096), rng.choice([0, 4, 32])
        else:
            c["used"] = rng.choice([0.2, 0.5, 0.8, 0.95])
        while c["seqs"] * (c["len"] + 2 * page) * c["layers"] * c["kv_heads"] * max(dim, 64) > 1 << 30:
            if c["layers"] > 1:
                c["layers"] //= 2
            elif c["seqs"] > 1:
                c["seqs"] //= 2
                if op == "regroup":
                    c["parents"] = min(c["parents"], c["seqs"])
            else:
                c["len"] //= 2
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------- inputs
def _width(dim):
    return next(w for w in (64, 96, 128, 192, 256) if w >= dim)


def _spread(most, count, ragged, least=1):
    """`count` sizes of at most `most`: all of them `most`, or spread over least..most with `most` among them."""
    if not ragged:
        return [most] * count
    return [max(least, most if i == 0 else int(most * ((i * 0.6180339887498949) % 1.0))) for i in range(count)]


def _sizes(c):
    """(lengths, new tokens) of the case's sequences; a ragged call has sequences without new tokens and with a single one."""
    new = _spread(c["new"], c["seqs"], c["ragged"] and c["new"] > 1, 0)
    lengths = [max(a, b) for a, b in zip(_spread(c["len"], c["seqs"], c["ragged"]), new)]
    return lengths, new


def _slots(tokens, page):
    return -(-tokens // page)


def _starts(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device=DEV)


def _codes(shape, channel, gen):
    """Codes as a quantiser leaves them: bell-shaped, a few channels (dimension `channel`) several times wider than the others."""
    n = shape[channel]
    spread = torch.exp(0.5 * torch.randn(n, device=DEV, generator=gen)) * 18
    out = torch.empty(shape, dtype=torch.uint8, device=DEV)
    view = [n if i == channel else 1 for i in range(1, len(shape))]
    for layer in range(shape[0]):
        for p0 in range(0, shape[1], 4096):
            x = torch.randn(min(4096, shape[1] - p0), *shape[2:], device=DEV, generator=gen)
            out[layer, p0: p0 + 4096] = (x * spread.view(view)).round_().clamp_(-127, 127).add_(128).to(torch.uint8)
    return out


def _pool(c, pages, gen, random_codes=True):
    layers, heads, page, w = c.get("layers", 1), c["kv_heads"], c["page"], _width(c["dim"])
    ks, vs = (layers, pages, heads, page, w), (layers, pages, heads, w, page)
    if random_codes:
        k, v = _codes(ks, 4, gen), _codes(vs, 3, gen)
    else:
        k, v = (torch.randint(0, 256, s, dtype=torch.uint8, device=DEV, generator=gen) for s in (ks, vs))
    scale = [torch.exp(0.3 * torch.randn(layers, pages, heads, device=DEV, generator=gen)) * f for f in (0.035, 0.02)]
    return {"k": k, "v": v, "k_scale": scale[0], "v_scale": scale[1]}


def _table(lengths, page, pages, slots, gen):
    """Pages in no order at all, as a pool hands them out after a while."""
    perm = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)
    need = [_slots(n, page) for n in lengths]
    table = torch.full((len(lengths), slots), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at: at + n]
        at += n
    return table


def prepare(case, seed):
    c, gen = case, torch.Generator(device=DEV)
    gen.manual_seed(seed)
    page = c["page"]
    s = {"case": c}
    if c["op"] in ("attend", "append"):
        lengths, new = _sizes(c)
        slots = _slots(max(lengths), page)
        pages = sum(_slots(n, page) for n in lengths) + 3
        s.update(_pool(c, pages, gen))
        s["table"] = _table(lengths, page, pages, slots, gen)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        s["start"], s["tokens"], s["max_new"], s["max_len"] = _starts(new), sum(new), max(new), max(lengths)
        dtype = TYPES[c["type"]]
        if c["op"] == "attend":
            s["q"] = (1.3 * torch.randn(s["tokens"], c["q_heads"], c["dim"], device=DEV, generator=gen)).to(dtype)
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(s["tokens"], c["q_heads"], device=DEV)
        else:
            wide = torch.exp(0.5 * torch.randn(c["dim"], device=DEV, generator=gen))
            s["k_new"] = (torch.randn(s["tokens"], c["kv_heads"], c["dim"], device=DEV, generator=gen) * wide).to(dtype)
            s["v_new"] = torch.randn(s["tokens"], c["kv_heads"], c["dim"], device=DEV, generator=gen).to(dtype)
            # the whole of every block that is written to comes back
            back = [n and length - (length - n) // page * page for length, n in zip(lengths, new)]
            s["back_start"], s["back_tokens"], s["back_max"] = _starts(back), sum(back), max(back)
            s["k_back"], s["v_back"] = (torch.zeros(s["back_tokens"], c["kv_heads"], c["dim"], dtype=dtype, device=DEV) for _ in "kv")
    else:
        lengths = _spread(c["len"], c["seqs"] if c["op"] == "compact" else c["parents"], c["ragged"])
        grow = c.get("grow", 0)
        used = sum(_slots(n, page) for n in lengths)
        if c["op"] == "regroup":
            # every row may need a page to copy its open one to, and pages for what it grows by
            pages = used + c["seqs"] * (1 + _slots(grow + page - 1, page)) + 5
            slots = _slots(max(lengths) + grow, page) + 1
            rows = c["seqs"]
        else:
            pages, slots, rows = max(used + 1, int(used / c["used"])), _slots(max(lengths), page), c["seqs"]
        s.update(_pool(c, pages, gen, random_codes=False))
        s["table"] = _table(lengths, page, pages, slots, gen)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        if c["op"] == "regroup":
            s["parent"] = torch.randint(0, c["parents"], (rows,), dtype=torch.int32, device=DEV, generator=gen)
            s["parent"][torch.rand(rows, device=DEV, generator=gen) < 0.05] = -1          # a row in twenty has ended
            s["grow"] = torch.full((rows,), grow, dtype=torch.int32, device=DEV)
        s["next_table"] = torch.zeros(rows, slots, dtype=torch.int32, device=DEV)
        s["next_lengths"] = torch.zeros(rows, dtype=torch.int32, device=DEV)
        s["status"] = torch.zeros(4, dtype=torch.int32, device=DEV)
    if own:                                                    # a program makes its descriptors once, beside its buffers
        s["call"] = _handle(s)
    return s


def _handle(s):
    """The descriptors and the workspace that a program keeps beside its buffers, as a function that makes the calls of a pass."""
    import paper_2505_02380_amd as E
    c = s["case"]
    cache = E.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], page_tokens=c["page"], head_dim=c["dim"])
    table = E.CacheTable(s["table"], s["lengths"])

    def room(n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)

    if c["op"] == "attend":
        query = E.CacheQuery(s["q"], s["out"], s["start"], lse=s["lse"], scale=_scale(c), window=c["window"], sinks=c["sinks"],
                             max_new=s["max_new"], max_len=s["max_len"])
        ws = room(E.entro_cache_attend_workspace_bytes(cache, table, query))
        return lambda: E.entro_cache_attend(cache, table, query, ws)
    if c["op"] == "append":
        rows = E.CacheRows(s["k_new"], s["v_new"], s["start"], max_new=s["max_new"])
        back = E.CacheRows(s["k_back"], s["v_back"], s["back_start"], max_new=s["back_max"])

        def write_and_read():
            E.entro_cache_append(cache, table, rows)
            E.entro_cache_read(cache, table, back)
        return write_and_read
    following = E.CacheTable(s["next_table"], s["next_lengths"])
    ws, status = room(E.entro_cache_pages_workspace_bytes(cache, table, following)), s["status"]
    if c["op"] == "regroup":
        parent, grow = s["parent"], s["grow"]
        return lambda: E.entro_cache_regroup(cache, table, following, status, ws, parent=parent, grow=grow,
                                             window=c["window"], sinks=c["sinks"])
    return lambda: E.entro_cache_compact(cache, table, following, status, ws)


def _scale(c):
    return 1.0 / math.sqrt(c["dim"])


# ----------------------------------------------------------------------------------------------------------------- a pass
def run(state):
    s, op = state, state["case"]["op"]
    if own:
        s["call"]()
    else:
        {"attend": _plain_attend, "append": _plain_append, "regroup": _plain_regroup, "compact": _plain_compact}[op](s)
    if op == "attend":
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        return {"k": s["k_back"], "v": s["v_back"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return {"table": s["next_table"], "lengths": s["next_lengths"], "status": s["status"], "k": s["k"], "v": s["v"],
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _rows_of(start, tokens):
    """(sequence, offset) of every row of a tensor of `tokens` rows."""
    row = torch.arange(tokens, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(start, row, right=True) - 1
    return seq, row - start[seq]


def _plain_attend(s):
    c = s["case"]
    page, dim, groups = c["page"], c["dim"], c["q_heads"] // c["kv_heads"]
    n_seqs, slots = s["table"].shape
    new, span, heads = s["max_new"], slots * page, c["kv_heads"]
    pages = s["table"].clamp(min=0).long()
    k = (s["k"][0][pages][..., :dim].float() - 128) * s["k_scale"][0][pages][..., None, None]          # [seq, slot, head, token, dim]
    v = (s["v"][0][pages][..., :dim, :].float() - 128) * s["v_scale"][0][pages][..., None, None]       # [seq, slot, head, dim, token]
    k = k.permute(0, 2, 4, 1, 3).reshape(n_seqs, heads, dim, span)
    v = v.permute(0, 2, 1, 4, 3).reshape(n_seqs, heads, span, dim)
    offset = torch.arange(new, device=DEV)
    at = (s["start"][:-1, None] + offset).clamp(max=s["tokens"] - 1)
    q = s["q"][at].float().view(n_seqs, new, heads, groups, dim).permute(0, 2, 3, 1, 4).reshape(n_seqs, heads, groups * new, dim)
    score = torch.matmul(q, k).mul_(_scale(c)).view(n_seqs, heads, groups, new, span)
    here = (s["lengths"] - (s["start"][1:] - s["start"][:-1]))[:, None] + offset                       # position of each query
    key = torch.arange(span, device=DEV)
    seen = key <= here[..., None]
    if c["window"]:
        seen &= (here[..., None] - key < c["window"]) | (key < c["sinks"])
    seen &= (s["table"] >= 0).repeat_interleave(page, 1)[:, None]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n_seqs, heads, groups * new, span), v).view(n_seqs, heads, groups, new, dim) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)[..., 0]
    seq, off = _rows_of(s["start"], s["tokens"])
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(n_seqs, new, c["q_heads"], dim)[seq, off])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(n_seqs, new, c["q_heads"])[seq, off])


def _plain_blocks(x, old, s_old, is_new, is_old):
    """New codes and scales of blocks: x new values, old codes less 128, both [blocks, head, token, dim] in 32 bits."""
    s_old = torch.where(is_old.any(1)[:, None], s_old, 0.0)
    x = torch.where(is_new[:, None, :, None], x, 0.0)
    most = torch.where(torch.isfinite(x), x.abs(), 0.0).amax((2, 3))
    scale = torch.maximum(s_old, most / 127)
    by = torch.where(scale > 0, scale, 1.0)[..., None, None]
    fresh = torch.nan_to_num(torch.round(x / by), nan=0.0, posinf=127, neginf=-127).clamp(-127, 127) * (scale > 0)[..., None, None]
    kept = torch.round(old * s_old[..., None, None] / by)
    return torch.where(is_new[:, None, :, None], fresh, torch.where(is_old[:, None, :, None], kept, old)) + 128, scale


def _plain_append(s):
    c = s["case"]
    page, dim = c["page"], c["dim"]
    count = s["start"][1:] - s["start"][:-1]
    first = s["lengths"] - count                                                                        # position of the first new token
    block = torch.div(first, page, rounding_mode="floor")[:, None] + torch.arange((s["max_new"] + page - 2) // page + 1, device=DEV)
    seq, which = torch.nonzero((block * page < s["lengths"][:, None]) & (count > 0)[:, None], as_tuple=True)
    block = block[seq, which]
    pages = s["table"][seq, block].long()
    pos = block[:, None] * page + torch.arange(page, device=DEV)
    is_new = (pos >= first[seq][:, None]) & (pos < s["lengths"][seq][:, None])
    is_old = pos < first[seq][:, None]
    row = (s["start"][seq][:, None] + pos - first[seq][:, None]).clamp(0, s["tokens"] - 1)
    k = s["k"][0][pages][..., :dim].float() - 128
    v = s["v"][0][pages][..., :dim, :].float().transpose(2, 3) - 128
    k, ks = _plain_blocks(s["k_new"][row].float().transpose(1, 2), k, s["k_scale"][0][pages], is_new, is_old)
    v, vs = _plain_blocks(s["v_new"][row].float().transpose(1, 2), v, s["v_scale"][0][pages], is_new, is_old)
    s["k"][0, pages, :, :, :dim] = k.to(torch.uint8)
    s["v"][0, pages, :, :dim, :] = v.transpose(2, 3).to(torch.uint8)
    s["k_scale"][0, pages], s["v_scale"][0, pages] = ks, vs
    back, off = _rows_of(s["back_start"], s["back_tokens"])
    pos = (s["lengths"] - (s["back_start"][1:] - s["back_start"][:-1]))[back] + off
    pages, at = s["table"][back, torch.div(pos, page, rounding_mode="floor")].long(), torch.remainder(pos, page)
    s["k_back"].copy_((s["k"][0][pages, :, at, :dim].float() - 128) * s["k_scale"][0][pages][..., None])
    s["v_back"].copy_((s["v"][0][pages, :, :dim, at].float() - 128) * s["v_scale"][0][pages][..., None])


def _plain_move(s, src, dst):
    s["k"][:, dst], s["v"][:, dst] = s["k"][:, src], s["v"][:, src]
    s["k_scale"][:, dst], s["v_scale"][:, dst] = s["k_scale"][:, src], s["v_scale"][:, src]


def _plain_regroup(s):
    c = s["case"]
    page, slots, pages = c["page"], s["table"].shape[1], s["k"].shape[1]
    parent = s["parent"].long()
    rows = torch.arange(len(parent), device=DEV)
    alive = parent >= 0
    old = torch.where(alive, s["lengths"][parent.clamp(min=0)], 0)
    grow = torch.where(alive, s["grow"], 0)
    length = (old + grow).clamp(min=0)
    kept = torch.minimum(old, length)
    slot = torch.arange(slots, device=DEV)
    table = s["table"][parent.clamp(min=0)].clone()
    table[~alive] = -1
    table[slot >= _ceil(kept, page)[:, None]] = -1
    if c["window"]:
        table[((slot + 1) * page + c["window"] <= kept[:, None] + 1) & (slot * page >= c["sinks"])] = -1
    # a page that is only partly filled belongs to one row: the lowest, unless a row holds it as a full one
    open_slot = torch.div(kept, page, rounding_mode="floor")
    is_open = (slot == open_slot[:, None]) & (torch.remainder(kept, page) > 0)[:, None] & (table >= 0)
    owner = torch.full((pages,), len(parent), dtype=torch.int64, device=DEV)
    held = table >= 0
    claim = torch.where(is_open, rows[:, None], -1)
    owner.scatter_reduce_(0, table[held].long(), claim[held], "amin")
    open_page = table.gather(1, open_slot.clamp(max=slots - 1)[:, None])[:, 0]
    copies = is_open.any(1) & (owner[open_page.clamp(min=0).long()] != rows)
    used = (owner < len(parent)).to(torch.int32)
    fresh = torch.argsort(used, stable=True)                                                            # free pages first, lowest first
    need = copies.long() + (_ceil(length, page) - _ceil(kept, page))
    first = torch.cumsum(need, 0) - need
    is_copy = is_open & copies[:, None]
    is_grown = (slot >= _ceil(kept, page)[:, None]) & (slot < _ceil(length, page)[:, None])
    nth = first[:, None] + torch.where(is_grown, copies.long()[:, None] + slot - _ceil(kept, page)[:, None], 0)
    nxt = torch.where(is_copy | is_grown, fresh[nth.clamp(max=pages - 1)].to(torch.int32), table)
    _plain_move(s, table[is_copy].long(), nxt[is_copy].long())
    s["next_table"].copy_(nxt)
    s["next_lengths"].copy_(length)
    in_use = used.sum() + need.sum()
    s["status"].copy_(torch.stack([torch.zeros_like(in_use), in_use, pages - in_use, copies.sum()]))


def _ceil(tokens, page):
    return torch.div(tokens + page - 1, page, rounding_mode="floor")


def _plain_compact(s):
    pages = s["k"].shape[1]
    held = s["table"] >= 0
    used = torch.zeros(pages, dtype=torch.int32, device=DEV)
    used[s["table"][held].long()] = 1
    total = used.sum()
    at = torch.arange(pages, device=DEV)
    src, dst = at[(used > 0) & (at >= total)], at[(used == 0) & (at < total)]
    to = at.to(torch.int32)
    to[src] = dst.to(torch.int32)
    _plain_move(s, src, dst)
    s["next_table"].copy_(torch.where(held, to[s["table"].clamp(min=0).long()], -1))
    s["next_lengths"].copy_(s["lengths"])
    s["status"].copy_(torch.stack([torch.zeros_like(total), total, pages - total, torch.full_like(total, len(src))]))


# ------------------------------------------------------------------------------------------------------------------ work
def _seen(c, length, new):
    """(keys that any of the last `new` tokens of a sequence see, pairs of a query and a key that it sees)."""
    if not new:
        return 0, 0
    w, k = c["window"], c["sinks"]
    if not w:
        return length, sum(range(length - new + 1, length + 1))
    first = max(0, length - new - w + 1)
    pairs = sum(min(p + 1, w + min(k, max(0, p + 1 - w))) for p in range(length - new, length))
    return length - first + min(k, first), pairs


def work(case):
    c = case
    w = c["dim"]
    if c["op"] == "attend":
        lengths, new = _sizes(c)
        seen = [_seen(c, a, b) for a, b in zip(lengths, new)]
        keys, pairs, rows = sum(k for k, _ in seen), sum(p for _, p in seen), sum(new) * c["q_heads"]
        size = 2 if c["type"] == "bf16" else 4
        return {"bytes": keys * c["kv_heads"] * 2 * (w + 4 / c["page"]) + rows * (2 * w * size + 4), "flops": 4.0 * pairs * c["q_heads"] * w}
    if c["op"] == "append":
        lengths, new = _sizes(c)
        size = 2 if c["type"] == "bf16" else 4
        rows = sum(new)
        blocks = sum(_slots(a, c["page"]) - (a - b) // c["page"] for a, b in zip(lengths, new) if b)
        back = sum(a - (a - b) // c["page"] * c["page"] for a, b in zip(lengths, new) if b)
        # new rows read once and written once in 8 bits; the blocks that they touch read and given back as values
        return {"bytes": 2.0 * c["kv_heads"] * (rows * w * (size + 1) + back * w * (1 + size) + blocks * 8), "flops": 0}
    lengths = _spread(c["len"], c["seqs"] if c["op"] == "compact" else c["parents"], c["ragged"])
    one = c["layers"] * c["kv_heads"] * 2 * (c["page"] * _width(w) + 4)
    used = sum(_slots(n, c["page"]) for n in lengths)
    if c["op"] == "compact":
        pages = max(used + 1, int(used / c["used"]))
        moved = used * (pages - used) / pages                  # as many as there are holes among the first `used`, on average
        return {"bytes": 2.0 * moved * one + 8.0 * used, "flops": 0}
    # rows that share a parent's open page: all but one of them copy it
    shared = [n % c["page"] > 0 for n in lengths]
    share = sum(shared) / len(lengths)
    copies = share * max(0.0, 0.95 * c["seqs"] - c["parents"] * (1 - (1 - 1 / c["parents"]) ** (0.95 * c["seqs"])))
    return {"bytes": 2.0 * copies * one + 8.0 * c["seqs"] * used / len(lengths), "flops": 0}


# ----------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions in 64 bits, a sequence at a time. Pages that only move have no computed numbers."""
    c = case
    if c["op"] in ("regroup", "compact"):
        return None
    s = prepare(c, seed)
    return _exact_attend(s) if c["op"] == "attend" else _exact_append(s)


def _exact_values(s, b, first, last):
    """Keys and values of positions first..last-1 of sequence b: [tokens, head, dim]."""
    page, dim = s["case"]["page"], s["case"]["dim"]
    pos = torch.arange(first, last, device=DEV)
    p, t = s["table"][b][pos // page].long(), pos % page
    k = (s["k"][0][p, :, t, :dim].double() - 128) * s["k_scale"][0][p].double()[..., None]
    v = (s["v"][0][p, :, :dim, t].double() - 128) * s["v_scale"][0][p].double()[..., None]
    return k, v


def _exact_attend(s):
    c = s["case"]
    lengths, new = _sizes(c)
    per = c["q_heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for b in range(c["seqs"]):
        if not new[b]:
            continue
        k, v = _exact_values(s, b, 0, lengths[b])
        j = torch.arange(lengths[b], device=DEV)
        for r0 in range(0, new[b], 1024):
            r1 = min(new[b], r0 + 1024)
            i = torch.arange(lengths[b] - new[b] + r0, lengths[b] - new[b] + r1, device=DEV)[:, None]
            ok = j[None] <= i
            if c["window"]:
                ok &= (i - j[None] < c["window"]) | (j[None] < c["sinks"])
            for h in range(c["q_heads"]):
                z = s["q"][row + r0: row + r1, h].double() @ k[:, h // per].T.contiguous() * _scale(c)
                z = torch.where(ok, z, -math.inf)
                out[row + r0: row + r1, h] = torch.softmax(z, -1) @ v[:, h // per].contiguous()
                lse[row + r0: row + r1, h] = torch.logsumexp(z, -1)
        row += new[b]
    return {"out": out, "lse": lse}


def _exact_append(s):
    c = s["case"]
    page, dim = c["page"], c["dim"]
    lengths, new = _sizes(c)
    back = {"k": [], "v": []}
    scales = {"k": s["k_scale"].double(), "v": s["v_scale"].double()}
    row = 0
    for b in range(c["seqs"]):
        if not new[b]:
            continue
        begin = lengths[b] - new[b]
        head = begin // page * page
        old = dict(zip("kv", _exact_values(s, b, head, begin)))
        pad = -(lengths[b] - head) % page
        pages = s["table"][b][head // page: _slots(lengths[b], page)].long()
        for x in "kv":
            fresh = s[x + "_new"][row: row + new[b]].double()
            all_new = torch.cat([torch.zeros_like(old[x]), fresh, torch.zeros(pad, *fresh.shape[1:], dtype=torch.float64, device=DEV)])
            blocks = all_new.view(-1, page, *fresh.shape[1:])
            scale = blocks.abs().amax((1, 3)) / 127
            if begin > head:
                scale[0] = torch.maximum(scale[0], s[x + "_scale"][0][pages[0]].double())
            scale = scale.float().double()                     # a scale is held in 32 bits
            values = torch.cat([old[x], fresh, all_new[begin - head + new[b]:]]).view(blocks.shape)
            values = torch.round(values / scale[:, None, :, None]) * scale[:, None, :, None]
            back[x].append(values.reshape(-1, *fresh.shape[1:])[: lengths[b] - head])
            scales[x][0][pages] = scale
        row += new[b]
    return {"k": torch.cat(back["k"]), "v": torch.cat(back["v"]), "k_scale": scales["k"], "v_scale": scales["v"]}
