"""Timed cases of positions and of shared prefixes: heads normed and rotated, written to the 8-bit token cache in that pass, and
attention for groups of sequences that begin with the same pages.

A case is a dict of plain values. Its "op" says what one pass does:

  rotate   entro_rotate: rows of queries and keys, normed per head or not, and rotated by their positions
  append   entro_cache_append_rotated, and entro_cache_read of every block it touched, so that what was written comes back as values
  attend   entro_cache_attend_shared: queries against the keys and values of their sequences, the tokens that a group's sequences
           share taken once for all of them
  shared   entro_cache_shared: how many tokens the sequences of each group share

The pool's layouts, "width" being the head's dimensions rounded up to 64, 96, 128, 192 or 256 (a value is (code - 128) * scale):

  k [layers][pages][kv_heads][page_tokens][width]      v [layers][pages][kv_heads][width][page_tokens]
  k_scale, v_scale [layers][pages][kv_heads]           table [sequences][slots], lengths [sequences]

Sizes of sequences and groups follow from the case alone, everything else from the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _turning(**kw):
    """How heads are normed and rotated: the first `rotated` of a head's dimensions, in pairs of halves or of neighbours."""
    c = {"q_heads": 32, "kv_heads": 8, "dim": 128, "rotated": 128, "layout": "halves", "norm": "none", "base": 10000.0, "scaling": "none",
         "factor": 1.0, "trained": 4096, "type": "bf16"}
    c.update(kw)
    return c


def _rotate(name, **kw):
    c = {"name": name, "op": "rotate", "tokens": 1, "runs": 1, "far": 4096, "packed": False}
    c.update(_turning(**kw))
    return c


def _append(name, **kw):
    c = {"name": name, "op": "append", "seqs": 1, "new": 1, "len": 1024, "ragged": False, "page": 64, "packed": False}
    c.update(_turning(**kw))
    return c


def _attend(name, **kw):
    c = {"name": name, "op": "attend", "groups": 1, "each": 4, "lone": 0, "prefix": 1000, "own": 100, "new": 1, "ragged": False, "q_heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64, "window": 0, "sinks": 0, "type": "bf16"}
    c.update(kw)
    return c


def _shared(name, **kw):
    c = {"name": name, "op": "shared", "groups": 16, "each": 4, "prefix": 1500, "own": 500, "ragged": True, "page": 64}
    c.update(kw)
    return c


def listed():
    return [
        # one user's next token: heads of the 7B set, a norm on each
        _rotate("rotate_token", tokens=1, far=131072, norm="rms"),
        # a prompt, its q, k and v rows side by side as one product leaves them, frequencies of a context four times as long as the trained one
        _rotate("rotate_prompt_8192", tokens=8192, far=1, packed=True, base=500000.0, scaling="parts", factor=4.0, trained=8192),
        # pieces of prompts far into their contexts, odd sizes, neighbours as pairs, part of the head, 32-bit in and out
        _rotate("rotate_pieces_f32_20x80", tokens=4999, runs=7, far=1 << 22, q_heads=20, kv_heads=4, dim=80, rotated=32, layout="pairs", norm="centred",
                type="f32"),
        # a serving step: a next token for each of many users, normed, rotated and written
        _append("append_64_users", seqs=64, len=8192, ragged=True, norm="rms", packed=True),
        # prompts of several users written at once
        _append("append_prompts", seqs=6, new=8192, len=9000, ragged=True),
        # prompts' pieces and single tokens in one call, heads of 96 of which half are rotated, small pages, 32-bit rows
        _append("append_pieces_f32_24x96", seqs=12, new=333, len=5000, ragged=True, q_heads=24, kv_heads=4, dim=96, rotated=48, layout="pairs", norm="rms",
                page=16, scaling="linear", factor=2.0, type="f32"),
        # beams that go on from one short prompt, heads of the 1.7B set
        _attend("beams_4_32x64", each=4, prefix=517, own=40, kv_heads=32, dim=64, page=16),
        # one prompt answered 48 times over, each answer some way on
        _attend("answers_48", each=48, prefix=4001, own=500, ragged=True),
        # many users behind one long common context
        _attend("users_64_behind_32k", each=64, prefix=32768, own=2048, ragged=True),
        # several requests with pieces of new tokens behind shared contexts, one sequence alone, a window, odd heads, 32-bit in and out
        _attend("pieces_f32_20x80", groups=5, each=6, lone=1, prefix=5000, own=400, new=150, ragged=True, q_heads=20, kv_heads=4, dim=80, page=16,
                window=3000, sinks=16, type="f32"),
        # after a step of beam search over 16 requests
        _shared("shared_beams"),
        # answers to a few very long documents in small pages
        _shared("shared_documents", groups=4, each=48, prefix=100000, own=9000, page=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _draw_turning(rng, c):
    c["dim"] = rng.choice([64, 96, 128, 128, 80, 112, 192, 256, rng.randint(16, 256)])
    c["rotated"] = rng.choice([c["dim"] // 2 * 2, c["dim"] // 2 * 2, c["dim"] // 4 * 2, 2 * rng.randint(1, c["dim"] // 2)])
    c["layout"], c["norm"] = rng.choice(["halves", "halves", "pairs"]), rng.choice(["none", "rms", "centred"])
    c["base"] = rng.choice([10000.0, 500000.0, 1000000.0])
    c["scaling"] = rng.choice(["none", "none", "linear", "parts"])
    c["factor"], c["trained"] = rng.choice([2.0, 4.0, 8.0, 32.0]), rng.choice([2048, 4096, 8192])
    c["kv_heads"] = rng.choice([1, 2, 4, 5, 8, 16, 32])
    c["q_heads"] = c["kv_heads"] * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if c["kv_heads"] * g <= 64])
    c["type"], c["packed"] = rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "attend", "attend", "attend", "shared"])
    ragged = rng.random() < 0.7
    if op == "rotate":
        c = _rotate("", tokens=_log_int(rng, 1, 16384), far=_log_int(rng, 1, 1 << 26))
        _draw_turning(rng, c)
        c["runs"] = rng.randint(1, min(c["tokens"], 20))
        while c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["dim"] > 1 << 25:
            c["tokens"] = c["tokens"] // 2
        c["runs"] = min(c["runs"], c["tokens"])
    elif op == "append":
        c = _append("", seqs=_log_int(rng, 1, 128), len=_log_int(rng, 1, 16384), ragged=ragged, page=rng.choice([16, 32, 64, 64, 128]))
        _draw_turning(rng, c)
        c["new"] = min(c["len"], rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 16, 8192)]))
        while (c["seqs"] * max(c["new"], c["page"]) * (c["kv_heads"] + c["q_heads"] / 4) * max(c["dim"], 64) > 1 << 25
               or c["seqs"] * c["len"] * c["kv_heads"] * max(c["dim"], 64) > 1 << 29):
            if c["seqs"] > 1:
                c["seqs"] = c["seqs"] // 2
            else:
                c["len"] = max(1, c["len"] // 2)
                c["new"] = min(c["new"], c["len"])
    elif op == "attend":
        c = _attend("", groups=rng.choice([1, 1, 2, 3, rng.randint(4, 16)]), each=_log_int(rng, 2, 96), lone=rng.choice([0, 0, 1, 3]),
                    prefix=_log_int(rng, 32, 65536), own=_log_int(rng, 1, 4096), ragged=ragged, page=rng.choice([16, 32, 64, 64, 128]),
                    dim=rng.choice([64, 96, 128, 128, 72, 80, 112, 192, 256, rng.randint(16, 256)]), type=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        c["kv_heads"] = rng.choice([1, 2, 4, 5, 8, 16, 32])
        c["q_heads"] = c["kv_heads"] * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if c["kv_heads"] * g <= 64])
        c["new"] = min(c["own"], rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 16, 256)]))
        if rng.random() < 0.25:
            c["window"], c["sinks"] = _log_int(rng, 16, 8192), rng.choice([0, 1, 4, 16, 100])

        def too_much():
            seqs, wide = c["groups"] * c["each"] + c["lone"], c["kv_heads"] * max(c["dim"], 64)
            keys = max(c["groups"] * c["prefix"], seqs * (c["own"] + c["page"]))
            return keys * wide > 1 << 27 or seqs * c["new"] * c["q_heads"] * (c["prefix"] + c["own"]) > 1 << 27 or seqs * c["new"] * c["q_heads"] * c["dim"] > 1 << 24
        while too_much():
            big = max(("groups", "each", "new"), key=lambda n: c[n])
            if c["groups"] * c["each"] > 2 and big != "new":
                c[big] = max(1 if big == "groups" else 2, c[big] // 2)
            else:
                c["prefix"], c["own"] = max(32, c["prefix"] // 2), max(1, c["own"] // 2)
                c["new"] = max(1, min(c["new"] // 2, c["own"]))
    else:
        c = _shared("", groups=_log_int(rng, 4, 64), each=_log_int(rng, 2, 96), own=_log_int(rng, 1, 16384), ragged=ragged, page=rng.choice([16, 32, 64, 128]))
        c["prefix"] = _log_int(rng, 16 * c["page"], 131072)
        while c["groups"] * c["each"] * _slots(c["prefix"] + c["own"], c["page"]) > 1 << 21:
            c["groups" if c["groups"] > 4 else "each"] //= 2
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


def _slots(tokens, page):
    return -(-tokens // page)


def _counts(c):
    """(lengths, new tokens) of the sequences of an append case; a ragged call has sequences without new tokens and with a single one."""
    new = _spread(c["new"], c["seqs"], c["ragged"] and c["new"] > 1, 0)
    return [max(a, b) for a, b in zip(_spread(c["len"], c["seqs"], c["ragged"]), new)], new


def _groups(c):
    """(sequences of each group, tokens each group begins with, tokens of each sequence after those, new ones among them); sequences that are in
    no group come last."""
    each = _spread(c["each"], c["groups"], c["ragged"], min(2, c["each"]))
    prefix = _spread(c["prefix"], c["groups"], c["ragged"])
    seqs = sum(each) + c.get("lone", 0)
    new = _spread(c.get("new", 1), seqs, c["ragged"] and c.get("new", 1) > 1, 0)
    return each, prefix, [max(a, b) for a, b in zip(_spread(c["own"], seqs, c["ragged"]), new)], new


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(counts):
    return _ints(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32).tolist())


def _codes(shape, channel, gen):
    """Codes as a quantiser leaves them: bell-shaped, a few channels (dimension `channel`) several times wider than the others."""
    n = shape[channel]
    spread = torch.exp(0.5 * torch.randn(n, device=DEV, generator=gen)) * 18
    view = [n if i == channel else 1 for i in range(len(shape))]
    return (torch.randn(shape, device=DEV, generator=gen) * spread.view(view)).round_().clamp_(-127, 127).add_(128).to(torch.uint8)


def _pool(c, pages, gen):
    heads, page, w = c["kv_heads"], c["page"], _width(c["dim"])
    s = {"k": _codes((1, pages, heads, page, w), 4, gen), "v": _codes((1, pages, heads, w, page), 3, gen)}
    s["k_scale"], s["v_scale"] = (torch.exp(0.3 * torch.randn(1, pages, heads, device=DEV, generator=gen)) * f for f in (0.035, 0.02))
    return s


def _scattered(need, pages, slots, gen):
    """Pages in no order at all, as a pool hands them out after a while: need[b] of them in row b."""
    perm = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)
    held = torch.arange(slots, device=DEV) < _ints(need)[:, None]
    table = torch.full((len(need), slots), -1, dtype=torch.int32, device=DEV)
    table[held] = perm[: sum(need)]
    return table


def _frequencies(c):
    """Radians a position, in 64 bits: base^(-2 i / rotated), scaled as the case says. Scaled by parts: pairs that turn less than once over the
    trained length are slowed down by the factor, those that turn more than four times are left, a ramp between them."""
    f = np.float64(c["base"]) ** (-np.arange(0, c["rotated"], 2, dtype=np.float64) / c["rotated"])
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "parts":
        left = np.clip((c["trained"] * f / (2 * np.pi) - 1.0) / 3.0, 0.0, 1.0)
        f = f * (left + (1 - left) / c["factor"])
    return f


def _amplitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "parts" else 1.0


def _heads(s, c, tokens, gen):
    """q, k, v rows as products leave them: on their own, or side by side in one tensor; some channels several times wider than others."""
    counts = (c["q_heads"], c["kv_heads"], c["kv_heads"])
    x = torch.randn(tokens, sum(counts), c["dim"], device=DEV, generator=gen)
    x *= torch.exp(0.5 * torch.randn(sum(counts), c["dim"], device=DEV, generator=gen))
    x = x.to(TYPES[c["type"]])
    parts = torch.split(x, counts, 1)
    s["q"], s["k_rows"], s["v_rows"] = parts if c["packed"] else [p.contiguous() for p in parts]
    s["q_out"] = torch.zeros(s["q"].shape, dtype=x.dtype, device=DEV)
    s["k_out"] = torch.zeros(s["k_rows"].shape, dtype=x.dtype, device=DEV)
    s["q_gain"], s["k_gain"] = (1 + 0.2 * torch.randn(c["dim"], device=DEV, generator=gen) for _ in "qk")
    s["frequencies"] = torch.from_numpy(_frequencies(c)).to(DEV)


def prepare(case, seed):
    c, gen = case, torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": c}
    if c["op"] == "rotate":
        count = np.diff(np.linspace(0, c["tokens"], c["runs"] + 1).astype(np.int64))
        begin = torch.randint(0, c["far"], (c["runs"],), device=DEV, generator=gen)
        run = torch.repeat_interleave(torch.arange(c["runs"], device=DEV), torch.from_numpy(count).to(DEV), output_size=c["tokens"])
        first = torch.from_numpy(np.cumsum(count) - count).to(DEV)
        s["positions"] = (begin[run] + torch.arange(c["tokens"], device=DEV) - first[run]).to(torch.int32)
        _heads(s, c, c["tokens"], gen)
    elif c["op"] == "append":
        page = c["page"]
        lengths, new = _counts(c)
        need = [_slots(n, page) for n in lengths]
        s.update(_pool(c, sum(need) + 3, gen))
        s["table"], s["lengths"] = _scattered(need, sum(need) + 3, max(need), gen), _ints(lengths)
        s["start"], s["tokens"], s["max_new"] = _starts(new), sum(new), max(new)
        _heads(s, c, s["tokens"], gen)
        # the whole of every block that is written to comes back, in bf16 whatever the rows' type
        back = [n and length - (length - n) // page * page for length, n in zip(lengths, new)]
        s["back_start"], s["back_tokens"], s["back_max"] = _starts(back), sum(back), max(back)
        s["k_back"], s["v_back"] = (torch.zeros(s["back_tokens"], c["kv_heads"], c["dim"], dtype=torch.bfloat16, device=DEV) for _ in "kv")
    else:
        page = c["page"]
        each, prefix, tail, new = _groups(c)
        lone = c.get("lone", 0)
        group = np.repeat(np.arange(len(each)), each)
        before = np.concatenate([np.array(prefix)[group], np.zeros(lone, np.int64)])               # tokens that a sequence has from its group
        lengths = (before + np.array(tail)).tolist()
        common = [p // page for p in prefix]                                                      # pages that a group's sequences share
        if c["op"] == "shared":                                                                   # where they part is what is asked
            common = [int(n * x) for n, x in zip(common, torch.rand(len(common), device=DEV, generator=gen).tolist())]
        kept = np.concatenate([np.array(common)[group], np.zeros(lone, np.int64)]).astype(np.int64)
        need = [_slots(n, page) for n in lengths]
        own_need = (np.array(need) - kept).tolist()
        pages, slots = sum(common) + sum(own_need) + 3, max(need)
        both = _scattered(common + own_need, pages, max(max(common), max(own_need)), gen)
        s["table"] = torch.full((len(lengths), slots), -1, dtype=torch.int32, device=DEV)
        slot, kept_dev = torch.arange(slots, device=DEV), torch.from_numpy(kept).to(DEV)[:, None]
        lead = torch.from_numpy(np.concatenate([group, np.zeros(lone, np.int64)])).to(DEV)
        at = torch.where(slot < kept_dev, slot, slot - kept_dev).clamp(0, both.shape[1] - 1)
        s["table"] = torch.where(slot < kept_dev, both[lead[:, None], at], both[len(each) + torch.arange(len(lengths), device=DEV)[:, None], at])
        s["table"][slot >= _ints(need)[:, None]] = -1
        s["lengths"], s["first"] = _ints(lengths), _starts(each)
        s["shared"] = _ints([n * page for n in common])
        s["max_each"], s["max_shared"], s["pages"] = max(each), max(common) * page, pages
        if c["op"] == "attend":
            s.update(_pool(c, pages, gen))
            s["start"], s["tokens"], s["max_new"], s["max_len"] = _starts(new), sum(new), max(new), max(lengths)
            s["max_own"] = max(n - k * page for n, k in zip(lengths, kept.tolist()))
            s["q"] = (1.3 * torch.randn(s["tokens"], c["q_heads"], c["dim"], device=DEV, generator=gen)).to(TYPES[c["type"]])
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(s["tokens"], c["q_heads"], device=DEV)
        else:
            s["shared"] = torch.zeros(len(each), dtype=torch.int32, device=DEV)
    if own:                                                    # a program makes its descriptors once, beside its buffers
        s["call"] = _handle(s)
    return s


def _rotary(E, s):
    c = s["case"]
    kind = {"none": E.ENTRO_CONTEXT_AS_TRAINED, "linear": E.ENTRO_CONTEXT_LINEAR, "parts": E.ENTRO_CONTEXT_BY_PARTS}[c["scaling"]]
    turns = E.entro_rotary_turns(c["rotated"], c["base"], kind, factor=c["factor"], trained=c["trained"], low=1.0, high=4.0)
    norm = {"none": E.ENTRO_NORM_NONE, "rms": E.ENTRO_NORM_RMS, "centred": E.ENTRO_NORM_CENTRED}[c["norm"]]
    layout = {"halves": E.ENTRO_ROTARY_HALVES, "pairs": E.ENTRO_ROTARY_PAIRS}[c["layout"]]
    return E.Rotary(torch.from_numpy(turns.view(np.int64)).to(DEV), c["rotated"], layout, amplitude=_amplitude(c), norm=norm, eps=EPS, q_gain=s["q_gain"],
                    k_gain=s["k_gain"])


def _handle(s):
    """The descriptors and the workspace that a program keeps beside its buffers, as a function that makes the calls of a pass."""
    import paper_2505_02380_amd as E
    c = s["case"]
    if c["op"] == "rotate":
        rotary, q, k, positions = _rotary(E, s), E.RotaryRows(s["q"], s["q_out"]), E.RotaryRows(s["k_rows"], s["k_out"]), s["positions"]
        return lambda: E.entro_rotate(rotary, q, k, positions)
    if c["op"] == "append":
        cache, table = E.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], page_tokens=c["page"], head_dim=c["dim"]), E.CacheTable(s["table"], s["lengths"])
        rotary, q = _rotary(E, s), E.RotaryRows(s["q"], s["q_out"])
        rows = E.CacheRows(s["k_rows"], s["v_rows"], s["start"], max_new=s["max_new"])
        back = E.CacheRows(s["k_back"], s["v_back"], s["back_start"], max_new=s["back_max"])

        def write_and_read():
            E.entro_cache_append_rotated(cache, table, rows, rotary, q)
            E.entro_cache_read(cache, table, back)
        return write_and_read
    table, groups = E.CacheTable(s["table"], s["lengths"]), E.CacheGroups(s["first"], s["shared"], max_seqs=s["max_each"], max_shared=s["max_shared"])
    if c["op"] == "shared":
        cache = E.Cache.empty(1, s["pages"], 1, c["page"], 64, DEV)
        return lambda: E.entro_cache_shared(cache, table, groups)
    cache = E.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], page_tokens=c["page"], head_dim=c["dim"])
    query = E.CacheQuery(s["q"], s["out"], s["start"], lse=s["lse"], scale=_scale(c), window=c["window"], sinks=c["sinks"], max_new=s["max_new"],
                         max_len=s["max_len"])
    ws = torch.empty(max(16, E.entro_cache_attend_shared_workspace_bytes(cache, table, query, groups)), dtype=torch.uint8, device=DEV)
    return lambda: E.entro_cache_attend_shared(cache, table, query, groups, ws)


def _scale(c):
    return 1.0 / math.sqrt(c["dim"])


# ----------------------------------------------------------------------------------------------------------------- a pass
def run(state):
    s, op = state, state["case"]["op"]
    if own:
        s["call"]()
    else:
        {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend, "shared": _plain_shared}[op](s)
    if op == "rotate":
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if op == "attend":
        return {"out": s["out"], "lse": s["lse"]}
    return {"shared": s["shared"]}


def _rows_of(start, tokens):
    """(sequence, offset) of every row of a tensor of `tokens` rows."""
    row = torch.arange(tokens, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(start, row, right=True) - 1
    return seq, row - start[seq]


def _plain_turned(s, x, gain, positions):
    """Heads [tokens][heads][dim] normed and rotated, in 32 bits; angles in 64."""
    c, r = s["case"], s["case"]["rotated"]
    x = x.float()
    if c["norm"] == "rms":
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    elif c["norm"] == "centred":
        x = x - x.mean(-1, keepdim=True)
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    angle = positions.double()[:, None] * s["frequencies"]
    cos, sin = ((f(angle) * _amplitude(c)).float()[:, None] for f in (torch.cos, torch.sin))
    u, w = (x[..., : r // 2], x[..., r // 2: r]) if c["layout"] == "halves" else (x[..., 0:r:2], x[..., 1:r:2])
    u, w = u * cos - w * sin, w * cos + u * sin
    turned = torch.cat([u, w], -1) if c["layout"] == "halves" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_rotate(s):
    s["q_out"].copy_(_plain_turned(s, s["q"], s["q_gain"], s["positions"]))
    s["k_out"].copy_(_plain_turned(s, s["k_rows"], s["k_gain"], s["positions"]))


def _plain_blocks(x, old, s_old, is_new, is_old):
    """New codes and scales of blocks: x new values, old codes less 128, both [blocks, head, token, dim] in 32 bits."""
    s_old = torch.where(is_old.any(1)[:, None], s_old, 0.0)
    x = torch.where(is_new[:, None, :, None], x, 0.0)
    scale = torch.maximum(s_old, x.abs().amax((2, 3)) / 127)
    by = torch.where(scale > 0, scale, 1.0)[..., None, None]
    fresh = torch.round(x / by).clamp(-127, 127)
    kept = torch.round(old * s_old[..., None, None] / by)
    return torch.where(is_new[:, None, :, None], fresh, torch.where(is_old[:, None, :, None], kept, old)) + 128, scale


def _plain_append(s):
    c = s["case"]
    page, dim = c["page"], c["dim"]
    at, off = _rows_of(s["start"], s["tokens"])
    count = s["start"][1:] - s["start"][:-1]
    first = s["lengths"] - count                                                                        # position of the first new token
    s["q_out"].copy_(_plain_turned(s, s["q"], s["q_gain"], first[at] + off))
    k_new = _plain_turned(s, s["k_rows"], s["k_gain"], first[at] + off)
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
    k, ks = _plain_blocks(k_new[row].transpose(1, 2), k, s["k_scale"][0][pages], is_new, is_old)
    v, vs = _plain_blocks(s["v_rows"][row].float().transpose(1, 2), v, s["v_scale"][0][pages], is_new, is_old)
    s["k"][0, pages, :, :, :dim] = k.to(torch.uint8)
    s["v"][0, pages, :, :dim, :] = v.transpose(2, 3).to(torch.uint8)
    s["k_scale"][0, pages], s["v_scale"][0, pages] = ks, vs
    back, off = _rows_of(s["back_start"], s["back_tokens"])
    pos = (s["lengths"] - (s["back_start"][1:] - s["back_start"][:-1]))[back] + off
    pages, at = s["table"][back, torch.div(pos, page, rounding_mode="floor")].long(), torch.remainder(pos, page)
    s["k_back"].copy_((s["k"][0][pages, :, at, :dim].float() - 128) * s["k_scale"][0][pages][..., None])
    s["v_back"].copy_((s["v"][0][pages, :, :dim, at].float() - 128) * s["v_scale"][0][pages][..., None])


def _plain_part(c, s, q, here, pages, begin, until):
    """Attention of queries q [sets, rows, q_heads, dim] at positions `here` [sets, rows] over the tokens of `pages` [sets, slots], which begin at the
    positions `begin` [sets]; those from `until` [sets] on are left out. (weighted values less their weights' sum, lse) of each row and head."""
    page, dim, heads, groups = c["page"], c["dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    sets, rows, span = q.shape[0], q.shape[1], pages.shape[1] * page
    held = pages.clamp(min=0).long()
    k = (s["k"][0][held][..., :dim].float() - 128) * s["k_scale"][0][held][..., None, None]             # [set, slot, head, token, dim]
    k = k.permute(0, 2, 4, 1, 3).reshape(sets, heads, dim, span)
    q = q.float().view(sets, rows, heads, groups, dim).permute(0, 2, 3, 1, 4).reshape(sets, heads, groups * rows, dim)
    score = torch.matmul(q, k).mul_(_scale(c)).view(sets, heads, groups, rows, span)
    del k
    key = begin[:, None] + torch.arange(span, device=DEV)                                               # [set, span]
    seen = (key[:, None] <= here[..., None]) & (key < until[:, None])[:, None]
    if c["window"]:
        seen &= (here[..., None] - key[:, None] < c["window"]) | (key < c["sinks"])[:, None]
    seen &= (pages >= 0).repeat_interleave(page, 1)[:, None]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score.sub_(torch.where(torch.isfinite(top), top, 0.0)))
    total = p.sum(-1, keepdim=True)
    v = (s["v"][0][held][..., :dim, :].float() - 128) * s["v_scale"][0][held][..., None, None]          # [set, slot, head, dim, token]
    v = v.permute(0, 2, 1, 4, 3).reshape(sets, heads, span, dim)
    o = torch.matmul(p.view(sets, heads, groups * rows, span), v).view(sets, heads, groups, rows, dim) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)[..., 0]
    return o.permute(0, 3, 1, 2, 4).reshape(sets, rows, c["q_heads"], dim), lse.permute(0, 3, 1, 2).reshape(sets, rows, c["q_heads"])


def _plain_attend(s):
    """The tokens that a group shares against all its rows at once, every sequence's own tokens against its rows, and the two joined."""
    c, page = s["case"], s["case"]["page"]
    seq, off = _rows_of(s["start"], s["tokens"])
    count = s["start"][1:] - s["start"][:-1]
    here = (s["lengths"] - count)[seq] + off
    n_seqs, n_groups = s["table"].shape[0], s["first"].numel() - 1
    group = torch.searchsorted(s["first"], torch.arange(n_seqs, device=DEV, dtype=torch.int32), right=True) - 1
    in_group = group < n_groups
    shared = torch.where(in_group, s["shared"][group.clamp(max=n_groups - 1)], 0)                       # [seqs]
    # own tokens
    slot = torch.div(shared, page, rounding_mode="floor")[:, None] + torch.arange(_slots(s["max_own"], page), device=DEV)
    pages = torch.where(slot < s["table"].shape[1], s["table"].gather(1, slot.clamp(max=s["table"].shape[1] - 1).long()), -1)
    row = (s["start"][:-1, None] + torch.arange(s["max_new"], device=DEV)).clamp(max=s["tokens"] - 1)
    o, lse = _plain_part(c, s, s["q"][row], here[row], pages, shared, s["lengths"])
    o, lse = o[seq, off], lse[seq, off]
    if s["max_shared"]:
        # shared ones
        begin = s["start"][s["first"].long()]
        row = (begin[:-1, None] + torch.arange(s["max_each"] * s["max_new"], device=DEV)).clamp(max=s["tokens"] - 1)
        pages = s["table"][s["first"][:-1].long(), : s["max_shared"] // page]
        o1, lse1 = _plain_part(c, s, s["q"][row], here[row], pages, torch.zeros_like(s["shared"]), s["shared"])
        g = group[seq].clamp(max=n_groups - 1)
        at = (torch.arange(s["tokens"], device=DEV) - begin[g]).clamp(max=row.shape[1] - 1)
        o1, lse1 = o1[g, at], torch.where(in_group[seq][:, None], lse1[g, at], -math.inf)
        top = torch.maximum(lse, lse1)
        base = torch.where(torch.isfinite(top), top, 0.0)
        a, b = torch.exp(lse - base), torch.exp(lse1 - base)
        total = a + b
        some = torch.where(total > 0, total, 1.0)
        o = o * (a / some)[..., None] + torch.where(in_group[seq][:, None, None], o1, 0.0) * (b / some)[..., None]
        lse = torch.where(total > 0, base + torch.log(some), -math.inf)
    s["out"].copy_(o)
    s["lse"].copy_(lse)


def _plain_shared(s):
    page, table = s["case"]["page"], s["table"]
    group = torch.searchsorted(s["first"], torch.arange(table.shape[0], device=DEV, dtype=torch.int32), right=True) - 1
    lead = table[s["first"][:-1].long()]
    slot = torch.arange(table.shape[1], device=DEV)
    same = (table == lead[group]) & (table >= 0) & (slot < torch.div(s["lengths"], page, rounding_mode="floor")[:, None])
    run = torch.cumprod(same.to(torch.int32), 1, dtype=torch.int32).sum(1).to(torch.int32) * page
    s["shared"].fill_(2 ** 31 - 1).scatter_reduce_(0, group, run, "amin")


# ------------------------------------------------------------------------------------------------------------------ work
def _pairs(c, length, new):
    """Pairs of one of the last `new` tokens of a sequence and a token that it sees."""
    w, k = c["window"], c["sinks"]
    if not w:
        return new * length - new * (new - 1) // 2
    return sum(min(p + 1, w + min(k, max(0, p + 1 - w))) for p in range(length - new, length))


def _seen(c, first, last, lo, hi):
    """Tokens lo..hi-1 that some query at first..last sees."""
    hi = min(hi, last + 1)
    if not c["window"]:
        return max(0, hi - lo)
    a = max(lo, first - c["window"] + 1)
    return max(0, hi - a) + max(0, min(c["sinks"], hi, a) - lo)


def work(case):
    c = case
    if c["op"] == "rotate":
        n = c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["dim"]
        return {"bytes": 2.0 * n * (2 if c["type"] == "bf16" else 4), "flops": 6.0 * n}
    if c["op"] == "append":
        lengths, new = _counts(c)
        page, w, rows = c["page"], c["dim"], sum(new)
        size = 2 if c["type"] == "bf16" else 4
        blocks = sum(_slots(a, page) - (a - b) // page for a, b in zip(lengths, new) if b)
        back = sum(a - (a - b) // page * page for a, b in zip(lengths, new) if b)
        # query rows read and written, new rows of keys and values read once and written once in 8 bits; the blocks that they touch read and given back
        return {"bytes": 2.0 * rows * c["q_heads"] * w * size + 2.0 * c["kv_heads"] * (rows * w * (size + 1) + back * w * 3 + blocks * 8), "flops": 0}
    each, prefix, tail, new = _groups(c)
    lone = c.get("lone", 0)
    lengths = [t + p for t, p in zip(tail, [p for n, p in zip(each, prefix) for _ in range(n)] + [0] * lone)]
    if c["op"] == "shared":
        first = np.concatenate([[0], np.cumsum(each)])
        read = sum((p // c["page"] / 2 + 1) * n for p, n in zip(prefix, each))    # on average up to the middle
        return {"bytes": 4.0 * (read + len(lengths) + int(first[-1]) + 2 * len(each)), "flops": 0}
    page, w, size = c["page"], c["dim"], 2 if c["type"] == "bf16" else 4
    keys = b = 0
    for n, p in zip(each, prefix):
        mine = [i for i in range(b, b + n) if new[i]]
        if mine:
            keys += _seen(c, min(lengths[i] - new[i] for i in mine), max(lengths[i] for i in mine) - 1, 0, p // page * page)
            keys += sum(_seen(c, lengths[i] - new[i], lengths[i] - 1, p // page * page, lengths[i]) for i in mine)
        b += n
    keys += sum(_seen(c, lengths[i] - new[i], lengths[i] - 1, 0, lengths[i]) for i in range(b, b + lone) if new[i])
    pairs, rows = sum(_pairs(c, a, n) for a, n in zip(lengths, new)), sum(new) * c["q_heads"]
    return {"bytes": keys * c["kv_heads"] * 2 * (w + 4 / page) + rows * (2 * w * size + 4), "flops": 4.0 * pairs * c["q_heads"] * w}


# ----------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions in 64 bits, a sequence and a head at a time."""
    if case["op"] == "shared":
        return None
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "attend": _exact_attend}[case["op"]](s)


def _exact_heads(c, x, gain, positions, frequencies):
    """One complex number for each pair of a head, turned by the position's angle."""
    y = x.double()
    if c["norm"] != "none":
        if c["norm"] == "centred":
            y = y - y.sum(-1, keepdim=True) / c["dim"]
        y = gain.double() * y / torch.sqrt(y.square().sum(-1, keepdim=True) / c["dim"] + EPS)
    r = c["rotated"]
    at = torch.arange(r, device=DEV).view(2, -1) if c["layout"] == "halves" else torch.arange(r, device=DEV).view(-1, 2).T.contiguous()
    z = torch.complex(y[..., at[0]], y[..., at[1]])
    turn = torch.polar(torch.full((), _amplitude(c), dtype=torch.float64, device=DEV).expand(len(positions), r // 2).contiguous(),
                       torch.outer(positions.double(), frequencies))
    z = z * turn[:, None]
    y = y.clone()
    y[..., at[0]], y[..., at[1]] = z.real, z.imag
    return y


def _exact_rotate(s):
    c = s["case"]
    return {"q": _exact_heads(c, s["q"], s["q_gain"], s["positions"], s["frequencies"]),
            "k": _exact_heads(c, s["k_rows"], s["k_gain"], s["positions"], s["frequencies"])}


def _exact_values(s, b, first, last):
    """Keys and values of positions first..last-1 of sequence b: [tokens, head, dim]."""
    page, dim = s["case"]["page"], s["case"]["dim"]
    pos = torch.arange(first, last, device=DEV)
    p, t = s["table"][b][pos // page].long(), pos % page
    k = (s["k"][0][p, :, t, :dim].double() - 128) * s["k_scale"][0][p].double()[..., None]
    v = (s["v"][0][p, :, :dim, t].double() - 128) * s["v_scale"][0][p].double()[..., None]
    return k, v


def _exact_append(s):
    c = s["case"]
    page = c["page"]
    lengths, new = _counts(c)
    q, back = [], {"k": [], "v": []}
    scales = {"k": s["k_scale"].double(), "v": s["v_scale"].double()}
    row = 0
    for b in range(c["seqs"]):
        if not new[b]:
            continue
        begin = lengths[b] - new[b]
        head = begin // page * page
        positions = torch.arange(begin, lengths[b], device=DEV)
        q.append(_exact_heads(c, s["q"][row: row + new[b]], s["q_gain"], positions, s["frequencies"]))
        rows = {"k": _exact_heads(c, s["k_rows"][row: row + new[b]], s["k_gain"], positions, s["frequencies"]), "v": s["v_rows"][row: row + new[b]].double()}
        old = dict(zip("kv", _exact_values(s, b, head, begin)))
        pad = -(lengths[b] - head) % page
        pages = s["table"][b][head // page: _slots(lengths[b], page)].long()
        for x in "kv":
            fresh = rows[x]
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
    return {"q": torch.cat(q), "k": torch.cat(back["k"]), "v": torch.cat(back["v"]), "k_scale": scales["k"], "v_scale": scales["v"]}


def _exact_attend(s):
    c = s["case"]
    lengths, start = s["lengths"].tolist(), s["start"].tolist()
    per = c["q_heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for b, length in enumerate(lengths):
        n = start[b + 1] - start[b]
        if not n:
            continue
        k, v = _exact_values(s, b, 0, length)
        j, i = torch.arange(length, device=DEV), torch.arange(length - n, length, device=DEV)[:, None]
        ok = j[None] <= i
        if c["window"]:
            ok &= (i - j[None] < c["window"]) | (j[None] < c["sinks"])
        for g in range(c["kv_heads"]):
            heads = slice(g * per, (g + 1) * per)
            z = s["q"][start[b]: start[b + 1], heads].double().reshape(-1, c["dim"]) @ k[:, g].T.contiguous() * _scale(c)
            z = torch.where(ok.repeat_interleave(per, 0), z, -math.inf)
            out[start[b]: start[b + 1], heads] = (torch.softmax(z, -1) @ v[:, g].contiguous()).view(n, per, -1)
            lse[start[b]: start[b + 1], heads] = torch.logsumexp(z, -1).view(n, per)
    return {"out": out, "lse": lse}
