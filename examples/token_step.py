"""Token generation with one attention layer: entropy-coded weights and an 8-bit token cache, in beams.

Every step multiplies each beam's x with the compressed q, k and v matrices (one prepared launch for all beams), takes the next page
table (forks, one more token), writes k and v into the cache, attends, and multiplies the result with the compressed output matrix. Products
and attention hand each other bf16 rows in place.

    python examples/token_step.py [--layer mistral|smol] [--prompt 1000] [--beams 4] [--steps 32] [--window 0] [--sinks 0]
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2505_02380_amd as E
import synth

LAYERS = {"mistral": (4, 32, 8, 128), "smol": (2, 32, 32, 64)}      # weight set, query heads, key heads, dimensions


class Layer:
    """q, k, v and o of one layer as compressed tensors on the device, with prepared products for `beams` rows."""

    def __init__(self, cfg: int, beams: int, device="cuda:0"):
        specs = [s for s in synth.config_tensors(cfg, 1) if s.name in "qkvo"]
        self.tensors = {}
        for s in specs:
            w = torch.from_numpy(synth.make_tensor(s)).to(device)
            self.tensors[s.name] = E.compress_on_device(w, s.bits, s.scheme, synth.config_chunk_symbols(s.cfg), s.rows, s.cols, s.name)
        rows = {name: t.enc.rows for name, t in self.tensors.items()}
        new = lambda n: torch.zeros(beams, n, dtype=torch.bfloat16, device=device)  # noqa: E731
        self.x, self.q, self.k, self.v = new(self.tensors["q"].enc.cols), new(rows["q"]), new(rows["k"]), new(rows["v"])
        self.attended, self.y = new(self.tensors["o"].enc.cols), new(rows["o"])
        self.plans = [self._plan([(name, getattr(self, name)[b], self.x[b]) for b in range(beams) for name in "qkv"]),
                      self._plan([("o", self.y[b], self.attended[b]) for b in range(beams)])]

    def _plan(self, products):
        ts = [self.tensors[name].ctensor(out, x) for name, out, x in products]
        ws = torch.empty(max(16, E.entro_workspace_bytes(ts, E.ENTRO_OP_GEMV)), dtype=torch.uint8, device=self.x.device)
        return E.entro_plan_init(ts, E.ENTRO_OP_GEMV, E.ENTRO_BF16, ws), ws


class Generation:
    """Beams over one layer: the cache, its two tables (of this step and of the next), and the step."""

    def __init__(self, layer: Layer, heads: int, kv_heads: int, dim: int, beams: int, most_tokens: int, page: int = 64, window: int = 0,
                 sinks: int = 0):
        dev = layer.x.device
        slots = -(-most_tokens // page) + 1
        self.layer, self.window, self.sinks = layer, window, sinks
        self.cache = E.Cache.empty(1, slots * (beams + 1), kv_heads, page, dim, dev)
        self.tables = [E.CacheTable.empty(beams, slots, dev) for _ in range(2)]
        self.status = torch.zeros(4, dtype=torch.int32, device=dev)
        self.room = torch.empty(E.entro_cache_pages_workspace_bytes(self.cache, *self.tables), dtype=torch.uint8, device=dev)
        start = torch.arange(beams + 1, dtype=torch.int32, device=dev)
        rows = lambda x, n: x.view(beams, n, dim)  # noqa: E731
        self.rows = E.CacheRows(rows(layer.k, kv_heads), rows(layer.v, kv_heads), start, 1)
        self.query = E.CacheQuery(rows(layer.q, heads), rows(layer.attended, heads), start, 1, most_tokens, window=window, sinks=sinks)
        need = E.entro_cache_attend_workspace_bytes(self.cache, self.tables[0], self.query)
        self.attend_room = torch.empty(max(16, need), dtype=torch.uint8, device=dev)
        self.one = torch.ones(beams, dtype=torch.int32, device=dev)

    @property
    def table(self) -> E.CacheTable:
        return self.tables[0]

    def next_table(self, parent=None, grow=None):
        E.entro_cache_regroup(self.cache, self.tables[0], self.tables[1], self.status, self.room, parent=parent, grow=grow,
                              window=self.window, sinks=self.sinks)
        self.tables.reverse()

    def prompt(self, k, v):
        """The first beam's keys and values [tokens][kv_heads][dim]; step() with parents of 0 forks the others from it."""
        n, beams = k.shape[0], self.one.numel()
        grow = torch.zeros(beams, dtype=torch.int32, device=k.device)
        grow[0] = n
        self.next_table(grow=grow)
        start = torch.full((beams + 1,), n, dtype=torch.int32, device=k.device)
        start[0] = 0
        E.entro_cache_append(self.cache, self.table, E.CacheRows(k, v, start, n))

    def step(self, parent=None):
        """One token for every beam: y from x. parent: the beams that these go on from (None: themselves)."""
        E.entro_plan_run(self.layer.plans[0][0])
        self.next_table(parent=parent, grow=self.one)
        E.entro_cache_append(self.cache, self.table, self.rows)
        E.entro_cache_attend(self.cache, self.table, self.query, self.attend_room)
        E.entro_plan_run(self.layer.plans[1][0])
        return self.layer.y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layer", choices=sorted(LAYERS), default="mistral")
    for name, value in (("prompt", 1000), ("beams", 4), ("steps", 32), ("window", 0), ("sinks", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    cfg, heads, kv_heads, dim = LAYERS[a.layer]
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    layer = Layer(cfg, a.beams)
    g = Generation(layer, heads, kv_heads, dim, a.beams, a.prompt + a.steps, window=a.window, sinks=a.sinks)
    g.prompt(*(torch.randn(a.prompt, kv_heads, dim, device="cuda:0", generator=gen).to(torch.bfloat16) for _ in "kv"))
    layer.x.copy_(torch.randn(layer.x.shape, device="cuda:0", generator=gen))
    parent = torch.zeros(a.beams, dtype=torch.int32, device="cuda:0")
    g.step(parent)                                                      # every beam forks from the prompt
    torch.cuda.synchronize()
    began = time.perf_counter()
    for i in range(1, a.steps):
        layer.x.copy_(torch.nn.functional.layer_norm(layer.y.float(), layer.y.shape[1:]))
        parent.copy_(torch.randint(0, a.beams, (a.beams,), device="cuda:0", generator=gen, dtype=torch.int32))
        g.step(parent)
    torch.cuda.synchronize()
    took = (time.perf_counter() - began) / max(1, a.steps - 1)
    status = g.status.tolist()
    if E.entro_cache_status(status[0]) != 0:
        raise RuntimeError("the pool has no page left")
    print(f"{a.steps} steps of {a.beams} beams after {a.prompt} tokens: {took * 1e6:.0f} us a step; "
          f"{status[1]} pages in use, {status[2]} free, {g.table.lengths.tolist()} tokens")
    return g


if __name__ == "__main__":
    main()
