"""Adapted self-attention of a layer over the paged key-value cache: the calls of
``lora`` and ``kv`` in the order in which a serving step makes them.

For the rows of a step (Section 2.2: one row per decoding request, a segment
of rows per prompt), with x [n_rows, hidden]:

    q, k, v = x W + s_g (x A_g) B_g      each row with its request's adapter
    cache  <- k, v                       at the rows' positions
    a       = attention(q, cache)
    y       = a W_o + s_g (a A_g) B_g

Position encodings belong between the first two lines and are the caller's: a
model that rotates q and k does it on ``q`` and ``k`` between ``project`` and
``attend``.  Run as a command on a GPU, the module serves a small random stack
of layers (prompts, branches, decode steps in a HIP graph, a window's pages given
back, compaction) and prints what each part took.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Sequence

import numpy as np

from . import kv as KV
from . import lora as L


@dataclass
class Projection:
    """A base weight, transposed ([h_out, h_in], as a linear layer keeps it), and
    the table of its adapters."""
    table: int
    wt: object

    @property
    def shape(self):
        return int(self.wt.shape[1]), int(self.wt.shape[0])


@dataclass
class Layer:
    q: Projection
    k: Projection
    v: Projection
    o: Projection


def _ordered(stream, device):
    """A context in which tensors are made in the order of the stream's launches: they
    may not be filled on another stream, nor be memory that one still uses."""
    import torch
    handle = L._stream(stream)
    return torch.cuda.stream(torch.cuda.ExternalStream(handle, device) if handle else torch.cuda.default_stream(device))


class Step:
    """What the layers of one step share: segment s of the batch holds the last
    rows of sequence s, and every sequence has a segment (of length 0 if it has no rows).
    Creation allocates and waits for ``stream``; ``run`` only enqueues, and may be
    recorded in a HIP graph."""

    def __init__(self, layers: Sequence[Layer], cache: KV.Cache, seg_lens: Sequence[int], seg_adapter: Sequence[int],
                 n_heads: int, window: int = 0, n_sinks: int = 0, stream=None):
        import torch
        self.layers, self.cache, self.n_heads, self.window, self.n_sinks = list(layers), cache, n_heads, window, n_sinks
        head_dim = int(cache.k.shape[4])
        self.scale = head_dim ** -0.5
        self.width, self.kv_width = n_heads * head_dim, int(cache.k.shape[2]) * head_dim
        offset = np.concatenate([[0], np.cumsum(seg_lens)]).astype(np.int32)
        self.n_rows = int(offset[-1])
        self.n_segments = len(seg_lens)
        if len(seg_adapter) != self.n_segments or min(seg_lens, default=0) < 0:
            raise ValueError("seg_lens and seg_adapter: a length of at least 0 and an adapter for every segment are needed")
        for i, layer in enumerate(self.layers):
            want = (("q", layer.q, 1, self.width), ("k", layer.k, 1, self.kv_width), ("v", layer.v, 1, self.kv_width),
                    ("o", layer.o, 0, self.width))
            for name, p, side, n in want:
                if p.shape[side] != n:
                    raise ValueError(f"layer {i}: the {name} projection is {p.shape}, the heads take {n}")
        self.single = all(n == 1 for n in seg_lens)      # one row per sequence: the decode form
        self.batch = L.Batch(offset, np.asarray(seg_adapter, np.int32), self.n_rows)
        dev, dt = cache.k.device, cache.k.dtype
        with _ordered(stream, dev):
            self.seg_offset = torch.from_numpy(offset).to(dev)
            self.q = torch.empty((self.n_rows, self.width), dtype=dt, device=dev)
            self.k = torch.empty((self.n_rows, self.kv_width), dtype=dt, device=dev)
            self.v = torch.empty_like(self.k)
            self.a = torch.empty_like(self.q)
        self._plans, self._plan_of = [], {}              # plans with their shapes; a table's plan
        try:
            for layer in self.layers:
                for p in (layer.q, layer.k, layer.v, layer.o):
                    self._plan_for(p, stream)
        except Exception:
            self.release()
            raise

    def _plan_for(self, p: Projection, stream):
        """One plan serves all tables of a shape whose adapters agree in rank."""
        if p.table in self._plan_of:
            return
        for shape, plan in self._plans:
            if shape == p.shape and self._fits(plan, p):
                break
        else:
            plan = L.lora_base_plan_create(p.table, self.batch, stream)
            self._plans.append((p.shape, plan))
        self._plan_of[p.table] = plan

    @staticmethod
    def _fits(plan: int, p: Projection) -> bool:
        # (a call without operands enqueues nothing: it is refused for the table where that does not
        # fit the plan, for the missing x where it does; a plan of no rows takes it)
        try:
            L.lora_base_plan_apply(plan, p.table, None, p.shape[0], None, p.shape[0], None, p.shape[1])
        except L.LoraError as e:
            return e.code == L.LORA_E_ARG
        return True

    def _apply(self, p: Projection, x, y, stream):
        L.lora_base_plan_apply(self._plan_of[p.table], p.table, x, x.stride(0), p.wt, p.wt.stride(0), y, y.stride(0),
                               stream)

    def _check_seqs(self, seqs: KV.Seqs):
        # (the launches read an offset per sequence)
        if seqs.n_seqs != self.n_segments:
            raise ValueError(f"a step of {self.n_segments} segments with {seqs.n_seqs} sequences: one segment per sequence "
                             "is needed, of no rows where it has none")

    def _check_rows(self, name: str, t, width: int):
        # (the launches read or write n_rows rows of this width)
        if t.dim() != 2 or t.shape[0] < self.n_rows or t.shape[1] < width or t.dtype != self.q.dtype or \
                t.device != self.q.device or t.stride(1) != 1:
            raise ValueError(f"{name}: a {self.q.dtype} tensor of [{self.n_rows}, {width}] or more on {self.q.device}, dense "
                             f"in the last dimension, is needed, not {t.dtype} {tuple(t.shape)} on {t.device}")

    def project(self, layer: int, x, stream=None) -> None:
        """q, k and v of the step's rows, into ``self.q``, ``self.k`` and ``self.v``."""
        w = self.layers[layer]
        self._check_rows("x", x, w.q.shape[0])
        for p, y in ((w.q, self.q), (w.k, self.k), (w.v, self.v)):
            self._apply(p, x, y, stream)

    def attend(self, attn: int, layer: int, seqs: KV.Seqs, y, stream=None) -> None:
        """The rows' keys and values into the cache, attention, the o projection."""
        self._check_seqs(seqs)
        self._check_rows("y", y, self.layers[layer].o.shape[1])
        one = self.single
        KV.lora_kv_append(self.cache, layer, seqs, None if one else self.seg_offset, self.n_rows, self.k,
                          self.kv_width, self.v, self.kv_width, stream)
        rows = (self.n_heads, self.q, self.width, self.a, self.width, self.scale, self.window, self.n_sinks, stream)
        if one:
            KV.lora_attn_decode(attn, self.cache, layer, seqs, *rows)
        else:
            KV.lora_attn_prompt(attn, self.cache, layer, seqs, self.seg_offset, self.n_rows, *rows)
        self._apply(self.layers[layer].o, self.a, y, stream)

    def run(self, attn: int, seqs: KV.Seqs, x, y, stream=None) -> None:
        """Every layer: the first reads x, the others what the one before wrote to y."""
        self._check_seqs(seqs)
        if self.layers:
            self._check_rows("y", y, self.layers[0].o.shape[1])
        for i in range(len(self.layers)):
            self.project(i, x if i == 0 else y, stream)
            self.attend(attn, i, seqs, y, stream)

    def release(self) -> None:
        """Frees the plans: no launch, recorded or enqueued, may still use them."""
        for _, plan in self._plans:
            L.lora_base_plan_destroy(plan)
        self._plans, self._plan_of = [], {}


class Server:
    """The sequences of a cache: pages, lengths, and the steps that use them.

    ``grow`` comes before each step: ``seqs``, which the step is run with, has the sequences
    that it gave their tokens (``step_lens``).  The others have no row in that step: nothing
    of theirs is stored, and attention gives their rows zeros.  No sequence grows past
    ``max_len`` tokens, whether or not its last page has room for more."""

    def __init__(self, cache: KV.Cache, n_seqs: int, max_len: int, stream=None):
        import torch
        dev = cache.k.device
        n_pages, page_rows = int(cache.k.shape[1]), int(cache.k.shape[3])
        ld = -(-max_len // page_rows)
        self.cache, self.stream, self.max_len = cache, stream, max_len
        i32 = dict(dtype=torch.int32, device=dev)
        with _ordered(stream, dev):
            self.tables = torch.full((n_seqs, ld), -1, **i32)
            self.lens = torch.zeros(n_seqs, **i32)
            self.step_lens = torch.zeros(n_seqs, **i32)
            self.refs = torch.zeros(n_pages, **i32)
            self.info = torch.zeros(2, **i32)
            self.book = KV.Book(self.tables, self.lens, self.refs, page_rows)
            self.seqs = KV.Seqs(self.tables, self.step_lens, max_len)
            self.ws_bytes = KV.lora_kv_workspace_bytes(self.book)
            self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self.attn = KV.lora_attn_create(dev.index or 0, stream)

    def grow(self, add) -> None:
        """``add``: int32 device tensor [n_seqs], the step's rows of each sequence.  ``info``
        then holds (pages taken, sequences that did not fit), ``step_lens`` 0 for those and
        for those without rows; to be read on the server's stream, which the host then waits for."""
        KV.lora_kv_grow_step(self.book, add, self.max_len, self.step_lens, self.info, self.ws, self.ws_bytes,
                             self.stream)

    def fork(self, parents, children) -> None:
        """Between a step and the next ``grow``: the children have no rows before it."""
        KV.lora_kv_fork_step(self.cache, self.book, parents, children, self.step_lens, self.info, self.ws,
                             self.ws_bytes, self.stream)

    def free(self, seqs) -> None:
        KV.lora_kv_free(self.book, seqs, self.stream)

    def trim(self, window: int, n_sinks: int = 0) -> None:
        """Between a step and the next ``grow``, which moves the window's end."""
        KV.lora_kv_trim(self.book, window, n_sinks, self.stream)

    def compact(self) -> None:
        KV.lora_kv_compact(self.cache, self.book, self.tables, self.refs, self.info, self.ws, self.ws_bytes,
                           self.stream)

    def release(self) -> None:
        KV.lora_attn_destroy(self.attn)
        self.attn = 0


def random_layers(n_layers: int, hidden: int, n_heads: int, n_kv_heads: int, head_dim: int, dtype, ranks, device,
                  seed: int = 0, stream=None):
    """Layers of random weights and adapters (scales 16 / r), and the tensors that
    the tables point at (keep them while the tables live)."""
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def draw(*shape):
        return (torch.randn(shape, generator=gen, device=device) * shape[-1] ** -0.5).to(dtype)

    code = L.LORA_F16 if dtype == torch.float16 else L.LORA_BF16
    index = torch.device(device).index or 0
    kept = []

    def projection(h_in, h_out):
        wt = draw(h_out, h_in)
        A = [draw(r, h_in).t().contiguous() for r in ranks]
        B = [(draw(h_out, r) * 0.25).t().contiguous() for r in ranks]
        scales = [16.0 / r for r in ranks]
        torch.cuda.synchronize(device)
        table = L.lora_register_adapters(index, h_in, h_out, code, [a.data_ptr() for a in A],
                                         [b.data_ptr() for b in B], ranks, scales, stream)
        kept.append((A, B, scales))
        return Projection(table, wt)

    w, kw = n_heads * head_dim, n_kv_heads * head_dim
    layers = [Layer(projection(hidden, w), projection(hidden, kw), projection(hidden, kw), projection(w, hidden))
              for _ in range(n_layers)]
    return layers, kept


def main() -> None:
    import time

    import torch
    dev, dt = torch.device("cuda:0"), torch.bfloat16
    n_layers, hidden, heads, kv_heads, dim = 4, 4096, 32, 32, 128
    window, sinks, max_len, n_seqs = 256, 16, 1536, 24
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        layers, kept = random_layers(n_layers, hidden, heads, kv_heads, dim, dt, [8, 16, 32, 64], dev, stream=st)
        shape = (n_layers, n_seqs * max_len // 16, kv_heads, 16, dim)
        cache = KV.Cache(torch.zeros(shape, dtype=dt, device=dev), torch.zeros(shape, dtype=dt, device=dev))
        srv = Server(cache, n_seqs, max_len, st)
        prompts = [203, 512, 64, 1000, 17, 300, 128, 700] + [0] * (n_seqs - 8)
        adapters = [s % 4 for s in range(n_seqs)]

        def timed(what, f, n=1):
            st.synchronize()
            t0 = time.perf_counter()
            f()
            st.synchronize()
            print(f"{what}: {1e3 * (time.perf_counter() - t0) / n:.3f} ms", flush=True)

        step = Step(layers, cache, prompts, adapters, heads, window, sinks, st)
        x = torch.randn((step.n_rows, hidden), device=dev).to(dt)
        y = torch.empty_like(x)
        add = torch.tensor(prompts, dtype=torch.int32, device=dev)
        srv.grow(add)
        timed(f"{step.n_rows} prompt rows, {n_layers} layers", lambda: step.run(srv.attn, srv.seqs, x, y, st))

        timed("8 prompts, each branched twice", lambda: srv.fork([s for s in range(8) for _ in range(2)],
                                                                 list(range(8, 24))))
        decode = Step(layers, cache, [1] * n_seqs, adapters, heads, window, sinks, st)
        dx = torch.randn((n_seqs, hidden), device=dev).to(dt)
        dy = torch.empty_like(dx)
        ones = torch.ones(n_seqs, dtype=torch.int32, device=dev)

        def token():
            srv.grow(ones)
            decode.run(srv.attn, srv.seqs, dx, dy, st)

        token()
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            token()
        timed(f"a token of {n_seqs} sequences, {n_layers} layers", lambda: [graph.replay() for _ in range(100)], 100)
        timed("pages behind the window given back", lambda: srv.trim(window, sinks))
        srv.free(list(range(0, n_seqs, 3)))
        timed("compaction", srv.compact)
        print("pages in use, pages moved:", srv.info.tolist(), "of", shape[1], flush=True)
        timed("a token after compaction", graph.replay)
        st.synchronize()
        del graph
        step.release()
        decode.release()
        srv.release()
        for layer in layers:
            for p in (layer.q, layer.k, layer.v, layer.o):
                L.lora_release_adapters(p.table)
    del kept


if __name__ == "__main__":
    main()
