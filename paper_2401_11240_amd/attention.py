"""Adapted self-attention of a layer over the paged key-value cache: the calls of
``lora``, ``kv``, ``mx`` and ``sample`` in the order in which a serving step makes them.

For the rows of a step (Section 2.2: one row per decoding request, a segment
of rows per prompt), with x [n_rows, hidden]:

    q, k, v = x W + s_g (x A_g) B_g      each row with its request's adapter
    cache  <- k, v                       at the rows' positions
    a       = attention(q, cache)
    y       = a W_o + s_g (a A_g) B_g

Position encodings belong between the first two lines and are the caller's: a
model that rotates q and k does it on ``q`` and ``k`` between ``project`` and
``attend``.

A layer may have a norm in front of it, whose weight it holds; a step of such layers keeps
the sum of its input and of what the layers gave (``total``), and a layer reads

    total  += what the layer before gave       (in 16 bits)
    h       = norm(total)

as its x.  A base weight may be in 4-bit blocks (``mx.Rows``).  Then x goes into 8-bit blocks for it,
y is rounded to 16 bits once behind the product and once behind the adapters' delta, which reads the
16-bit x.  A ``Head`` behind the last layer leads from a sequence's last row to its next token.

Run as a command on a GPU, the module serves two small random stacks of layers, of 16-bit weights
(prompts, branches, decode steps in a HIP graph, a window's pages given back, compaction) and of
4-bit weights with norms and a head (prompts, tokens in a HIP graph), and prints what each part took.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Sequence

import numpy as np

from . import kv as KV
from . import lora as L
from . import mx as MX
from . import sample as SA


@dataclass
class Projection:
    """A base weight, transposed ([h_out, h_in], as a linear layer keeps it; a tensor, or
    ``mx.Rows`` of 4-bit blocks), and the table of its adapters."""
    table: int
    wt: object

    @property
    def in_blocks(self):
        return isinstance(self.wt, MX.Rows)

    @property
    def shape(self):
        if self.in_blocks:
            return self.wt.h, self.wt.n_rows
        return int(self.wt.shape[1]), int(self.wt.shape[0])


@dataclass
class Layer:
    """``norm``: the weight [hidden] of the norm in front of q, k and v, or None for no norm."""
    q: Projection
    k: Projection
    v: Projection
    o: Projection
    norm: object = None


@dataclass
class Head:
    """The last norm's weight [hidden] and the weight of the vocabulary, ``mx.Rows`` of 4-bit
    blocks [n_vocab, hidden].  ``n_vocab``: the tokens, where the weight has more rows than those (the product
    takes a multiple of 8)."""
    norm: object
    wt: MX.Rows
    n_vocab: int = 0

    def __post_init__(self):
        self.n_vocab = self.n_vocab or self.wt.n_rows
        if not 0 < self.n_vocab <= self.wt.n_rows:
            raise ValueError(f"n_vocab is {self.n_vocab}, the weight has {self.wt.n_rows} rows")


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
                 n_heads: int, window: int = 0, n_sinks: int = 0, stream=None, head: Head = None, eps: float = 1e-5):
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
        self.head, self.eps = head, eps
        self.normed = any(layer.norm is not None for layer in self.layers)
        if any((layer.norm is not None) != self.normed for layer in self.layers) or (head and not self.normed):
            raise ValueError("a norm in front of every layer or of none is needed, and of every one with a head")
        self.single = all(n == 1 for n in seg_lens)      # one row per sequence: the decode form
        self.batch = L.Batch(offset, np.asarray(seg_adapter, np.int32), self.n_rows)
        dev, dt = cache.k.device, cache.k.dtype
        with _ordered(stream, dev):
            self.seg_offset = torch.from_numpy(offset).to(dev)
            self.q = torch.empty((self.n_rows, self.width), dtype=dt, device=dev)
            self.k = torch.empty((self.n_rows, self.kv_width), dtype=dt, device=dev)
            self.v = torch.empty_like(self.k)
            self.a = torch.empty_like(self.q)
            self._make_blocks(seg_lens)
        # plans with what they serve; the plan of a table behind weights of one kind (the same adapters may be behind
        # weights of both), or of three tables behind weights in blocks
        self._plans, self._plan_of = [], {}
        try:
            for layer in self.layers:
                one = self._plan_for_three(layer, stream)
                for p in (layer.o,) if one else (layer.q, layer.k, layer.v, layer.o):
                    self._plan_for(p, stream)
        except Exception:
            self.release()
            raise

    def _make_blocks(self, seg_lens):
        """What norms, weights in blocks and a head need beside q, k, v and a."""
        import torch
        dev, dt = self.q.device, self.q.dtype
        self.code = L.LORA_F16 if dt == torch.float16 else L.LORA_BF16
        self.hidden = self.layers[0].q.shape[0] if self.layers else 0
        self.total = self.h = self.hq = self.aq = self.last = None
        for i, layer in enumerate(self.layers):
            if self.normed and (layer.q.shape[0] != self.hidden or layer.o.shape[1] != self.hidden):
                raise ValueError(f"layer {i}: norms need layers of one width, {self.hidden}")
            if self.normed:
                self._check_weight(f"layer {i}", layer.norm)
            for p in (layer.q, layer.k, layer.v, layer.o):
                if p.in_blocks and (p.wt.fmt != MX.LORA_E2M1 or p.wt.device != dev):
                    raise ValueError(f"layer {i}: weights in blocks are LORA_E2M1, on {dev}")
        if self.normed:
            self.total = torch.empty((self.n_rows, self.hidden), dtype=dt, device=dev)
            self.h = torch.empty_like(self.total)
        need = [0]
        rows = {}
        for layer in self.layers:
            for p, name in ((layer.q, "hq"), (layer.k, "hq"), (layer.v, "hq"), (layer.o, "aq")):
                if p.in_blocks:
                    key = name, p.shape[0]
                    if key not in rows:
                        rows[key] = MX.empty_rows(self.n_rows, p.shape[0], MX.LORA_E4M3, dev)
                    need.append(MX.lora_mx_workspace_bytes(rows[key], p.wt))
        self._rows = rows                                # x and a in blocks, by width
        if self.head:
            self._check_weight("head", self.head.norm)
            wt, n = self.head.wt, self.n_segments
            if wt.fmt != MX.LORA_E2M1 or wt.device != dev or wt.h != self.hidden:
                raise ValueError(f"head: a weight in LORA_E2M1 blocks of {self.hidden} on {dev} is needed")
            ends = np.cumsum(seg_lens) - 1
            self.empty = torch.from_numpy(np.asarray(seg_lens) == 0).to(dev) if min(seg_lens, default=1) == 0 else None
            # (a segment of no rows takes some other row, and no token)
            self.last = None if self.single else torch.from_numpy(np.maximum(ends, 0).astype(np.int64)).to(dev)
            self.last_rows = [torch.zeros((n, self.hidden), dtype=dt, device=dev) for _ in range(2)]
            self.last_q = MX.empty_rows(n, self.hidden, MX.LORA_E4M3, dev)
            self.logits = torch.empty((n, wt.n_rows), dtype=torch.float32, device=dev)
            need.append(MX.lora_mx_workspace_bytes(self.last_q, wt))
            need.append(SA.lora_sample_workspace_bytes(n, self.head.n_vocab, SA.LORA_F32))
        self.ws_bytes = max(need)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)

    def _check_weight(self, what: str, w):
        if w.shape != (self.hidden,) or w.dtype != self.q.dtype or w.device != self.q.device or not w.is_contiguous():
            raise ValueError(f"{what}: a norm's weight is {self.q.dtype} [{self.hidden}] on {self.q.device}, contiguous")

    def _plan_for(self, p: Projection, stream):
        """One plan serves all tables of a shape and kind of weight whose adapters agree in rank."""
        if (p.table, p.in_blocks) in self._plan_of:
            return
        for kind, plan in self._plans:
            if kind == (p.shape, p.in_blocks) and self._fits(plan, p):
                break
        else:
            plan = (L.lora_plan_create if p.in_blocks else L.lora_base_plan_create)(p.table, self.batch, stream)
            self._plans.append(((p.shape, p.in_blocks), plan))
        self._plan_of[p.table, p.in_blocks] = plan

    def _plan_for_three(self, layer: Layer, stream) -> bool:
        """One plan, and one launch, for the deltas of q, k and v behind weights in blocks (a token of 24 sequences, 4
        layers of 4096: 551 us with three, 465 with one).  False where their adapters differ in rank."""
        three = (layer.q, layer.k, layer.v)
        tables = tuple(p.table for p in three)
        if not all(p.in_blocks for p in three):
            return False
        if tables in self._plan_of:
            return True
        kind = tuple(p.shape for p in three)
        for k, plan in self._plans:
            if k == kind and L.lora_plan_fits(plan, tables):
                break
        else:
            try:
                plan = L.lora_plan_create_multi(tables, self.batch, stream)
            except L.LoraError as e:
                if e.code in (L.LORA_E_RANK, L.LORA_E_SHAPE, L.LORA_E_INDEX):
                    return False                         # (what is wrong with the batch itself, a plan for one says too)
                raise
            self._plans.append((kind, plan))
        self._plan_of[tables] = plan
        return True

    @staticmethod
    def _fits(plan: int, p: Projection) -> bool:
        return L.lora_plan_fits(plan, (p.table,)) if p.in_blocks else L.lora_base_plan_fits(plan, p.table)

    def _apply(self, p: Projection, x, y, stream, rows=None, delta=True):
        """``rows``: x in blocks, for a weight in blocks; ``delta``: with the adapters' (there)."""
        plan = self._plan_of.get((p.table, p.in_blocks))
        if p.in_blocks:
            MX.lora_mx_apply(rows, p.wt, y, y.stride(0), self.code, self.ws, self.ws_bytes, stream)
            if self.n_rows and delta:                  # (without rows x and y have no memory, which the call refuses)
                L.lora_plan_apply(plan, p.table, x, x.stride(0), y, y.stride(0), stream)
        else:
            L.lora_base_plan_apply(plan, p.table, x, x.stride(0), p.wt, p.wt.stride(0), y, y.stride(0), stream)

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
        """q, k and v of the step's rows, into ``self.q``, ``self.k`` and ``self.v``.  With norms x
        begins ``total`` at layer 0 and is added to it at the others."""
        w = self.layers[layer]
        self._check_rows("x", x, w.q.shape[0])
        if self.normed:
            rows = self._rows.get(("hq", self.hidden)) if any(p.in_blocks for p in (w.q, w.k, w.v)) else None
            MX.lora_norm(x, x.stride(0), self.total if layer else None, self.hidden, w.norm, self.eps, self.n_rows, self.hidden,
                         self.code, self.total, self.hidden, self.h, self.hidden, rows, stream)
            x = self.h
        done = {self.hidden} if self.normed else set()   # widths of x that are in blocks already
        three = (w.q, w.k, w.v)
        tables = tuple(p.table for p in three)
        # the plan of the three deltas in one launch (a 16-bit weight's own launch adds its delta)
        together = self._plan_of.get(tables) if all(p.in_blocks for p in three) else None
        for p, y in zip(three, (self.q, self.k, self.v)):
            rows = self._rows.get(("hq", p.shape[0])) if p.in_blocks else None
            if rows is not None and p.shape[0] not in done:
                MX.lora_mx_quantize(x, x.stride(0), self.code, rows, stream)
                done.add(p.shape[0])
            self._apply(p, x, y, stream, rows, together is None)
        if together is not None and self.n_rows:
            ys = (self.q, self.k, self.v)
            L.lora_plan_apply_multi(together, tables, x, x.stride(0), ys, [y.stride(0) for y in ys], stream)

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
        o = self.layers[layer].o
        rows = self._rows[("aq", self.width)] if o.in_blocks else None
        if rows is not None:
            MX.lora_mx_quantize(self.a, self.width, self.code, rows, stream)
        self._apply(o, self.a, y, stream, rows)

    def run(self, attn: int, seqs: KV.Seqs, x, y, stream=None) -> None:
        """Every layer: the first reads x, the others what the one before wrote to y (which with norms they add
        to ``total``; the last one's is left to the head)."""
        self._check_seqs(seqs)
        if self.layers:
            self._check_rows("y", y, self.layers[0].o.shape[1])
        for i in range(len(self.layers)):
            self.project(i, x if i == 0 else y, stream)
            self.attend(attn, i, seqs, y, stream)

    def choose(self, y, params, u, tokens, probs=None, stream=None) -> None:
        """The next token of every sequence from its last row of ``total`` + y, y what ``run`` left: ``tokens``
        (int32 [n_segments]) and, unless None, ``probs``; -1 and 0 for a segment of no rows.  (Only the device
        knows which sequences did not fit, ``Server.step_lens`` is 0 for those: their tokens mean nothing.)
        ``params`` (``sample.Params`` or None) and ``u`` as ``lora_sample`` takes them."""
        import torch
        head, n, v = self.head, self.n_segments, self.head.wt.n_rows if self.head else 0
        if head is None:
            raise ValueError("a step without a head has no tokens")
        self._check_rows("y", y, self.hidden)
        x, total, ldy = y, self.total, y.stride(0)
        if self.last is not None and self.n_rows:
            with _ordered(stream, self.q.device):
                for src, dst in ((y[:, :self.hidden], self.last_rows[0]), (self.total, self.last_rows[1])):
                    torch.index_select(src, 0, self.last, out=dst)
        if self.last is not None:
            (x, total), ldy = self.last_rows, self.hidden
        MX.lora_norm(x, ldy, total, self.hidden, head.norm, self.eps, n, self.hidden, self.code, None, 0, None, 0, self.last_q,
                     stream)
        MX.lora_mx_apply(self.last_q, head.wt, self.logits, v, MX.LORA_F32, self.ws, self.ws_bytes, stream)
        SA.lora_sample(self.logits, v, SA.LORA_F32, n, head.n_vocab, params, u, tokens, probs, self.ws, self.ws_bytes, stream)
        if self.empty is not None:
            with _ordered(stream, self.q.device):
                tokens[:n].masked_fill_(self.empty, -1)
                if probs is not None:
                    probs[:n].masked_fill_(self.empty, 0.)

    def release(self) -> None:
        """Frees the plans: no launch, recorded or enqueued, may still use them."""
        for kind, plan in self._plans:
            (L.lora_base_plan_destroy if kind[-1] is False else L.lora_plan_destroy)(plan)
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
                  seed: int = 0, stream=None, in_blocks: bool = False):
    """Layers of random weights and adapters (scales 16 / r), and the tensors that
    the tables point at (keep them while the tables live).  ``in_blocks``: weights in 4-bit
    blocks, and a norm in front of every layer."""
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def draw(*shape):
        return (torch.randn(shape, generator=gen, device=device) * shape[-1] ** -0.5).to(dtype)

    code = L.LORA_F16 if dtype == torch.float16 else L.LORA_BF16
    index = torch.device(device).index or 0
    kept = []

    def projection(h_in, h_out):
        wt = in_4_bits(draw(h_out, h_in)) if in_blocks else draw(h_out, h_in)
        A = [draw(r, h_in).t().contiguous() for r in ranks]
        B = [(draw(h_out, r) * 0.25).t().contiguous() for r in ranks]
        scales = [16.0 / r for r in ranks]
        torch.cuda.synchronize(device)
        table = L.lora_register_adapters(index, h_in, h_out, code, [a.data_ptr() for a in A],
                                         [b.data_ptr() for b in B], ranks, scales, stream)
        kept.append((A, B, scales))
        return Projection(table, wt)

    w, kw = n_heads * head_dim, n_kv_heads * head_dim
    layers = [Layer(projection(hidden, w), projection(hidden, kw), projection(hidden, kw), projection(w, hidden),
                    1 + draw(hidden) if in_blocks else None)
              for _ in range(n_layers)]
    return layers, kept


def in_4_bits(wt) -> MX.Rows:
    """A 16-bit device tensor [h_out, h_in] in 4-bit blocks, on torch's current stream."""
    import torch
    code = L.LORA_F16 if wt.dtype == torch.float16 else L.LORA_BF16
    rows = MX.empty_rows(wt.shape[0], wt.shape[1], MX.LORA_E2M1, wt.device)
    MX.lora_mx_quantize(wt, wt.stride(0) if wt.shape[0] > 1 else wt.shape[1], code, rows, torch.cuda.current_stream(wt.device))
    return rows


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

        # weights in 4 bits, norms, and every sequence's token the input of its next step
        n_vocab, max_new = 32000, 100
        layers, kept = random_layers(n_layers, hidden, heads, kv_heads, dim, dt, [8, 16, 32, 64], dev, 1, st, in_blocks=True)
        embed = torch.randn((n_vocab, hidden), device=dev).to(dt)
        head = Head(torch.ones(hidden, device=dev, dtype=dt), in_4_bits((torch.randn_like(embed) * hidden ** -0.5).to(dt)))
        prompts = [203, 512, 64, 1000, 17, 300, 128, 700] * 3
        shape = (n_layers, sum((p + max_new + 16) // 16 + 1 for p in prompts), kv_heads, 16, dim)
        cache = KV.Cache(torch.zeros(shape, dtype=dt, device=dev), torch.zeros(shape, dtype=dt, device=dev))
        srv = Server(cache, n_seqs, max_len, st)
        tokens = torch.zeros(n_seqs, dtype=torch.int32, device=dev)
        chosen = torch.zeros((max_new + 2, n_seqs), dtype=torch.int32, device=dev)
        at = torch.zeros(1, dtype=torch.int64, device=dev)
        u = torch.rand(chosen.shape, device=dev)
        params = SA.Params(torch.full((n_seqs,), 0.8, device=dev), None, torch.full((n_seqs,), 0.95, device=dev))
        uu = torch.empty(n_seqs, device=dev)

        def choose(s, y):
            uu.copy_(torch.index_select(u, 0, at)[0])
            s.choose(y, params, uu, tokens, None, st)
            chosen.index_copy_(0, at, tokens[None])
            at.add_(1)

        step = Step(layers, cache, prompts, adapters, heads, window, sinks, st, head)
        x = torch.index_select(embed, 0, torch.randint(n_vocab, (step.n_rows,), device=dev))
        y = torch.empty_like(x)
        srv.grow(torch.tensor(prompts, dtype=torch.int32, device=dev))

        def first():
            step.run(srv.attn, srv.seqs, x, y, st)
            choose(step, y)

        first()                                          # (once untimed: code and memory are there from then on)
        at.zero_()
        timed(f"4-bit weights: {step.n_rows} prompt rows to {n_seqs} tokens, {n_layers} layers", first)
        decode = Step(layers, cache, [1] * n_seqs, adapters, heads, window, sinks, st, head)

        def token():
            srv.grow(ones)
            torch.index_select(embed, 0, tokens, out=dx)
            decode.run(srv.attn, srv.seqs, dx, dy, st)
            choose(decode, dy)

        token()
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            token()
        timed(f"4-bit weights: a token of {n_seqs} sequences, {n_layers} layers, {n_vocab} logits",
              lambda: [graph.replay() for _ in range(max_new)], max_new)
        print("sequence 0:", chosen[:8, 0].tolist(), "...", flush=True)
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
