"""The paged key-value cache and its attention, as cases that can be timed and
checked: what a step of continuous batching does beside the adapted projections.

A case is a dict of plain values.  ``op`` names the operator:

  "decode"   attention of one new token per sequence over its pages
  "prompt"   attention of prompt segments, the last rows of their sequences
  "append"   the rows' keys and values into the cache
  "fork"     sequences branch: full pages shared, last pages copied
  "compact"  pages in use move to the lowest ids, tables rewritten

  dtype, heads, kv_heads, head_dim, page_rows   "f16" / "bf16", q heads, cache heads, width, tokens per page
  layers     layers of the cache (attention and append run on one of them, the last)
  order      "head" pages of [kv_heads, page_rows, head_dim], "row" pages of [page_rows, kv_heads, head_dim]
  seqs, len_lo, len_hi   sequences and the range of their lengths (logarithmically uniform)
  rows       rows per sequence: 1, or 0 for whole prompts, or a chunk at the end of each sequence
  window, sinks   tokens a row sees behind itself (0 for all), first tokens that stay visible
  children   fork: children of every sequence
  spare      pages in use by nobody, as a share of those in use
  batch      seed of lengths and tables

Keys, values and queries are normal, queries times 1.5 so that rows attend
unevenly; pages are handed out in random order, as after some time of service.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

TORCH_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}


def _case(op, dtype, heads, kv_heads, head_dim, page_rows, *, layers=1, order="head", seqs=1, len_lo=1, len_hi=1,
          rows=1, window=0, sinks=0, children=0, spare=0.05, batch=0, name=None):
    c = dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page_rows=page_rows,
             layers=layers, order=order, seqs=seqs, len_lo=len_lo, len_hi=len_hi, rows=rows, window=window,
             sinks=sinks, children=children, spare=spare, batch=batch)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One request alone on a 4096-wide model with 32 heads: latency counts.
        _case("decode", "f16", 32, 32, 128, 16, layers=2, seqs=1, len_lo=300, len_hi=300, name="decode_one_300"),
        # A 13B-shaped decode batch (40 heads of their own keys), prompt lengths of a chat service.
        _case("decode", "bf16", 40, 40, 128, 16, seqs=128, len_lo=64, len_hi=1024, batch=3, name="decode_13b_t128"),
        # The decode rows of a 70B-shaped step (8 heads share keys), lengths from short to long.
        _case("decode", "bf16", 64, 8, 128, 64, seqs=256, len_lo=64, len_hi=8192, batch=4, name="decode_70b_t256"),
        # Long conversations that see a window and the first tokens, on one shard of four.
        _case("decode", "f16", 16, 2, 128, 32, seqs=8, len_lo=20000, len_hi=100000, window=4096, sinks=4, batch=5,
              name="decode_window_tp4"),
        # One short prompt, as it arrives beside decoding requests.
        _case("prompt", "f16", 32, 32, 128, 16, seqs=1, len_lo=203, len_hi=203, rows=0, name="prompt_one_203"),
        # Sixteen prompts of a prompt step, 4096 wide.
        _case("prompt", "bf16", 32, 32, 128, 16, seqs=16, len_lo=256, len_hi=1024, rows=0, batch=2,
              name="prompt_16seg"),
        # A 2048-token chunk of a long 70B-shaped prompt behind what is cached already.
        _case("prompt", "bf16", 64, 8, 128, 64, seqs=1, len_lo=16384, len_hi=16384, rows=2048,
              name="prompt_chunk_70b"),
        # Prompts under a window with sinks, narrow heads, rows stored across heads.
        _case("prompt", "f16", 24, 8, 64, 32, order="row", seqs=4, len_lo=2500, len_hi=6000, rows=0, window=1024,
              sinks=16, batch=6, name="prompt_window_d64"),
        # The new token's keys and values of every decoding request.
        _case("append", "bf16", 64, 8, 128, 64, layers=2, seqs=256, len_lo=64, len_hi=400, batch=4,
              name="append_decode_t256"),
        # Those of a whole prompt step.
        _case("append", "bf16", 32, 32, 128, 16, seqs=16, len_lo=256, len_hi=1024, rows=0, batch=2,
              name="append_16seg"),
        # Sixteen requests branch into three more each (sampled answers from one prompt), every layer's tail copied.
        _case("fork", "bf16", 64, 8, 128, 32, layers=16, seqs=16, len_lo=100, len_hi=1500, children=3, spare=0.5,
              batch=7, name="fork_16x3"),
        # A cache with holes after requests have ended: the pages in use gathered at the front.
        _case("compact", "bf16", 64, 8, 128, 16, layers=16, seqs=48, len_lo=33, len_hi=700, spare=0.7, batch=8,
              name="compact_48"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng: random.Random):
    """One more case of the listed ones' ranges."""
    while True:
        op = rng.choice(("decode", "decode", "decode", "prompt", "prompt", "prompt", "append", "fork", "compact"))
        head_dim = rng.choice((64, 128, 128, 128, 80, 96, 256))
        kv_heads, group = rng.choice(((32, 1), (40, 1), (8, 8), (2, 8), (8, 3), (8, 4), (1, 16), (4, 7), (1, 20)))
        c = dict(dtype=rng.choice(("f16", "bf16")), head_dim=head_dim, kv_heads=kv_heads, heads=kv_heads * group,
                 page_rows=rng.choice((16, 16, 32, 64, 128, 256)), order=rng.choice(("head", "head", "row")),
                 batch=rng.randrange(1 << 20))
        window = rng.choice((0, 0, _log_int(rng, 17, 8192)))
        sinks = rng.choice((0, 4, _log_int(rng, 1, 200))) if window else 0
        if op == "decode":
            lo = _log_int(rng, 1, 20000)
            c.update(seqs=_log_int(rng, 1, 256), len_lo=lo, len_hi=lo + _log_int(rng, 1, 100000 - lo),
                     window=window, sinks=sinks, layers=rng.choice((1, 2)))
        elif op == "prompt":
            lo = _log_int(rng, 1, 8192)
            c.update(seqs=_log_int(rng, 1, 16), len_lo=lo, len_hi=lo + _log_int(rng, 1, 8192),
                     rows=rng.choice((0, 0, _log_int(rng, 2, 2048))), window=window, sinks=sinks)
        elif op == "append":
            lo = _log_int(rng, 1, 1024)
            c.update(seqs=_log_int(rng, 1, 256), len_lo=lo, len_hi=lo + _log_int(rng, 1, 1024),
                     rows=rng.choice((0, 1, _log_int(rng, 2, 512))), layers=rng.choice((1, 2)))
        else:
            lo = _log_int(rng, 1, 512)
            c.update(seqs=_log_int(rng, 1, 48), len_lo=lo, len_hi=lo + _log_int(rng, 1, 1024),
                     layers=_log_int(rng, 1, 16), spare=rng.uniform(0.3, 1.0),
                     children=_log_int(rng, 1, 4) if op == "fork" else 0)
        case = _case(op, **c)
        w = work(case)
        pool = _plan(case)["n_pages"] * case["layers"] * _page_elements(case) * 4
        if w["bytes"] <= 1.7e9 and w["flops"] <= 1.0e12 and pool <= 4e9 and (op in ("decode", "prompt") or pool <= 1.5e9):
            return case


# ---------------------------------------------------------------------------
# lengths, tables and work of a case
# ---------------------------------------------------------------------------

def _page_elements(case):
    return case["kv_heads"] * case["page_rows"] * case["head_dim"]


def _plan(case):
    """Lengths, rows and tables of the case: the same for every seed."""
    rng = np.random.default_rng(case["batch"])
    n, pr = case["seqs"], case["page_rows"]
    lens = np.exp(rng.uniform(np.log(case["len_lo"]), np.log(case["len_hi"] + 0.49), size=n)).round().astype(np.int64)
    lens = lens.clip(case["len_lo"], case["len_hi"])
    rows = lens if case["rows"] == 0 else np.minimum(lens, case["rows"])
    pages = -(-lens // pr)
    used = int(pages.sum())
    n_child = n * case["children"]
    n_pages = used + int(used * case["spare"]) + n_child + 1
    ids = rng.permutation(n_pages)[:used].astype(np.int32)
    ld = int(pages.max()) + 1
    tables = np.full((n + n_child, ld), -1, dtype=np.int32)
    at = 0
    for s in range(n):
        tables[s, :pages[s]] = ids[at:at + pages[s]]
        at += pages[s]
    refs = np.zeros(n_pages, dtype=np.int32)
    refs[ids] = 1
    all_lens = np.zeros(n + n_child, dtype=np.int64)
    all_lens[:n] = lens
    parents = np.repeat(np.arange(n, dtype=np.int32), case["children"])
    return dict(lens=lens, rows=rows, pages=pages, n_pages=n_pages, ld=ld, tables=tables, refs=refs,
                all_lens=all_lens, parents=parents, children=n + np.arange(n_child, dtype=np.int32))


def _visible(pos, window, sinks):
    """How many tokens the rows at positions ``pos`` see."""
    seen = pos + 1
    if window:
        first = np.maximum(0, pos + 1 - window)
        seen = np.minimum(seen, window) + np.minimum(first, sinks)
    return seen


def work(case):
    """Every key and value that some row sees read once, queries read and outputs
    written once, 4 head_dim operations for each visible pair and head; the
    bytes of the rows or pages moved, read and written, and of the tables."""
    p = _plan(case)
    d, h, kvh = case["head_dim"], case["heads"], case["kv_heads"]
    win, sinks = case["window"], case["sinks"]
    row = 2 * 2 * kvh * d                      # a token's key and value, all heads, bytes
    if case["op"] in ("decode", "prompt"):
        rows = np.ones_like(p["rows"]) if case["op"] == "decode" else p["rows"]
        tokens = pairs = 0
        for ln, q in zip(p["lens"], rows):
            pos = np.arange(ln - q, ln)
            pairs += int(_visible(pos, win, sinks).sum())
            first = int(max(0, ln - q + 1 - win)) if win else 0
            tokens += int(ln) - first + min(first, sinks if win else 0)
        return {"bytes": tokens * row + 2 * 2 * int(rows.sum()) * h * d + 4 * int(p["pages"].sum()),
                "flops": 4 * d * h * pairs}
    if case["op"] == "append":
        return {"bytes": 2 * int(p["rows"].sum()) * row, "flops": 0}
    if case["op"] == "fork":
        tail = int((p["lens"] % case["page_rows"]).sum()) * case["children"]
        tables = 4 * 2 * int(p["pages"].sum()) * case["children"]
        return {"bytes": 2 * tail * row * case["layers"] + tables + 4 * p["n_pages"], "flops": 0}
    live = p["refs"] > 0
    moved = int(live[int(live.sum()):].sum())
    return {"bytes": 2 * moved * case["page_rows"] * row * case["layers"] + 8 * p["tables"].size + 8 * p["n_pages"],
            "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _cache(case, p, gen):
    shape = [case["layers"], p["n_pages"], case["kv_heads"], case["page_rows"], case["head_dim"]]
    if case["order"] == "row":
        shape[2], shape[3] = shape[3], shape[2]
    out = []
    for _ in range(2):
        t = torch.empty(shape, dtype=TORCH_DTYPE[case["dtype"]], device="cuda:0")
        for layer in t:
            layer.copy_(torch.randn(shape[1:], generator=gen, device="cuda:0", dtype=torch.float32))
        out.append(t.transpose(2, 3) if case["order"] == "row" else t)
    return out                                  # [layers, pages, heads, rows, dim] views


class _State:
    """Inputs on the GPU, and what a program keeps from step to step."""

    def __init__(self, case, seed):
        self.case, self.op = case, case["op"]
        p = self.plan = _plan(case)
        dev = torch.device("cuda:0")
        dtype = TORCH_DTYPE[case["dtype"]]
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)
        self.layer = case["layers"] - 1
        self.k, self.v = _cache(case, p, gen)
        i32 = dict(dtype=torch.int32, device=dev)
        self.tables = torch.tensor(p["tables"], **i32)
        self.lens = torch.tensor(p["all_lens"], **i32)
        self.refs = torch.tensor(p["refs"], **i32)
        self.scale = case["head_dim"] ** -0.5
        rows = np.ones_like(p["rows"]) if self.op == "decode" else p["rows"]
        off = np.concatenate([[0], np.cumsum(rows)])
        self.offset, self.n_rows = [int(v) for v in off], int(off[-1])
        self.seq_lens = [int(v) for v in p["lens"]]
        self.seg_offset = torch.tensor(off, **i32)

        def normal(shape, std=1.0):
            return (torch.randn(shape, generator=gen, device=dev, dtype=torch.float32) * std).to(dtype)

        if self.op in ("decode", "prompt"):
            self.q = normal((self.n_rows, case["heads"] * case["head_dim"]), 1.5)
            self.out = torch.zeros_like(self.q)
        elif self.op == "append":
            self.k_new = normal((self.n_rows, case["kv_heads"] * case["head_dim"]))
            self.v_new = normal((self.n_rows, case["kv_heads"] * case["head_dim"]))
        elif self.op == "fork":
            self.parents = torch.tensor(p["parents"], dtype=torch.int64, device=dev)
            self.children = torch.tensor(p["children"], dtype=torch.int64, device=dev)
        else:
            self.tables_out = torch.empty_like(self.tables)
            self.refs_out = torch.empty_like(self.refs)
        self.attn = 0
        if own:
            from paper_2401_11240_amd import kv as KV
            self.KV = KV
            self.stream = torch.cuda.current_stream()
            self.cache = KV.Cache(self.k, self.v)
            self.seqs = KV.Seqs(self.tables, self.lens, max(self.seq_lens))
            if self.op in ("decode", "prompt"):
                self.attn = KV.lora_attn_create(0, self.stream)
            elif self.op in ("fork", "compact"):
                self.book = KV.Book(self.tables, self.lens, self.refs, case["page_rows"])
                n = KV.lora_kv_workspace_bytes(self.book)
                self.ws = torch.empty(n, dtype=torch.uint8, device=dev)
                self.info = torch.zeros(2, **i32)

    def __del__(self):
        try:
            if self.attn:
                torch.cuda.synchronize()
                self.KV.lora_attn_destroy(self.attn)
        except Exception:
            pass


def prepare(case, seed):
    return _State(case, seed)


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    KV, c = s.KV, s.case
    if s.op == "decode":
        KV.lora_attn_decode(s.attn, s.cache, s.layer, s.seqs, c["heads"], s.q, s.q.shape[1], s.out, s.out.shape[1],
                            s.scale, c["window"], c["sinks"], s.stream)
        return s.out
    if s.op == "prompt":
        KV.lora_attn_prompt(s.attn, s.cache, s.layer, s.seqs, s.seg_offset, s.n_rows, c["heads"], s.q, s.q.shape[1],
                            s.out, s.out.shape[1], s.scale, c["window"], c["sinks"], s.stream)
        return s.out
    if s.op == "append":
        KV.lora_kv_append(s.cache, s.layer, s.seqs, None if c["rows"] == 1 else s.seg_offset, s.n_rows,
                          s.k_new, s.k_new.shape[1], s.v_new, s.v_new.shape[1], s.stream)
        return [s.k, s.v]
    if s.op == "fork":
        KV.lora_kv_fork(s.cache, s.book, s.plan["parents"], s.plan["children"], s.info, s.ws, s.ws.numel(), s.stream)
        return [s.k, s.v, s.tables, s.lens, s.refs]
    KV.lora_kv_compact(s.cache, s.book, s.tables_out, s.refs_out, s.info, s.ws, s.ws.numel(), s.stream)
    return [s.k, s.v, s.tables_out, s.refs_out]


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _tokens(s, seq, first, last, sinks):
    """Tokens of a sequence that rows from position ``first`` see up to ``last``, and where they lie."""
    win = s.case["window"]
    lo = max(0, first + 1 - win) if win else 0
    j = torch.arange(lo, last + 1, device=s.k.device)
    if lo and sinks:
        j = torch.cat([torch.arange(min(lo, sinks), device=s.k.device), j])
    page = s.tables[seq].long()[j // s.case["page_rows"]]
    return j, page, j % s.case["page_rows"]


def _attend(s, seq, q, first):
    """q [rows, heads, dim] at positions first, first + 1, ... of a sequence; float32 throughout."""
    c = s.case
    rows, group = q.shape[0], c["heads"] // c["kv_heads"]
    j, page, slot = _tokens(s, seq, first, first + rows - 1, c["sinks"])
    k = s.k[s.layer][page, :, slot].float()     # [tokens, kv_heads, dim]
    v = s.v[s.layer][page, :, slot].float()
    qg = q.float().view(rows, c["kv_heads"], group, -1).permute(1, 2, 0, 3).reshape(c["kv_heads"], group * rows, -1)
    w = torch.matmul(qg, k.permute(1, 2, 0).contiguous()) * s.scale
    if rows > 1:
        p = (first + torch.arange(rows, device=j.device)).repeat(group)[:, None]
        seen = j[None, :] <= p
        if c["window"]:
            seen &= (j[None, :] > p - c["window"]) | (j[None, :] < c["sinks"])
        w = w.masked_fill_(~seen, float("-inf"))
    w = torch.exp(w - w.amax(-1, keepdim=True))
    o = torch.matmul(w, v.transpose(0, 1).contiguous()) / w.sum(-1, keepdim=True)
    return o.view(c["kv_heads"], group, rows, -1).permute(2, 0, 1, 3).reshape(rows, -1)


def _run_plain(s):
    c = s.case
    if s.op in ("decode", "prompt"):
        q = s.q.view(s.n_rows, c["heads"], c["head_dim"])
        for seq, ln in enumerate(s.seq_lens):
            lo, hi = s.offset[seq], s.offset[seq + 1]
            step = max(1, (1 << 28) // (c["heads"] * ln))      # scores of a part stay near 1 GB
            for r in range(lo, hi, step):
                e = min(hi, r + step)
                s.out[r:e] = _attend(s, seq, q[r:e], ln - (hi - r)).to(s.out.dtype)
        return s.out
    if s.op == "append":
        rows = s.seg_offset[1:] - s.seg_offset[:-1]
        n_seq = len(s.seq_lens)
        seq = torch.repeat_interleave(torch.arange(n_seq, device=s.k.device), rows.long(), output_size=s.n_rows)
        pos = s.lens.long()[seq] - s.seg_offset[1:].long()[seq] + torch.arange(s.n_rows, device=s.k.device)
        page = s.tables[seq, pos // c["page_rows"]].long()
        slot = pos % c["page_rows"]
        s.k[s.layer][page, :, slot] = s.k_new.view(s.n_rows, c["kv_heads"], -1)
        s.v[s.layer][page, :, slot] = s.v_new.view(s.n_rows, c["kv_heads"], -1)
        return [s.k, s.v]
    if s.op == "fork":
        return _fork_plain(s)
    live = s.refs > 0
    n_live = live.sum()
    ids = torch.arange(s.refs.numel(), device=s.k.device)
    src = torch.nonzero(live & (ids >= n_live)).flatten()
    dst = torch.nonzero(~live & (ids < n_live)).flatten()
    to = torch.where(live, ids, -1)
    to[src] = dst
    s.refs_out.copy_(torch.where(ids < n_live, s.refs, 0))
    s.refs_out[dst] = s.refs[src]
    n_held = (s.lens + c["page_rows"] - 1) // c["page_rows"]
    held = torch.arange(s.tables.shape[1], device=s.k.device)[None, :] < n_held[:, None]
    s.tables_out.copy_(torch.where(held & (s.tables >= 0), to[s.tables.clamp(min=0).long()], -1))
    for t in (s.k, s.v):
        t[:, dst] = t[:, src]
    return [s.k, s.v, s.tables_out, s.refs_out]


def _fork_plain(s):
    pr = s.case["page_rows"]
    entry = torch.arange(s.tables.shape[1], device=s.k.device)[None, :]
    # what the children held is released
    old = s.tables[s.children]
    held = (entry < ((s.lens[s.children] + pr - 1) // pr)[:, None]) & (old >= 0)
    s.refs.index_add_(0, old.clamp(min=0).long().flatten(), -held.flatten().int())
    # the lowest free pages go to the pairs with a partly filled last page
    ln = s.lens[s.parents]
    tail = ln % pr
    order = torch.cumsum((tail > 0).int(), 0)
    free = torch.cumsum((s.refs == 0).int(), 0)
    fresh = torch.searchsorted(free, order)
    rows = s.tables[s.parents]
    full = (ln // pr)[:, None]
    shared = (entry < full) & (rows >= 0)
    s.refs.index_add_(0, rows.clamp(min=0).long().flatten(), shared.flatten().int())
    own_page = (entry == full) & (tail > 0)[:, None]
    new = torch.where(shared, rows, torch.where(own_page, fresh[:, None].int(), -1))
    s.tables[s.children] = new.to(torch.int32)
    s.lens[s.children] = ln
    pair = torch.nonzero(tail > 0).flatten()
    src = rows[pair].gather(1, full[pair].long()).flatten().long()
    dst = fresh[pair]
    s.refs[dst] = 1
    used = (torch.arange(pr, device=s.k.device)[None, :] < tail[pair][:, None])[None, :, None, :, None]
    for t in (s.k, s.v):
        t[:, dst] = torch.where(used, t[:, src], t[:, dst])
    return [s.k, s.v, s.tables, s.lens, s.refs]


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    """Attention of every row and head by its definition; None for what only moves bits."""
    if case["op"] not in ("decode", "prompt"):
        return None
    p = _plan(case)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    k, v = _cache(case, p, gen)
    rows = np.ones_like(p["rows"]) if case["op"] == "decode" else p["rows"]
    heads, d = case["heads"], case["head_dim"]
    group = heads // case["kv_heads"]
    q = (torch.randn((int(rows.sum()), heads * d), generator=gen, device="cuda:0", dtype=torch.float32) * 1.5)
    q = q.to(TORCH_DTYPE[case["dtype"]]).double().view(-1, heads, d)
    out = torch.zeros_like(q)
    at = 0
    for seq, (ln, n) in enumerate(zip(p["lens"].tolist(), rows.tolist())):
        pages = torch.from_numpy(p["tables"][seq, :int(p["pages"][seq])].astype(np.int64)).to(k.device)
        # [kv_heads, tokens, dim], tokens in order
        ks, vs = (t[case["layers"] - 1][pages].transpose(0, 1).reshape(case["kv_heads"], -1, d)[:, :ln] for t in (k, v))
        for lo in range(0, n, 1024):
            hi = min(n, lo + 1024)
            pos = torch.arange(ln - n + lo, ln - n + hi, device=k.device)[:, None]
            j = torch.arange(ln, device=k.device)[None, :]
            hidden = j > pos
            if case["window"]:
                hidden |= (j <= pos - case["window"]) & (j >= case["sinks"])
            first = 0
            if case["window"] and not case["sinks"]:
                first = max(0, ln - n + lo + 1 - case["window"])
            hidden = hidden[:, first:]
            for kh in range(case["kv_heads"]):
                kd, vd = ks[kh, first:].double(), vs[kh, first:].double()
                for h in range(kh * group, (kh + 1) * group):
                    score = (q[at + lo:at + hi, h] @ kd.t()) / math.sqrt(d)
                    score[hidden] = -math.inf
                    prob = torch.softmax(score, dim=1)
                    out[at + lo:at + hi, h] = prob @ vd
        at += n
    return out.view(-1, heads * d)
