"""Steps in which not every sequence has a row: sequences that found no page or no
room in their table, and sequences that pause.  What they hold, and what others share with
them, stays as it is bit for bit; the rows of the others are stored and attend as always."""
import numpy as np
import pytest

import kv_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2401_11240_amd import attention as T  # noqa: E402
from paper_2401_11240_amd import kv as KV  # noqa: E402
from paper_2401_11240_amd import lora as L  # noqa: E402

DEV = torch.device("cuda:0")
HIDDEN, HEADS, KV_HEADS, DIM, LAYERS, PR = 128, 4, 2, 32, 2, 16


def f64(t):
    return t.double().cpu().numpy()


class Stack:
    """A server of n_pages pages and its book in Python lists."""

    def __init__(self, n_seqs, n_pages, max_len, dtype=torch.bfloat16):
        self.n_seqs, self.max_len, self.dtype = n_seqs, max_len, dtype
        self.st = torch.cuda.current_stream(DEV)
        self.layers, self.kept = T.random_layers(LAYERS, HIDDEN, HEADS, KV_HEADS, DIM, dtype, [4, 8], DEV, 3, self.st)
        self.gen = torch.Generator().manual_seed(n_pages)
        shape = (LAYERS, n_pages, KV_HEADS, PR, DIM)
        self.k, self.v = (torch.randn(shape, generator=self.gen).to(dtype).to(DEV) for _ in range(2))
        self.srv = T.Server(KV.Cache(self.k, self.v), n_seqs, max_len, self.st)
        ld = self.srv.tables.shape[1]
        self.ref = R.Book([[-1] * ld for _ in range(n_seqs)], [0] * n_seqs, n_pages, PR)
        self.steps = {}

    def step(self, rows):
        if tuple(rows) not in self.steps:
            self.steps[tuple(rows)] = T.Step(self.layers, self.srv.cache, rows, [s % 2 for s in range(self.n_seqs)], HEADS,
                                             stream=self.st)
        return self.steps[tuple(rows)]

    def x(self, n):
        return torch.randn((n, HIDDEN), generator=self.gen).to(self.dtype).to(DEV)

    def grown(self, add):
        """The Python book grown: info, and which sequences have their rows."""
        before = list(self.ref.lens)
        past = len(self.ref.t[0]) * PR + 1       # (the list book knows the table's end alone)
        info = self.ref.grow([past if a > 0 and n + a > self.max_len else a for n, a in zip(before, add)])
        return info, [b > a for a, b in zip(before, self.ref.lens)]

    def token(self, add, rows, launch=None):
        """grow(add) and a step of these rows; launch() does both from a recorded graph."""
        step, n = self.step(rows), sum(rows)
        before = self.k.clone(), self.v.clone()
        if launch is None:
            self.srv.grow(torch.tensor(add, dtype=torch.int32, device=DEV))
            step.run(self.srv.attn, self.srv.seqs, self.x(n), torch.empty((n, HIDDEN), dtype=self.dtype, device=DEV),
                     self.st)
        else:
            launch()
        torch.cuda.synchronize()
        info, has = self.grown(add)
        assert self.srv.info.tolist() == info
        assert self.srv.lens.tolist() == self.ref.lens and self.srv.refs.tolist() == self.ref.refs
        table = self.srv.tables.cpu().numpy()
        k, v = f64(self.k[-1]), f64(self.v[-1])
        newk, newv = (t.view(-1, KV_HEADS, DIM) for t in (step.k, step.v))
        written = torch.zeros((before[0].shape[1], PR), dtype=torch.bool)
        q, a, at = f64(step.q).reshape(-1, HEADS, DIM), f64(step.a).reshape(-1, HEADS, DIM), 0
        for s, r in enumerate(rows):
            if not has[s]:
                assert (a[at:at + r] == 0).all(), (s, "rows of a sequence that got nothing")
            else:
                first = self.ref.lens[s] - r
                for i in range(r):
                    page, row = int(table[s, (first + i) // PR]), (first + i) % PR
                    assert self.ref.refs[page] == 1
                    assert torch.equal(self.k[-1, page, :, row], newk[at + i])
                    assert torch.equal(self.v[-1, page, :, row], newv[at + i])
                    written[page, row] = True
                o, m, reach = R.attention(q[at:at + r], k, v, table[s], self.ref.lens[s], first, step.scale, 0, 0)
                tol = R.allowance(o, m, reach, DIM, self.ref.lens[s], self.dtype == torch.bfloat16)
                assert (np.abs(a[at:at + r] - o) <= tol).all(), s
            at += r
        keep = ~written.to(DEV)[None, :, None, :, None].expand_as(self.k)
        for t, b in zip((self.k, self.v), before):
            assert torch.equal(t[keep].view(torch.int16), b[keep].view(torch.int16)), "a token that is no row's was changed"
        return has

    def close(self):
        torch.cuda.synchronize()
        for s in self.steps.values():
            s.release()
        self.srv.release()
        for layer in self.layers:
            for p in (layer.q, layer.k, layer.v, layer.o):
                L.lora_release_adapters(p.table)


@pytest.fixture
def stack(request):
    s = Stack(*request.param)
    yield s
    s.close()


@pytest.mark.parametrize("stack", [(4, 3, 64)], indirect=True)
@pytest.mark.parametrize("recorded", [False, True])
def test_forked_sequences_without_a_page_for_their_token(stack, recorded):
    # 32 tokens in two full pages that three sequences share, and one page for three tokens
    s, st = stack, stack.st
    assert s.token([32, 0, 0, 0], [32, 0, 0, 0])[0]
    s.srv.fork([0, 0], [1, 2])
    s.ref.fork([0, 0], [1, 2])
    rows = [1] * 4
    launch = None
    if recorded:
        step, x, y = s.step(rows), s.x(4), torch.empty((4, HIDDEN), dtype=s.dtype, device=DEV)
        add = torch.zeros(4, dtype=torch.int32, device=DEV)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        s.srv.stream = side
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.srv.grow(add)
            step.run(s.srv.attn, s.srv.seqs, x, y, side)
        s.srv.stream = st

    def token(a):
        def replay():
            add.copy_(torch.tensor(a, dtype=torch.int32))
            x.copy_(s.x(4))
            torch.cuda.synchronize()
            graph.replay()
        return s.token(a, rows, replay if recorded else launch)

    for _ in range(3):
        assert token([1, 1, 1, 0]) == [True, False, False, False]
    assert token([0, 1, 0, 1]) == [False] * 4        # one pauses, one has no page, one is empty and gets none
    s.srv.free([0])
    s.ref.free([0])
    assert token([0, 1, 1, 0]) == [False, True, False, False]
    assert token([1, 1, 1, 0]) == [False, True, False, False]
    if recorded:
        del graph


@pytest.mark.parametrize("stack", [(3, 12, 48)], indirect=True)
def test_full_tables_and_chunks_without_room(stack):
    s = stack
    assert s.token([40, 32, 5], [40, 32, 5]) == [True] * 3
    assert s.token([9, 7, 0], [9, 7, 0]) == [False, True, False]       # 49 tokens do not fit a table of 48
    assert s.token([8, 0, 20], [8, 0, 20]) == [True, False, True]
    assert s.token([1, 9, 1], [1, 9, 1]) == [False, True, True]
    assert s.token([1, 1, 1], [1, 1, 1]) == [False, False, True]       # the first two are at 48
    assert s.token([0, 0, 0], [1, 1, 1]) == [False] * 3


@pytest.mark.parametrize("stack", [(3, 40, 100), (3, 40, 33)], indirect=True)
def test_the_longest_length_ends_inside_a_page(stack):
    s, m = stack, stack.max_len
    assert s.token([m - 3, m, 7], [m - 3, m, 7]) == [True] * 3
    for i in range(5):
        assert s.token([1, 1, 1], [1, 1, 1]) == [i < 3, False, True], i
    assert s.token([1, 1, 9], [4, 2, 9]) == [False, False, True]         # chunks
    assert s.token([1, 1, m - 20], [4, 2, m - 20]) == [False, False, False]
    assert s.token([0, 0, m - 21], [1, 1, m - 21]) == [False, False, True]
    assert s.srv.lens.tolist() == [m] * 3


@pytest.mark.parametrize("stack", [(4, 9, 64)], indirect=True)
def test_a_child_has_no_row_before_it_grows(stack):
    # the children were in the step before the fork, with lengths of their own
    s = stack
    assert s.token([32, 20, 3, 0], [32, 20, 3, 0]) == [True, True, True, False]
    s.srv.fork([0, 0], [1, 2])
    s.ref.fork([0, 0], [1, 2])
    before = s.k.clone(), s.v.clone()
    assert s.srv.step_lens.tolist()[1:3] == [0, 0]
    assert s.token([1, 1, 1, 1], [1] * 4) == [True] * 4
    pages = s.srv.tables[0, :2].tolist()
    for t, b in zip((s.k, s.v), before):
        assert torch.equal(t[:, pages].view(torch.int16), b[:, pages].view(torch.int16))


def test_grow_step_against_the_book():
    n, n_pages = 1300, 700
    i32 = dict(dtype=torch.int32, device=DEV)
    tables, lens, refs = torch.full((n, 6), -1, **i32), torch.zeros(n, **i32), torch.zeros(n_pages, **i32)
    step_lens, info = torch.full((n,), -3, **i32), torch.zeros(2, **i32)
    book = KV.Book(tables, lens, refs, PR)
    nb = KV.lora_kv_workspace_bytes(book)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    ref = R.Book(tables.tolist(), [0] * n, n_pages, PR)
    rng = np.random.default_rng(4)
    for rep in range(5):
        add = [int(x) for x in rng.choice([0, 1, 1, 5, 16, 40, -3, 100], size=n)]
        before = list(ref.lens)
        KV.lora_kv_grow_step(book, torch.tensor(add, **i32), 6 * PR, step_lens, info, ws, nb,
                             torch.cuda.current_stream())
        assert info.tolist() == ref.grow(add)
        assert lens.tolist() == ref.lens and refs.tolist() == ref.refs
        assert step_lens.tolist() == [b if b > a else 0 for a, b in zip(before, ref.lens)], rep


@pytest.mark.parametrize("n_pages,kids", [(100, 120), (30, 200), (3, 239), (70, 600)])
def test_more_children_than_pages(n_pages, kids):
    # one short parent whose last page every child wants a copy of, and one of a full page
    from test_gpu_kv import Pages
    for rep in range(4):
        p = Pages(kids + 2, 2, n_pages, PR, [5, 16], seed=rep)
        children = [int(c) for c in np.random.default_rng(rep).permutation(np.arange(2, kids + 2))]
        parents = [int(i % 7 == 3) for i in range(kids)]
        k, v = p.k.clone(), p.v.clone()
        KV.lora_kv_fork(p.cache, p.book, parents, children, p.info, p.ws, p.nb, torch.cuda.current_stream())
        info, copies = p.ref.fork(parents, children)
        assert p.info.tolist() == info
        p.same()
        for src, dst, rows in copies:
            for w, t in ((k, p.k), (v, p.v)):
                w[:, dst, :, :rows] = w[:, src, :, :rows].clone()
        assert torch.equal(p.k.view(torch.int16), k.view(torch.int16))
        assert torch.equal(p.v.view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("stack", [(3, 12, 48)], indirect=True)
@pytest.mark.parametrize("rows", [[3, 2], [1, 1], [1, 1, 1, 1], [4]])
def test_a_segment_per_sequence_is_needed(stack, rows):
    s = stack
    step = T.Step(s.layers, s.srv.cache, rows, [0] * len(rows), HEADS, stream=s.st)
    s.steps[tuple(rows)] = step
    x = s.x(sum(rows))
    y = torch.empty_like(x)
    k = s.k.clone()
    for call in (lambda: step.run(s.srv.attn, s.srv.seqs, x, y, s.st),
                 lambda: step.attend(s.srv.attn, 0, s.srv.seqs, y, s.st)):
        with pytest.raises(ValueError, match="segments"):
            call()
    assert torch.equal(k, s.k)


@pytest.mark.parametrize("stack", [(2, 12, 48)], indirect=True)
def test_rows_and_projections_of_other_sizes_are_refused(stack):
    s, st = stack, stack.st
    for rows, adapters in (([2, 3], [0]), ([2, 3], [0, 1, 0]), ([2, -1], [0, 1])):
        with pytest.raises(ValueError, match="segment"):
            T.Step(s.layers, s.srv.cache, rows, adapters, HEADS, stream=st)
    for heads in (2, 8):
        with pytest.raises(ValueError, match="projection"):
            T.Step(s.layers, s.srv.cache, [1, 1], [0, 1], heads, stream=st)
    step = s.step([2, 3])
    s.srv.grow(torch.tensor([2, 3], dtype=torch.int32, device=DEV))
    x, y, k = s.x(5), torch.zeros((5, HIDDEN), dtype=s.dtype, device=DEV), s.k.clone()
    wide = torch.zeros((5, 2 * HIDDEN), dtype=s.dtype, device=DEV)
    for bad in (x[:4], x[:, :64], x.half(), x.float(), x.cpu(), wide[:, ::2], x.view(-1)):
        for args in ((bad, y), (x, bad)):
            with pytest.raises(ValueError):
                step.run(s.srv.attn, s.srv.seqs, *args, st)
        with pytest.raises(ValueError):
            step.attend(s.srv.attn, 0, s.srv.seqs, bad, st)
        with pytest.raises(ValueError):
            step.project(0, bad, st)
    assert torch.equal(k, s.k) and (y == 0).all()
    wide[:, :HIDDEN] = x
    step.run(s.srv.attn, s.srv.seqs, wide, y, st)            # rows further apart
    other = torch.zeros_like(y)
    step.run(s.srv.attn, s.srv.seqs, x, other, st)
    assert torch.equal(y, other) and not (y == 0).all()


@pytest.mark.parametrize("form", ["torch", "handle", "default"])
def test_a_server_on_a_stream_that_is_not_current(form):
    # the current stream is busy while the server is made and used on the other one
    n_seqs, rows, dt = 3, [5, 20, 1], torch.bfloat16
    layers, kept = T.random_layers(1, HIDDEN, HEADS, KV_HEADS, DIM, dt, [4, 8], DEV, 3, torch.cuda.current_stream())
    gen = torch.Generator().manual_seed(2)
    x = torch.randn((sum(rows), HIDDEN), generator=gen).to(dt).to(DEV)
    add = torch.tensor(rows, dtype=torch.int32, device=DEV)
    busy = torch.randn((8192, 8192), device=DEV)
    shape = (1, 6, KV_HEADS, PR, DIM)

    def serve(stream):
        cache = KV.Cache(*(torch.zeros(shape, dtype=dt, device=DEV) for _ in range(2)))
        y = torch.zeros_like(x)
        torch.cuda.synchronize()
        if stream is not None:
            for _ in range(12):
                torch.mm(busy, busy)             # some milliseconds each in float32
        srv = T.Server(cache, n_seqs, 32, stream)
        step = T.Step(layers, cache, rows, [0, 1, 0], HEADS, stream=stream)
        srv.grow(add)
        step.run(srv.attn, srv.seqs, x, y, stream)
        torch.cuda.synchronize()
        out = [t.clone() for t in (y, cache.k, cache.v, srv.tables, srv.lens, srv.refs, srv.info)]
        torch.cuda.synchronize()
        step.release()
        srv.release()
        return out

    want = serve(None)                           # everything on the default stream
    assert want[4].tolist() == rows and want[6].tolist() == [4, 0] and not (want[0] == 0).all()
    side = torch.cuda.Stream()
    if form == "default":                        # a side stream is current, and the default one is used
        with torch.cuda.stream(side):
            for _ in range(12):
                torch.mm(busy, busy)
            got = serve(None)
    else:
        got = serve(side if form == "torch" else side.cuda_stream)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    for layer in layers:
        for p in (layer.q, layer.k, layer.v, layer.o):
            L.lora_release_adapters(p.table)
    del kept


def test_projections_of_one_shape_and_other_ranks():
    # q, k, v and o are all HIDDEN x HIDDEN here; their adapters differ in rank, between layers too
    dt, st = torch.float16, torch.cuda.current_stream()
    heads, dim, n = 4, HIDDEN // 4, [3, 20, 1]
    parts = [T.random_layers(1, HIDDEN, heads, heads, dim, dt, ranks, DEV, i, st)
             for i, ranks in enumerate([[4, 8], [8, 4], [16, 8], [4, 8], [4, 8, 2]])]
    one = [p[0][0] for p in parts]
    layers = [T.Layer(one[0].q, one[1].k, one[2].v, one[3].o), T.Layer(one[3].q, one[0].k, one[0].v, one[1].o),
              T.Layer(one[4].q, one[4].k, one[4].v, one[4].o)]
    cache = KV.Cache(*(torch.zeros((3, 9, heads, PR, dim), dtype=dt, device=DEV) for _ in range(2)))
    srv = T.Server(cache, 3, 32, st)
    step = T.Step(layers, cache, n, [0, 1, 0], heads, stream=st)
    x = torch.randn((sum(n), HIDDEN), generator=torch.Generator().manual_seed(1)).to(dt).to(DEV)
    y = torch.empty_like(x)
    srv.grow(torch.tensor(n, dtype=torch.int32, device=DEV))

    def alone(p, src):                           # the projection's one call, without a plan
        batch = L.Batch(step.batch.seg_offset, [0, 1, 0], sum(n))
        nb = L.lora_base_workspace_bytes(p.table, batch)
        ws, out = torch.empty(nb, dtype=torch.uint8, device=DEV), torch.empty_like(src)
        L.lora_base_apply(p.table, batch, src, HIDDEN, p.wt, HIDDEN, out, HIDDEN, ws, nb, st)
        torch.cuda.synchronize()
        return out

    src = x
    for i, layer in enumerate(layers):
        step.project(i, src, st)
        step.attend(srv.attn, i, srv.seqs, y, st)
        torch.cuda.synchronize()
        for p, a, b in ((layer.q, src, step.q), (layer.k, src, step.k), (layer.v, src, step.v), (layer.o, step.a, y)):
            assert torch.equal(alone(p, a), b), i
        src = y.clone()
    done = y.clone()
    step.run(srv.attn, srv.seqs, x, y, st)
    assert torch.equal(done, y)
    assert len(step._plans) == 3                 # ranks (4, 8), (8, 4), (16, 8): the third adapter is in no segment
    torch.cuda.synchronize()
    step.release()
    with pytest.raises(L.LoraError):             # an adapter that a table lacks: nothing is left behind
        T.Step(layers, cache, n, [0, 2, 0], heads, stream=st)
    srv.release()
    for layer in one:
        for p in (layer.q, layer.k, layer.v, layer.o):
            L.lora_release_adapters(p.table)


def test_trim_of_more_sequences_than_a_grid_takes():
    n, held = (1 << 20) + 300, 400               # the last ones have three pages each
    i32 = dict(dtype=torch.int32, device=DEV)
    tables, lens = torch.full((n, 3), -1, **i32), torch.zeros(n, **i32)
    tables[n - held:] = torch.randperm(3 * held, generator=torch.Generator().manual_seed(0)).view(held, 3).to(DEV)
    lens[n - held:] = torch.arange(33, 33 + 16, device=DEV).repeat(held // 16).int()
    refs = torch.ones(3 * held, **i32)
    before = tables.clone()
    KV.lora_kv_trim(KV.Book(tables, lens, refs, PR), 10, 1, torch.cuda.current_stream())
    gone = lens[n - held:] - 10 >= 31            # the second page; the first holds the sink
    want = before.clone()
    want[n - held:, 1] = torch.where(gone, -1, before[n - held:, 1])
    assert torch.equal(tables, want)
    assert gone.any() and refs.sum().item() == 3 * held - int(gone.sum())


@pytest.mark.parametrize("stack", [(6, 20, 90), (6, 11, 70), (6, 64, 90)], indirect=True)
@pytest.mark.parametrize("seed", range(2))
def test_service_on_a_pool_that_runs_out(stack, seed):
    # prompts, chunks, tokens, branches, ends and compactions in random order
    s, rng = stack, np.random.default_rng(seed)
    granted = refused = 0
    for _ in range(40):
        what = rng.integers(6)
        if what == 0:
            gone = [int(i) for i in rng.permutation(6)[:rng.integers(3)]]
            s.srv.free(gone)
            s.ref.free(gone)
        elif what == 1:
            ids = [int(i) for i in rng.permutation(6)]
            parents, kids = ids[:2], ids[2:2 + rng.integers(3)]
            pairs = [parents[int(i)] for i in rng.integers(0, 2, len(kids))]
            s.srv.fork(pairs, kids)
            s.ref.fork(pairs, kids)
        elif what == 2:
            s.srv.compact()
            s.ref.compact()
        form = rng.integers(3)
        if form == 0:
            add = [int(a) for a in rng.choice([0, 1, 1, 1], size=6)]
            rows = [1] * 6
        else:
            rows = [int(a) for a in rng.choice([0, 1, 3, 16, 17, 40], size=6)]
            add = [r if rng.integers(5) else 0 for r in rows]
        has = s.token(add, rows)
        granted += sum(has)
        refused += sum(1 for a, h in zip(add, has) if a and not h)
    assert granted and refused
