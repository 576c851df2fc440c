"""Serving steps of layers with norms, weights in 4-bit blocks and a head: every stage against
its definition in 64 bits, fed with what the stage itself read, and a recorded step from token to
token against the eager one over several replays."""
import numpy as np
import pytest

import kv_reference as KR
import mx_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2401_11240_amd import attention as T  # noqa: E402
from paper_2401_11240_amd import kv as KV  # noqa: E402
from paper_2401_11240_amd import lora as L  # noqa: E402
from paper_2401_11240_amd import mx as MX  # noqa: E402
from paper_2401_11240_amd import sample as SA  # noqa: E402

DEV = torch.device("cuda:0")
HIDDEN, HEADS, KV_HEADS, DIM, LAYERS, N_SEQS, MAX_LEN, VOCAB = 256, 6, 2, 64, 2, 5, 160, 1000
RANKS, ADAPTERS = [4, 16, 40], [0, 1, 2, -1, 1]
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
EPS = 1e-5


def f64(t):
    return t.detach().double().cpu().numpy()


def values(q):
    return R.values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.fmt, q.h)


def largest_of_8(q):
    """As the product's cut-off counts: the largest magnitude of every eight elements, none below the
    format's smallest normal one (of whole blocks here)."""
    v = np.abs(values(q)).reshape(q.n_rows, -1, 4, 8).max(3)
    unit = np.ldexp(1.0, q.scales.cpu().numpy()[:, :v.shape[1]].astype(int) - 127)[..., None]
    return np.maximum(v, unit * (2.0 ** -6 if q.fmt == R.E4M3 else 1)).reshape(q.n_rows, -1)


def product(x, w):
    """(x W, its bound before the output's rounding): additions, and what is cut off below 2^-13 of the
    largest of eight products."""
    vx, vw = values(x), values(w)
    return vx @ vw.T, (x.h + 16) * 2.0 ** -24 * (np.abs(vx) @ np.abs(vw).T) + 7 * 2.0 ** -13 * (largest_of_8(x) @ largest_of_8(w).T)


class Stack:
    def __init__(self, dt):
        self.dt = dt
        self.st = torch.cuda.current_stream(DEV)
        self.layers, self.kept = T.random_layers(LAYERS, HIDDEN, HEADS, KV_HEADS, DIM, dt, RANKS, DEV, 5, self.st, in_blocks=True)
        gen = torch.Generator().manual_seed(9)
        self.embed = torch.randn((VOCAB, HIDDEN), generator=gen).to(dt).to(DEV)
        out = (torch.randn((VOCAB, HIDDEN), generator=gen) * 0.2).to(dt).to(DEV)
        self.head = T.Head((1 + 0.1 * torch.randn(HIDDEN, generator=gen)).to(dt).to(DEV), T.in_4_bits(out), VOCAB - 5)
        nan = float("nan")
        self.cache = KV.Cache(*(torch.full((LAYERS, 60, KV_HEADS, 16, DIM), nan, dtype=dt, device=DEV) for _ in range(2)))
        self.srv = T.Server(self.cache, N_SEQS, MAX_LEN, self.st)
        self.steps = []

    def step(self, seg_lens):
        s = T.Step(self.layers, self.cache, seg_lens, ADAPTERS, HEADS, 0, 0, self.st, self.head, EPS)
        self.steps.append(s)
        return s

    def grow(self, add):
        self.srv.grow(torch.tensor(add, dtype=torch.int32, device=DEV))

    def close(self):
        torch.cuda.synchronize()
        for s in self.steps:
            s.release()
        self.srv.release()
        for layer in self.layers:
            for p in (layer.q, layer.k, layer.v, layer.o):
                L.lora_release_adapters(p.table)

    def check_norm(self, x, residual, weight, total, h, q):
        half = HALF[self.dt]
        s, y = R.norm(f64(x), None if residual is None else residual, f64(weight), np.float64(np.float32(EPS)))
        # float32 before the outputs' rounding: chains of at most h / 64 + 64 additions, halved by the root,
        # and eight roundings besides
        slack = (HIDDEN / 64 + 64) * 2.0 ** -25 + 8 * 2.0 ** -24
        if total is not None:
            assert (np.abs(f64(total) - s) <= np.abs(s) * (half + 2.0 ** -24) + 2.0 ** -25).all()
        if h is not None:
            assert (np.abs(f64(h) - y) <= np.abs(y) * (half + slack) + 2.0 ** -25).all()
        # half a step of a code, or the distance to the largest one (448 of up to 512), in units of the block
        unit = np.repeat(np.ldexp(1.0, q.scales.cpu().numpy()[:, :HIDDEN // 32].astype(int) - 127), 32, 1)
        a = np.abs(y) / unit
        bound = np.maximum(np.maximum(a * 2.0 ** -4, 2.0 ** -10), a - 448) + a * slack
        assert (a < 512 * (1 + slack)).all() and (np.abs(values(q) - y) <= bound * unit).all()

    def check_projection(self, name, layer, proj, seg_lens, x, q, y):
        at = ("q", "k", "v", "o").index(name)
        A, B, scales = self.kept[4 * layer + at]
        base, bound = product(q, proj.wt)
        half = HALF[self.dt]
        want, err = base.copy(), bound + half * (np.abs(base) + bound)          # rounded behind the product
        x = f64(x)
        row = 0
        for n, g in zip(seg_lens, ADAPTERS):
            r = slice(row, row + n)
            row += n
            if g < 0 or n == 0:
                continue
            a, b = f64(A[g]), f64(B[g])
            v, s = x[r] @ a, scales[g]
            want[r] += s * (v @ b)
            # the delta's operands in two 16-bit parts, and float32 sums over h_in and the rank
            err[r] += 2.0 ** -14 * s * (np.abs(v) @ np.abs(b)) + (x.shape[1] + a.shape[1]) * 2.0 ** -24 * s * (np.abs(x[r]) @ np.abs(a) @ np.abs(b))
            err[r] += half * (np.abs(want[r]) + err[r])                        # and rounded again
        worst = float((np.abs(f64(y) - want) / (err + 2.0 ** -25)).max(initial=0.0))
        assert worst <= 1, (name, layer, worst)

    def check_attention(self, layer, step, seg_lens):
        lens, table = self.srv.lens.cpu().numpy(), self.srv.tables.cpu().numpy()
        k, v = f64(self.cache.k[layer]), f64(self.cache.v[layer])
        a, q = f64(step.a).reshape(-1, HEADS, DIM), f64(step.q).reshape(-1, HEADS, DIM)
        at = 0
        for s, n in enumerate(seg_lens):
            if n:
                o, m, reach = KR.attention(q[at:at + n], k, v, table[s], int(lens[s]), int(lens[s]) - n, step.scale, 0, 0)
                tol = KR.allowance(o, m, reach, DIM, int(lens[s]), self.dt == torch.bfloat16)
                assert (np.abs(a[at:at + n] - o) <= tol).all(), (layer, s)
            at += n

    def run_checked(self, step, seg_lens, x):
        """Every layer of a step, each stage against its definition; y and the tokens' check are the caller's."""
        y, src, before = torch.empty_like(x), x, None
        for i, layer in enumerate(self.layers):
            step.project(i, src, self.st)
            torch.cuda.synchronize()
            hq = step._rows["hq", HIDDEN]
            self.check_norm(src, before, layer.norm, step.total, step.h, hq)
            for name, got in (("q", step.q), ("k", step.k), ("v", step.v)):
                self.check_projection(name, i, getattr(layer, name), seg_lens, step.h, hq, got)
            before = f64(step.total)
            step.attend(self.srv.attn, i, self.srv.seqs, y, self.st)
            torch.cuda.synchronize()
            self.check_attention(i, step, seg_lens)
            aq = step._rows["aq", HEADS * DIM]
            codes, scales = R.quantize(f64(step.a), R.E4M3)
            assert np.array_equal(aq.codes.cpu().numpy(), codes)
            assert np.array_equal(aq.scales.cpu().numpy()[:, :scales.shape[1]], scales)
            self.check_projection("o", i, layer.o, seg_lens, step.a, aq, y)
            src = y.clone()
        return y

    def check_choice(self, step, seg_lens, y, par, u, tokens, probs):
        ends = [int(np.sum(seg_lens[:s + 1])) - 1 for s in range(N_SEQS) if seg_lens[s]]
        rows = [s for s in range(N_SEQS) if seg_lens[s]]
        q = step.last_q
        pick = MX.Rows(q.codes[rows].contiguous(), q.scales[rows].contiguous(), q.fmt, q.h)
        self.check_norm(y[ends], f64(step.total)[ends], self.head.norm, None, None, pick)
        want, bound = product(pick, self.head.wt)
        logits = f64(step.logits)
        assert (np.abs(logits[rows] - want) <= bound + 2.0 ** -24 * (np.abs(want) + bound)).all()
        t, k, p, m = (x.cpu().numpy() for x in (par.temperature, par.top_k, par.top_p, par.min_p))
        for s in range(N_SEQS):
            if not seg_lens[s]:
                assert tokens[s].item() == -1 and probs[s].item() == 0
                continue
            token, own, total = R.sample(logits[s][:VOCAB - 5], t[s], int(k[s]), p[s], m[s], np.float32(u[s].item()))
            assert tokens[s].item() == token
            assert abs(probs[s].item() - own / total) <= own / total * (2.0 ** -24 + 2.0 ** -50)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_from_prompts_to_tokens(dt):
    s = Stack(dt)
    srv, st = s.srv, s.st
    rng = np.random.default_rng(11)
    dev = lambda a, d: torch.from_numpy(np.asarray(a, d)).to(DEV)  # noqa: E731
    par = SA.Params(dev([1, 0.7, 0, 1.3, 1], np.float32), dev([0, 40, 0, 5, 0], np.int32), dev([1, 0.9, 1, 0.8, 0.5], np.float32),
                    dev([0, 0, 0, 0.05, 0.1], np.float32))
    u = torch.empty(N_SEQS, device=DEV)
    tokens = torch.zeros(N_SEQS + 1, dtype=torch.int32, device=DEV)
    probs = torch.zeros(N_SEQS + 1, device=DEV)
    tokens[N_SEQS], probs[N_SEQS] = 77, 77

    def draw():
        u.copy_(dev(rng.random(N_SEQS), np.float32))

    try:
        for seg_lens in ([37, 16, 1, 0, 50], [0, 0, 20, 9, 0], [1] * N_SEQS):
            step = s.step(seg_lens)
            x = s.embed[dev(rng.integers(0, VOCAB, sum(seg_lens)), np.int64)]
            s.grow(seg_lens)
            y = s.run_checked(step, seg_lens, x)
            whole = torch.empty_like(y)
            step.run(srv.attn, srv.seqs, x, whole, st)
            assert torch.equal(whole, y)
            draw()
            step.choose(y, par, u, tokens, probs, st)
            torch.cuda.synchronize()
            s.check_choice(step, seg_lens, y, par, u, tokens, probs)
            assert tokens[N_SEQS] == 77 and probs[N_SEQS] == 77

        decode, ones = s.steps[-1], torch.ones(N_SEQS, dtype=torch.int32, device=DEV)
        x, y = torch.empty((N_SEQS, HIDDEN), dtype=dt, device=DEV), torch.empty((N_SEQS, HIDDEN), dtype=dt, device=DEV)

        def token(stream):
            srv.grow(ones)
            torch.index_select(s.embed, 0, tokens[:N_SEQS], out=x)
            decode.run(srv.attn, srv.seqs, x, y, stream)
            decode.choose(y, par, u, tokens, probs, stream)

        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        srv.stream = side
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            token(side)
        srv.stream = st
        state = [srv.tables, srv.lens, srv.refs, tokens]
        for i in range(8):
            draw()
            before = [t.clone() for t in state]
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (tokens, probs, y, decode.logits)]
            for t, b in zip(state, before):
                t.copy_(b)
            y.zero_()
            token(st)
            assert all(torch.equal(t, g) for t, g in zip((tokens, probs, y, decode.logits), got)), i
            s.check_choice(decode, [1] * N_SEQS, y, par, u, tokens, probs)
        assert srv.lens.tolist() == [n + 9 for n in (37, 16, 21, 9, 50)]
        del graph
    finally:
        s.close()


def test_weights_in_blocks_without_norms_and_beside_others():
    """A layer whose q and o are in blocks and k and v are not: x is quantised for q alone."""
    s = Stack(torch.float16)
    try:
        seg_lens = [3, 0, 2, 1, 4]
        blocks = s.layers[0]
        plain, kept = T.random_layers(1, HIDDEN, HEADS, KV_HEADS, DIM, s.dt, RANKS, DEV, 6, s.st)
        layer = T.Layer(blocks.q, plain[0].k, plain[0].v, blocks.o)
        step = T.Step([layer], s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st)
        x = s.embed[:sum(seg_lens)].contiguous()
        s.grow(seg_lens)
        y = torch.empty_like(x)
        step.run(s.srv.attn, s.srv.seqs, x, y, s.st)
        torch.cuda.synchronize()
        hq, aq = step._rows["hq", HIDDEN], step._rows["aq", HEADS * DIM]
        for q, v in ((hq, x), (aq, step.a)):
            codes, scales = R.quantize(f64(v), R.E4M3)
            assert np.array_equal(q.codes.cpu().numpy(), codes)
            assert np.array_equal(q.scales.cpu().numpy()[:, :scales.shape[1]], scales)
        s.check_projection("q", 0, layer.q, seg_lens, x, hq, step.q)
        s.check_projection("o", 0, layer.o, seg_lens, step.a, aq, y)
        s.check_attention(0, step, seg_lens)
        with pytest.raises(ValueError):
            step.choose(y, None, None, None)
        step.release()
        with pytest.raises(ValueError):       # a head behind layers without norms
            T.Step([layer], s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st, s.head)
        with pytest.raises(ValueError):       # a norm in front of one layer alone
            T.Step([layer, s.layers[1]], s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st)
        bad = T.Layer(blocks.q, blocks.k, blocks.v, blocks.o, blocks.norm[:-8])
        with pytest.raises(ValueError):
            T.Step([bad], s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st)
        with pytest.raises(ValueError):       # a head of another width
            T.Step(s.layers, s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st, T.Head(s.head.norm, blocks.o.wt))
        for p in (plain[0].q, plain[0].k, plain[0].v, plain[0].o):
            L.lora_release_adapters(p.table)
        for n in (-8, VOCAB + 1):             # tokens that the weight has not
            with pytest.raises(ValueError):
                T.Head(s.head.norm, s.head.wt, n)
        empty = s.step([0] * N_SEQS)          # a step without rows
        s.grow([0] * N_SEQS)
        y = torch.empty((0, HIDDEN), dtype=s.dt, device=DEV)
        empty.run(s.srv.attn, s.srv.seqs, y, y, s.st)
        tokens = torch.zeros(N_SEQS, dtype=torch.int32, device=DEV)
        empty.choose(y, None, torch.zeros(N_SEQS, device=DEV), tokens, None, s.st)
        assert tokens.tolist() == [-1] * N_SEQS
    finally:
        s.close()


def test_norms_in_front_of_16_bit_weights():
    """The stages are the calls by themselves, bit for bit."""
    s = Stack(torch.bfloat16)
    plain, kept = T.random_layers(2, HIDDEN, HEADS, KV_HEADS, DIM, s.dt, RANKS, DEV, 6, s.st)
    seg_lens, steps = [3, 0, 2, 1, 4], []
    try:
        layers = [T.Layer(p.q, p.k, p.v, p.o, b.norm) for p, b in zip(plain, s.layers)]
        step = T.Step(layers, s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st, s.head, EPS)
        bare = T.Step(plain, s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st)
        steps += [step, bare]
        n = sum(seg_lens)
        x = s.embed[:n].contiguous()
        s.grow(seg_lens)
        y, want = torch.empty_like(x), torch.empty_like(x)
        step.run(s.srv.attn, s.srv.seqs, x, y, s.st)
        total, h, src = torch.empty_like(x), torch.empty_like(x), x
        for i in range(2):
            MX.lora_norm(src, HIDDEN, total if i else None, HIDDEN, layers[i].norm, EPS, n, HIDDEN, L.LORA_BF16, total, HIDDEN,
                         h, HIDDEN, None, s.st)
            bare.project(i, h, s.st)
            bare.attend(s.srv.attn, i, s.srv.seqs, want, s.st)
            src = want
        assert torch.equal(y, want) and torch.equal(step.total, total) and torch.equal(step.h, h)
        tokens, probs = torch.zeros(N_SEQS, dtype=torch.int32, device=DEV), torch.zeros(N_SEQS, device=DEV)
        step.choose(y, None, torch.zeros(N_SEQS, device=DEV), tokens, probs, s.st)
        assert tokens[1] == -1 and (tokens[[0, 2, 3, 4]] >= 0).all() and (probs[[0, 2, 3, 4]] > 0).all()
    finally:
        torch.cuda.synchronize()
        for t in steps:
            t.release()
        for layer in plain:
            for p in (layer.q, layer.k, layer.v, layer.o):
                L.lora_release_adapters(p.table)
        s.close()


def test_layers_of_other_ranks():
    """q, k and v share a launch where their adapters agree in rank, layers a plan where theirs do; every
    delta is its own table's either way."""
    s = Stack(torch.float16)
    others, kept = T.random_layers(2, HIDDEN, HEADS, KV_HEADS, DIM, s.dt, [7, 24, 40], DEV, 6, s.st, in_blocks=True)
    seg_lens, step = [3, 0, 2, 1, 4], None
    try:
        a, b = s.layers[0], others[0]
        mixed = T.Layer(a.q, b.k, a.v, b.o, a.norm)
        layers = [a, b, s.layers[1], others[1], mixed]
        cache = KV.Cache(*(torch.zeros((5, 60, KV_HEADS, 16, DIM), dtype=s.dt, device=DEV) for _ in range(2)))
        step = T.Step(layers, cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st)
        # a plan of three and one for o for either ranks; q, k and v of the mixed layer on their own (k and v are of one shape)
        assert len(step._plans) == 4 + 3
        x = s.embed[:sum(seg_lens)].contiguous()
        s.kept = [s.kept[0], s.kept[1], s.kept[2], s.kept[3], *kept[:4], *s.kept[4:], *kept[4:], s.kept[0], kept[1], s.kept[2], kept[3]]
        for i, layer in enumerate(layers):
            step.project(i, x, s.st)
            torch.cuda.synchronize()
            for name, got in (("q", step.q), ("k", step.k), ("v", step.v)):
                s.check_projection(name, i, getattr(layer, name), seg_lens, step.h, step._rows["hq", HIDDEN], got)
    finally:
        torch.cuda.synchronize()
        if step:
            step.release()
        for layer in others:
            for p in (layer.q, layer.k, layer.v, layer.o):
                L.lora_release_adapters(p.table)
        s.close()
