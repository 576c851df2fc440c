"""A step in which the same adapters' tables stand behind 16-bit weights and behind weights in 4-bit blocks."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_mx_step import ADAPTERS, DEV, DIM, EPS, HEADS, HIDDEN, KV_HEADS, RANKS, Stack  # noqa: E402

from paper_2401_11240_amd import attention as T  # noqa: E402
from paper_2401_11240_amd import lora as L  # noqa: E402


@pytest.mark.parametrize("norms", [False, True], ids=["bare", "norms"])
@pytest.mark.parametrize("order", [(0, 1, 2), (1, 0, 2), (2, 1, 0)])
def test_the_same_adapters_behind_weights_of_both_kinds(order, norms):
    """Every layer of the step gives the bits that a step of its own gives: a layer in blocks, one of 16-bit weights and
    one whose q and o are in blocks, all with the adapters of the first."""
    s = Stack(torch.float16)
    plain, kept = T.random_layers(1, HIDDEN, HEADS, KV_HEADS, DIM, s.dt, RANKS, DEV, 6, s.st)
    steps, seg_lens = [], [3, 0, 2, 1, 4]
    try:
        a, b = s.layers[0], plain[0]
        norm = a.norm if norms else None
        wide = [T.Projection(p.table, w.wt) for p, w in zip((a.q, a.k, a.v, a.o), (b.q, b.k, b.v, b.o))]
        kinds = [T.Layer(a.q, a.k, a.v, a.o, norm), T.Layer(*wide, norm), T.Layer(a.q, wide[1], wide[2], a.o, norm)]
        layers = [kinds[i] for i in order]
        cache = T.KV.Cache(*(torch.zeros((3, 60, KV_HEADS, 16, DIM), dtype=s.dt, device=DEV) for _ in range(2)))
        together = T.Step(layers, cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st, eps=EPS)
        steps.append(together)
        x = s.embed[:sum(seg_lens)].contiguous()
        y, want = torch.zeros_like(x), torch.zeros_like(x)
        s.grow(seg_lens)
        for i, layer in enumerate(layers):
            alone = T.Step([layer], cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st, eps=EPS)
            steps.append(alone)
            if norms:
                together.total.zero_()               # (a layer behind others adds its x to what is there)
            together.project(i, x, s.st)
            alone.project(0, x, s.st)
            for got, one in ((together.q, alone.q), (together.k, alone.k), (together.v, alone.v)):
                assert torch.equal(got, one) and not (one == 0).all()
            together.attend(s.srv.attn, i, s.srv.seqs, y, s.st)
            alone.attend(s.srv.attn, 0, s.srv.seqs, want, s.st)
            assert torch.equal(y, want) and not (want == 0).all()
    finally:
        torch.cuda.synchronize()
        for t in steps:
            t.release()
        for layer in plain:
            for p in (layer.q, layer.k, layer.v, layer.o):
                L.lora_release_adapters(p.table)
        s.close()
