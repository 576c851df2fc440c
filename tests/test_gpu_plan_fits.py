"""lora_plan_fits and lora_base_plan_fits: what they say is what the plan's launches do, and a step shares plans by it."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_mx_step import ADAPTERS, DEV, DIM, HEADS, HIDDEN, KV_HEADS, N_SEQS, RANKS, Stack  # noqa: E402

from paper_2401_11240_amd import attention as T  # noqa: E402
from paper_2401_11240_amd import lora as L  # noqa: E402


class Tables:
    def __init__(self):
        self.kept, self.made = [], []

    def table(self, ranks, h_in=64, h_out=128, dtype=torch.float16):
        A = [torch.randn((h_in, r), device=DEV).to(dtype) for r in ranks]
        B = [torch.randn((r, h_out), device=DEV).to(dtype) for r in ranks]
        torch.cuda.synchronize()
        code = L.LORA_F16 if dtype == torch.float16 else L.LORA_BF16
        t = L.lora_register_adapters(0, h_in, h_out, code, A, B, ranks, [1.0] * len(ranks))
        self.kept.append((A, B))
        self.made.append(t)
        return t


@pytest.fixture
def tables():
    t = Tables()
    yield t
    torch.cuda.synchronize()
    for x in t.made:
        L.lora_release_adapters(x)


def agrees(says, run):
    """The answer, and the launch's that was asked about."""
    try:
        run()
        ran = True
    except L.LoraError as e:
        assert e.code in (L.LORA_E_SHAPE, L.LORA_E_RANK, L.LORA_E_INDEX)
        ran = False
    torch.cuda.synchronize()
    assert says == ran
    return says


@pytest.mark.parametrize("n", [0, 5])
def test_answers_are_the_launches(tables, n):
    batch = L.Batch([0, n], [1], n)
    own = tables.table([4, 8])
    others = {tables.table([4, 8]): True, tables.table([7, 8]): True,                 # (the first adapter is in no segment)
              tables.table([4, 9]): n == 0, tables.table([4]): n == 0,                 # (nor is any of a batch of no rows)
              tables.table([4, 8], h_in=72): False, tables.table([4, 8], h_out=136): False,
              tables.table([4, 8], dtype=torch.bfloat16): False, own: True}
    x, wt = torch.ones((8, 72), dtype=torch.float16, device=DEV), torch.ones((136, 72), dtype=torch.float16, device=DEV)
    y, z = torch.zeros((8, 136), dtype=torch.float16, device=DEV), torch.zeros((8, 136), dtype=torch.float16, device=DEV)
    plan, base = L.lora_plan_create(own, batch), L.lora_base_plan_create(own, batch)
    two = L.lora_plan_create_multi([own, own], batch)
    for t, want in others.items():
        assert agrees(L.lora_plan_fits(plan, (t,)), lambda: L.lora_plan_apply(plan, t, x, 72, y, 136)) == want
        assert agrees(L.lora_base_plan_fits(base, t), lambda: L.lora_base_plan_apply(base, t, x, 72, wt, 72, y, 136)) == want
        for pair in ((own, t), (t, own)):
            assert agrees(L.lora_plan_fits(two, pair), lambda: L.lora_plan_apply_multi(two, pair, x, 72, (y, z), (136, 136))) == want
    assert L.lora_plan_fits(plan, (None,)) and L.lora_base_plan_fits(base, None) and L.lora_plan_fits(two, (None, own))
    for call in (lambda: L.lora_plan_fits(plan, (own, own)), lambda: L.lora_plan_fits(two, (own,)), lambda: L.lora_plan_fits(two, (own, None)),
                 lambda: L.lora_plan_fits(plan, ())):
        with pytest.raises(L.LoraError) as e:
            call()
        assert e.value.code == L.LORA_E_ARG
    for p in (plan, two):
        L.lora_plan_destroy(p)
    L.lora_base_plan_destroy(base)


@pytest.mark.parametrize("seg_lens", [[3, 0, 2, 1, 4], [1] * N_SEQS, [0] * N_SEQS])
def test_steps_share_plans(seg_lens):
    """Layers of one shape and equal ranks: a plan for three and one for o, or with 16-bit weights one for each shape, with rows
    or without."""
    s = Stack(torch.float16)
    plain, kept = T.random_layers(2, HIDDEN, HEADS, KV_HEADS, DIM, s.dt, RANKS, DEV, 6, s.st)
    try:
        for layers, want in ((s.layers, 2), (plain, len({p.shape for p in (plain[0].q, plain[0].k, plain[0].o)}))):
            step = T.Step(layers, s.cache, seg_lens, ADAPTERS, HEADS, 0, 0, s.st)
            assert len(step._plans) == want
            step.release()
    finally:
        torch.cuda.synchronize()
        for layer in plain:
            for p in (layer.q, layer.k, layer.v, layer.o):
                L.lora_release_adapters(p.table)
        s.close()
