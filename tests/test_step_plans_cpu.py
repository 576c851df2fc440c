"""Which plan a step takes for which projection, on the host: the library's calls are stand-ins that
check what they are given, and no GPU is needed."""
import contextlib
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2401_11240_amd import attention as T  # noqa: E402
from paper_2401_11240_amd import build as B  # noqa: E402
from paper_2401_11240_amd import kv as KV  # noqa: E402
from paper_2401_11240_amd import lora as L  # noqa: E402
from paper_2401_11240_amd import mx as MX  # noqa: E402

HIDDEN, HEADS, DIM = 64, 2, 32
BASE, DELTA, THREE = "base plan", "plan", "plan of three"


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(B.lib_path()):
        B.build()
    L.load()


class Library:
    """Plans are (kind, tables they were made for); every table fits every plan of its kind.  ``ran`` lists what a step
    enqueued, as (call, table)."""

    def __init__(self, monkeypatch):
        self.ran = []

        def create(kind):
            return lambda tables, batch, stream=None: (kind, tables)

        def fits(plan, tables, want):
            assert plan[0] == want, f"{plan} asked for {tables}"
            return True

        def base(plan, table, x, ldx, wt, ldw, y, ldy, stream=None):
            if x is None:
                raise L.LoraError(L.LORA_E_ARG, "x is NULL")
            assert plan is not None and plan[0] == BASE, f"{plan} for a 16-bit weight"
            self.ran.append(("base", table))

        def delta(plan, table, x, ldx, y, ldy, stream=None):
            if isinstance(x, int):
                raise L.LoraError(L.LORA_E_ALIGN, "x not aligned")
            assert plan is not None and plan[0] == DELTA, f"{plan} for a delta"
            self.ran.append(("delta", table))

        def three(plan, tables, x, ldx, ys, ldys, stream=None):
            if ys[2] is None:
                raise L.LoraError(L.LORA_E_ARG, "y 2 is NULL")
            assert plan[0] == THREE, f"{plan} for three deltas"
            self.ran.extend(("delta", t) for t in tables)

        for name, f in dict(lora_base_plan_create=create(BASE), lora_plan_create=create(DELTA), lora_plan_create_multi=create(THREE),
                            lora_base_plan_apply=base, lora_plan_apply=delta, lora_plan_apply_multi=three,
                            lora_base_plan_fits=lambda p, t: fits(p, t, BASE),
                            lora_plan_fits=lambda p, ts: fits(p, ts, THREE if len(ts) == 3 else DELTA),
                            lora_base_plan_destroy=lambda p: fits(p, None, BASE),
                            lora_plan_destroy=lambda p: self.destroyed(p)).items():
            monkeypatch.setattr(L, name, f, raising=False)
        monkeypatch.setattr(MX, "lora_norm", lambda *a: None)
        monkeypatch.setattr(MX, "lora_mx_quantize", lambda *a: None)
        monkeypatch.setattr(MX, "lora_mx_apply", lambda x, w, *a: self.ran.append(("product", w)))
        monkeypatch.setattr(T, "_ordered", lambda stream, device: contextlib.nullcontext())

    @staticmethod
    def destroyed(plan):
        assert plan[0] in (DELTA, THREE), plan


@pytest.fixture
def library(monkeypatch):
    return Library(monkeypatch)


def layer(tables, in_blocks, norm=False):
    def weight():
        return MX.empty_rows(HIDDEN, HIDDEN, MX.LORA_E2M1, "cpu") if in_blocks else torch.zeros((HIDDEN, HIDDEN), dtype=torch.float16)
    return T.Layer(*(T.Projection(t, weight()) for t in tables), torch.ones(HIDDEN, dtype=torch.float16) if norm else None)


def step_of(layers, rows=3):
    cache = KV.Cache(*(torch.zeros((len(layers), 2, HEADS, 16, DIM), dtype=torch.float16) for _ in range(2)))
    return T.Step(layers, cache, [rows], [0], HEADS)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("order", ["blocks first", "16 bits first"])
def test_tables_behind_weights_of_both_kinds(library, order, norm):
    """The adapters of one layer on two, one with its weights in blocks: every projection gets a plan of its own kind
    and its delta once."""
    tables = (11, 12, 13, 14)
    layers = [layer(tables, True, norm), layer(tables, False, norm)]
    if order != "blocks first":
        layers.reverse()
    step = step_of(layers)
    x, y = (torch.zeros((3, HIDDEN), dtype=torch.float16) for _ in range(2))
    for i, one in enumerate(layers):
        library.ran.clear()
        step.project(i, x)
        step._apply(one.o, x, y, None, object())
        if one.q.in_blocks:
            assert sorted(t for call, t in library.ran if call == "delta") == list(tables)
            assert [w for call, w in library.ran if call == "product"] == [p.wt for p in (one.q, one.k, one.v, one.o)]
            assert not any(call == "base" for call, _ in library.ran)
        else:
            assert library.ran == [("base", t) for t in tables]
    step.release()


def test_a_layer_partly_in_blocks_behind_one_that_is_wholly(library):
    """q, k and v with a plan for three in one layer, and with weights of both kinds in the next."""
    tables = (11, 12, 13, 14)
    whole, plain = layer(tables, True), layer(tables, False)
    mixed = T.Layer(whole.q, plain.k, whole.v, plain.o)
    step = step_of([whole, mixed])
    x = torch.zeros((3, HIDDEN), dtype=torch.float16)
    step.project(1, x)
    assert library.ran == [("product", whole.q.wt), ("delta", 11), ("base", 12), ("product", whole.v.wt), ("delta", 13)]
    step.release()


def test_a_step_asks_for_plans_and_runs_nothing(library, monkeypatch):
    """Layers of one shape share plans, which the library is asked about: nothing that could enqueue is called before
    the step runs."""
    asked = []

    def runs(*a, **k):
        raise AssertionError("a step that is being made runs something")

    def fits(plan, tables):
        asked.append((plan, tables))
        return True

    for name in ("lora_plan_apply", "lora_plan_apply_multi", "lora_base_plan_apply", "lora_plan_shrink", "lora_plan_expand"):
        monkeypatch.setattr(L, name, runs)
    monkeypatch.setattr(L, "lora_plan_fits", fits)
    monkeypatch.setattr(L, "lora_base_plan_fits", lambda plan, table: fits(plan, (table,)))
    step = step_of([layer((1, 2, 3, 4), True), layer((5, 6, 7, 8), True), layer((9, 10, 11, 12), False)])
    three, o = (THREE, (1, 2, 3)), (DELTA, 4)
    assert asked == [(three, (5, 6, 7)), (o, (8,)), ((BASE, 9), (10,)), ((BASE, 9), (11,)), ((BASE, 9), (12,))]
    assert [plan for _, plan in step._plans] == [three, o, (BASE, 9)]
    step.release()


def test_questions_about_no_plan():
    for call in (lambda: L.lora_plan_fits(None, (None,)), lambda: L.lora_plan_fits(None, ()), lambda: L.lora_base_plan_fits(None, None)):
        with pytest.raises(L.LoraError) as e:
            call()
        assert e.value.code == L.LORA_E_ARG
