"""The products of mx_forms.py get the kernels that they are there for (on a stand-in runtime; no GPU is needed)."""
import pytest

from launches import Calls
from mx_forms import FORMS

from paper_2401_11240_amd import lora as L


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    L.load()
    return Calls(tmp_path_factory.mktemp("launches"))


@pytest.mark.parametrize("form", FORMS, ids=lambda f: f.name)
def test_form(calls, form):
    launched, need = calls.product(form.rows, form.h, form.h_out, form.fmt, L.LORA_BF16)
    kind, sizes = form.kernel.split()
    p, q = sizes.split("x")
    assert launched[0].kernel.startswith(f"lora_mx_{kind}_kernel<{form.fmt}, {p}, {q}")
    blocks, sixteens = -(-form.h // 32), -(-form.h // 512)
    assert blocks % 16                                    # a last turn of scales that is not whole
    if kind == "stream":
        assert -(-blocks // 8) > 2 * launched[0].threads // 64 and blocks % 8      # more than two units for a wave, the last not whole
        assert len(launched) == 1 and form.ranges == 1
        return
    assert launched[0].grid[1] == form.ranges and len(launched) == (1 if form.ranges == 1 else 2)
    assert need == (16 if form.ranges == 1 else 4 * form.ranges * form.rows * form.h_out)
    # steps of 4 blocks of the first range: at least two turns of the scales
    each = next(16 * -(-sixteens // n) for n in (1, 2, 4, 8) if -(-blocks // (16 * -(-sixteens // n))) == form.ranges)
    steps = -(-min(each, blocks) // 4)
    assert steps >= 8
    one_row = form.rows <= int(q)
    if form.turned:                                       # more workgroups than XCDs, and more than one turn to begin at
        assert one_row and steps % 4 == 0 and steps > 4 and -(-form.h_out // int(p)) > 8


def test_every_form_is_there(calls):
    """Every product kernel that there is, and for tiles one and several ranges of K and one and several rows of tiles."""
    have = {calls.product(f.rows, f.h, f.h_out, f.fmt, L.LORA_BF16)[0][0].kernel for f in FORMS}
    assert have == {k for k in calls.kernels() if k.startswith(("lora_mx_stream", "lora_mx_tile"))}
    for fmt in (0, 1):
        for tile in ("64x64", "128x64", "128x128", "256x256"):
            of = [f for f in FORMS if f.fmt == fmt and f.kernel == f"tile {tile}"]
            assert {(f.ranges > 1) for f in of} == {False, True} and any(f.turned for f in of) and any(not f.turned for f in of)
