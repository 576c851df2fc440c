"""What the device's arrays hold leads nowhere outside the buffers, and a launch sized for
more tokens than there are gives what one sized for them gives."""
import itertools

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2401_11240_amd import kv as KV  # noqa: E402
from test_gpu_kv import DEV, Case, say, stream  # noqa: E402


@pytest.fixture(scope="module")
def attn():
    a = KV.lora_attn_create(0, stream())
    yield a
    torch.cuda.synchronize()
    KV.lora_attn_destroy(a)


def guarded(t, fill):
    """t in the middle of a larger tensor of `fill`; the larger one and the part that is t."""
    big = torch.full((t.numel() + 2 * 65536,), fill, dtype=t.dtype, device=t.device)
    inner = big[65536:65536 + t.numel()].view(t.shape)
    inner.copy_(t)
    return big, inner


def bits(t):
    return t.view(torch.int16)


@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 2, 128), (68, 4, 64), (4, 1, 256)])
@pytest.mark.parametrize("page_rows", [16, 64])
def test_offsets_out_of_order_stay_inside(attn, heads, kv_heads, dim, page_rows):
    n_rows, lens = 100, [100, 130, 64]
    c = Case("bf16", heads, kv_heads, dim, page_rows, lens, [60, 30, 10], seed=11, spare=5)
    (kbig, kd), (vbig, vd), (obig, out) = guarded(c.kd, 3.0), guarded(c.vd, 3.0), guarded(c.out, 7.0)
    cache = KV.Cache(kd, vd)
    held = torch.tensor(sorted({int(p) for row in c.table for p in row if p >= 0}), device=DEV)
    free = torch.tensor([p for p in range(c.n_pages) if p not in set(held.tolist())], device=DEV)
    w = kv_heads * dim
    new = torch.randn((n_rows, w), device=DEV).bfloat16()
    big = 1 << 30
    bad = list(itertools.product((0, -7, 100, big), (-3, 20, 100, 150), (90, 5, -(1 << 31), big), (100, 40, (1 << 31) - 1)))
    for off in bad:
        say("offsets", off)
        off_d = torch.tensor(off, dtype=torch.int32, device=DEV)
        before = (kd[:, free].clone(), vd[:, free].clone())
        KV.lora_attn_prompt(attn, cache, 0, c.seqs, off_d, n_rows, heads, c.qd, c.ld, out, c.ld, c.scale, 0, 0, stream())
        KV.lora_attn_prompt(attn, cache, 0, c.seqs, off_d, n_rows, heads, c.qd, c.ld, out, c.ld, c.scale, 20, 3, stream())
        KV.lora_kv_append(cache, 0, c.seqs, off_d, n_rows, new, w, -new, w, stream())
        torch.cuda.synchronize()
        for guard, fill in ((kbig, 3.0), (vbig, 3.0), (obig, 7.0)):
            assert (guard[:65536] == fill).all() and (guard[-65536:] == fill).all()
        for t, b in zip((kd, vd), before):
            assert torch.equal(bits(t[:, free]), bits(b)), "a page that no sequence has"
    # the handle's counters are as they were: an ordinary launch
    c.prompt(attn)
    c.check(what="after offsets out of order")


@pytest.mark.parametrize("lens,rows", [([203], [203]), ([203, 1, 0, 40], [100, 1, 0, 40]), ([1], [1])])
@pytest.mark.parametrize("heads,kv_heads,dim", [(32, 32, 128), (4, 2, 64), (64, 2, 128), (8, 1, 256), (72, 1, 64)])
@pytest.mark.parametrize("max_len,window,sinks", [(1024, 0, 0), (32768, 0, 0), (1 << 20, 0, 0), (32768, 50, 3)])
def test_capacity_far_above_the_lengths(attn, lens, rows, heads, kv_heads, dim, max_len, window, sinks):
    # most parts of such a launch have no token
    c = Case("bf16", heads, kv_heads, dim, 16, lens, rows, seed=len(lens))
    tables = torch.full((len(lens), max_len // 16), -1, dtype=torch.int32, device=DEV)
    tables[:, :c.tables.shape[1]] = c.tables
    c.seqs = KV.Seqs(tables, c.lens_d, max_len)
    c.prompt(attn, window, sinks)
    c.check(window, sinks, f"prompt {rows} behind {lens}, capacity {max_len}, {heads}/{kv_heads} x {dim}")
    c = Case("f16", heads, kv_heads, dim, 16, lens, [1] * len(lens), seed=len(lens))
    c.seqs = KV.Seqs(tables, c.lens_d, max_len)
    tables[:, :c.tables.shape[1]] = c.tables
    c.decode(attn, window, sinks)
    c.check(window, sinks, f"decode {lens}, capacity {max_len}")
