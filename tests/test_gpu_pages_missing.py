"""Attention where a row's table names pages that are not there, and the bytes that nobody has written are the worst there are."""
import pytest
import torch

from tests import pages_reference as ref
from tests.test_gpu_pages import fill, ints, pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new,cap", [([1, 1, 1], 12), ([1, 1, 1], 100), ([9, 12, 5], 100), ([130, 150, 33], 12), ([300, 150, 190], 100)],
                         ids=["one", "one-long-table", "some", "prompts", "longer-prompts"])
@pytest.mark.parametrize("dim", [64, 192])
def test_scales_of_missing_pages(dim, new, cap, dtype):
    heads, group = 8, 8
    lengths = [n + 60 for n in new]
    p, pool = pair(1, 60, 3, cap, heads, dim, 32)
    p.codes.view(torch.uint8).fill_(0x7f)
    p.scales.fill_(255)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    fill(p, pool, lengths, 1)
    gone = [[0, 1], [(lengths[1] - 1) // 32], list(range(cap))]      # the first ones; the last; all of a row
    p.codes.view(torch.uint8)[:, 0] = 0x7f
    p.scales[:, 0] = 255
    for r, places in enumerate(gone):
        for j in places:
            p.tables[r, j] = (-1, 60, 1 << 30)[j % 3]
    g = torch.Generator("cuda").manual_seed(2)
    q = torch.randn(sum(new), heads * group, dim, device="cuda", generator=g).to(dtype)
    starts = ints([sum(new[:r]) for r in range(4)])
    for window in (0, 45):
        got, at = p.attend(0, q, starts, max(new), window=window, out_dtype=torch.float32).double().cpu(), 0
        assert bool(torch.isfinite(got).all())
        for r, n in enumerate(new):
            kv = pool.values(0, r)
            for i in {0, n // 2, n - 1}:
                place = lengths[r] - n + i
                seen = [t for t in range(max(0, place - window + 1) if window else 0, place + 1) if t // 32 not in gone[r]]
                x = q[at + i:at + i + 1].double().cpu()
                want = ref.attend(x, kv[:, :, seen], group, dim ** -0.5)[0] if seen else torch.zeros(heads * group, dim, dtype=torch.float64)
                # weights to 2^-17 at least, scores of some tens of steps of 2^-24 each over dim terms: 2^-12 of the values' size, which is below 8
                assert float((got[at + i] - want).abs().max()) <= 8 * 2.0 ** -12, (r, i, window)
            at += n
