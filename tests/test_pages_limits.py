"""The ends of what the rotary positions and attention over pages take, as the header states them."""
import pytest
import torch

from paper_2002_02645_amd import binding
from tests.test_gpu_pages import ints, pair
from tests.test_pages_refusals import GB, P, at, pool

EINVAL = binding.FREEZE_EINVAL


@pytest.mark.parametrize("scale,taken", [(1e-38, True), (2e38, True), (2.01e38, False), (3e38, False), (0.0, False), (-1e-38, False)])
def test_scale(scale, taken):
    p = pool()
    got = binding.lib().freeze_pages_attend(at(p), 0, P(6 * GB), 1, 240, 40, 2, 0, None, 0, scale, 0, P(7 * GB), 1, 240, 40, P(8 * GB), GB, None)
    assert got == (0 if taken else EINVAL)


@pytest.mark.parametrize("factor,taken", [(3e38, True), (-3e38, True), (3.01e38, False), (-3.01e38, False)])
def test_factor(factor, taken):
    h = binding.FreezeHeads(GB, 2 * GB, 1, 3, 24, 8, 24, 8)
    assert binding.lib().freeze_rotate_positions(at(h), 1, 0, 8, P(8 * GB), P(9 * GB), 4, 0, factor, 0, None) == (0 if taken else EINVAL)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [[1, 1], [5, 3], [300, 260]])
def test_largest_scale(new, dtype):
    """Scores of 0 are 0 whatever they are multiplied by: keys of every size against queries of zeros, and of the largest scale against the smallest keys."""
    lengths = [n + 40 for n in new]
    p, want = pair(1, 40, 2, 12, 8, 32, 32)
    assert p.reserve(ints(lengths)).tolist() == want.reserve(lengths)
    g = torch.Generator("cuda").manual_seed(1)
    k, v = (torch.randn(sum(lengths), 8, 32, device="cuda", generator=g) for _ in range(2))
    starts = ints([0, new[0], sum(new)])
    for k, q_size in ((k, 0.0), (k * 1e30, 0.0), (k * 0, 1.0)):
        p.append(0, k, v, ints([0, lengths[0], sum(lengths)]))
        want.append(0, k.cpu(), v.cpu(), lengths)
        q = torch.full((sum(new), 64, 32), q_size, device="cuda", dtype=dtype)
        got, first = p.attend(0, q, starts, scale=2e38, out_dtype=torch.float32).double().cpu(), 0
        for r, n in enumerate(new):
            mean = want.values(0, r)[1].cumsum(1) / torch.arange(1, lengths[r] + 1)[:, None]          # [heads, places, dim]
            mean = mean[:, lengths[r] - n:].transpose(0, 1).repeat_interleave(8, 1)
            # equal weights are exact; sums of up to 340 values below 8 and of as many weights, in fp32: 2^-24 of the sum of sizes for each addition
            assert float((got[first:first + n] - mean).abs().max()) <= 2 * 340 * 2.0 ** -24 * 8
            first += n
