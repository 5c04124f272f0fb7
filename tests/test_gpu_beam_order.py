"""The order of continuations that are worth the same, and values far from zero: against the definition, order and all."""
import numpy as np
import pytest
import torch

from paper_2002_02645_amd import binding

pytestmark = pytest.mark.gpu

INF = float("inf")
# log of a sum of fp32 exponentials: two units in the last place each, a sum of 32 a lane and batch, its rescaling: 40 * 2^-24; the rounded
# score: 2^-24 of itself
NEAR = 4e-6


def _best(logits, scores, beams, k):
    """Per group the k best (total, row in the batch, token): best first, then the lower row, the larger value, the lower token.  A total is the
    score so far and the log of a share of the row's sum: neither cancels against the row's largest value."""
    x, scores = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    out = []
    for first in range(0, x.shape[0], beams):
        cand = []
        for r in range(first, first + beams):
            if scores[r] == -INF or not (x[r] > -INF).any():
                continue
            top = x[r].max()
            offset = scores[r] - np.log(np.exp(x[r] - top).sum())
            for v in np.lexsort((np.arange(x.shape[1]), -x[r]))[:k]:
                if x[r, v] > -INF:
                    cand.append((offset + (x[r, v] - top), r, x[r, v], int(v)))
        cand.sort(key=lambda c: (-c[0], c[1], -c[2], c[3]))
        out.append([(c[0], c[1], c[3]) for c in cand[:k]])
    return out


def _run(logits, scores, beams, k):
    fc = binding.FreezeCache(1)
    try:
        out = {key: v.cpu().numpy() for key, v in fc.beam_select(logits, scores, beams, k).items()}
    finally:
        fc.close()
    for g, best in enumerate(_best(logits, scores, beams, k)):
        assert list(zip(out["parent"][g], out["token"][g]))[:len(best)] == [(r, t) for _, r, t in best], g
        for i, (total, _, _) in enumerate(best):
            assert abs(out["score"][g, i] - total) <= NEAR + 2.0 ** -24 * abs(total), (g, i, out["score"][g, i], total)
        assert (out["score"][g, len(best):] == -INF).all()


def _noise(rows, vocab, seed):
    return torch.randn(rows, vocab, generator=torch.Generator().manual_seed(seed)) * 2.5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1003, 30522, 50257, 50021, 7, 32000])
def test_rows_alike(vocab, dtype):
    # the rows of a group are the same and lie at every place within 16 bytes: their sums are the same to the last bit, so that rows go by number
    for seed in range(4):
        rows = _noise(3, vocab, 31 + seed).repeat_interleave(4, 0).to(dtype).cuda()
        _run(rows, torch.full((12,), -1.25, device="cuda"), 4, 8)
    wide = torch.zeros(8, vocab + 9, dtype=dtype, device="cuda")
    wide[:, 3:3 + vocab] = rows[:1]
    _run(wide[:, 3:3 + vocab], torch.zeros(8, device="cuda"), 8, 16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e7, 3e9, 1e10, 1e20, 1e37, 1e38])
def test_values_far_from_zero(size, dtype):
    # 50,021 values of 1e7 and more away from zero, some of them alike: a row is worth its score and the log of a share of its sum
    g = torch.Generator().manual_seed(8)
    for sign in (1, -1):
        x = sign * size * (1 + torch.rand(8, 50021, generator=g))
        for r in range(8):
            x[r, torch.randint(0, 50021, (3,), generator=g)] = x[r].max()
        _run(x.to(dtype).cuda(), -torch.rand(8, generator=g).cuda(), 4, 9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fill", ["lowest", "highest", "lowest_and_few"])
def test_rows_of_the_type_s_ends(fill, dtype):
    # a row whose every value is the mark of a forbidden token: all tokens alike, none of them better than the other rows' best
    x = _noise(12, 5003, 6).to(dtype)
    info = torch.finfo(dtype)
    if fill == "lowest_and_few":
        x[torch.rand(x.shape, generator=torch.Generator().manual_seed(1)) < 0.999] = info.min
    x[1] = x[6] = info.max if fill == "highest" else info.min
    _run(x.cuda(), -torch.arange(12).float().cuda() / 8, 4, 12)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("beams,vocab,k", [(4, 50021, 1), (4, 50021, 2), (4, 50021, 12), (1, 131075, 64), (8, 20000, 16), (64, 700, 64), (3, 300, 5)])
def test_totals_that_swallow_the_values(beams, vocab, k, dtype):
    # marks of rows that are out of use, and values that a total of -10 does not resolve: the values themselves decide within a row
    x = _noise(2 * beams, vocab, 3 + beams).to(dtype).cuda()
    for mark in (-1e30, torch.finfo(torch.float32).min):
        scores = torch.full((2 * beams,), mark, device="cuda")
        _run(x, scores, beams, k)
        scores[beams + beams // 2] = -2.0
        _run(x, scores, beams, k)
    tiny = torch.zeros(2 * beams, vocab)
    for i in range(min(5, vocab)):
        tiny[:, (i * 977 + 131) % vocab] = (i + 1) * 1e-18
    _run(tiny.to(dtype).cuda(), torch.zeros(2 * beams, device="cuda"), beams, k)
