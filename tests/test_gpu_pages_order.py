"""Rows whose tokens overlap those of a row before: appending and every kernel of attention pass over the same rows, and do the others whole."""
import random

import pytest
import torch

from tests import pages_reference as ref
from tests.test_gpu_pages import ints, pair, same_codes
from tests.test_gpu_pages_attend import bounds


def in_order(starts, tokens, most=0):
    """(row, first token, tokens) of the rows that count: in order by themselves, and not beginning before the end of one before that is so."""
    floor, rows = 0, []
    for r, (a, b) in enumerate(zip(starts, starts[1:])):
        if 0 <= a < b <= tokens and (most == 0 or b - a <= most):
            if a >= floor:
                rows.append((r, a, b - a))
            floor = max(floor, b)
    return rows


def test_the_rule():
    assert in_order([0, 9, 0, 9, 0, 9], 9) == [(0, 0, 9)]
    assert in_order([0, 2, 9, 3, 5, 9, 12], 12) == [(0, 0, 2), (1, 2, 7), (5, 9, 3)]
    assert in_order([0, 9, 4, 6, 6, 9], 9, 4) == [(2, 4, 2), (4, 6, 3)]


def many(rows, tokens, seed):
    """Starts of many rows, most in order, some thrown back, forward or out."""
    rng = random.Random(seed)
    starts, at = [], 0
    for _ in range(rows + 1):
        starts.append(at if rng.random() < 0.9 else rng.choice([rng.randrange(tokens), 0, -1, tokens + 3, max(0, at - 3)]))
        at = min(tokens, at + rng.choice([0, 0, 1, 1, 2, 3]))
    return starts


CASES = [([0, 70, 0, 70, 0, 70], 70), ([0, 40, 10, 50, 20, 70], 70), ([0, 2, 60, 3, 5, 62, 70], 70), (many(40, 50, 1), 50), (many(700, 400, 2), 400), (many(3000, 900, 3), 900)]


@pytest.mark.gpu
@pytest.mark.parametrize("starts,tokens", CASES, ids=[f"{len(s) - 1}-rows" + ("" if i else "-same") for i, (s, _) in enumerate(CASES)])
@pytest.mark.parametrize("most", [0, 65])
def test_append_and_attention(starts, tokens, most):
    rows, heads, group, dim = len(starts) - 1, 2, 3, 24
    done = in_order(starts, tokens, most)
    lengths = [75 + r % 40 if rows < 100 else 6 + r % 30 for r in range(rows)]
    p, pool = pair(1, sum(-(-n // 32) for n in lengths) + 3, rows, 5, heads, dim, 32)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    g = torch.Generator("cuda").manual_seed(rows)
    first = [sum(lengths[:r]) for r in range(rows + 1)]
    k, v = (torch.randn(first[-1], heads, dim, device="cuda", generator=g) for _ in range(2))
    p.append(0, k, v, ints(first))
    pool.append(0, k.cpu(), v.cpu(), lengths)
    same_codes(p, pool)
    k, v = (torch.randn(tokens, heads, dim, device="cuda", generator=g) * 2 for _ in range(2))
    p.append(0, k, v, ints(starts), most)
    new = [0] * rows
    for r, _, n in done:
        new[r] = n
    mine = [t for _, a, n in done for t in range(a, a + n)]
    pool.append(0, k[mine].cpu(), v[mine].cpu(), new)
    same_codes(p, pool)
    for dtype in (torch.bfloat16, torch.float32):
        q = torch.randn(tokens, heads * group, dim, device="cuda", generator=g).to(dtype)
        out = torch.full((tokens, heads * group, dim), 7.0, device="cuda")
        p.attend(0, q, ints(starts), most, out=out)
        x = q[mine].cpu()
        off = (out[mine].double().cpu() - pool.attend(0, x, new, group, dim ** -0.5)).abs()
        assert bool((off <= bounds(pool, 0, x, new, group, dim ** -0.5, dtype) + 1e-30).all())
        others = sorted(set(range(tokens)) - set(mine))
        assert bool((out[others] == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("starts,tokens,cap", [([0, 300, 0, 300, 0, 300], 300, 12), ([0, 40, 0, 260, 190, 280, 200, 300], 300, 12), ([0, 1, 0, 600, 2, 40, 600, 640], 640, 100)],
                         ids=["same", "some", "longer"])
def test_prompts(starts, tokens, cap, dtype):
    rows, heads, group, dim = len(starts) - 1, 8, 8, 24
    done = in_order(starts, tokens)
    lengths = [max(0, b - a) + 30 for a, b in zip(starts, starts[1:])]
    p, pool = pair(1, 140, rows, cap if cap > 60 else 12, heads, dim, 32)
    lengths = [min(n, 12 * 32) if cap < 60 else n for n in lengths]
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    g = torch.Generator("cuda").manual_seed(rows)
    first = [sum(lengths[:r]) for r in range(rows + 1)]
    k, v = (torch.randn(first[-1], heads, dim, device="cuda", generator=g) for _ in range(2))
    p.append(0, k, v, ints(first))
    pool.append(0, k.cpu(), v.cpu(), lengths)
    q = torch.randn(tokens, heads * group, dim, device="cuda", generator=g).to(dtype)
    out = torch.full((tokens, heads * group, dim), 7.0, device="cuda")
    p.attend(0, q, ints(starts), out=out)
    written = torch.zeros(tokens, dtype=torch.bool)
    for r, a, n in done:
        written[a:a + n] = True
        kv = pool.values(0, r)
        for i in sorted({0, 1, n // 3, n // 2, n - 2, n - 1} & set(range(n))):
            seen = lengths[r] - n + i + 1
            want = ref.attend(q[a + i:a + i + 1].double().cpu(), kv[:, :, :seen], group, dim ** -0.5)[0]
            # weights to 2^-17 at least, scores of some tens of steps of 2^-24 each over dim terms: 2^-12 of the values' size, which is below 8
            assert float((out[a + i].double().cpu() - want).abs().max()) <= 8 * 2.0 ** -12, (r, i)
    assert bool((out.cpu()[~written] == 7).all()) and bool((out.cpu()[written] != 7).any(2).any(1).all())
