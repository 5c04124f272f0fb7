"""Attention over pages at sizes that take its other kernels: 32 columns a wave (many rows of several columns), and the prompts' kernel (a row's many new tokens), in
every width, against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2002_02645_amd import binding
from tests.test_gpu_pages import fill, ints, pair

pytestmark = pytest.mark.gpu

HEADS, GROUP = 8, 8     # of 64 heads in all: 64 new tokens are 4,096 columns, 256 are 16,384
WIDE = [8, 5, 13, 0, 8, 11, 8, 12]
PROMPTS = [130, 5, 64, 0, 33, 200]


def exact(pool, q, new, scale, window, seen=None):
    """Outputs, and sums of |weight| |value|, in 64 bits; seen(row, token): tokens that do not count are False."""
    out, size, at = [], [], 0
    for r, n in enumerate(new):
        x = q[at:at + n].double().view(n, HEADS, GROUP, pool.dim)
        at += n
        if n == 0:
            continue
        k, v = pool.values(0, r)
        length = k.shape[1]
        place = length - n + torch.arange(n)[:, None]
        token = torch.arange(length)[None, :]
        hidden = (token > place) | (token <= place - window if window else token < 0)
        if seen is not None:
            hidden = hidden | ~torch.tensor([seen(r, t) for t in range(length)], dtype=torch.bool)[None, :]
        s = scale * torch.einsum("nhgd,htd->nhgt", x, k).masked_fill(hidden[:, None, None, :], -math.inf)
        w = torch.softmax(s, -1).nan_to_num(0.0) if length else s
        out.append(torch.einsum("nhgt,htd->nhgd", w, v).reshape(n, -1, pool.dim))
        size.append(torch.einsum("nhgt,htd->nhgd", w, v.abs()).reshape(n, -1, pool.dim))
    return torch.cat(out), torch.cat(size)


def check(p, pool, new, dtype, seed, window=0, out_dtype=None, strided=False, seen=None, most=0):
    g = torch.Generator("cuda").manual_seed(seed)
    total, heads, dim, scale = sum(new), HEADS * GROUP, pool.dim, pool.dim ** -0.5
    if strided:
        q = torch.randn(total, heads + 1, dim + 3, device="cuda", generator=g).to(dtype)[:, 1:, 2:dim + 2]
        out = torch.full((total + 2, heads, dim + 5), 9.0, device="cuda", dtype=out_dtype or dtype)
    else:
        q, out = torch.randn(total, heads, dim, device="cuda", generator=g).to(dtype), None
    starts = ints([sum(new[:r]) for r in range(len(new) + 1)])
    got = p.attend(0, q, starts, most, window=window, out_dtype=None if strided else out_dtype, out=out[1:-1, :, 1:dim + 1] if strided else None)
    if strided:
        assert bool((out[0] == 9).all()) and bool((out[-1] == 9).all()) and bool((out[..., 0] == 9).all()) and bool((out[..., dim + 1:] == 9).all())
    want, size = exact(pool, q.cpu(), new, scale, window, seen)
    # weights: rounded to bf16 once (2^-8 of a step of the sum at most) with bf16 q; fp32's share: scores of some tens, a few hundred terms
    rel = (2.0 ** -8 if dtype == torch.bfloat16 else 0) + (dim / 8 + 400) * 2.0 ** -24 * 8
    bound = size * rel + want.abs() * torch.finfo(got.dtype).eps / 2 + 1e-30
    off = (got.double().cpu() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [WIDE, PROMPTS], ids=["wide", "prompts"])
@pytest.mark.parametrize("dim", [17, 64, 96, 128, 160, 192, 200, 256])
def test_every_width(dim, new, dtype):
    lengths = [n + m for n, m in zip(new, [140, 0, 33, 70, 96, 1, 31, 5])]
    p, pool = pair(1, 120, len(new), 12, HEADS, dim, 32)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    fill(p, pool, lengths, dim, 0, dtype)
    check(p, pool, new, dtype, 1)
    check(p, pool, new, dtype, 2, window=45, out_dtype=torch.float32, most=max(new))
    check(p, pool, new, dtype, 3, window=1, strided=True)


@pytest.mark.parametrize("group", [1, 3, 16, 40])
def test_groups(group, monkeypatch):
    monkeypatch.setitem(globals(), "GROUP", group)
    new = [130, 5, 64, 0, 33, 200 * 8]
    lengths = [n + 40 for n in new]
    p, pool = pair(1, 140, 6, 60, HEADS, 64, 32)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    fill(p, pool, lengths, 5, 0, torch.bfloat16)
    check(p, pool, new, torch.bfloat16, 1)


@pytest.mark.parametrize("new", [WIDE, PROMPTS], ids=["wide", "prompts"])
def test_pages_outside_the_pool(new):
    """First, middle and last pages that are not there; a row of nothing but such."""
    lengths = [n + 100 for n in new]
    p, pool = pair(1, 120, len(new), 12, HEADS, 64, 32)
    p.reserve(ints(lengths))
    pool.reserve(lengths)
    fill(p, pool, lengths, 3)
    gone = {(0, 0), (0, 3), (1, 1), (2, (lengths[2] - 1) // 32)} | {(4, j) for j in range(12)}
    for r, j in gone:
        p.tables[r, j] = (120, -1, 1 << 30)[j % 3]
    p.codes.view(torch.uint8)[:, pool.tables[0][0]] = 0x7f     # (nor does what lies there matter)
    check(p, pool, new, torch.bfloat16, 1, seen=lambda r, t: (r, t // 32) not in gone)


@pytest.mark.parametrize("new", [WIDE, PROMPTS], ids=["wide", "prompts"])
def test_not_a_number(new):
    """NaN in keys and values that some tokens see and some do not: later ones, ones before the window, in whole blocks and at edges."""
    lengths = [n + 100 for n in new]
    p, pool = pair(1, 120, len(new), 12, HEADS, 64, 32)
    p.codes.view(torch.uint8).fill_(0x7f)                      # what nobody has written
    p.reserve(ints(lengths))
    pool.reserve(lengths)
    g = torch.Generator("cuda").manual_seed(4)
    k, v = (torch.randn(sum(lengths), HEADS, 64, device="cuda", generator=g) for _ in range(2))
    first = [sum(lengths[:r]) for r in range(len(new) + 1)]
    for r in range(len(new)):
        v[first[r] + 40, 1, 7] = float("nan")
        k[first[r] + lengths[r] - 1, 2, 3] = float("inf")
        v[first[r] + lengths[r] - 2, 3, 60] = -float("inf")
        v[first[r] + max(0, lengths[r] - 40), 0, 20] = float("nan")
    p.append(0, k, v, ints(first))
    pool.append(0, k.cpu(), v.cpu(), lengths)
    q = torch.randn(sum(new), HEADS * GROUP, 64, device="cuda", generator=g).to(torch.bfloat16)
    starts = ints([sum(new[:r]) for r in range(len(new) + 1)])
    for window in (0, 37):
        got, at = p.attend(0, q, starts, window=window).double().cpu(), 0
        for r, n in enumerate(new):
            kk, vv = pool.values(0, r)
            for i in range(n):
                place = lengths[r] - n + i
                lo = max(0, place - window + 1) if window else 0
                bad = torch.isnan(kk[:, lo:place + 1]).any(2).any(1)[:, None] | torch.isnan(vv[:, lo:place + 1]).any(1)
                assert torch.equal(torch.isnan(got[at + i]).view(HEADS, GROUP, 64), bad[:, None].expand(HEADS, GROUP, 64)), (r, i, window)
            at += n


def test_more_new_tokens_than_places_and_empty_rows():
    p, pool = pair(1, 40, 4, 8, HEADS, 64, 32)
    lengths = [0, 100, 7, 200]
    p.reserve(ints(lengths))
    pool.reserve(lengths)
    fill(p, pool, lengths, 3)
    new = [150, 160, 90, 10]
    q = torch.randn(410, HEADS * GROUP, 64, device="cuda").to(torch.bfloat16)
    got = p.attend(0, q, ints([0, 150, 310, 400, 410])).double().cpu()
    assert bool((got[:150 + 60] == 0).all()) and bool((got[310:310 + 83] == 0).all())
    want, size = exact(pool, q[210:310].cpu(), [0, 100, 0, 0], 0.125, 0)
    assert bool(((got[210:310] - want).abs() <= size * 2.0 ** -7).all())
    want, size = exact(pool, q[393:400].cpu(), [0, 0, 7, 0], 0.125, 0)
    assert bool(((got[393:400] - want).abs() <= size * 2.0 ** -7).all())


def test_rising_scores():
    """Scores that rise along the row: the running reference moves in most blocks."""
    n = 600
    p, pool = pair(1, 30, 1, 25, HEADS, 64, 32)
    p.reserve(ints([n]))
    pool.reserve([n])
    g = torch.Generator("cuda").manual_seed(8)
    k = torch.randn(n, HEADS, 64, device="cuda", generator=g) * torch.linspace(0.01, 30, n, device="cuda")[:, None, None]
    v = torch.randn(n, HEADS, 64, device="cuda", generator=g)
    p.append(0, k, v, ints([0, n]))
    pool.append(0, k.cpu(), v.cpu(), [n])
    check(p, pool, [300], torch.bfloat16, 1)
    check(p, pool, [64], torch.bfloat16, 1)


@pytest.mark.parametrize("new", [WIDE, PROMPTS, [1] * 8], ids=["wide", "prompts", "one"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_keys_of_zeros_and_tiny_scales(new, dtype):
    """Scores that are all as good as 0: every visible token has the same weight, hidden ones none."""
    lengths = [n + 40 for n in new]
    p, pool = pair(1, 120, len(new), 12, HEADS, 64, 32)
    p.reserve(ints(lengths))
    pool.reserve(lengths)
    g = torch.Generator("cuda").manual_seed(4)
    v = torch.randn(sum(lengths), HEADS, 64, device="cuda", generator=g)
    first = ints([sum(lengths[:r]) for r in range(len(new) + 1)])
    q = torch.randn(sum(new), HEADS * GROUP, 64, device="cuda", generator=g).to(dtype)
    starts = ints([sum(new[:r]) for r in range(len(new) + 1)])
    for k, scale in ((torch.zeros_like(v), 0.125), (torch.zeros_like(v), 1e-30), (torch.full_like(v, 1e-38), 1.0), (v, 1e-37), (v * 1e-30, 1e-20)):
        p.append(0, k, v, first)
        pool.append(0, k.cpu(), v.cpu(), lengths)
        want, size = exact(pool, q.cpu(), new, 1e-200, 0)   # (0 times a hidden token's -inf would be no number)
        off = (p.attend(0, q, starts, scale=scale, out_dtype=torch.float32).double().cpu() - want).abs()
        assert bool((off <= size * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -18)).all()), scale


def test_same_results_every_time():
    p, pool = pair(1, 300, 6, 45, HEADS, 128, 64)
    p.reserve(ints([2000, 300, 64, 0, 900, 1200]))
    g = torch.Generator("cuda").manual_seed(8)
    k, v = (torch.randn(4464, HEADS, 128, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    p.append(0, k, v, ints([0, 2000, 2300, 2364, 2364, 3264, 4464]))
    for new in ([700, 100, 64, 0, 9, 400], [9, 8, 15, 0, 12, 30]):
        q = torch.randn(sum(new), HEADS * GROUP, 128, device="cuda", generator=g).to(torch.bfloat16)
        starts = ints([sum(new[:r]) for r in range(7)])
        first = p.attend(0, q, starts)
        for _ in range(4):
            assert torch.equal(first, p.attend(0, q, starts))


@pytest.mark.parametrize("dim", [17, 64, 96, 128, 160, 200, 256])
def test_longer_prompts(dim):
    """632 new tokens of 64 heads are 40,448 columns: 32 columns a wave in the prompts' kernel where the heads allow it."""
    new = [130, 5, 64, 0, 33, 400]
    lengths = [n + m for n, m in zip(new, [140, 0, 33, 70, 96, 1])]
    p, pool = pair(1, 120, len(new), 14, HEADS, dim, 32)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    fill(p, pool, lengths, dim, 0, torch.bfloat16)
    check(p, pool, new, torch.bfloat16, 1)
    check(p, pool, new, torch.bfloat16, 2, window=45, out_dtype=torch.float32, most=max(new))
    check(p, pool, new, torch.bfloat16, 3, window=1, strided=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [[130, 5, 64, 0, 33, 40], PROMPTS, [130, 5, 64, 0, 33, 400]], ids=["17408", "27648", "40448"])
def test_prompts_in_long_tables(new, dtype):
    """Tables that could hold more than 64 blocks a row: sizes between go to the kernel that splits rows over workgroups."""
    lengths = [n + m for n, m in zip(new, [140, 0, 33, 70, 96, 1])]
    p, pool = pair(1, 120, len(new), 100, HEADS, 128, 32)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    fill(p, pool, lengths, 7, 0, dtype)
    check(p, pool, new, dtype, 4)
    check(p, pool, new, dtype, 5, window=45, most=max(new))
