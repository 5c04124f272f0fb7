"""Pages of keys and values on the GPU: bookkeeping against lists, appending against plain loops in 64 bits."""
import random

import pytest
import torch

from paper_2002_02645_amd import binding
from tests import pages_reference as ref

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def pair(*sizes):
    return binding.FreezePages(*sizes), ref.Pool(*sizes)


def same_book(p, want):
    assert p.tables.tolist() == want.tables
    assert p.lengths.tolist() == want.lengths
    assert p.refs.tolist() == want.refs


def same_codes(p, want, pages=None):
    """Codes, as numbers, and exponents of the pages in use."""
    at = ref.places(want.dim).view(2, -1)
    got = p.codes.double().cpu()
    got = torch.stack([got[..., 0, :][..., at[0]], got[..., 1, :][..., at[1]]], 4).view(want.codes.shape)
    for page in range(want.num_pages) if pages is None else pages:
        if want.refs[page]:
            assert torch.equal(torch.nan_to_num(got[:, page], 999.0), torch.nan_to_num(want.codes[:, page], 999.0)), page
            assert torch.equal(p.scales[:, page].cpu().long() - 127, want.exps[:, page]), page


@pytest.mark.parametrize("rows,max_pages,num_pages,page,seed", [(1, 1, 1, 32, 1), (3, 4, 9, 32, 2), (8, 6, 30, 64, 3), (17, 5, 60, 32, 4), (70, 9, 400, 32, 5), (1500, 3, 5000, 32, 6)])
def test_bookkeeping(rows, max_pages, num_pages, page, seed):
    """Random reservations, forks, cuts and compactions, every state as the lists say."""
    rng = random.Random(seed)
    p, want = pair(1, num_pages, rows, max_pages, 1, 8, page)
    for step in range(25 if rows < 1000 else 6):
        what = rng.choice(["reserve", "reserve", "one", "fork", "truncate", "compact"])
        if what == "reserve":
            add = [rng.choice([0, -3, 1, rng.randint(0, 2 * page), rng.randint(0, max_pages * page + 5)]) for _ in range(rows)]
            assert p.reserve(ints(add)).tolist() == want.reserve(add), step
        elif what == "one":
            assert p.reserve().tolist() == want.reserve([1] * rows), step
        elif what == "fork":
            parents = [rng.choice([r, rng.randrange(rows), rng.randrange(rows), -1, rows]) for r in range(rows)]
            p.fork(ints(parents))
            want.fork(parents)
        elif what == "truncate":
            keep = [rng.choice([-1, 0, rng.randint(0, max_pages * page), n, n + 1]) for n in want.lengths]
            p.truncate(ints(keep))
            want.truncate(keep)
        else:
            assert p.compact().tolist() == [want.compact()], step
        same_book(p, want)


def test_many_rows_and_pages():
    """As many rows as there may be, several thousand pages: the lists of more than one round of the single workgroup."""
    rows, pages = 16384, 40000
    p, want = pair(1, pages, rows, 2, 1, 8, 32)
    rng = random.Random(7)
    for add in ([rng.randint(0, 40) for _ in range(rows)], [rng.randint(0, 64) for _ in range(rows)], [64] * rows):
        assert p.reserve(ints(add)).tolist() == want.reserve(add)
        same_book(p, want)
    parents = [rng.randrange(rows) for _ in range(rows)]
    p.fork(ints(parents))
    want.fork(parents)
    assert p.compact().tolist() == [want.compact()]
    assert p.reserve().tolist() == want.reserve([1] * rows)
    same_book(p, want)


def fill(p, want, new, seed, layer=0, dtype=torch.bfloat16, size=1.0, granted=None, strided=False, most=0):
    g = torch.Generator("cuda").manual_seed(seed)
    total, heads, dim = sum(new), want.heads, want.dim
    shape = (total, heads, dim)
    if strided:
        both = (torch.randn(total, 2 * heads + 1, dim + 3, device="cuda", generator=g) * size).to(dtype)
        k, v = both[:, 1:heads + 1, 2:dim + 2], both[:, heads + 1:, 1:dim + 1]
    else:
        k, v = ((torch.randn(shape, device="cuda", generator=g) * size).to(dtype) for _ in range(2))
    starts = None
    if not (all(n == 1 for n in new) and total == want.rows):
        starts = ints([sum(new[:r]) for r in range(len(new) + 1)])
    p.append(layer, k, v, starts, most, None if granted is None else ints(granted))
    want.append(layer, k.cpu(), v.cpu(), new, granted)
    return k, v


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,page", [(1, 1, 32), (8, 2, 32), (32, 1, 64), (37, 3, 32), (64, 2, 128), (80, 2, 32), (96, 1, 64), (128, 3, 64), (160, 1, 32), (192, 2, 32), (200, 1, 32), (256, 1, 64)])
def test_append(dim, heads, page, dtype):
    """A prompt of odd length, then tokens one by one and some at once; larger values make exponents grow over what is there."""
    rows = 4
    p, want = pair(2, 40, rows, 6, heads, dim, page)
    for step, (new, size) in enumerate([([1, 0, 31, 70], 1.0), ([1, 1, 1, 1], 0.01), ([1, 1, 1, 1], 300.0), ([33, 5, 0, 2], 1e-3), ([1, 1, 1, 1], 1e5), ([0, 64, 32, 0], 1e-30)]):
        assert p.reserve(ints(new)).tolist() == want.reserve(new) == new
        for layer in (0, 1):
            fill(p, want, new, 10 * step + layer, layer, dtype, size, strided=step % 2 == 1, most=(0, 70, max(new))[step % 3])
        same_codes(p, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_ends_of_the_range(dtype):
    """Zeros, the smallest and largest numbers, infinities and NaN beside ordinary values."""
    p, want = pair(1, 4, 1, 2, 1, 32, 32)
    tiny, huge = 2.0 ** -149 if dtype == torch.float32 else 2.0 ** -133, float(torch.finfo(dtype).max)
    for values in ([0.0, -0.0], [tiny, -tiny], [2.0 ** -126, 448 * 2.0 ** -126], [448 * 2.0 ** -126 * 1.01], [448.0, -449.0, 0.3], [float("nan"), 1.0], [float("inf"), 3.0, -float("inf")],
                   [huge, 1.0, -huge], [2.0 ** 40, 2.0 ** 30, 1e-20]):
        x = torch.zeros(1, 1, 32, dtype=dtype, device="cuda")
        x[0, 0, 3:3 + len(values)] = torch.tensor(values, dtype=dtype)
        p.reserve()
        want.reserve([1])
        p.append(0, x, x.flip(2).contiguous())
        want.append(0, x.cpu(), x.flip(2).cpu(), [1])
        same_codes(p, want)


def test_append_leaves_others_alone():
    """Rows that got no room, that are shared, that have too many tokens or starts out of order are not written; nor is any byte of another page."""
    p, want = pair(1, 12, 6, 2, 2, 64, 32)
    new = [40, 20, 20, 0, 10, 64]
    p.reserve(ints(new))
    want.reserve(new)
    fill(p, want, new, 1)
    p.fork(ints([0, 1, 1, 3, 4, 5]))
    want.fork([0, 1, 1, 3, 4, 5])
    before, scales = p.codes.view(torch.uint8).clone(), p.scales.clone()
    k = torch.randn(200, 2, 64, device="cuda", dtype=torch.bfloat16)
    p.append(0, k[:12], k[:12], ints([0, 0, 6, 12, 12, 12, 12]), granted=ints([0, 6, 6, 0, 0, 0]))   # shared pages
    p.append(0, k[:12], k[:12], ints([0, 6, 6, 6, 6, 6, 12]), granted=ints([0, 0, 0, 0, 0, 5]))      # refused rows
    p.append(0, k[:12], k[:12], ints([0, 6, 6, 6, 6, 6, 12]), most=5)                                # more than the most
    p.append(0, k[:12], k[:12], ints([-1, -1, -1, -1, -1, 5, 13]))                                   # outside the tokens
    p.append(0, k[:12], k[:12], ints([12, 6, 6, 6, 5, 3, 0]))                                        # out of order
    p.append(0, k[:11], k[:11], ints([0, 0, 0, 0, 0, 11, 11]))                                       # more tokens than the row has
    assert torch.equal(before, p.codes.view(torch.uint8)) and torch.equal(scales, p.scales)
    p.tables[0, 1] = 12                                                                              # outside the pool
    p.tables[5, 1] = -7
    p.append(0, k[:16], k[:16], ints([0, 8, 8, 8, 8, 8, 16]))
    assert torch.equal(before, p.codes.view(torch.uint8)) and torch.equal(scales, p.scales)


def test_shared_pages_are_copied():
    """Beams of one parent: the next tokens go into pages of their own, what came before is copied, in every layer; unfilled blocks of the copies are left."""
    p, want = pair(3, 40, 6, 4, 2, 48, 64)
    new = [70, 0, 100, 128, 30, 1]
    p.reserve(ints(new))
    want.reserve(new)
    for layer in range(3):
        fill(p, want, new, layer, layer)
    parents = [0, 0, 0, 3, 3, 5]
    p.fork(ints(parents))
    want.fork(parents)
    p.codes.view(torch.uint8)[:, p.refs == 0] = 0x2b      # (pages that the fork left free are given out again)
    assert p.reserve().tolist() == want.reserve([1] * 6) == [1] * 6
    same_book(p, want)
    for r in (0, 1, 2):   # 6 tokens of 64 in the last page: its second block is not the copy's
        assert bool((p.codes.view(torch.uint8)[:, want.tables[r][1], :, 1] == 0x2b).all())
    for layer in range(3):
        fill(p, want, [1] * 6, 50 + layer, layer)
    same_codes(p, want, [t for r in (1, 2) for t in want.tables[r][:1]] + [want.tables[5][0]])
    for layer in range(3):
        at = ref.places(48).view(2, -1)
        for r in range(6):
            n = want.lengths[r]
            ids = want.tables[r][: want.pages(n)]
            x = p.codes[layer].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double().cpu()
            x = torch.stack([x[..., 0, :][..., at[0]], x[..., 1, :][..., at[1]]], 3).view(*x.shape[:4], 32, 64)
            x = x * torch.exp2(p.scales[layer, ids].cpu().double() - 127)[..., None, None]
            x = x.permute(3, 1, 0, 2, 4, 5).reshape(2, 2, -1, 64)[:, :, :n, :48]
            assert torch.equal(x, want.values(layer, r)), (layer, r)


def test_compaction_moves_what_pages_hold():
    p, want = pair(2, 50, 5, 5, 2, 40, 32)
    for step in range(3):
        new = [33, 20, 50, 1, 30]
        p.reserve(ints(new))
        want.reserve(new)
        for layer in (0, 1):
            fill(p, want, new, step * 2 + layer, layer)
    p.truncate(ints([0, 40, -1, 0, 64]))
    want.truncate([0, 40, -1, 0, 64])
    assert p.compact().tolist() == [want.compact()]
    same_book(p, want)
    same_codes(p, want)
    assert p.compact().tolist() == [want.compact()]
    same_book(p, want)
    p.truncate(ints([0] * 5))
    assert p.compact().tolist() == [0] and int(p.refs.abs().sum()) == 0 and bool((p.tables == -1).all())


def test_bad_tables_are_not_followed():
    """Page numbers outside the pool in tables that a caller wrote."""
    p, _ = pair(1, 5, 3, 3, 1, 16, 32)
    p.reserve(ints([40, 0, 10]))
    p.tables[0, 1] = 5
    p.tables[1, 0] = 1 << 30
    p.tables[2, 1] = -9
    p.fork(ints([2, 1, 0]))
    p.truncate(ints([0, 0, 0]))
    p.compact()
    p.lengths.copy_(ints([1 << 30, -5, 96]))
    assert p.reserve().tolist() == [0, 1, 0]
    torch.cuda.synchronize()
