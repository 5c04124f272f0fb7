"""Attention over pages of 8 bits on the GPU, against the definition in 64 bits on the values that the codes stand for."""
import pytest
import torch

from paper_2002_02645_amd import binding
from tests import pages_reference as ref
from tests.test_gpu_pages import fill, ints, pair

pytestmark = pytest.mark.gpu


def bounds(pool, layer, q, new, group, scale, dtype, window=0):
    """How far an output may be off: the sum of |weight| |value| times
      bf16 q: a weight's rounding to bf16 (2^-9 .. 2^-8 of it at most), and fp32's share as below;
      fp32: scores of products exact to 2^-24, summed in fp32 over dim terms and turned to powers of two: an absolute error of
            (dim / 8 + 16) 2^-24 of the sum of |scale q k|, log2(e) times it in the exponent, relative in the weight;
    then the output's own rounding."""
    out, at = torch.zeros(q.shape, dtype=torch.float64), 0
    for r, n in enumerate(new):
        if n:
            kv = pool.values(layer, r)
            x = q[at:at + n].double()
            big = ref.attend(x, torch.stack([kv[0], kv[1].abs()]), group, scale, window)
            reach = scale * torch.stack([(x[:, j].abs() @ kv[0, j // group].abs().t()).amax(1) if kv.shape[2] else torch.zeros(n, dtype=torch.float64) for j in range(x.shape[1])], 1)
            rel = (pool.dim / 8 + 16) * 2.0 ** -24 * (1 + reach) * 3 + kv.shape[2] * 2.0 ** -26 + (2.0 ** -8 if dtype == torch.bfloat16 else 0)
            out[at:at + n] = big * rel[..., None]
        at += n
    return out


def check(p, pool, new, group, dtype, seed, window=0, scale=None, out_dtype=None, layer=0, packed=None, most=0, strided=False):
    g = torch.Generator("cuda").manual_seed(seed)
    total, heads = sum(new), pool.heads * group
    scale = pool.dim ** -0.5 if scale is None else scale
    if strided:
        q = torch.randn(total, heads + 2, pool.dim + 5, device="cuda", generator=g).to(dtype)[:, 1:heads + 1, 3:pool.dim + 3]
    else:
        q = torch.randn(total, heads, pool.dim, device="cuda", generator=g).to(dtype)
    packed = not (all(n == 1 for n in new) and total == pool.rows) if packed is None else packed
    starts = ints([sum(new[:r]) for r in range(len(new) + 1)]) if packed else None
    got = p.attend(layer, q, starts, most, scale, window, out_dtype)
    want = pool.attend(layer, q.cpu(), new, group, scale, window)
    bound = bounds(pool, layer, q.cpu(), new, group, scale, dtype, window)
    bound = bound + want.abs() * torch.finfo(got.dtype).eps / 2 + 1e-40
    off = (got.double().cpu() - want).abs()
    assert bool((off <= bound).all()), (float((off / bound).nan_to_num(9e9).max()), got.shape)
    return got


def grown(sizes, lengths, seed=1, dtype=torch.bfloat16, size=1.0):
    p, pool = pair(*sizes)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    fill(p, pool, lengths, seed, 0, dtype, size)
    return p, pool


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,group,page", [(128, 2, 4, 64), (1, 1, 1, 32), (8, 2, 3, 32), (32, 1, 16, 64), (37, 3, 2, 32), (64, 2, 8, 128), (80, 1, 5, 32), (96, 2, 1, 64),
                                                  (130, 1, 2, 32), (192, 1, 4, 32), (224, 1, 1, 64), (256, 2, 2, 32), (128, 1, 17, 64), (128, 1, 40, 32), (256, 1, 33, 32)])
def test_one_token_a_row(dim, heads, group, page, dtype):
    lengths = [1, 32, 33, 2, 150, 64, 31, 257]
    p, pool = grown((1, 60, 8, 12, heads, dim, page), lengths)
    check(p, pool, [1] * 8, group, dtype, 2)
    check(p, pool, [1] * 8, group, dtype, 3, packed=True, most=1, strided=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,group,page", [(128, 2, 4, 64), (64, 1, 1, 32), (80, 3, 5, 32), (256, 1, 2, 32), (31, 1, 3, 128)])
@pytest.mark.parametrize("new", [[1, 3, 0, 2, 8], [40, 1, 17, 0, 90], [130, 5, 64, 33, 200]])
def test_several_tokens_a_row(new, dim, heads, group, page, dtype):
    """Prompts from nothing (a row's whole length is new) and behind what is there; rows without new tokens; windows."""
    lengths = [max(n, m) for n, m in zip(new, [140, 5, 64, 33, 200])]
    p, pool = grown((1, 60, 5, 8, heads, dim, page), lengths)
    check(p, pool, new, group, dtype, 4, most=max(new))
    check(p, pool, new, group, dtype, 5, window=37, out_dtype=torch.float32, strided=True)
    check(p, pool, new, group, dtype, 6, window=1, most=1000)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_blocks_over_many_workgroups(dtype):
    """Long rows beside short ones: tiles that two, and many, workgroups meet in."""
    lengths = [5000, 1, 0, 700, 33, 2100]
    p, pool = grown((1, 300, 6, 160, 2, 64, 32), lengths)
    for seed, new in ((1, [1, 1, 0, 1, 1, 1]), (2, [4, 1, 0, 2, 1, 7])):
        for window in (0, 1000):
            check(p, pool, new, 2, dtype, seed, window)
            check(p, pool, new, 3, dtype, seed, window, out_dtype=torch.bfloat16)


def test_empty_rows_and_places_before_the_first():
    """Rows of no tokens at all, and more new tokens than a row has places: nothing to attend to gives zeros; rows without new tokens are left."""
    p, pool = grown((1, 20, 4, 4, 1, 32, 32), [0, 5, 40, 0])
    q = torch.randn(20, 2, 32, device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(q, 7.0)
    p.attend(0, q, ints([0, 3, 11, 11, 14]), out=out)     # row 1: 8 tokens, 5 places
    assert bool((out[:6] == 0).all()) and bool((out[11:14] == 0).all()) and bool((out[14:] == 7).all())
    want = ref.attend(q[6:11].double().cpu(), pool.values(0, 1), 2, 32 ** -0.5)
    assert float((out[6:11].double().cpu() - want).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
    out.fill_(7.0)
    p.attend(0, q, ints([0, -1, 3, 2, 21]), out=out)      # none as it should be
    assert bool((out == 7).all())
    p.attend(0, q, ints([0, 3, 11, 11, 14]), most=2, out=out)
    assert bool((out == 7).all())


@pytest.mark.parametrize("new", [[1, 1], [4, 4], [50, 3]])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_not_a_number_stays_with_those_that_see_it(new, dtype):
    """NaN and infinities in later tokens, before the window, in the rest of a block, in pages of nobody."""
    p, pool = pair(1, 10, 2, 4, 1, 64, 32)
    p.codes.view(torch.uint8).fill_(0x7f)                 # what free pages hold
    p.reserve(ints([90, 70]))
    pool.reserve([90, 70])
    g = torch.Generator("cuda").manual_seed(3)
    k, v = (torch.randn(160, 1, 64, device="cuda", generator=g) for _ in range(2))
    k[10, 0, 5], v[20, 0, 7], v[88, 0, 40], k[89, 0, 1], v[90 + 69, 0, 3] = (float(x) for x in ("nan", "inf", "nan", "inf", "-inf"))
    p.append(0, k, v, ints([0, 90, 160]))
    pool.append(0, k.cpu(), v.cpu(), [90, 70])
    q = torch.randn(sum(new), 2, 64, device="cuda", generator=g).to(dtype)
    starts = ints([0, new[0], sum(new)])
    for window in (0, 60, 2, 1):
        got = p.attend(0, q, starts, window=window).double().cpu()
        want = pool.attend(0, q.cpu(), new, 2, 0.125, window)
        assert torch.equal(torch.isnan(got), torch.isnan(want)), window
        fine = ~torch.isnan(want)
        assert bool(((got - want)[fine].abs() <= 2.0 ** -6 * (1 + want[fine].abs())).all())
    q2 = q.clone()
    q2[0, 0, 0] = float("nan")
    got, other = p.attend(0, q2, starts, window=60), p.attend(0, q, starts, window=60)
    assert bool(torch.isnan(got[0, 0]).all()) and torch.equal(got[0, 1].isnan(), other[0, 1].isnan()) and torch.equal(torch.nan_to_num(got[1:]), torch.nan_to_num(other[1:]))


def test_large_scores_and_exponents():
    """Scores of several hundred, of either sign and rising along a row (the running reference moves all the time), keys and values far from one."""
    p, pool = pair(1, 40, 2, 20, 1, 64, 32)
    n = 600
    p.reserve(ints([n, n]))
    pool.reserve([n, n])
    g = torch.Generator("cuda").manual_seed(8)
    k = torch.randn(2 * n, 1, 64, device="cuda", generator=g) * torch.linspace(0.01, 30, 2 * n, device="cuda")[:, None, None]
    v = torch.randn(2 * n, 1, 64, device="cuda", generator=g) * 1e-20
    starts = ints([0, n, 2 * n])
    p.append(0, k, v, starts)
    pool.append(0, k.cpu(), v.cpu(), [n, n])
    for dtype in (torch.float32, torch.bfloat16):
        check(p, pool, [1, 1], 4, dtype, 1, scale=2.0)
        check(p, pool, [7, 30], 4, dtype, 2, scale=1.0)


def test_pages_outside_the_pool_do_not_count():
    p, pool = grown((1, 20, 1, 8, 2, 32, 32), [200])
    q = torch.randn(1, 2, 32, device="cuda")
    for j, bad in ((1, 20), (3, -1), (6, 1 << 30)):
        p.tables[0, j] = bad
    kv = pool.values(0, 0)
    seen = [t for t in range(200) if t // 32 not in (1, 3, 6)]
    want = ref.attend(q.double().cpu(), kv[:, :, seen], 1, 32 ** -0.5)
    assert float((p.attend(0, q).double().cpu() - want).abs().max()) < 1e-5
    p.tables.fill_(-1)
    assert bool((p.attend(0, q) == 0).all())


def test_same_results_every_time():
    p, _ = grown((1, 300, 6, 160, 2, 64, 32), [5000, 1, 0, 700, 33, 2100])
    q = torch.randn(6, 8, 64, device="cuda", dtype=torch.bfloat16)
    first = p.attend(0, q)
    for _ in range(5):
        assert torch.equal(first, p.attend(0, q))
