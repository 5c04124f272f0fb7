"""Rows of few new tokens beside prompts in one call of attention: each row goes to the kernel that its own number of tokens asks for."""
import pytest
import torch

from tests.test_gpu_pages import fill, ints, pair
from tests.test_gpu_pages_variants import GROUP, HEADS, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,dim", [(512, 64), (600, 40)])
def test_one_token_a_row_whatever_is_said_of_it(rows, dim, dtype):
    """The plain form, the packed one, and the packed one without the most that a row has: the same kernel, the same shares, the same bits."""
    g = torch.Generator("cuda").manual_seed(rows)
    lengths = [1 + (r * 37) % 90 for r in range(rows)]
    p, pool = pair(1, 3 * rows, rows, 3, HEADS, dim, 32)
    assert p.reserve(ints(lengths)).tolist() == lengths
    k, v = (torch.randn(sum(lengths), HEADS, dim, device="cuda", generator=g).to(dtype) for _ in range(2))
    p.append(0, k, v, ints([sum(lengths[:r]) for r in range(rows + 1)]))
    q = torch.randn(rows, HEADS * GROUP, dim, device="cuda", generator=g).to(dtype)      # 32,768 columns and heads, and more
    starts = ints(list(range(rows + 1)))
    plain = p.attend(0, q)
    assert torch.equal(plain, p.attend(0, q, starts, 1))
    assert torch.equal(plain, p.attend(0, q, starts))
    assert torch.equal(plain, p.attend(0, q, starts, rows))


NEW = {"long": [600, 1, 3, 8, 0, 9, 1], "some": [500, 8, 9, 1, 7, 40, 2], "first": [1, 1, 0, 2, 560, 1, 8], "ones": [70, 1, 1] + [1] * 450}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", list(NEW.values()), ids=list(NEW))
@pytest.mark.parametrize("dim", [64, 100, 160, 256])
def test_mixed(dim, new, dtype):
    """8 tokens of a row are 64 columns, 9 are not; rows behind up to 2,100 places beside ones of nothing else."""
    behind = [5, 2100, 90, 0, 40, 700, 33]
    lengths = [n + behind[r % 7] * (r < 7) for r, n in enumerate(new)]
    p, pool = pair(1, sum(-(-n // 32) for n in lengths) + 2, len(new), 80, HEADS, dim, 32)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    fill(p, pool, lengths, dim, 0, dtype)
    check(p, pool, new, dtype, 1)
    check(p, pool, new, dtype, 2, window=45, out_dtype=torch.float32, most=max(new))
    check(p, pool, new, dtype, 3, strided=True, most=max(new))
    # rows that are not there are not written, in either kernel
    q = torch.randn(sum(new), HEADS * GROUP, dim, device="cuda").to(dtype)
    starts = [sum(new[:r]) for r in range(len(new) + 1)]
    out = torch.full_like(q, 7.0)
    p.attend(0, q, ints(starts[:1] + [-1] + starts[2:]), out=out)
    assert bool((out[:starts[2]] == 7).all()) and bool((out[starts[2]:] != 7).any(2).any(1).all())
