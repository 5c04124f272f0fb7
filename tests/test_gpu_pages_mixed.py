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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured(dtype):
    """Both kernels of a mixed call in a graph, replayed beside eager calls and over other lengths and starts."""
    new = [600, 1, 3, 8, 0, 9, 1]
    lengths = [n + 700 for n in new]
    p, _ = pair(1, 200, 7, 80, HEADS, 64, 32)
    assert p.reserve(ints(lengths)).tolist() == lengths
    g = torch.Generator("cuda").manual_seed(1)
    k, v = (torch.randn(sum(lengths), HEADS, 64, device="cuda", generator=g).to(dtype) for _ in range(2))
    p.append(0, k, v, ints([sum(lengths[:r]) for r in range(8)]))
    q = torch.randn(sum(new), HEADS * GROUP, 64, device="cuda", generator=g).to(dtype)
    starts = ints([sum(new[:r]) for r in range(8)])
    p.attend(0, q, starts)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = p.attend(0, q, starts)
    for turn, order in enumerate((new, [1, 600, 8, 3, 9, 0, 1], [0, 0, 622, 0, 0, 0, 0], new)):
        starts.copy_(ints([sum(order[:r]) for r in range(8)]))
        q.copy_(torch.randn(q.shape, device="cuda", generator=g))
        out.fill_(9.0)
        want = p.attend(0, q, starts)
        graph.replay()
        assert torch.equal(out, want), turn
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(out, want), turn


def test_rows_without_room():
    """A row that got no place for its new token attends from its last old place, as the header says: `granted` tells whose outputs count."""
    p, pool = pair(1, 5, 3, 3, HEADS, 64, 32)
    lengths = [64, 32, 40]
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths      # all five pages
    fill(p, pool, lengths, 1)
    granted = p.reserve()
    assert granted.tolist() == pool.reserve([1, 1, 1]) == [0, 0, 1]
    k, v = (torch.randn(3, HEADS, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    p.append(0, k, v, granted=granted)
    pool.append(0, k.cpu(), v.cpu(), [1, 1, 1], [0, 0, 1])
    check(p, pool, [1, 1, 1], torch.bfloat16, 1)
