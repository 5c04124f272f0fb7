"""Rotary positions on the GPU against the formula in 64 bits."""
import pytest
import torch

from paper_2002_02645_amd import binding
from tests import pages_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cache():
    c = binding.FreezeCache(1)
    yield c
    c.close()


def _close(got, want, x, factor, dtype):
    # Two products and a sum in fp32, the sine and cosine of an angle that fp64 holds to 2^-52 of its turns (10^6 radians: 2^-33) and fp32 to 2^-24 of a
    # turn (2 pi 2^-25 radians after rounding, then the functions' own two units): under 8 * 2^-24 of |x_a| + |x_b|, then the output's rounding.
    size = x.abs().amax(-1, keepdim=True).double().cpu() * 2 * abs(factor)
    bound = 8 * 2.0 ** -24 * size + want.abs() * torch.finfo(dtype).eps / 2
    assert bool(((got.double().cpu() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,pairs", [(1, 1, 2, 1), (1, 8, 128, 64), (5, 3, 70, 17), (33, 2, 64, 32), (7, 5, 37, 18), (3, 1, 256, 0), (130, 4, 96, 24), (2, 3, 4096, 2048)])
def test_rotate(cache, tokens, heads, dim, pairs, interleaved, dtype):
    g = torch.Generator("cuda").manual_seed(tokens * 1000 + dim)
    x = torch.randn(tokens, heads, dim, device="cuda", generator=g).to(dtype)
    positions = torch.randint(-5, 1000000, (tokens,), device="cuda", generator=g, dtype=torch.int32)
    positions[0] = 0
    f = binding.rotary_frequencies(pairs)
    for inverse in (False, True):
        got = cache.rotate_positions(x, positions, f, interleaved, 1.25, inverse)
        want = ref.rotate(x.double().cpu(), positions.cpu(), f.cpu(), interleaved, 1.25, inverse)
        _close(got, want, x, 1.25, dtype)
        assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])
    if not pairs:
        assert torch.equal(got, x)


def test_largest_places(cache):
    positions = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1], device="cuda", dtype=torch.int32)
    f = torch.tensor([1.0, 0.37, 1e-9], dtype=torch.float64, device="cuda")
    x = torch.randn(3, 2, 6, device="cuda")
    _close(cache.rotate_positions(x, positions, f), ref.rotate(x.double().cpu(), positions.cpu(), f.cpu(), False), x, 1.0, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_several_strided_in_place_and_misaligned(cache, dtype, interleaved):
    tokens, dim = 19, 64
    big = torch.randn(tokens, 12 * dim + 5, device="cuda").to(dtype)
    f = binding.rotary_frequencies(16, stretch=4.0, trained=64)
    positions = torch.arange(tokens, device="cuda", dtype=torch.int32)
    before = big.clone()
    for shift in (0, 1, 5):
        big.copy_(before)
        q = big[:, shift:shift + 8 * dim].view(tokens, 8, dim)
        k = big[:, shift + 8 * dim:shift + 10 * dim].view(tokens, 2, dim)
        turned = cache.rotate_positions((q, k.transpose(0, 1).contiguous().transpose(0, 1)), positions, f, interleaved)
        cache.rotate_positions((q, k), positions, f, interleaved, out=(q, k))
        assert torch.equal(q, turned[0]) and torch.equal(k, turned[1])
        assert torch.equal(big[:, :shift], before[:, :shift]) and torch.equal(big[:, shift + 10 * dim:], before[:, shift + 10 * dim:])
        _close(q, ref.rotate(before[:, shift:shift + 8 * dim].reshape(tokens, 8, dim).double().cpu(), positions.cpu(), f.cpu(), interleaved), q, 2.0, dtype)


def test_inverse_is_the_gradient(cache):
    """<R x, y> = <x, R^T y>, against differences of a pass too."""
    f, positions = binding.rotary_frequencies(20), torch.arange(9, device="cuda", dtype=torch.int32) * 77
    x, y = torch.randn(9, 3, 48, device="cuda"), torch.randn(9, 3, 48, device="cuda")
    forward = lambda t: cache.rotate_positions(t, positions, f, factor=0.75)
    grad = cache.rotate_positions(y, positions, f, factor=0.75, inverse=True).double()
    grad[..., 40:] = y[..., 40:].double()
    a, b = (forward(x).double() * y.double()).sum(), (x.double() * grad).sum()
    size = (x.abs().double() * y.abs().double()).sum() * 2
    assert abs(float(a - b)) <= 16 * 2.0 ** -24 * float(size)
    d = torch.zeros_like(x)
    d[4, 1, 7] = 1.0      # linear: a difference of one is the derivative
    rise = ((forward(x + d) - forward(x)).double() * y.double()).sum()
    assert abs(float(rise - grad[4, 1, 7])) <= 64 * 2.0 ** -24 * float((x[4, 1].abs().max() + 1) * y[4, 1].abs().sum())


def test_not_finite_stays_in_its_pair(cache):
    x = torch.randn(3, 2, 32, device="cuda")
    x[1, 0, 3] = float("nan")
    x[2, 1, 5] = float("inf")
    f, positions = binding.rotary_frequencies(16), torch.tensor([0, 3, 9], device="cuda", dtype=torch.int32)
    y = cache.rotate_positions(x, positions, f)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, 0, [3, 19]] = True
    want[2, 1, [5, 21]] = True
    assert torch.equal(bad, want)


def test_nothing_to_do(cache):
    f, none = binding.rotary_frequencies(2), torch.empty(0, dtype=torch.int32, device="cuda")
    assert cache.rotate_positions(torch.empty(0, 3, 8, device="cuda"), none, f).shape == (0, 3, 8)
    assert cache.rotate_positions(torch.empty(2, 0, 8, device="cuda"), none.new_zeros(2), f).shape == (2, 0, 8)
    assert cache.rotate_positions((), none, f) == []


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(128, 64), (72, 36), (100, 50), (66, 33), (80, 36), (68, 18), (34, 14), (22, 0), (33, 16)])
def test_every_piece(cache, dim, pairs, interleaved, dtype):
    """Heads that come in pieces of 16, 8 or 4 bytes or by elements, from addresses of every alignment, into others: the same bytes."""
    tokens, heads = 21, 3
    x = torch.randn(tokens, heads, dim, device="cuda").to(dtype)
    positions, f = torch.arange(tokens, device="cuda", dtype=torch.int32) * 5, binding.rotary_frequencies(pairs)
    want = None
    for row in (dim, dim + 1, dim + 2, dim + 4):
        for shift in (0, 1, 2, 4):
            src = torch.zeros(tokens * heads * row + 8, device="cuda", dtype=dtype)
            dst = torch.full_like(src, 7.0)
            view = lambda t: t[shift:shift + tokens * heads * row].view(tokens, heads, row)[:, :, :dim]
            view(src).copy_(x)
            cache.rotate_positions(view(src), positions, f, interleaved, out=view(dst))
            if want is None:
                want = view(dst).clone()
                _close(want, ref.rotate(x.double().cpu(), positions.cpu(), f.cpu(), interleaved), x, 1.0, dtype)
            assert torch.equal(view(dst), want), (row, shift)
            view(dst).fill_(7.0)
            assert bool((dst == 7).all())
