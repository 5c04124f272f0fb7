"""How many bits attention over pages keeps of weights and queries: every token attends to two places through one element of its head, so that little but the parts
that weights and queries are taken in stands between an output and the definition in 64 bits."""
import pytest
import torch

from tests import pages_reference as ref
from tests.test_gpu_pages import ints, pair

HEADS, GROUP = 8, 8


def bound(parts, reach):
    """Relative to the sum of |weight| |value|.
      weights in n parts: of a number from 2^e on, below 2^(e + 1), bf16's steps are 2^(e - 7), so the first part leaves at most half of one, 2^(e - 8), of either sign.
            Numbers below 2^(e - 8) have steps of 2^(e - 16) at most, so the next part leaves 2^(e - 17), and each further one 2^-9 of that: 2^-(9n - 1) of the number;
            with fp32 queries, in as many parts, as much of the score, reach at most;
      fp32's share, in steps of 2^-24: a score (sums of the parts' products 3, the factor and its product 2, the exponent's sum 1, the reference's own product 1) 7 of reach; the
      exponential 2; the factor of a reference that moved 3; sums of values' products and of weights, two or three parts of two tokens each, over four waves and
      their factors: 6 and 6; the quotient and its product 3."""
    taken = 2.0 ** -(9 * parts - 1) * (1 + (reach if parts > 2 else 0))
    return taken + (7 * reach + 20) * 2.0 ** -24


def in_parts(x, n):
    """x as the sum of n bf16 numbers."""
    out, rest = torch.zeros_like(x), x.clone()
    for _ in range(n):
        part = rest.float().bfloat16().double()
        out, rest = out + part, rest - part
    return out


def two_places(s, v, parts):
    """Outputs and sums of |weight| |value| of two places' scores [..., 2] and values [..., 2], the weights in parts (0: as they are)."""
    w = torch.exp(s - s.amax(-1, keepdim=True))
    u = in_parts(w, parts) if parts else w
    return (u * v).sum(-1) / w.sum(-1), (w * v.abs()).sum(-1) / w.sum(-1)


def test_bounds_tell_the_parts_apart():
    """Weights in one part less than there should be pass neither bound, weights in as many do."""
    g = torch.Generator().manual_seed(1)
    s = torch.rand(200000, 2, dtype=torch.float64, generator=g)
    v = torch.randn(200000, 2, dtype=torch.float64, generator=g)
    want, size = two_places(s, v, 0)
    for parts in (2, 3):
        assert bool(((two_places(s, v, parts)[0] - want).abs() <= size * bound(parts, 1.0)).all())
        assert not bool(((two_places(s, v, parts - 1)[0] - want).abs() <= size * bound(parts, 1.0)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new,cap", [([1] * 8, 20), ([1] * 8, 200), ([8, 5, 13, 1, 8, 11, 8, 12], 200), ([130, 5, 64, 1, 33, 40], 20), ([130, 5, 64, 1, 33, 200], 20),
                                     ([130, 5, 64, 1, 33, 400], 200)],
                         ids=["one", "one-long-table", "some", "prompts-17472", "prompts-27712", "prompts-40512"])
@pytest.mark.parametrize("dim", [1, 64, 96, 128, 160, 192, 256])
def test_parts_of_weights_and_queries(dim, new, cap, dtype):
    lengths = [n + m for n, m in zip(new, [40, 31, 2, 70, 33, 5, 64, 1])]
    p, pool = pair(1, 80, len(new), cap, HEADS, dim, 32)
    assert p.reserve(ints(lengths)).tolist() == pool.reserve(lengths) == lengths
    g = torch.Generator("cuda").manual_seed(dim)
    total = sum(lengths)
    k = torch.zeros(total, HEADS, dim, device="cuda")
    k[:, :, 0] = torch.randn(total, HEADS, device="cuda", generator=g).clamp(-1, 1)
    v = torch.randn(total, HEADS, dim, device="cuda", generator=g)
    first = [sum(lengths[:r]) for r in range(len(new) + 1)]
    p.append(0, k, v, ints(first))
    pool.append(0, k.cpu(), v.cpu(), lengths)
    q = torch.zeros(sum(new), HEADS * GROUP, dim, device="cuda")
    q[:, :, 0] = torch.randn(sum(new), HEADS * GROUP, device="cuda", generator=g).clamp(-1, 1)
    q = q.to(dtype)
    starts = ints([sum(new[:r]) for r in range(len(new) + 1)])
    got = p.attend(0, q, starts, max(new), 1.0, 2, torch.float32).double().cpu()
    at = 0
    for r, n in enumerate(new):
        kv = pool.values(0, r)
        place = lengths[r] - n + torch.arange(n)
        pairs = torch.stack([place - 1, place], 1)                                      # (every token has one before it)
        kk, vv = (x[:, pairs] for x in kv)                                              # [heads, n, 2, dim]
        x = q[at:at + n, :, 0].double().cpu().view(n, HEADS, GROUP).permute(1, 2, 0)    # [heads, group, n]
        s = x[..., None] * kk[:, None, :, :, 0]                                         # [heads, group, n, 2]
        want, size = two_places(s[..., None, :], vv.transpose(2, 3)[:, None], 0)        # [heads, group, n, dim]
        off = (got[at:at + n].view(n, HEADS, GROUP, dim).permute(1, 2, 0, 3) - want).abs()
        limit = size * bound(2 if dtype == torch.bfloat16 else 3, float(s.abs().max()))
        assert bool((off <= limit).all()), (r, float((off / limit).max()))
        at += n
