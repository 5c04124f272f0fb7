"""The operators of a generating model together, as its decoding uses them: prompts, then steps over beams (rotary positions, appending, attention, the 8-bit
output layer, the choice of tokens, the pages following the chosen parents); captured steps; several streams."""
import pytest
import torch

from paper_2002_02645_amd import binding
from tests import pages_reference as ref
from tests.test_gpu_pages import ints, pair, same_book

pytestmark = pytest.mark.gpu

LAYERS, HEADS, GROUP, DIM, VOCAB, BEAMS, GROUPS = 2, 2, 2, 64, 97, 3, 2
ROWS, WIDTH = BEAMS * GROUPS, HEADS * GROUP * DIM


class Model:
    def __init__(self, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, device="cuda", generator=g)
        self.embed = rand(VOCAB, WIDTH)
        self.qkv = [(rand(WIDTH, WIDTH + 2 * HEADS * DIM) / WIDTH ** 0.5).to(torch.bfloat16) for _ in range(LAYERS)]
        self.cache = binding.FreezeCache(1)
        self.cache.build_quantised(0, rand(VOCAB, WIDTH) * 0.3)
        self.frequencies = binding.rotary_frequencies(DIM // 2)

    def step(self, pages, tokens, positions, starts=None, most=0, seen=None):
        """Hidden rows of the tokens; seen(layer, q, k, v, out) is shown what a layer computed."""
        x = self.embed[tokens]
        n = x.shape[0]
        for layer in range(LAYERS):
            # (the heads lie side by side in one buffer and are turned in place)
            qkv = (x.to(torch.bfloat16) @ self.qkv[layer]).view(n, HEADS * (GROUP + 2), DIM)
            q, k, v = qkv.split([HEADS * GROUP, HEADS, HEADS], 1)
            self.cache.rotate_positions((q, k), positions, self.frequencies, out=(q, k))
            pages.append(layer, k, v, starts, most)
            out = pages.attend(layer, q, starts, most, out_dtype=torch.float32)
            if seen:
                seen(layer, q, k, v, out)
            x = x + out.reshape(n, WIDTH)
        return x


def test_decoding_with_beams():
    model = Model(1)
    p, pool = pair(LAYERS, 60, ROWS, 6, HEADS, DIM, 32)
    worst = []

    def seen(new):
        def check(layer, q, k, v, out):
            pool.append(layer, k.cpu(), v.cpu(), new)
            want = pool.attend(layer, q.cpu(), new, GROUP, DIM ** -0.5)
            worst.append(float((out.double().cpu() - want).abs().max() / want.abs().max()))
        return check

    # prompts of the groups' first beams, the others go on from them
    new = [0] * ROWS
    new[0], new[BEAMS] = 41, 17
    assert p.reserve(ints(new)).tolist() == pool.reserve(new) == new
    starts = ints([sum(new[:r]) for r in range(ROWS + 1)])
    tokens = torch.randint(0, VOCAB, (sum(new),), device="cuda")
    x = model.step(p, tokens, torch.cat([torch.arange(41), torch.arange(17)]).int().cuda(), starts, 41, seen(new))
    first = [r // BEAMS * BEAMS for r in range(ROWS)]
    p.fork(ints(first))
    pool.fork(first)
    rows = x[torch.tensor([40, 57], device="cuda")].repeat_interleave(BEAMS, 0)
    scores = torch.full((ROWS,), -float("inf"), device="cuda")
    scores[::BEAMS] = 0
    for _ in range(40):
        best = model.cache.beam_select(model.cache.quantised_project(0, rows), scores, BEAMS, BEAMS)
        parents, scores = best["parent"].view(-1), best["score"].reshape(-1)
        p.fork(parents)
        pool.fork(parents.tolist())
        positions = p.lengths.clone()
        assert p.reserve().tolist() == pool.reserve([1] * ROWS) == [1] * ROWS
        rows = model.step(p, best["token"].view(-1).long(), positions, seen=seen([1] * ROWS))
        same_book(p, pool)
    # weights rounded to bf16 (2^-9 of each on average at most), codes alike: outputs within 2^-7 of the largest
    assert max(worst) < 2.0 ** -7
    p.truncate(ints([-1, 0, 0] * GROUPS))
    pool.truncate([-1, 0, 0] * GROUPS)
    assert p.compact().tolist() == [pool.compact()]
    same_book(p, pool)
    model.cache.close()


def _step(model, p, parents, q, k, v, granted):
    p.fork(parents)
    positions = p.lengths.clone()
    granted.copy_(p.reserve())
    q, k = model.cache.rotate_positions((q, k), positions, model.frequencies)
    for layer in range(LAYERS):
        p.append(layer, k, v, granted=granted)
    return p.attend(0, q), p.attend(1, q, window=20)


def _grown(seed):
    p = binding.FreezePages(LAYERS, 80, ROWS, 8, HEADS, DIM, 32)
    new = [60, 3, 33, 0, 31, 64]
    p.reserve(ints(new))
    g = torch.Generator("cuda").manual_seed(seed)
    k, v = (torch.randn(sum(new), HEADS, DIM, device="cuda", generator=g) for _ in range(2))
    for layer in range(LAYERS):
        p.append(layer, k, v, ints([sum(new[:r]) for r in range(ROWS + 1)]))
    return p


def test_captured_steps():
    """A whole step in a graph, replayed beside eager steps of another pool with the same inputs, eager work of the graph's own holder between the replays."""
    model = Model(2)
    a, b = _grown(5), _grown(5)
    g = torch.Generator("cuda").manual_seed(9)
    q = torch.zeros(ROWS, HEADS * GROUP, DIM, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.zeros(ROWS, HEADS, DIM, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    parents, granted = torch.arange(ROWS, device="cuda", dtype=torch.int32), torch.zeros(ROWS, dtype=torch.int32, device="cuda")
    start = a.book.clone(), a.codes.clone(), a.scales.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(model, a, parents, q, k, v, granted)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(model, a, parents, q, k, v, granted)
    a.book.copy_(start[0])
    a.codes.view(torch.uint8).copy_(start[1].view(torch.uint8))
    a.scales.copy_(start[2])
    for step in range(70):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        parents.copy_(torch.randint(0, ROWS, (ROWS,), device="cuda", generator=g))
        graph.replay()
        got = [t.clone() for t in out] + [granted.clone()]
        a.attend(0, q)                                     # eager work of the same holder
        other = torch.zeros_like(granted)
        want = list(_step(model, b, parents, q, k, v, other)) + [other]
        if step % 7 == 0:
            torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), step
        for x, y in ((a.book, b.book), (a.scales, b.scales)):
            assert torch.equal(x, y), step
    assert torch.equal(a.codes.view(torch.uint8)[:, a.refs > 0], b.codes.view(torch.uint8)[:, a.refs > 0])
    model.cache.close()


def test_two_streams_and_two_graphs():
    """Calls of one holder on two streams at once, and replays of two graphs of it, share no scratch memory."""
    p = binding.FreezePages(1, 700, 2, 320, 4, 64, 32)
    p.reserve(ints([10000, 10000]))
    k, v = (torch.randn(20000, 4, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    p.append(0, k, v, ints([0, 10000, 20000]))
    qs = [torch.randn(2, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    want = [p.attend(0, q) for q in qs]
    torch.cuda.synchronize()
    streams, outs, graphs = [torch.cuda.Stream() for _ in qs], [torch.empty_like(q) for q in qs], []
    for q, o in zip(qs, outs):
        p.attend(0, q, out=o)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.attend(0, q, out=o)
        graphs.append(graph)
    for turn in range(20):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                graphs[i].replay() if turn % 2 else p.attend(0, qs[i], out=outs[i])
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


def test_refused_by_the_holder():
    p, cache = binding.FreezePages(1, 8, 2, 2, 2, 32, 32), binding.FreezeCache(1)
    x = torch.randn(2, 2, 32, device="cuda")
    f, at = binding.rotary_frequencies(16), ints([0, 1])
    refused = [lambda: p.append(0, x.cpu(), x), lambda: p.append(0, x, x.bfloat16()), lambda: p.append(0, x[:, :1], x[:, :1]), lambda: p.append(0, x.half(), x.half()),
               lambda: p.append(0, x.transpose(1, 2), x), lambda: p.append(0, x, x, ints([0, 1])), lambda: p.append(0, x, x, granted=ints([1])),
               lambda: p.attend(0, x[..., :16]), lambda: p.attend(0, x[:, :1]), lambda: p.attend(0, x, out=x.new_empty(2, 2, 31)), lambda: p.attend(0, x, ints([0, 1, 2]).long()),
               lambda: p.attend(0, x.half()), lambda: p.reserve(ints([1])), lambda: p.reserve(torch.ones(2, device="cuda")), lambda: p.fork(ints([1, 1, 1])),
               lambda: p.truncate(torch.zeros(2, dtype=torch.int32)), lambda: cache.rotate_positions(x, at.long(), f), lambda: cache.rotate_positions(x, at, f.float()),
               lambda: cache.rotate_positions(x, ints([0]), f), lambda: cache.rotate_positions(x, at, binding.rotary_frequencies(17)), lambda: cache.rotate_positions(x.half(), at, f),
               lambda: cache.rotate_positions(x, at, f, out=x[:1]), lambda: cache.rotate_positions((x, x[..., :16]), at, f)]
    for call in refused:
        with pytest.raises((AssertionError, KeyError)):
            call()
    for call in (lambda: p.append(1, x, x), lambda: p.append(0, x[:1], x[:1]), lambda: p.attend(1, x), lambda: p.attend(0, x, scale=-1.0), lambda: p.attend(0, x, window=-1),
                 lambda: p.attend(0, x, out=x), lambda: p.append(0, x, x, most=-1), lambda: binding.FreezePages(1, 8, 2, 2, 2, 300), lambda: binding.FreezePages(1, 8, 2, 2, 2, 32, 48)):
        with pytest.raises(binding.FreezeError):
            call()
    cache.close()


def test_far_pages():
    """A layer of more than 4 GiB whose last pages are in use: the same codes and outputs as in a small pool, through appending, copies, attention of each kind and a
    compaction that brings the pages to the front."""
    sizes = dict(rows=3, max_pages=8, heads=8, head_dim=128, page_tokens=64)
    far, near = binding.FreezePages(1, 40000, **sizes), binding.FreezePages(1, 40, **sizes)
    assert far.codes.numel() > 4 << 30
    far.refs[:39970] = 1                                  # somebody else's
    g = torch.Generator("cuda").manual_seed(3)
    k, v = (torch.randn(600, 8, 128, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(600, 64, 128, device="cuda", generator=g).to(torch.bfloat16)
    starts = ints([0, 300, 410, 600])

    def outputs(p):
        return [p.attend(0, q[:3]), p.attend(0, q[:36], ints([0, 12, 24, 36])), p.attend(0, q, starts), p.attend(0, q[:36].float(), ints([0, 12, 24, 36]))]

    for p in (far, near):
        assert p.reserve(ints([300, 110, 190])).tolist() == [300, 110, 190]
        p.append(0, k, v, starts)
    assert int(far.tables.max()) > 39975 and torch.equal(far.tables - 39970, torch.where(near.tables >= 0, near.tables, -1 - 39970))
    for step in range(2):
        assert all(torch.equal(a, b) for a, b in zip(outputs(far), outputs(near)))
        assert torch.equal(far.codes.view(torch.uint8)[:, 39970:39990], near.codes.view(torch.uint8)[:, :20])
        for p in (far, near):                             # shared last pages are copied
            p.fork(ints([0, 0, 1]))
            assert p.reserve().tolist() == [1] * 3
            p.append(0, k[step * 3:step * 3 + 3], v[step * 3:step * 3 + 3])
    want = outputs(far)
    far.refs[:39970] = 0
    assert far.compact().tolist() == near.compact().tolist()
    assert int(far.tables.max()) < 40 and all(torch.equal(a, b) for a, b in zip(outputs(far), want))
