"""The choice of the next tokens over beams and vocabulary, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2002_02645_amd import binding
from tests import decode_reference as ref

pytestmark = pytest.mark.gpu

INF = float("inf")
# log of a sum of fp32 exponentials: two units in the last place each, a sum of 32 a lane and batch, its rescaling: 40 * 2^-24
NEAR = 4e-6


def _check(logits, scores, finished, beams, k, end, out):
    want = ref.beam_select(logits.double().cpu().numpy(), scores.double().cpu().numpy(),
                           None if finished is None else finished.cpu().numpy(), beams, end, k)
    got = {key: v.cpu().numpy() for key, v in out.items()}
    vocab = logits.shape[1]
    for g, best in enumerate(want):
        seen = set()
        for i, (total, row, token) in enumerate(best):
            s, r, t = got["score"][g, i], int(got["parent"][g, i]), int(got["token"][g, i])
            assert 0 <= t < vocab and g * beams <= r < (g + 1) * beams
            assert bool(got["finished"][g, i]) == (t == end)
            if total == -INF:
                assert s == -INF and (r, t) == (row, token)
                continue
            assert (r, t) not in seen
            seen.add((r, t))
            assert abs(s - total) <= NEAR + 2.0 ** -24 * abs(total), (g, i, s, total)
            if (r, t) != (row, token):
                # another one only where rows' totals cannot be told apart
                same = [c for c in best if (c[1], c[2]) == (r, t)]
                assert row != r or same, (g, i, (r, t), (row, token))
                assert not same or abs(same[0][0] - total) <= 2 * NEAR
        order = got["score"][g]
        assert (order[:-1] >= order[1:]).all()


def _run(logits, scores, beams, k, finished=None, end=-1):
    fc = binding.FreezeCache(1)
    try:
        out = fc.beam_select(logits, scores, beams, k, finished=finished, end_token=end)
        torch.cuda.synchronize()
    finally:
        fc.close()
    _check(logits, scores, finished, beams, k, end, out)
    return out


def _make(rows, vocab, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g) * 2.5).to(dtype).cuda(), (-8 * torch.rand(rows, generator=g)).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,beams,vocab,k", [
    (1, 1, 1, 1), (1, 1, 1, 5), (2, 3, 2, 4), (1, 4, 5, 8), (3, 2, 63, 4), (1, 5, 64, 64), (2, 1, 1000, 64), (7, 4, 1023, 4),
    (1, 4, 1024, 8), (2, 8, 1025, 16), (1, 64, 300, 64), (1, 3, 4097, 6), (33, 4, 2050, 4), (1, 4, 32000, 4), (2, 8, 50021, 16),
    (1, 2, 131075, 63), (130, 16, 700, 16), (1, 1, 300001, 1),
])
def test_sizes(groups, beams, vocab, k, dtype):
    logits, scores = _make(groups * beams, vocab, dtype, 7 * groups + beams + vocab + k)
    _run(logits, scores, beams, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["equal", "few_values", "rising", "falling", "lowest", "huge_spread"])
def test_orders_and_ties(kind, dtype):
    rows, vocab, beams, k = 8, 5003, 4, 12
    g = torch.Generator().manual_seed(5)
    if kind == "equal":
        x = torch.full((rows, vocab), 1.5)
    elif kind == "few_values":
        x = torch.randint(-3, 3, (rows, vocab), generator=g).float()
    elif kind == "rising":
        x = torch.arange(vocab).float().repeat(rows, 1) / 64
    elif kind == "falling":
        x = -torch.arange(vocab).float().repeat(rows, 1) / 64
    elif kind == "lowest":
        x = torch.randn(rows, vocab, generator=g)
        x[torch.rand(rows, vocab, generator=g) < 0.999] = torch.finfo(dtype).min
        x[3] = torch.finfo(dtype).min
    else:
        x = torch.randn(rows, vocab, generator=g) * 1e4
    scores = -torch.arange(rows).float()   # (rows that differ by their scores alone)
    _run(x.to(dtype).cuda(), scores.cuda(), beams, k)


def test_equal_rows_go_by_row_then_token():
    x = torch.zeros(6, 2048, device="cuda")
    out = _run(x, torch.zeros(6, device="cuda"), 3, 8)
    assert out["token"].cpu().tolist() == [list(range(8))] * 2
    assert out["parent"].cpu().tolist() == [[0] * 8, [3] * 8]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_empty_and_finished_rows(dtype):
    groups, beams, vocab, k, end = 7, 4, 3001, 6, 2
    logits, scores = _make(groups * beams, vocab, dtype, 9)
    g = torch.Generator().manual_seed(10)
    logits[torch.rand(logits.shape, generator=g).cuda() < 0.5] = -INF
    done = torch.zeros(groups * beams, dtype=torch.uint8)
    logits[4:8] = -INF                        # group 1: nothing at all
    logits[8:12] = -INF                       # group 2: three tokens in all
    logits[9, 100], logits[9, 7], logits[11, 2] = 0.5, 0.5, -3.0
    scores[12:15] = -INF                      # group 3: a first step
    done[16:20] = 1                           # group 4: all ended
    scores[17] = -INF
    done[20:22] = 1                           # group 5: two ended, their logits no numbers
    logits[20:22] = float("nan")
    scores[24:28] = -INF                      # group 6: empty
    logits[24] = float("nan")
    _run(logits, scores, beams, k, finished=done.cuda(), end=end)
    logits[20:22] = 0
    logits[24] = 0
    _run(logits, scores, beams, k)
    _run(logits, scores, beams, k, finished=torch.zeros_like(done).cuda(), end=vocab - 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_apart_and_off_alignment(dtype):
    wide, scores = _make(6, 9100, dtype, 12)
    for view in (wide[:, 1:9000], wide[:, 3:4], wide[:, 5:1029], wide[:, 8:8200], wide[:, 2:1026]):
        _run(view, scores, 3, 5)
    _run(wide[::2, 7:7007], scores[::2].contiguous(), 3, 5)


def test_exact_workspace_and_guards():
    for groups, beams, vocab, k, dtype in ((3, 5, 2500, 7, torch.float32), (2, 3, 40000, 64, torch.bfloat16), (90, 8, 1100, 3, torch.bfloat16)):
        logits, scores = _make(groups * beams, vocab, dtype, 13)
        need = binding.freeze_beam_workspace_bytes(groups, beams, vocab, k)
        raw = torch.full((need + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        n = groups * k
        o = torch.full((4, n + 64), -5, dtype=torch.int32, device="cuda")
        fin = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        binding.freeze_beam_select(logits, scores, None, beams, 5, k, o[0, 32:32 + n].view(torch.float32), o[1, 32:32 + n], o[2, 32:32 + n],
                                   fin[32:32 + n], raw[4096:4096 + need])
        torch.cuda.synchronize()
        assert (raw[:4096] == 0xA5).all() and (raw[-4096:] == 0xA5).all()
        assert (o[:, :32] == -5).all() and (o[:, 32 + n:] == -5).all() and (fin[:32] == 0x5A).all() and (fin[32 + n:] == 0x5A).all()
        _check(logits, scores, None, beams, k, 5, dict(score=o[0, 32:32 + n].view(torch.float32).view(groups, k), token=o[1, 32:32 + n].view(groups, k),
                                                      parent=o[2, 32:32 + n].view(groups, k), finished=fin[32:32 + n].view(groups, k)))
        with pytest.raises(binding.FreezeError):
            binding.freeze_beam_select(logits, scores, None, beams, 5, k, o[0, :n].view(torch.float32), o[1, :n], o[2, :n], None,
                                       raw[4096:4096 + need - 256])


def test_logits_beyond_4_gib():
    # 1.2e9 fp32 values: the last group's rows lie behind byte 4.7e9
    groups, beams, vocab, k = 300, 4, 1000003, 5
    logits = torch.zeros(groups * beams, vocab, device="cuda")
    rows = [0, 1, 1073, 1074, 1196, 1197, 1198, 1199]
    for n, r in enumerate(rows):
        logits[r, vocab - 1 - n] = 20.0 + n
        logits[r, n] = 18.0
    scores = torch.zeros(groups * beams, device="cuda")
    fc = binding.FreezeCache(1)
    try:
        out = fc.beam_select(logits, scores, beams, k)
    finally:
        fc.close()
    for g in (0, 268, 299):
        part = slice(g * beams, (g + 1) * beams)
        _check(logits[part], scores[part], None, beams, k, -1, dict(score=out["score"][g:g + 1], token=out["token"][g:g + 1],
                                                                   parent=out["parent"][g:g + 1] - g * beams, finished=out["finished"][g:g + 1]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_large_value_before_many_small_ones(dtype):
    # the small ones are a fifth of the sum, each 4e-7 of the large one
    logits = torch.zeros(4, 500009, device="cuda")
    logits[:, 0] = 14.75
    logits[2, 0] = 0
    logits[2, -1] = 14.75
    _run(logits.to(dtype), torch.zeros(4, device="cuda"), 2, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_whole_rows_to_a_wave(dtype):
    # 4,000 rows: a piece is a row of several runs of batches; the best ones last, first, spread, all alike, and within one load
    groups, beams, vocab, k = 1000, 4, 50021, 6
    g = torch.Generator(device="cuda").manual_seed(12)
    logits = torch.randn(groups * beams, vocab, generator=g, device="cuda").to(dtype)
    logits[0] = torch.linspace(-9, 9, vocab).to(dtype)
    logits[1] = torch.linspace(9, -9, vocab).to(dtype)
    logits[2] = 0.5
    logits[3] = torch.where(torch.arange(vocab) % 4001 == 17, 4.0, -1.0).to(dtype)
    logits[3996, 16384 * 2 + 8:16384 * 2 + 16] = 7.0
    logits[3997, :] = -INF
    logits[3997, 50020] = -2.0
    logits[3998, vocab // 2:] = -INF
    scores = -torch.rand(groups * beams, generator=g, device="cuda")
    fc = binding.FreezeCache(1)
    try:
        out = fc.beam_select(logits, scores, beams, k)
    finally:
        fc.close()
    for n in (0, 500, 999):
        part = slice(n * beams, (n + 1) * beams)
        _check(logits[part], scores[part], None, beams, k, -1, dict(score=out["score"][n:n + 1], token=out["token"][n:n + 1],
                                                                   parent=out["parent"][n:n + 1] - n * beams, finished=out["finished"][n:n + 1]))


@pytest.mark.parametrize("seed", range(12))
def test_random_sizes(seed):
    rng = np.random.RandomState(100 + seed)
    beams, vocab = int(rng.choice([1, 2, 3, 5, 8, 16, 33])), int(2 ** rng.uniform(0, 15.5))
    groups, k = int(2 ** rng.uniform(0, 5)), int(rng.choice([1, 2, beams, 2 * beams, 64]))
    k = min(k, 64)
    dtype = [torch.float32, torch.bfloat16][seed % 2]
    logits, scores = _make(groups * beams, vocab, dtype, 200 + seed)
    g = torch.Generator().manual_seed(300 + seed)
    if rng.rand() < 0.6:
        logits[torch.rand(logits.shape, generator=g).cuda() < rng.uniform(0, 1)] = -INF
    done = (torch.rand(groups * beams, generator=g) < 0.2).to(torch.uint8).cuda()
    scores[torch.rand(groups * beams, generator=g).cuda() < 0.1] = -INF
    _run(logits, scores, beams, k, finished=done, end=int(rng.randint(vocab)))


def test_replays_and_other_streams():
    groups, beams, vocab, k = 3, 4, 20000, 8
    sets = [_make(groups * beams, vocab, torch.float32, 20 + i) for i in range(3)]
    fc = binding.FreezeCache(1)
    try:
        want = [{key: v.clone() for key, v in fc.beam_select(l, s, beams, k, end_token=3).items()} for l, s in sets]
        logits, scores = sets[0][0].clone(), sets[0][1].clone()
        ws = torch.empty(binding.freeze_beam_workspace_bytes(groups, beams, vocab, k), dtype=torch.uint8, device="cuda")
        out = {key: torch.empty_like(v) for key, v in want[0].items()}

        def call(stream=None):
            binding.freeze_beam_select(logits, scores, None, beams, 3, k, out["score"], out["token"], out["parent"], out["finished"], ws,
                                       stream=stream)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        call(side)
        side.synchronize()
        assert all(torch.equal(out[key], want[0][key]) for key in out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for i in (1, 2, 0, 1):
            logits.copy_(sets[i][0])
            scores.copy_(sets[i][1])
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[key], want[i][key]) for key in out)
            again = fc.beam_select(*sets[i], beams, k, end_token=3)
            assert all(torch.equal(again[key], want[i][key]) for key in out)
    finally:
        fc.close()
