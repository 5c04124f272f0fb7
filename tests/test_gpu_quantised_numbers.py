"""What numbers the dense layer in 8 bits gives: sums that cancel, bf16 outputs, infinities and no numbers, the smallest values."""
import pytest
import torch

from paper_2002_02645_amd import binding

pytestmark = pytest.mark.gpu


def _noise(rows, d, seed):
    return torch.randn(rows, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("b,d,m", [(1, 4096, 1000), (40, 1000, 131), (150, 700, 259), (300, 1100, 258), (1100, 1024, 1040), (2500, 1152, 1032),
                                   (1000, 515, 4104), (4096, 2048, 2048)])
@pytest.mark.parametrize("relu", [False, True])
def test_bf16_outputs_are_the_fp32_ones_rounded(b, d, m, relu):
    x, w = _noise(b, d, b + d) * torch.where(_noise(1, d, 5).abs() > 2.3, 20.0, 1.0), _noise(m, d, m) / d ** 0.5
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w, torch.linspace(-1, 1, m, device="cuda"))
        want = fc.quantised_project(0, x, relu=relu).to(torch.bfloat16)
        got = fc.quantised_project(0, x, relu=relu, out_dtype=torch.bfloat16)
        assert torch.equal(got, want), (got != want).float().mean().item()
    finally:
        fc.close()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_sums_that_cancel(out):
    # Each output: neighbours 1 and -1 times 448, which cancel, beside products of 2^-9 * k: whole numbers of 2^-9 below 2^24, so that every
    # order of fp32 sums of exact products gives them without rounding
    b, d, m = 4096, 512, 2048
    x = torch.zeros(b, d, device="cuda")
    x[:, 0::8], x[:, 1::8] = 448.0, -448.0
    x[:, 2::8] = 2.0 ** -9 * (1 + torch.arange(b, device="cuda") % 7).view(-1, 1)
    w = torch.zeros(m, d, device="cuda")
    w[:, 0::8], w[:, 1::8], w[:, 2::8] = 1.0, 1.0, 1.0
    w[:, 3] = 448.0   # (x: zero) every block's exponent is 0
    want = (x.double() @ w.double().t().contiguous()).to(out)
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w)
        assert torch.equal(fc.quantised_project(0, x, out_dtype=out), want)
    finally:
        fc.close()


@pytest.mark.parametrize("m,d", [(8192, 8192), (32768, 4096)])
def test_one_workspace_for_a_batch_that_shrinks(m, d):
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, _noise(m, d, 1))
        ws = torch.empty(binding.freeze_quantised_workspace_bytes(fc.ctx, 0, 400, binding.FREEZE_F32), dtype=torch.uint8, device="cuda")
        x = _noise(400, d, 2)
        for b in (400, 375, 257, 256, 129, 39, 33, 17, 1):
            for out in (torch.full((b, m), 7.0, device="cuda"), torch.full((b, m), 7.0, device="cuda", dtype=torch.bfloat16)):
                binding.freeze_quantised_project(fc.ctx, 0, x[:b], None, d, False, out, ws)
                assert torch.equal(out, fc.quantised_project(0, x[:b].clone(), out_dtype=out.dtype))
    finally:
        fc.close()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,d,m", [(1, 256, 40), (7, 256, 500), (9, 4097, 200), (70, 300, 300), (300, 1024, 1000), (2100, 512, 1032)])
def test_no_numbers_show_in_their_rows_alone(b, d, m, xt, out):
    inf, nan = float("inf"), float("nan")
    x, w, bias = _noise(b, d, 11), _noise(m, d, 12), torch.linspace(-1, 1, m, device="cuda")
    x = x.to(xt)
    clean = x.clone()
    bad = {b // 2: nan, b - 1: inf, 0: -inf}
    for row, value in bad.items():
        x[row, (row * 37 + 5) % d] = value
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w, bias)
        codes, scales = fc.quantise_rows(x)
        assert (scales[:, :-(-d // 128)].amax(1)[list(bad)] >= 247).all()
        for relu in (False, True):
            want = fc.quantised_project(0, clean, relu=relu, out_dtype=out)
            rows = torch.tensor([r not in bad for r in range(b)], device="cuda")
            for got in (fc.quantised_project(0, x, relu=relu, out_dtype=out), fc.quantised_project(0, codes, scales, relu=relu, out_dtype=out)):
                assert torch.isnan(got[list(bad)]).all() and torch.equal(got[rows], want[rows])
        # in the weights: their output alone, for every row
        w[m // 3, d // 2], w[m - 1, 0] = nan, inf
        fc.build_quantised(0, w, bias)
        got = fc.quantised_project(0, clean, relu=True, out_dtype=out)
        assert torch.isnan(got[:, [m // 3, m - 1]]).all()
        keep = torch.tensor([c not in (m // 3, m - 1) for c in range(m)], device="cuda")
        assert torch.equal(got[:, keep], want[:, keep])
        # (a bias that is no number; infinite outputs)
        bias[3], w[:] = nan, 1.0
        w[5], w[6] = 3e38, -3e38
        fc.build_quantised(0, w, bias)
        got = fc.quantised_project(0, torch.full((b, d), 4.0, device="cuda").to(xt), relu=True, out_dtype=out)
        assert torch.isnan(got[:, 3]).all() and (got[:, 5] == inf).all() and (got[:, 6] == 0).all()
    finally:
        fc.close()


@pytest.mark.parametrize("b", [1, 40, 300])
def test_the_ends_of_the_range(b):
    """Values below 2^-126 count as the nearest multiple of 2^-133 (off by 2^-134 at most), beside weights that make them matter; a row of fp32's
    largest numbers is held as 2^128."""
    d, m = 512, 260
    w = _noise(m, d, 3)
    w = w.clamp(-3.5, 3.5) * 2.0 ** 100
    x = _noise(b, d, 4) * torch.exp2(torch.tensor([-118.0, -120.0, -124.0, -128.0], device="cuda")).repeat_interleave(128)
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w)
        values = []
        for t in (x, w):
            codes, scales = fc.quantise_rows(t)
            values.append((codes.double().view(-1, d // 128, 128) * torch.exp2(scales.double() - 127).unsqueeze(2)).view(-1, d))
        xv, wv = values
        assert ((xv != 0) & (xv.abs() < 2.0 ** -130)).any()
        y, size = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
        # d / 32 + 16 roundings of fp32 sums, and what the smallest values lose
        tol = (16 + d / 32) * 2.0 ** -24 * size + 2.0 ** -134 * wv.abs().sum(1)
        off = (fc.quantised_project(0, x).double() - y).abs()
        assert (off <= tol).all(), (off / tol).max().item()
        nearest = torch.where(xv.abs() < 2.0 ** -126, torch.round(xv * 2.0 ** 133) * 2.0 ** -133, xv)
        off = (fc.quantised_project(0, x).double() - nearest @ wv.t().contiguous()).abs()
        assert (off <= (16 + d / 32) * 2.0 ** -24 * size).all()
        fc.build_quantised(0, torch.full((m, d), 2.0 ** -100, device="cuda"))
        assert (fc.quantised_project(0, torch.full((b, d), torch.finfo(torch.float32).max, device="cuda")) == float("inf")).all()
        large = torch.full((b, d), 240.0 * 2.0 ** 120, device="cuda")
        assert (fc.quantised_project(0, large) == d * 240.0 * 2.0 ** 20).all()
    finally:
        fc.close()
