"""Rows in 8 bits and the dense layer on them, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2002_02645_amd import binding
from tests import decode_reference as ref

pytestmark = pytest.mark.gpu


def _bits(codes):
    return codes.view(torch.uint8).cpu().numpy()


def _inputs(b, d, dtype, seed, channels=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(b, d, generator=g) * torch.exp(torch.randn(b, 1, generator=g))
    if channels:
        x *= torch.where(torch.rand(1, d, generator=g) < 0.02, 30.0, 1.0)
    return x.to(dtype)


def _check_codes(x, codes, scales):
    want_codes, want_scales = ref.quantise(x.double().cpu().numpy())
    got = _bits(codes)
    # (a value that rounds to nothing may keep its sign or not)
    assert np.array_equal(np.where(got == 128, 0, got), np.where(want_codes == 128, 0, want_codes))
    assert np.array_equal(scales.cpu().numpy(), want_scales)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,d", [(1, 1), (3, 7), (2, 127), (5, 128), (4, 129), (1, 8192), (17, 1000), (33, 517), (9, 2048),
                                 (2, 16391), (300, 384), (1, 65536 + 8)])
def test_codes(b, d, dtype):
    x = _inputs(b, d, dtype, 5 + b + d)
    fc = binding.FreezeCache(1)
    try:
        _check_codes(x, *fc.quantise_rows(x.cuda()))
    finally:
        fc.close()


def test_codes_of_every_kind_of_block():
    rows = []
    for top in (448.0, 448.0 * (1 + 2.0 ** -22), 449.0, 256.0, 255.99, 1.75, 1.7500001, 3.4028234e38, 2.0 ** -126, 1e-40, 1e-45, 0.0, 2.0 ** -118,
                1.75 * 2.0 ** -118, 1.8 * 2.0 ** -118):
        r = torch.zeros(256, dtype=torch.float32)
        # halfway cases of every binade below the top, both signs; subnormal codes; a lone value in the second block
        i = torch.arange(100)
        r[:100] = top * ((17 + 2 * (i % 8)).float() / 32) * torch.exp2(-(i // 8).float()) * (1 - 2 * (i % 2))
        r[100] = top
        r[101:110] = top * 2.0 ** -17 * torch.arange(1, 10)
        r[200] = -top
        rows.append(r)
    x = torch.stack(rows)
    fc = binding.FreezeCache(1)
    try:
        _check_codes(x, *fc.quantise_rows(x.cuda()))
        h = x[:7].to(torch.bfloat16)
        _check_codes(h, *fc.quantise_rows(h.cuda()))
    finally:
        fc.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_of_rows_apart_and_off_alignment(dtype):
    fc = binding.FreezeCache(1)
    try:
        base = _inputs(12, 700, dtype, 3).cuda()
        for view in (base[:, :512], base[:, 1:514], base[1:, 4:300], base[::3, 3:131], base[5:6, 9:20]):
            _check_codes(view, *fc.quantise_rows(view))
    finally:
        fc.close()


def test_codes_stay_within_their_buffers():
    x = _inputs(7, 300, torch.float32, 8).cuda()
    raw = torch.full((7 * 384 + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    raw_s = torch.full((7 * 4 + 32,), 0xA5, dtype=torch.uint8, device="cuda")
    binding.freeze_quantise_rows(x, raw[256:256 + 7 * 384].view(7, 384).view(torch.float8_e4m3fn), raw_s[16:16 + 28].view(7, 4))
    torch.cuda.synchronize()
    assert (raw[:256] == 0xA5).all() and (raw[-256:] == 0xA5).all() and (raw_s[:16] == 0xA5).all() and (raw_s[-16:] == 0xA5).all()


# ---- the dense layer --------------------------------------------------------------------------------

def _tolerance(xv, wv, bias, y, d_pad, out_dtype):
    """fp32: an instruction adds 32 exact products to a sum and rounds; 16 more roundings for its parts, the bias and the sums of cut depths.
    bf16: half a step of the output; the products of eight neighbours cut off 13 bits below the power of two of the largest: 7 * 2^-13 of it
    at most a group, twice that for groups that reach over two exponents."""
    size = xv.abs() @ wv.abs().t().contiguous()
    if bias is not None:
        size = size + bias.abs()
    tol = (16 + d_pad / 32) * 2.0 ** -24 * size
    if out_dtype == torch.bfloat16:
        cut = torch.zeros_like(y)
        w8 = wv.float().view(wv.shape[0], -1, 8)
        for r in range(xv.shape[0]):
            cut[r] = (xv[r].float().view(1, -1, 8) * w8).abs().amax(2).sum(1).double()
        tol = tol + 2.0 ** -8 * (y.abs() + tol) + 14 * 2.0 ** -13 * cut
    return tol + 1e-37


def _check_layer(fc, slot, x, w, bias, relu, out_dtype, given_x, got, d):
    wc, ws = ref.quantise(w.double().cpu().numpy())
    xc, xs = ref.quantise(x.double().cpu().numpy())
    xv, wv = (torch.from_numpy(ref.values(c, s)).cuda() for c, s in ((xc, xs), (wc, ws)))
    y = xv @ wv.t().contiguous()
    if bias is not None:
        y = y + bias.double().cuda()
    tol = _tolerance(xv, wv, None if bias is None else bias.double().cuda(), y, xv.shape[1], out_dtype)
    if relu:
        y = y.clamp(min=0)
    off = (got.double() - y).abs()
    assert torch.isfinite(got).all()
    assert (off <= tol).all(), (off / tol).max().item()


CASES = [
    # b, d, m, x, out, relu, bias, given
    (1, 1, 1, torch.float32, torch.float32, False, True, False),
    (1, 128, 16, torch.float32, torch.float32, False, False, False),
    (2, 129, 17, torch.bfloat16, torch.float32, True, True, False),
    (1, 4096, 1000, torch.bfloat16, torch.float32, False, False, False),
    (1, 16391, 130, torch.float32, torch.bfloat16, False, True, True),
    (5, 1030, 257, torch.float32, torch.float32, False, True, False),
    (15, 2050, 63, torch.bfloat16, torch.bfloat16, True, False, False),
    (16, 512, 128, torch.float32, torch.float32, False, False, True),
    (17, 640, 129, torch.bfloat16, torch.float32, False, True, False),
    (32, 4100, 300, torch.float32, torch.float32, True, True, False),
    (33, 4100, 511, torch.bfloat16, torch.bfloat16, False, True, False),
    (64, 1000, 1025, torch.float32, torch.float32, False, False, True),
    (65, 1000, 1, torch.float32, torch.float32, False, True, False),
    (100, 8192, 100, torch.bfloat16, torch.float32, False, False, False),
    (128, 384, 700, torch.float32, torch.bfloat16, True, True, False),
    (129, 384, 255, torch.bfloat16, torch.float32, False, True, False),
    (200, 20000, 65, torch.bfloat16, torch.float32, False, False, False),
    (255, 900, 256, torch.float32, torch.bfloat16, False, False, True),
    (256, 2048, 257, torch.float32, torch.float32, False, True, False),
    (257, 2048, 511, torch.bfloat16, torch.bfloat16, True, True, False),
    (301, 1639, 1501, torch.float32, torch.float32, False, True, True),
    (513, 130, 1000, torch.bfloat16, torch.bfloat16, False, False, False),
    (700, 5000, 70, torch.float32, torch.float32, True, False, False),
    (1100, 1024, 1040, torch.bfloat16, torch.bfloat16, False, True, False),
    (1100, 1024, 1040, torch.bfloat16, torch.float32, False, True, False),
    (40, 256, 20011, torch.bfloat16, torch.float32, False, False, False),
    (3, 65536, 64, torch.bfloat16, torch.float32, False, True, False),
    (300, 30000, 300, torch.bfloat16, torch.bfloat16, False, True, False),
]


@pytest.mark.parametrize("b,d,m,xt,ot,relu,with_bias,given", CASES)
def test_layer(b, d, m, xt, ot, relu, with_bias, given):
    g = torch.Generator().manual_seed(11 + b + d + m)
    x = _inputs(b, d, xt, 900 + b + d + m)
    w = torch.randn(m, d, generator=g) / d ** 0.5
    bias = torch.randn(m, generator=g) * 0.2 if with_bias else None
    fc = binding.FreezeCache(2)
    try:
        if given:
            wc, ws = fc.quantise_rows(w.cuda())
            fc.build_quantised(1, wc, None if bias is None else bias.cuda(), scales=ws, d=d)
            xc, xs = fc.quantise_rows(x.cuda())
            got = fc.quantised_project(1, xc, xs, relu=relu, out_dtype=ot)
        else:
            fc.build_quantised(1, w.cuda(), None if bias is None else bias.cuda())
            got = fc.quantised_project(1, x.cuda(), relu=relu, out_dtype=ot)
        assert got.dtype == ot
        _check_layer(fc, 1, x, w, bias, relu, ot, given, got, d)
    finally:
        fc.close()


def _values64(x):
    """The values that rows of x are held as, in 64 bits on the GPU (for sizes that numpy takes long for)."""
    rows, d = x.shape
    t = torch.zeros(rows, -(-d // 128) * 128, dtype=torch.float64, device="cuda")
    t[:, :d] = x
    t = t.view(rows, -1, 128)
    e = torch.ceil(torch.log2(t.abs().amax(2, keepdim=True) / 448)).clamp(min=-126)
    t = t / torch.exp2(e)
    step = torch.exp2(torch.frexp(t).exponent.double().clamp(min=-5) - 4)
    return (torch.round(t / step) * step * torch.exp2(e)).view(rows, -1)


def test_the_two_references_agree():
    x = _inputs(20, 700, torch.float32, 2)
    assert torch.equal(_values64(x.cuda()).cpu(), torch.from_numpy(ref.values(*ref.quantise(x.double().numpy()))))


@pytest.mark.parametrize("b,d,m,ot", [
    # every shape of tiles, whole and cut along the depth
    (1466, 64, 16, torch.float32), (3, 1466, 16, torch.float32), (4363, 64, 141, torch.float32), (106, 2553, 273, torch.float32),
    (5442, 68, 291, torch.float32), (5486, 4172, 22, torch.float32), (1, 392, 61910, torch.float32), (18, 5647, 16, torch.float32),
    (4138, 2193, 130, torch.float32), (17, 7390, 5298, torch.float32), (39, 697, 65486, torch.float32), (328, 3871, 2063, torch.float32),
    (73, 64, 32879, torch.float32), (66, 4137, 11021, torch.float32), (144, 70, 33170, torch.float32), (132, 9715, 7318, torch.float32),
    (166, 69, 35740, torch.float32), (176, 7477, 11082, torch.float32), (214, 72, 32799, torch.float32), (194, 8149, 18562, torch.float32),
    (73, 64, 32879, torch.bfloat16), (166, 3941, 3744, torch.bfloat16), (144, 70, 33170, torch.bfloat16), (135, 5904, 11349, torch.bfloat16),
    (214, 72, 32799, torch.bfloat16), (5496, 63304, 27, torch.bfloat16),
    (1000, 515, 4104, torch.bfloat16), (1000, 515, 4104, torch.float32), (2500, 1152, 1032, torch.float32),
])
def test_every_tile(b, d, m, ot):
    x = _inputs(b, d, torch.bfloat16, 70 + b + d).cuda()
    w = _inputs(m, d, torch.bfloat16, 71 + m + d, channels=False).cuda()
    bias = torch.linspace(-1, 1, m, device="cuda")
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w, bias)
        got = fc.quantised_project(0, x, out_dtype=ot)
        again = fc.quantised_project(0, x, out_dtype=ot)
        assert torch.equal(got, again)
        xv, wv = _values64(x), _values64(w)
        y = xv @ wv.t().contiguous() + bias.double()
        tol = _tolerance(xv, wv, bias.double(), y, xv.shape[1], ot)
        off = (got.double() - y).abs()
        assert (off <= tol).all(), (off / tol).max().item()
    finally:
        fc.close()


def test_weights_and_rows_beyond_4_gib():
    # 4.4e9 codes of weights, then as many of rows: the last ones and a few between
    d, n = 8192, 540007
    g = torch.Generator(device="cuda").manual_seed(3)
    codes = torch.randint(0, 0x7F, (n, d), generator=g, dtype=torch.uint8, device="cuda")
    scales = torch.randint(100, 130, (n, 64), generator=g, dtype=torch.uint8, device="cuda")
    few = torch.randn(3, d, generator=g, device="cuda")
    table = torch.from_numpy(np.nan_to_num(ref.CODE_VALUES)).cuda()
    some = torch.tensor([0, 1, 255, 256, 131071, 262144, 300001, 524287, 524288, n - 2, n - 1], device="cuda")
    at = (table[codes[some].long()].view(-1, 64, 128) * torch.exp2(scales[some].double() - 127).unsqueeze(2)).view(-1, d)
    fc = binding.FreezeCache(2)
    try:
        fc.build_quantised(0, codes.view(torch.float8_e4m3fn), scales=scales)
        fc.build_quantised(1, few)
        vf = _values64(few)
        y = vf @ at.t().contiguous()
        tol = _tolerance(vf, at, None, y, d, torch.float32)
        assert ((fc.quantised_project(0, few)[:, some].double() - y).abs() <= tol).all()
        del fc.storage[0]
        got = fc.quantised_project(1, codes.view(torch.float8_e4m3fn), scales)[some]
        assert ((got.double() - y.t()).abs() <= tol.t()).all()
        del codes, scales, got
        x = torch.zeros(n - 400000, d, device="cuda")     # 4.6e9 bytes of fp32
        x[-5:] = torch.randn(5, d, generator=g, device="cuda")
        c, s = fc.quantise_rows(x)
        want = ref.quantise(x[-5:].double().cpu().numpy())
        assert np.array_equal(_bits(c[-5:]), want[0]) and np.array_equal(s[-5:].cpu().numpy(), want[1])
    finally:
        fc.close()


@pytest.mark.parametrize("b,d,m,ot", [(1, 300, 70, torch.float32), (40, 1000, 131, torch.bfloat16), (150, 700, 259, torch.float32),
                                      (300, 1100, 258, torch.bfloat16), (300, 1100, 258, torch.float32)])
def test_rows_apart_exact_workspace_and_guards(b, d, m, ot):
    x = _inputs(b, d + 13, torch.float32, 40 + b)[:, 5:5 + d]
    w = _inputs(m, d, torch.bfloat16, 41 + b, channels=False)
    bias = torch.linspace(-1, 1, m)
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w.cuda(), bias.cuda())
        wide = _inputs(b, d + 13, torch.float32, 40 + b).cuda()
        out = torch.full((b + 2, m + 9), 77.0, dtype=ot, device="cuda")
        need = binding.freeze_quantised_workspace_bytes(fc.ctx, 0, b, binding.FREEZE_F32 if ot == torch.float32 else binding.FREEZE_BF16)
        raw = torch.full((need + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        binding.freeze_quantised_project(fc.ctx, 0, wide[:, 5:5 + d], None, d, False, out[1:b + 1, 3:3 + m], raw[4096:4096 + need])
        torch.cuda.synchronize()
        assert (raw[:4096] == 0xA5).all() and (raw[-4096:] == 0xA5).all()
        edge = torch.ones(b + 2, m + 9, dtype=torch.bool, device="cuda")
        edge[1:b + 1, 3:3 + m] = False
        assert (out[edge] == 77.0).all()
        _check_layer(fc, 0, x, w, bias, False, ot, False, out[1:b + 1, 3:3 + m].contiguous(), d)
        with pytest.raises(binding.FreezeError):
            binding.freeze_quantised_project(fc.ctx, 0, wide[:, 5:5 + d], None, d, False, out[1:b + 1, 3:3 + m], raw[4096:4096 + need - 256])
    finally:
        fc.close()


def test_far_apart_scales():
    # blocks of 2^100 against blocks of 2^-100, rows of zeros, the smallest values: each block's product at its own size
    b, d, m = 20, 512, 48
    x, w = _inputs(b, d, torch.float32, 1, channels=False), _inputs(m, d, torch.float32, 2, channels=False)
    s = torch.exp2(torch.tensor([100.0, -100.0, 0.0, 40.0])).repeat_interleave(128)
    x, w = x * s, w / s
    x[3] = 0
    w[5] = 0
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w.cuda())
        got = fc.quantised_project(0, x.cuda())
        _check_layer(fc, 0, x, w, None, False, torch.float32, False, got, d)
        assert (got[3] == 0).all() and (got[:, 5] == 0).all()
    finally:
        fc.close()


def test_output_over_its_input():
    x = _inputs(50, 256, torch.float32, 4).cuda()
    w = _inputs(256, 256, torch.float32, 5, channels=False).cuda()
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w)
        want = fc.quantised_project(0, x)
        fc.quantised_project(0, x, out=x)
        assert torch.equal(x, want)
        # the same over given codes and scales
        buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
        codes, scales = fc.quantise_rows(want)
        wanted = fc.quantised_project(0, codes, scales)
        buf[:50 * 256] = codes.view(torch.uint8).view(-1)
        buf[50 * 256:50 * 260] = scales.view(-1)
        got = fc.quantised_project(0, buf[:50 * 256].view(50, 256).view(torch.float8_e4m3fn), buf[50 * 256:50 * 260].view(50, 4),
                                   out=buf[:4 * 50 * 256].view(torch.float32).view(50, 256))
        assert torch.equal(got, wanted)
    finally:
        fc.close()


@pytest.mark.parametrize("ot", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_few_rows_straight_from_values(dtype, ot):
    # quantised within the product or before it: the same codes, so the same outputs bit by bit.  Sizes around what a workgroup holds (16 rows
    # of 768 values, not 13 of 1,056), cut and whole depths, rows apart, rows off 16 bytes and odd depths (before it), output over x
    fc = binding.FreezeCache(1)
    try:
        for b, d, m in [(1, 16, 1), (1, 128, 300), (1, 4096, 5000), (1, 14208, 700), (1, 14224, 33000), (1, 14464, 33000), (1, 40960, 33000), (2, 4096, 33000),
                        (2, 7040, 33000), (2, 7168, 33000), (3, 4736, 33000), (7, 1936, 9000), (8, 1024, 40000), (13, 1056, 40000), (16, 768, 40000),
                        (16, 1024, 40000), (1, 4100, 33000), (16, 16, 129)]:
            w = torch.randn(m, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d))
            fc.build_quantised(0, w, torch.linspace(-1, 1, m, device="cuda"))
            for pad in (0, 16, 3):
                x = _inputs(b, d + pad, dtype, 50 + b).cuda()[:, pad:]
                codes, scales = fc.quantise_rows(x)
                want = fc.quantised_project(0, codes, scales, relu=True, out_dtype=ot)
                got = fc.quantised_project(0, x, relu=True, out_dtype=ot)
                assert torch.equal(got.view(torch.uint8), want.view(torch.uint8)), (b, d, m, pad)
        x = torch.randn(2, 256, device="cuda").to(ot)
        fc.build_quantised(0, torch.randn(256, 256, device="cuda"))
        want = fc.quantised_project(0, x, out_dtype=ot)
        fc.quantised_project(0, x, out=x)
        assert torch.equal(x, want)
    finally:
        fc.close()


def test_workspace_over_operands_is_refused():
    b, d, m = 50, 256, 256
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, _inputs(m, d, torch.float32, 5, channels=False).cuda())
        need = binding.freeze_quantised_workspace_bytes(fc.ctx, 0, b, binding.FREEZE_F32)
        size = b * 256 * 4
        buf = torch.zeros(2 * need + 2 * size, dtype=torch.uint8, device="cuda")
        ws, other = buf[size:size + need], torch.zeros(b, 256, device="cuda")
        codes, scales = fc.quantise_rows(other)
        for at in (size - 256, size + need // 256 * 256 - 256):   # over the first and the last bytes
            rows = buf[at:at + size].view(torch.float32).view(b, 256)
            given = buf[at:at + b * 256].view(torch.float8_e4m3fn).view(b, 256), buf[at:at + b * 4].view(b, 4)
            for x, sc, out in ((rows, None, other), (other, None, rows), (given[0], scales, other), (codes, given[1] if at >= size else None, other)):
                if x is codes and sc is None:
                    continue
                with pytest.raises(binding.FreezeError):
                    binding.freeze_quantised_project(fc.ctx, 0, x, sc, d, False, out, ws)
        torch.cuda.synchronize()
        assert (buf == 0).all()
    finally:
        fc.close()


def test_a_row_does_not_depend_on_its_batch():
    # the same sums for a row alone and in the middle of others of the same tile
    x = _inputs(48, 1000, torch.bfloat16, 6).cuda()
    w = _inputs(500, 1000, torch.bfloat16, 7, channels=False).cuda()
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w)
        both = [fc.quantised_project(0, x) for _ in range(3)]
        assert torch.equal(both[0], both[1]) and torch.equal(both[0], both[2])
        y = x.clone()
        y[:10] = 0
        assert torch.equal(fc.quantised_project(0, y)[10:], both[0][10:])
    finally:
        fc.close()


def test_other_streams_and_replays():
    b, d, m = 24, 1100, 900
    w = _inputs(m, d, torch.float32, 9, channels=False).cuda()
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w)
        xs = [_inputs(b, d, torch.bfloat16, 100 + i).cuda() for i in range(4)]
        want = [fc.quantised_project(0, x).clone() for x in xs]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        ws = torch.empty(binding.freeze_quantised_workspace_bytes(fc.ctx, 0, b, binding.FREEZE_F32), dtype=torch.uint8, device="cuda")
        out = torch.empty(b, m, device="cuda")
        binding.freeze_quantised_project(fc.ctx, 0, xs[0], None, d, False, out, ws, stream=side)
        side.synchronize()
        assert torch.equal(out, want[0])
        x = xs[0].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.freeze_quantised_project(fc.ctx, 0, x, None, d, False, out, ws)
        for i in (1, 2, 3, 1, 0):
            x.copy_(xs[i])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[i])
            ws.fill_(255)
            assert torch.equal(fc.quantised_project(0, xs[i]), want[i])
    finally:
        fc.close()


def test_two_streams_at_once():
    w = _inputs(3000, 900, torch.float32, 30, channels=False).cuda()
    fc = binding.FreezeCache(1)
    try:
        fc.build_quantised(0, w)
        xs = [_inputs(b, 900, torch.bfloat16, 31 + b).cuda() for b in (40, 300)]
        want = [fc.quantised_project(0, x).clone() for x in xs]
        outs = [torch.empty_like(y) for y in want]
        ws = [torch.empty(binding.freeze_quantised_workspace_bytes(fc.ctx, 0, x.shape[0], binding.FREEZE_F32), dtype=torch.uint8, device="cuda") for x in xs]
        streams = [torch.cuda.Stream() for _ in xs]
        torch.cuda.synchronize()
        for _ in range(5):
            for x, out, w8, s in zip(xs, outs, ws, streams):
                binding.freeze_quantised_project(fc.ctx, 0, x, None, 900, False, out, w8, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    finally:
        fc.close()


def test_slots_and_rebuilds():
    w = _inputs(40, 200, torch.float32, 12, channels=False).cuda()
    x = _inputs(6, 200, torch.float32, 13).cuda()
    fc = binding.FreezeCache(2)
    try:
        fc.build_quantised(0, w)
        with pytest.raises(binding.FreezeError):
            fc.lookup(0, x, 1, 1)
        with pytest.raises(binding.FreezeError):
            fc.project(0, x)
        with pytest.raises(binding.FreezeError):
            binding.freeze_quantised_project(fc.ctx, 1, x, None, 200, False, torch.empty(6, 40, device="cuda"),
                                             torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
        fc.build_layer(0, w, torch.zeros(40, dtype=torch.int32, device="cuda"), 1)
        assert fc.lookup(0, w[7:8].contiguous(), 1, 1)["idx"].item() == 7
        assert binding.freeze_quantised_workspace_bytes(fc.ctx, 0, 6, binding.FREEZE_F32) == 0
        fc.build_quantised(0, w[:30].contiguous(), torch.ones(30, device="cuda"))
        _check_layer(fc, 0, x, w[:30], torch.ones(30), False, torch.float32, False, fc.quantised_project(0, x), 200)
        assert fc.quantised_project(0, x[:0]).shape == (0, 30)
    finally:
        fc.close()
