"""Arguments that the 8-bit layer, the choice of tokens and the reordering of states refuse, before anything is enqueued (no GPU),
and the definitions that their GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2002_02645_amd import binding
from tests import decode_reference as ref

EINVAL, ELAYER, ENOTBUILT, EWORKSPACE = (binding.FREEZE_EINVAL, binding.FREEZE_ELAYER, binding.FREEZE_ENOTBUILT, binding.FREEZE_EWORKSPACE)
P = ctypes.c_void_p


@pytest.fixture()
def ctx():
    h = binding.freeze_create(2)
    yield h
    binding.freeze_destroy(h)


def test_strides_and_sizes(ctx):
    L = binding.lib()
    for d, c, s in ((1, 128, 4), (128, 128, 4), (129, 256, 4), (512, 512, 4), (513, 640, 8), (1 << 22, 1 << 22, 1 << 15)):
        assert binding.freeze_quantised_code_stride(d) == c and binding.freeze_quantised_scale_stride(d) == s
    for d in (0, -1, (1 << 22) + 1):
        assert binding.freeze_quantised_code_stride(d) == 0 and binding.freeze_quantised_scale_stride(d) == 0
        assert binding.freeze_quantised_storage_bytes(5, d) == 0
    up = lambda x: (x + 255) // 256 * 256
    assert binding.freeze_quantised_storage_bytes(1000, 129) == 1024 * 256 + 1024 * 4 + up(4000)   # rows in tiles of 256
    assert binding.freeze_quantised_storage_bytes(0, 8) == 0 and binding.freeze_quantised_storage_bytes(2147483647, 8) == 0
    assert L.freeze_quantised_workspace_bytes(ctx, 0, 4, 0) == 0     # nothing built


def test_quantise_refusals():
    f = binding.lib().freeze_quantise_rows
    x, c, s = P(1 << 20), P(1 << 21), P(1 << 22)
    assert f(x, 0, 0, 8, 8, c, s, None) == 0
    assert f(None, 0, 0, 8, 8, None, None, None) == 0
    for args in ((None, 0, 2, 8, 8, c, s), (x, 0, 2, 8, 8, None, s), (x, 0, 2, 8, 8, c, None), (x, 2, 2, 8, 8, c, s), (x, -1, 2, 8, 8, c, s),
                 (x, 0, -1, 8, 8, c, s), (x, 0, 2, 0, 8, c, s), (x, 0, 2, 8, 7, c, s), (x, 0, 2, (1 << 22) + 1, 1 << 23, c, s),
                 (P((1 << 20) + 2), 0, 2, 8, 8, c, s), (P((1 << 20) + 1), 1, 2, 8, 8, c, s), (x, 0, 2, 8, 8, P((1 << 21) + 8), s),
                 (x, 0, 2, 8, 8, c, P((1 << 22) + 2)), (x, 0, (1 << 30) + 1, 8, 8, c, s), (x, 0, 2, 8, 1 << 40, c, s),
                 (x, 0, 2, 8, 8, x, s), (x, 0, 2, 8, 8, c, P((1 << 20) + 32)), (x, 0, 2, 8, 8, c, P((1 << 21) + 128))):
        assert f(*args, None) == EINVAL, args


def test_layer_refusals(ctx):
    L = binding.lib()
    w, st, sc = P(1 << 20), P(1 << 24), P(1 << 22)
    build = L.freeze_quantised_build
    assert build(None, 0, w, 0, None, 4, 8, None, st, 1 << 20, None) == EINVAL
    assert build(ctx, 2, w, 0, None, 4, 8, None, st, 1 << 20, None) == ELAYER
    assert build(ctx, 0, None, 0, None, 4, 8, None, st, 1 << 20, None) == EINVAL
    assert build(ctx, 0, w, 0, None, 4, 8, None, None, 1 << 20, None) == EINVAL
    assert build(ctx, 0, w, 3, None, 4, 8, None, st, 1 << 20, None) == EINVAL
    assert build(ctx, 0, w, 0, sc, 4, 8, None, st, 1 << 20, None) == EINVAL       # scales without codes
    assert build(ctx, 0, w, 2, None, 4, 8, None, st, 1 << 20, None) == EINVAL     # codes without scales
    assert build(ctx, 0, w, 0, None, 0, 8, None, st, 1 << 20, None) == EINVAL
    assert build(ctx, 0, w, 0, None, 4, 0, None, st, 1 << 20, None) == EINVAL
    assert build(ctx, 0, w, 0, None, 4, 8, None, st, 100, None) == EWORKSPACE
    assert build(ctx, 0, w, 0, None, 4, 8, None, P((1 << 24) + 16), 1 << 20, None) == EWORKSPACE
    assert build(ctx, 0, P((1 << 20) + 8), 2, sc, 4, 8, None, st, 1 << 20, None) == EINVAL
    x, out, ws = P(1 << 25), P(1 << 26), P(1 << 27)
    assert L.freeze_quantised_project(ctx, 0, x, 0, None, 2, 8, 0, out, 0, 4, ws, 1 << 20, None) == ENOTBUILT
    need = binding.freeze_quantised_storage_bytes(4, 8)
    for at in ((1 << 24) - 64, (1 << 24) + need - 64):      # weights, bias, codes and scales that reach into the storage
        assert build(ctx, 0, P(at), 0, None, 4, 8, None, st, 1 << 20, None) == EINVAL
        assert build(ctx, 0, w, 0, None, 32, 8, P(at), st, 1 << 20, None) == EINVAL
        assert build(ctx, 0, P(at), 2, sc, 4, 8, None, st, 1 << 20, None) == EINVAL
        assert build(ctx, 0, w, 2, P(at), 32, 8, None, st, 1 << 20, None) == EINVAL
    assert L.freeze_quantised_project(ctx, 5, x, 0, None, 2, 8, 0, out, 0, 4, ws, 1 << 20, None) == ELAYER
    assert L.freeze_quantised_project(None, 0, x, 0, None, 2, 8, 0, out, 0, 4, ws, 1 << 20, None) == EINVAL


def test_beam_refusals():
    L = binding.lib()
    assert binding.freeze_beam_workspace_bytes(1, 4, 1000, 4) > 0
    for args in ((-1, 4, 10, 4), (1, 0, 10, 4), (1, 65, 10, 4), (1, 4, 0, 4), (1, 4, 10, 0), (1, 4, 10, 65), (1, 4, 2147483647, 4),
                 ((1 << 20) // 4 + 1, 4, 10, 4)):
        assert binding.freeze_beam_workspace_bytes(*args) == 0, args
    lo, sc, fi, o, ws = P(1 << 20), P(1 << 21), P(1 << 22), P(1 << 23), P(1 << 24)
    need = binding.freeze_beam_workspace_bytes(2, 4, 1000, 4)
    good = [lo, 0, 2, 4, 1000, 1000, sc, fi, 5, 4, o, o, o, None, ws, need, None]

    def call(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return L.freeze_beam_select(*a)
    for kw in (dict(a0=None), dict(a1=2), dict(a2=-1), dict(a3=0), dict(a4=0), dict(a5=999), dict(a6=None), dict(a8=-1), dict(a8=1000), dict(a8=-2),
               dict(a9=0), dict(a9=65), dict(a10=None), dict(a11=None), dict(a12=None), dict(a14=None), dict(a0=P((1 << 20) + 2))):
        assert call(**kw) == EINVAL, kw
    assert call(a15=need - 1) == EWORKSPACE and call(a14=P((1 << 24) + 8)) == EWORKSPACE
    assert call(a2=0, a0=None, a14=None) == 0


def test_beam_outputs_over_other_buffers():
    # 2 groups of 4 rows, k = 4: 8 places of 4 bytes each; every buffer alone, then one of them moved over another one's last byte
    L = binding.lib()
    need = binding.freeze_beam_workspace_bytes(2, 4, 1000, 4)
    lo, sc, fi, oS, oT, oP, oF, ws = (n << 20 for n in range(1, 9))
    at = dict(lo=(lo, 8 * 1000 * 4), sc=(sc, 32), fi=(fi, 8), oS=(oS, 32), oT=(oT, 32), oP=(oP, 32), oF=(oF, 8), ws=(ws, need))

    def call(**moved):
        p = {k: P(moved.get(k, v[0])) for k, v in at.items()}
        return L.freeze_beam_select(p["lo"], 0, 2, 4, 1000, 1000, p["sc"], p["fi"], 5, 4, p["oS"], p["oT"], p["oP"], p["oF"], p["ws"], need, None)
    for out in ("oS", "oT", "oP", "oF"):
        for other, (begin, size) in at.items():
            if other != out:
                assert call(**{out: begin}) == EINVAL, (out, other)
                assert call(**{out: begin + (size - 1) // 4 * 4}) == EINVAL, (out, other)
    for other in ("lo", "sc", "fi"):
        assert call(**{other: ws + 256}) == EINVAL
    for name in ("sc", "oS", "oT", "oP"):
        assert call(**{name: at[name][0] + 2}) == EINVAL


def test_reorder_refusals():
    f = binding.lib().freeze_reorder_states

    def call(states, parents=P(4096), rows=4, src_rows=4):
        arr = (binding.FreezeState * max(1, len(states)))(*states)
        return f(ctypes.cast(arr, P), len(states), parents, rows, src_rows, None)
    S = binding.FreezeState
    a, b = 1 << 20, 1 << 24
    assert call([]) == 0 and call([S(a, b, 1, 0, 64, 1, 0, 64)], rows=0) == 0
    assert f(None, 1, P(4096), 4, 4, None) == EINVAL and f(None, 1025, P(4096), 4, 4, None) == EINVAL and f(None, -1, P(4096), 4, 4, None) == EINVAL
    for st in (S(a, b, -1, 0, 64, 1, 0, 64), S(a, b, 1, 0, -64, 1, 0, 64), S(a, b, 1, 0, 64, 1, 0, -1), S(None, b, 1, 0, 64, 1, 0, 64),
               S(a, None, 1, 0, 64, 1, 0, 64), S(a, b, 1, 0, 63, 1, 0, 64),              # rows that reach into each other
               S(a, b, 1, 0, 64, 2, 16, 32), S(a, b, 2, 128, 64, 1, 0, 64), S(a, b, 1 << 20, 1 << 30, 64, 1 << 20, 1 << 10, 64),
               S(a, a, 1, 0, 64, 1, 0, 64), S(a, a + 255, 1, 0, 64, 1, 0, 64), S(a, b, 1, 0, 1 << 60, 1, 0, 64), S(a, b, 1, 0, 64, 1, 0, 1 << 60)):
        assert call([st]) == EINVAL
    good = S(a, b, 1, 0, 64, 1, 0, 64)
    assert call([good], parents=None) == EINVAL and call([good], rows=-1) == EINVAL and call([good], src_rows=-1) == EINVAL
    assert call([good, S(b + 100, 1 << 26, 1, 0, 64, 1, 0, 64)]) == EINVAL         # a source within another's destination
    assert call([good, S(1 << 27, b + 200, 1, 0, 64, 1, 0, 64)]) == EINVAL         # two destinations
    assert call([good], parents=P(b + 252)) == EINVAL and call([good], parents=P(4098)) == EINVAL


def test_state_of_layouts():
    t, u = torch.zeros(2, 3, 4, 5, 6, dtype=torch.bfloat16), torch.zeros(2, 3, 4, 5, 6, dtype=torch.bfloat16)
    s = binding.state_of(t, u, used=2, row_dim=1)
    assert (s.outer, s.outer_stride, s.row_stride, s.pieces, s.piece_stride, s.piece_bytes) == (2, 720, 240, 4, 60, 24)
    s = binding.state_of(t[0], u[0])
    assert (s.outer, s.row_stride, s.pieces, s.piece_stride, s.piece_bytes) == (1, 240, 4, 60, 60)
    s = binding.state_of(t[0, 0, 0], u[0, 0, 0])
    assert (s.row_stride, s.pieces, s.piece_bytes) == (12, 1, 12)
    with pytest.raises(AssertionError):
        binding.state_of(t, u.transpose(0, 1), row_dim=1)
    with pytest.raises(AssertionError):
        binding.state_of(t[..., ::2], u[..., ::2], row_dim=1)
    with pytest.raises(AssertionError):
        binding.state_of(t, u, used=6, row_dim=1)


def test_reference_codes():
    x = np.random.RandomState(1).randn(4, 300) * 100
    codes, scales = ref.quantise(x)
    via = torch.from_numpy(np.pad(x, ((0, 0), (0, 84)))).view(4, 3, 128) / torch.exp2(torch.from_numpy(scales[:, :3].astype(np.float64)) - 127)[:, :, None]
    # (to fp32 first: these values have few enough bits left of the border for that not to matter)
    assert np.array_equal(codes.reshape(4, 3, 128), via.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    err = np.abs(ref.values(codes, scales)[:, :300] - x)
    assert (err <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * np.exp2(scales[:, :3].astype(float) - 127).repeat(128, 1)[:, :300])).all()
    assert (via.abs().amax(2) > 224).all() and (via.abs().amax(2) <= 448).all()


def test_reference_choice():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]]))
    best = ref.beam_select(x, [0.0, np.log(0.5)], None, 2, -1, 4)[0]
    assert [(r, t) for _, r, t in best] == [(0, 0), (1, 1), (0, 1), (0, 2)]
    assert np.allclose(np.exp([s for s, _, _ in best]), [0.5, 0.4, 0.25, 0.25])
    best = ref.beam_select(x, [0.0, -0.1], [0, 1], 2, 2, 2)[0]
    assert best == [(-0.1, 1, 2), (pytest.approx(np.log(0.5)), 0, 0)]
    assert ref.beam_select(x, [-np.inf, -np.inf], None, 2, 1, 1)[0] == [(-np.inf, 0, 1)]
