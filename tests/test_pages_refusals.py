"""Arguments that the rotary positions and the pages of keys and values refuse, before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

from paper_2002_02645_amd import binding
from tests import pages_reference as ref

EINVAL, EWORKSPACE = binding.FREEZE_EINVAL, binding.FREEZE_EWORKSPACE
P = ctypes.c_void_p
GB = 1 << 30


def pool(**kw):
    base = dict(codes=1 * GB, scales=2 * GB, refs=3 * GB, tables=4 * GB, lengths=5 * GB, num_pages=100, rows=4, max_pages=10, layers=2, heads=3, head_dim=40, page_tokens=64)
    base.update(kw)
    return binding.FreezePagesPool(*(base[f[0]] for f in binding.FreezePagesPool._fields_))


at = ctypes.addressof

SIZES = [dict(layers=0), dict(layers=1025), dict(heads=0), dict(heads=1025), dict(head_dim=0), dict(head_dim=257), dict(page_tokens=0), dict(page_tokens=16), dict(page_tokens=48),
         dict(page_tokens=2048), dict(page_tokens=-64), dict(num_pages=0), dict(num_pages=(1 << 24) + 1), dict(rows=0), dict(rows=16385), dict(max_pages=0),
         dict(max_pages=(1 << 20) + 1), dict(page_tokens=1024, max_pages=1 << 21), dict(num_pages=1 << 24, layers=1024, heads=1024)]
POINTERS = [dict(codes=None), dict(codes=GB + 8), dict(scales=None), dict(scales=2 * GB + 1), dict(refs=None), dict(refs=3 * GB + 2), dict(tables=None), dict(tables=4 * GB + 1),
            dict(lengths=None), dict(lengths=5 * GB + 2)]


def test_sizes():
    L = binding.lib()
    p = pool()
    assert binding.freeze_pages_bytes(p) == 2 * 100 * 3 * 2 * 2 * 32 * 64
    assert binding.freeze_pages_workspace_bytes(p) == 3 * 512 + 256 + 2 * 256 + 256
    assert L.freeze_pages_bytes(None) == 0 and L.freeze_pages_workspace_bytes(None) == 0
    for kw in SIZES:
        assert binding.freeze_pages_bytes(pool(**kw)) == 0 and binding.freeze_pages_workspace_bytes(pool(**kw)) == 0, kw
        assert binding.freeze_pages_attend_workspace_bytes(pool(**kw), 4, 4) == 0, kw
    last = 0
    for tokens in (0, 1, 4, 5, 9, 40, 1000):      # the bytes for some tokens serve fewer
        n = binding.freeze_pages_attend_workspace_bytes(p, 4, tokens)
        assert n >= last > -1
        last = n
    for most in (0, 1, 7, 30):
        assert binding.freeze_pages_attend_workspace_bytes(p, 4, 30, most) <= binding.freeze_pages_attend_workspace_bytes(p, 4, 30)
    assert binding.freeze_pages_attend_workspace_bytes(p, 4, 4, 0, False) > 0
    for group, tokens, most in ((0, 4, 0), (1025, 4, 0), (4, -1, 0), (4, 1 << 31, 0), (4, 4, -1), (1024, 1 << 17, 0)):
        assert binding.freeze_pages_attend_workspace_bytes(p, group, tokens, most) == 0


def test_bookkeeping_refusals():
    L = binding.lib()
    a, g, w = P(6 * GB), P(7 * GB), P(8 * GB)
    for kw in SIZES + POINTERS:
        p = pool(**kw)
        assert L.freeze_pages_reserve(at(p), a, g, w, 1 << 30, None) == EINVAL, kw
        assert L.freeze_pages_fork(at(p), a, None) == EINVAL, kw
        assert L.freeze_pages_truncate(at(p), a, None) == EINVAL, kw
        assert L.freeze_pages_compact(at(p), g, w, 1 << 30, None) == EINVAL, kw
    p = pool()
    n = binding.freeze_pages_workspace_bytes(p)
    assert L.freeze_pages_reserve(at(p), a, g, w, n - 1, None) == EWORKSPACE and L.freeze_pages_compact(at(p), g, w, n - 1, None) == EWORKSPACE
    assert L.freeze_pages_reserve(at(p), a, g, P(8 * GB + 16), n, None) == EWORKSPACE and L.freeze_pages_compact(at(p), g, P(8 * GB + 128), n, None) == EWORKSPACE
    codes = binding.freeze_pages_bytes(p)
    inside = (GB, GB + codes - 4, 2 * GB, 3 * GB + 396, 4 * GB, 5 * GB + 12)
    for args in [(a, None, w), (a, g, None), (P(6 * GB + 2), g, w), (a, P(7 * GB + 1), w), (g, g, w), (P(7 * GB + 12), g, w), (a, P(8 * GB + 256), w)] + [(P(x), g, w) for x in inside[:1] + inside[3:]] + [(a, P(x), w) for x in inside]:
        assert L.freeze_pages_reserve(at(p), *args, n, None) == EINVAL, args
    for x in (GB, 2 * GB, 3 * GB, 4 * GB, 5 * GB):
        assert L.freeze_pages_reserve(at(p), a, g, P(x), n, None) == EINVAL and L.freeze_pages_compact(at(p), g, P(x), n, None) == EINVAL
    for x in (None, P(6 * GB + 1), P(3 * GB), P(4 * GB + 8), P(5 * GB)):
        assert L.freeze_pages_fork(at(p), x, None) == EINVAL and L.freeze_pages_truncate(at(p), x, None) == EINVAL
    for x in (None, P(7 * GB + 2), P(GB), P(5 * GB), P(8 * GB + 256)):
        assert L.freeze_pages_compact(at(p), x, w, n, None) == EINVAL
    # two of the pool's own over one another
    for kw in (dict(refs=4 * GB + 16), dict(lengths=3 * GB), dict(tables=GB), dict(scales=GB + 64)):
        p = pool(**kw)
        assert L.freeze_pages_reserve(at(p), a, g, w, n, None) == EINVAL, kw


def test_append_refusals():
    L = binding.lib()
    k, v, st, gr = P(6 * GB), P(7 * GB), P(8 * GB), P(9 * GB)
    ok = dict(layer=0, k=k, kt=120, kh=40, v=v, vt=120, vh=40, dtype=1, tokens=9, starts=st, most=0, granted=gr)

    def call(p=None, **kw):
        a, p = {**ok, **kw}, p or pool()
        return L.freeze_pages_append(at(p), a["layer"], a["k"], a["kt"], a["kh"], a["v"], a["vt"], a["vh"], a["dtype"], a["tokens"], a["starts"], a["most"], a["granted"], None)

    assert call(tokens=0) == 0 and call(tokens=0, k=None, v=None, starts=None) == 0
    for kw in SIZES + POINTERS:
        assert call(pool(**kw)) == EINVAL, kw
    for kw in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(dtype=2), dict(dtype=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(tokens=1 << 28, kt=0, vt=0), dict(most=-1), dict(starts=None),
               dict(starts=None, tokens=3), dict(k=P(6 * GB + 1)), dict(v=P(7 * GB + 2), dtype=0), dict(starts=P(8 * GB + 2)), dict(granted=P(9 * GB + 1)), dict(kt=-1), dict(vh=-1),
               dict(kt=1 << 45), dict(k=P(GB)), dict(v=P(2 * GB)), dict(starts=P(GB + 64)), dict(granted=P(2 * GB))):
        assert call(**kw) == EINVAL, kw


def test_attend_refusals():
    L = binding.lib()
    q, o, w, st = P(6 * GB), P(7 * GB), P(8 * GB), P(9 * GB)
    n = binding.freeze_pages_attend_workspace_bytes(pool(), 2, 9)
    ok = dict(layer=0, q=q, qd=1, qt=240, qh=40, group=2, tokens=9, starts=st, most=0, scale=0.1, window=0, out=o, od=1, ot=240, oh=40, ws=w, bytes=n)

    def call(p=None, **kw):
        a, p = {**ok, **kw}, p or pool()
        return L.freeze_pages_attend(at(p), a["layer"], a["q"], a["qd"], a["qt"], a["qh"], a["group"], a["tokens"], a["starts"], a["most"], a["scale"], a["window"], a["out"],
                                     a["od"], a["ot"], a["oh"], a["ws"], a["bytes"], None)

    assert call(tokens=0) == 0
    for kw in SIZES + POINTERS:
        assert call(pool(**kw), bytes=GB) == EINVAL, kw
    for kw in (dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(ws=None), dict(qd=2), dict(od=2), dict(qd=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(group=0),
               dict(group=1025), dict(most=-1), dict(starts=None), dict(starts=None, tokens=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(window=-1), dict(window=1 << 31), dict(q=P(6 * GB + 1)), dict(q=P(6 * GB + 2), qd=0), dict(out=P(7 * GB + 1)), dict(out=P(7 * GB + 2), od=0), dict(starts=P(9 * GB + 2)),
               dict(qt=-1), dict(qh=-8), dict(ot=-1), dict(oh=-8), dict(ot=239), dict(oh=39), dict(ot=0), dict(oh=0), dict(out=q), dict(out=P(6 * GB + 8)), dict(out=P(GB)), dict(out=P(3 * GB)),
               dict(out=P(4 * GB)), dict(out=P(5 * GB)), dict(out=w), dict(out=P(9 * GB)), dict(ws=P(6 * GB)), dict(ws=P(GB)), dict(ws=P(4 * GB))):
        assert call(**kw) == EINVAL, kw
    assert call(bytes=n - 1) == EWORKSPACE and call(ws=P(8 * GB + 64)) == EWORKSPACE


def test_rotate_refusals():
    L = binding.lib()
    f, pos, freq = L.freeze_rotate_positions, P(8 * GB), P(9 * GB)

    def call(tensors, tokens=5, dim=8, positions=pos, frequencies=freq, pairs=4, factor=1.0, num=None):
        arr = (binding.FreezeHeads * max(1, len(tensors)))(*tensors)
        return f(at(arr), len(tensors) if num is None else num, tokens, dim, positions, frequencies, pairs, 0, factor, 0, None)

    H = binding.FreezeHeads
    good = H(GB, 2 * GB, 1, 3, 24, 8, 24, 8)
    assert call([]) == 0 and call([good], tokens=0) == 0 and call([H(None, None, 1, 0, 0, 0, 0, 0)]) == 0
    assert f(None, 1, 5, 8, pos, freq, 4, 0, 1.0, 0, None) == EINVAL
    assert call([good] * 9) == EINVAL and call([good], num=-1) == EINVAL
    for kw in (dict(tokens=-1), dict(tokens=1 << 31), dict(dim=0), dict(dim=4097, pairs=4), dict(pairs=-1), dict(pairs=5), dict(positions=None), dict(frequencies=None),
               dict(positions=P(8 * GB + 2)), dict(frequencies=P(9 * GB + 4)), dict(factor=float("nan")), dict(factor=float("inf"))):
        assert call([good], **kw) == EINVAL, kw
    for h in (H(None, 2 * GB, 1, 3, 24, 8, 24, 8), H(GB, None, 1, 3, 24, 8, 24, 8), H(GB, 2 * GB, 2, 3, 24, 8, 24, 8), H(GB, 2 * GB, 1, -1, 24, 8, 24, 8), H(GB, 2 * GB, 1, 8193, 24, 8, 24, 8),
              H(GB + 1, 2 * GB, 1, 3, 24, 8, 24, 8), H(GB, 2 * GB + 2, 0, 3, 24, 8, 24, 8), H(GB, 2 * GB, 1, 3, -1, 8, 24, 8), H(GB, 2 * GB, 1, 3, 24, 8, 23, 8), H(GB, 2 * GB, 1, 3, 24, 8, 24, 7),
              H(GB, 2 * GB, 1, 3, 24, 8, 0, 8), H(GB, GB, 1, 3, 24, 8, 48, 8), H(GB, GB + 16, 1, 3, 24, 8, 24, 8), H(GB, 8 * GB, 1, 3, 24, 8, 24, 8), H(GB, 9 * GB, 1, 3, 24, 8, 24, 8)):
        assert call([h]) == EINVAL
    assert call([good, H(3 * GB, 2 * GB, 1, 3, 24, 8, 24, 8)]) == EINVAL                       # two tensors to one place
    assert call([good, H(2 * GB + 16, 4 * GB, 1, 3, 24, 8, 24, 8)]) == EINVAL                  # one reads what another writes
    side = H(GB, GB, 1, 3, 40, 8, 40, 8)
    assert call([side, H(GB + 32, GB + 32, 1, 3, 40, 8, 40, 8)]) == EINVAL                     # side by side in one buffer, 8 bytes of each row shared


def test_frequencies():
    f = binding.rotary_frequencies(4, 10000.0, device="cpu")
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15)
    assert torch.allclose(binding.rotary_frequencies(4, stretch=4.0, device="cpu"), f / 4, rtol=1e-15)
    g = binding.rotary_frequencies(4, stretch=4.0, trained=2000, device="cpu")
    turns = 2000 * f / 6.283185307179586                                                        # 318, 31.8, 3.18, 0.318
    assert torch.allclose(g[:2], f[:2], rtol=1e-15) and torch.allclose(g[3:], f[3:] / 4, rtol=1e-15)
    keep = float((turns[2] - 1) / 3)
    assert abs(float(g[2]) - float(f[2]) * (keep + (1 - keep) / 4)) < 1e-15
    assert binding.rotary_frequencies(0, device="cpu").numel() == 0
    for kw in (dict(pairs=-1), dict(pairs=2, base=0.0), dict(pairs=2, stretch=0.0), dict(pairs=2, trained=5, low=4.0, high=4.0)):
        with pytest.raises(AssertionError):
            binding.rotary_frequencies(device="cpu", **kw)


def test_reference():
    """The oracle against itself in other words: rounding against the type's own, bytes of a block each used once, attention against a matrix form."""
    x = torch.cat([torch.randn(20000) * 10.0 ** torch.randint(-4, 3, (20000,)), torch.arange(-448, 449) / 2.0])
    x = x.clamp(-448, 448)
    assert torch.equal(ref.nearest(x.double()).float(), x.to(torch.float8_e4m3fn).float())
    for dim in (1, 32, 40, 256):
        for kv in (0, 1):
            assert sorted(ref.places(dim)[kv].flatten().tolist()) == list(range(32 * ref.width(dim)))
    assert [ref.exponent(a) for a in (0.0, 448.0, 448.1, 1.75, 1.76, 2.0 ** -130)] == [-126, 0, 1, -8, -7, -126]
    q, kv = torch.randn(3, 4, 5, dtype=torch.float64), torch.randn(2, 2, 7, 5, dtype=torch.float64)
    full = torch.stack([torch.softmax((q[:, j] @ kv[0, j // 2].t()).masked_fill(torch.arange(7)[None] > torch.arange(4, 7)[:, None], -float("inf")), 1) @ kv[1, j // 2] for j in range(4)], 1)
    assert torch.allclose(ref.attend(q, kv, 2, 1.0), full, rtol=1e-12)
    p = ref.Pool(1, 4, 2, 2, 1, 8, 32)
    assert p.reserve([33, 0]) == [33, 0] and p.tables == [[0, 1], [-1, -1]]
    p.fork([0, 0])
    assert p.refs == [2, 2, 0, 0] and p.reserve([1, 1]) == [1, 1] and p.tables == [[0, 2], [0, 3]] and p.refs == [2, 0, 1, 1]
    p.truncate([0, 40])
    assert p.refs == [1, 0, 0, 1] and p.compact() == 2 and p.tables == [[-1, -1], [0, 1]]
