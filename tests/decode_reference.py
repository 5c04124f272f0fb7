"""The definitions behind freeze_quantise_rows, freeze_quantised_project and freeze_beam_select in 64 bits, in plain loops and
numpy, for the tests."""
import numpy as np

BLOCK = 128


def code_values():
    """The 256 numbers that codes of 1 sign, 4 exponent (bias 7) and 3 mantissa bits stand for; 0x7f and 0xff: no number."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[c] = -x if c & 128 else x
    v[0x7F] = v[0xFF] = np.nan
    return v


CODE_VALUES = code_values()


def nearest_code(x):
    """Codes of the numbers |x| <= 448 rounded to nearest, halfway cases to the even code."""
    mags = CODE_VALUES[:0x7F]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(mags, a), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - mags[lo], mags[hi] - a
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantise(x):
    """codes [rows, d_pad] uint8, scale bytes [rows, sd] uint8 of an array of rows."""
    x = np.asarray(x, np.float64)
    rows, d = x.shape
    nb = -(-d // BLOCK)
    sd = -(-nb // 4) * 4
    t = np.zeros((rows, nb * BLOCK))
    t[:, :d] = x
    t = t.reshape(rows, nb, BLOCK)
    e = np.full((rows, nb), -126)
    amax = np.abs(t).max(2)
    for i in range(-126, 128):
        e = np.where(amax > 448 * 2.0 ** i, i + 1, e)
    codes = nearest_code(t / np.exp2(e.astype(np.float64))[:, :, None]).reshape(rows, nb * BLOCK)
    scales = np.ones((rows, sd), np.uint8)
    scales[:, :nb] = e + 127
    return codes, scales


def values(codes, scales):
    rows, d_pad = codes.shape
    nb = d_pad // BLOCK
    return (CODE_VALUES[codes].reshape(rows, nb, BLOCK) * np.exp2(scales[:, :nb].astype(np.float64) - 127)[:, :, None]).reshape(rows, d_pad)


def beam_select(logits, scores, finished, beams, end, k):
    """Per group the k best (total, row in the batch, token), best first, then fillers (-inf, first row, end or 0)."""
    logits, scores = np.asarray(logits, np.float64), np.asarray(scores, np.float64)
    rows, vocab = logits.shape
    out = []
    for g in range(rows // beams):
        cand = []
        for r in range(g * beams, (g + 1) * beams):
            if scores[r] == -np.inf:
                continue
            if finished is not None and finished[r]:
                cand.append((scores[r], r, end))
                continue
            x = logits[r]
            if not (x > -np.inf).any():
                continue
            offset = scores[r] - np.log(np.exp(x - x.max()).sum())   # (beside x.max() itself a score would be lost where that is far from zero)
            best = np.lexsort((np.arange(vocab), -x))[:k]
            cand += [(offset + (x[v] - x.max()), r, int(v)) for v in best if x[v] > -np.inf]
        cand.sort(key=lambda c: (-c[0], c[1], c[2]))
        cand = cand[:k]
        out.append(cand + [(-np.inf, g * beams, max(end, 0))] * (k - len(cand)))
    return out
