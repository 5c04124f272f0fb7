"""Keys and values of a generating model in pages of 8 bits, as cases for timing and comparison: rotary positions, appending to the
pages, attention over them, and the bookkeeping of pages that beams share.

Every case is a dict of plain values; its "kind" says which public entry points a pass goes through:

  rotate   queries and keys turned by their positions (pairs side by side or in halves, a part of the head, scaled frequencies)
  append   new keys and values of ragged rows, quantised (e4m3, a power of two for each block of 32 tokens and head), into pages
  attend   attention of new queries (one a row, a few, or a prompt's) over the pages of their rows
  fork     rows go on as their parents' continuations: tables and counts follow, pages that are shared and written are copied
  compact  the pages in use move together at the front
  step     fork, a place for each row's token, and rotate, append and attend in every layer, as a step of decoding does

Heads of 64, 80 and 128 values and up to 32 rows of beams are those of the repository's other decoding cases; lengths are generic,
from one token to long ones.  A pass that changes the bookkeeping starts from the same one each time.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 32


def listed():
    return [
        # a decoding step of a small batch: launches and latencies count
        dict(name="rotate_tokens", kind="rotate", tokens=16, q_heads=32, heads=8, dim=128, rot=128, inter=False, bf16=True, far=8192, scaled=False),
        # packed prompts, the largest: half of each head is turned, pairs side by side, far positions with scaled frequencies
        dict(name="rotate_prompts", kind="rotate", tokens=32768, q_heads=32, heads=8, dim=128, rot=64, inter=True, bf16=True, far=500000, scaled=True),
        # a decoding step of a batch: one token a row, most blocks partly filled
        dict(name="append_tokens", kind="append", rows=64, heads=8, dim=128, page=64, bf16=True, past=1500, new=1, salt=1),
        # prompts of very different lengths behind what the rows hold already
        dict(name="append_prompts", kind="append", rows=24, heads=8, dim=128, page=64, bf16=True, past=600, new=4096, salt=2),
        # one request at the start of its answer: latency counts
        dict(name="attend_one", kind="attend", rows=1, heads=8, group=4, dim=128, page=64, bf16=True, past=700, new=1, window=0, salt=3),
        # one request with a long context: the work is split over its tokens
        dict(name="attend_long", kind="attend", rows=1, heads=8, group=8, dim=128, page=128, bf16=True, past=131071, new=1, window=0, salt=4),
        # a serving batch of ragged lengths, the most bytes
        dict(name="attend_batch", kind="attend", rows=64, heads=8, group=4, dim=128, page=64, bf16=True, past=16000, new=1, window=0, even=True, salt=5),
        # packed pieces of prompts behind what was read already: bound by the matrix pipes
        dict(name="attend_prompts", kind="attend", rows=5, heads=8, group=4, dim=128, page=64, bf16=True, past=4000, new=4096, window=0, salt=6),
        # odd sizes: fp32, a few guessed tokens a row, five heads a group, a window
        dict(name="attend_odd", kind="attend", rows=13, heads=3, group=5, dim=80, page=32, bf16=False, past=3001, new=5, window=1000, salt=7),
        # beams of a batch follow their parents: shared last pages are copied in every layer
        dict(name="fork_beams", kind="fork", groups=8, beams=4, layers=32, heads=8, dim=128, page=64, past=2000, spare=1.3, salt=8),
        # a pool with holes, a third of it in use, gives its upper part back
        dict(name="compact_pool", kind="compact", rows=32, layers=16, heads=8, dim=128, page=64, past=3000, spare=3.0, salt=9),
        # a step of decoding for the beams of a batch, four layers
        dict(name="step_beams", kind="step", groups=8, beams=4, layers=4, heads=8, group=4, dim=128, page=64, past=2000, spare=1.5, salt=10),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "append", "append", "attend", "attend", "attend", "attend", "attend", "fork", "compact", "step"])
    salt, dim, page = rng.randrange(1 << 30), rng.choice([64, 128, 128, 8 * rng.randint(4, 16), rng.randint(20, 128)]), rng.choice([32, 64, 128])
    heads, bf16 = rng.choice([1, 2, 3, 8]), rng.random() < 0.75
    if kind == "rotate":
        dim += dim % 2
        rot = rng.choice([dim, dim, dim // 4 * 2])
        q_heads = heads * rng.choice([1, 4, 5])
        tokens = _log(rng, 1, max(2, 1.3e8 // (dim * (heads + q_heads)) // (1 if bf16 else 2)))
        return dict(kind=kind, tokens=min(tokens, 60000), q_heads=q_heads, heads=heads, dim=dim, rot=rot, inter=rng.random() < 0.5, bf16=bf16,
                    far=_log(rng, 100, 1000000), scaled=rng.random() < 0.5)
    if kind == "append":
        rows = _log(rng, 1, 64)
        new = rng.choice([1, 1, _log(rng, 1, 4096)])
        return dict(kind=kind, rows=rows if new < 600 else max(1, rows // 4), heads=heads, dim=dim, page=page, bf16=bf16, past=_log(rng, 1, 2000), new=new, salt=salt)
    if kind == "attend":
        group = rng.choice([1, 4, 5, 8])
        if rng.random() < 0.65:
            rows = _log(rng, 1, 64)
            new = rng.choice([1, 1, 1, rng.randint(2, 8)])
            past = _log(rng, 1, min(131071, 0.6e9 // (rows * heads * dim)))
        else:
            rows, new = rng.randint(1, 5), _log(rng, 9, 4096)
            past = _log(rng, 1, 4000)
            bf16, group = bf16 or new > 1000, min(group, 5)
        return dict(kind=kind, rows=rows, heads=heads, group=group, dim=dim, page=page, bf16=bf16, past=past, new=new,
                    window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]), even=rng.random() < 0.4, salt=salt)
    past = _log(rng, 1, 2000)
    if kind == "compact":
        return dict(kind=kind, rows=_log(rng, 1, 32), layers=rng.choice([1, 4, 16]), heads=heads, dim=dim, page=page, past=past,
                    spare=rng.choice([1.1, 2.0, 3.0]), salt=salt)
    case = dict(kind=kind, groups=_log(rng, 1, 8), beams=rng.choice([1, 3, 4]), layers=rng.choice([1, 4, 16]), heads=heads, dim=dim, page=page, past=past,
                spare=rng.choice([1.3, 2.0]), salt=salt)
    return dict(case, layers=min(4, case["layers"]), group=rng.choice([1, 4, 5]), dim=dim + dim % 2) if kind == "step" else case


# ---- sizes that follow from a case ------------------------------------------------------------------

def _rows(case):
    return case["rows"] if "rows" in case else case["groups"] * case["beams"]


def _spread(rng, most, rows, even=False):
    """Lengths spread over 0 .. most (over their logarithm; even: over its upper three quarters), the longest among them."""
    got = [rng.randint(most // 4, most) for _ in range(rows)] if even else [int(round(math.exp(rng.uniform(0, math.log(most + 1))))) - 1 for _ in range(rows)]
    got[rng.randrange(rows)] = most
    return got


def _lengths(case):
    """(tokens that each row holds before a pass, new tokens of each row); a group's beams are equally long."""
    rng, rows = random.Random(case["salt"]), _rows(case)
    if "groups" in case:
        past = [n for n in _spread(rng, case["past"], case["groups"]) for _ in range(case["beams"])]
        return past, [1] * rows
    past = _spread(rng, case["past"], rows, case.get("even", False))
    if case["kind"] == "compact":
        return past, [0] * rows
    new = case["new"]
    return past, [1] * rows if new == 1 else [1 + n for n in _spread(rng, new - 1, rows)]


def _pages(n, page):
    return -(-n // page)


def _pool(case):
    """(places of a row's table, pages of the pool)"""
    past, new = _lengths(case)
    most = max(_pages(p + n, case["page"]) for p, n in zip(past, new)) + 1
    used = sum(_pages(p + n, case["page"]) for p, n in zip(past, new))
    return most, max(used + 2 * len(past), int(used * case.get("spare", 1.1))) + 3


def _padded(case):
    return _pages(case["dim"], 32) * 32


class State:
    pass


# ---- rows in 8 bits, and the layout of their blocks --------------------------------------------------

def _exponent(amax):
    """The smallest E >= -126 with amax <= 448 2^E."""
    bits = amax.view(torch.int32)
    return ((bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp_(min=-126)


def _power(e):
    return ((e + 127) << 23).view(torch.float32)   # e in -126 .. 126


def _pack(x):
    """Blocks [..., 2 (keys, values), 32 tokens, padded dims] in the order in which they lie in a page, [..., 2, bytes]."""
    lead, dims = x.shape[:-3], x.shape[-1]
    n, c = len(lead), dims // 32
    k = x[..., 0, :, :].reshape(*lead, 2, 16, c, 4, 8)        # half, token, chunk, group, dim
    k = k.permute(*range(n), n + 2, n + 3, n + 1, n, n + 4)
    v = x[..., 1, :, :].reshape(*lead, 2, 4, 4, c, 2, 16)     # half, group, token, chunk, half of the chunk, dim
    v = v.permute(*range(n), n + 3, n + 1, n + 5, n + 4, n, n + 2)
    return torch.stack([k.reshape(*lead, 32 * dims), v.reshape(*lead, 32 * dims)], -2)


def _unpack(x, dims):
    """The inverse of _pack, as the numbers that the codes are."""
    lead = x.shape[:-2]
    n, c = len(lead), dims // 32
    k = x[..., 0, :].reshape(*lead, c, 4, 16, 2, 8).permute(*range(n), n + 3, n + 2, n, n + 1, n + 4)
    v = x[..., 1, :].reshape(*lead, c, 4, 16, 2, 2, 4).permute(*range(n), n + 4, n + 1, n + 5, n, n + 3, n + 2)
    return torch.stack([k.reshape(*lead, 32, dims), v.reshape(*lead, 32, dims)], -3).view(torch.float8_e4m3fn).float()


# ---- states ------------------------------------------------------------------------------------------

def _cache(s, case, g, filled):
    """Pages, tables and counts of the rows, in s.codes [layers, pages, heads, blocks, 2, bytes], s.scales, s.tables, s.lengths, s.refs;
    s.book holds the last three in one run of memory."""
    rows, layers = _rows(case), case.get("layers", 1)
    places, pool = _pool(case)
    heads, dim, page = case["heads"], case["dim"], case["page"]
    dims, blocks = _padded(case), case["page"] // BLOCK
    if own:
        from paper_2002_02645_amd import binding

        s.pages = binding.FreezePages(layers, pool, rows, places, heads, dim, page, DEV)
        s.codes, s.scales, s.book = s.pages.codes, s.pages.scales, s.pages.book
    else:
        s.codes = torch.zeros(layers, pool, heads, blocks, 2, BLOCK * dims, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
        s.scales = torch.full((layers, pool, heads, blocks, 2), 1, dtype=torch.uint8, device=DEV)
        s.book = torch.zeros(rows * places + rows + pool, dtype=torch.int32, device=DEV)
    s.tables, s.lengths, s.refs = s.book.split([rows * places, rows, pool])
    s.tables = s.tables.view(rows, places)
    # tables: pages from all over the pool; the beams of a group share the pages of its common start
    past, new = _lengths(case)
    rng = random.Random(case["salt"] + 1)
    free = list(range(pool))
    rng.shuffle(free)
    tables, refs = [[-1] * places for _ in range(rows)], [0] * pool
    after = case["kind"] == "attend"      # the new tokens are there already
    held = [p + n if after else p for p, n in zip(past, new)]
    for r in range(rows):
        beam = r % case["beams"] if "beams" in case else 0
        for j in range(_pages(held[r], page)):
            shared = beam and j < held[r] // page and j < _pages(held[r], page) * 3 // 4
            tables[r][j] = tables[r - 1][j] if shared else free.pop()
            refs[tables[r][j]] += 1
    s.tables.copy_(torch.tensor(tables, dtype=torch.int32))
    s.lengths.copy_(torch.tensor(held, dtype=torch.int32))
    s.refs.copy_(torch.tensor(refs, dtype=torch.int32))
    s.start = s.book.clone()
    s.add = torch.tensor(new, dtype=torch.int32, device=DEV)
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    s.starts = torch.tensor(at, dtype=torch.int32, device=DEV)
    s.total, s.most = at[-1], max(new)
    if filled:   # values of one size for each token and head, a few dims far larger
        one = (dims, blocks * 2 * BLOCK * heads)
        for layer in range(layers):
            for p in range(0, pool, max(1, (1 << 27) // (one[0] * one[1]))):
                to = slice(p, min(pool, p + max(1, (1 << 27) // (one[0] * one[1]))))
                x = torch.randn(to.stop - to.start, heads, blocks, 2, BLOCK, dims, generator=g, device=DEV)
                x *= torch.exp(0.5 * torch.randn(to.stop - to.start, heads, blocks, 2, BLOCK, 1, generator=g, device=DEV))
                x *= torch.where(torch.arange(dims, device=DEV) < dim, 1.0, 0.0) * torch.where(torch.arange(dims, device=DEV) % 61 == 7, 4.0, 1.0)
                e = _exponent(x.abs().amax((-1, -2)))
                s.codes[layer, to].copy_(_pack((x * _power(-e)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)).view(torch.float8_e4m3fn))
                s.scales[layer, to].copy_((e + 127).to(torch.uint8))


def _normal(shape, g, half, by_row=True):
    x = torch.randn(shape, generator=g, device=DEV)
    if by_row:
        x *= torch.exp(0.5 * torch.randn(shape[0], 1, 1, generator=g, device=DEV))
    return x.to(torch.bfloat16) if half else x


def _frequencies(rot, scaled):
    """Radians per position of each pair; scaled: long wavelengths stretched eightfold, short ones kept, a ramp between them."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if scaled:
        turns = 8192 * f / (2 * math.pi)
        keep = ((turns - 1) / (4 - 1)).clamp(0, 1)
        f = f * (keep + (1 - keep) / 8)
    return f


def _prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(1000003 * seed + 29)
    s = State()
    s.case, kind = case, case["kind"]
    if kind == "rotate":
        s.q = _normal((case["tokens"], case["q_heads"], case["dim"]), g, case["bf16"])
        s.k = _normal((case["tokens"], case["heads"], case["dim"]), g, case["bf16"])
        s.positions = torch.randint(0, case["far"], (case["tokens"],), generator=g, device=DEV, dtype=torch.int32)
        s.frequencies, s.factor = _frequencies(case["rot"], case["scaled"]), 1.1 if case["scaled"] else 1.0
        return s
    _cache(s, case, g, filled=True)
    heads, dim = case["heads"], case["dim"]
    if kind == "append":
        s.k, s.v = (_normal((s.total, heads, dim), g, case["bf16"]) for _ in range(2))
    if kind == "attend":
        s.q = _normal((s.total, heads * case["group"], dim), g, case["bf16"])
    if kind in ("fork", "step"):   # each row goes on from a row of its own group
        rows, beams = _rows(case), case["beams"]
        first = torch.arange(rows, device=DEV) // beams * beams
        s.parents = (first + torch.randint(0, beams, (rows,), generator=g, device=DEV)).int()
    if kind == "step":
        s.q = [_normal((s.total, heads * case["group"], dim), g, True) for _ in range(case["layers"])]
        s.k, s.v = ([_normal((s.total, heads, dim), g, True) for _ in range(case["layers"])] for _ in range(2))
        s.frequencies = _frequencies(dim, False)
        s.positions = s.lengths.clone()
    return s


def prepare(case, seed):
    s = _prepare(case, seed)
    if own and case["kind"] in ("rotate", "step"):
        from paper_2002_02645_amd import binding

        s.cache = binding.FreezeCache(1, DEV)
    return s


# ---- plain forms -------------------------------------------------------------------------------------

def _rotate(x, positions, frequencies, inter, factor=1.0):
    rot = 2 * frequencies.numel()
    angle = positions.double()[:, None, None] * frequencies       # 64 bits: far positions
    cos, sin = (angle.cos() * factor).float(), (angle.sin() * factor).float()
    t = x[..., :rot].float()
    a, b = (t[..., ::2], t[..., 1::2]) if inter else t.chunk(2, -1)
    a, b = a * cos - b * sin, a * sin + b * cos
    t = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
    return torch.cat([t.to(x.dtype), x[..., rot:]], -1)


def _append(s, layer, k, v, lengths):
    """Every block that gets a token is taken out of its page, given its new exponent and put back."""
    case = s.case
    rows, heads, dim, page = _rows(case), case["heads"], case["dim"], case["page"]
    dims, per = _padded(case), page // BLOCK
    first = lengths - s.add                                                   # where the new tokens begin
    j = torch.arange(s.most // BLOCK + 2, device=DEV)
    block = first[:, None] // BLOCK + j                                       # [rows, blocks of the most]
    r, b = ((block * BLOCK < lengths[:, None]) & (s.add[:, None] > 0)).nonzero(as_tuple=True)
    block = block[r, b]
    at = s.tables[r, block // per].long(), block % per
    token = block[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)          # [n, 32]
    old, fresh = (token < first[r, None]), (token >= first[r, None]) & (token < lengths[r, None])
    source = (s.starts[r, None] + token - first[r, None]).clamp(0, s.total - 1)
    x = torch.stack([k[source], v[source]], 1).float().movedim(3, 1)          # [n, heads, 2, 32, dim]
    x = torch.nn.functional.pad(x, (0, dims - dim)) * fresh[:, None, None, :, None]
    codes, scales = s.codes[layer].view(torch.uint8), s.scales[layer]
    was = _unpack(codes[at[0], :, at[1]], dims) * old[:, None, None, :, None]
    e_was = torch.where(old.any(1)[:, None, None], scales[at[0], :, at[1]].int() - 127, -126)
    e = torch.maximum(e_was, _exponent(x.abs().amax((-1, -2))))
    x = x * _power(-e)[..., None, None] + was * torch.exp2((e_was - e).float())[..., None, None]
    codes[at[0], :, at[1]] = _pack(x.to(torch.float8_e4m3fn).view(torch.uint8))
    scales[at[0], :, at[1]] = (e + 127).to(torch.uint8)


def _attend(s, layer, q, lengths):
    case = s.case
    rows, heads, dim, page, window = _rows(case), case["heads"], case["dim"], case["page"], case.get("window", 0)
    dims, group, new = _padded(case), case["group"], s.most
    at = s.tables.long().clamp(min=0)
    codes = _unpack(s.codes[layer].view(torch.uint8)[at], dims)               # [rows, places, heads, blocks, 2, 32, dims]
    x = codes * _power(s.scales[layer][at].int() - 127)[..., None, None]
    x = x[..., :dim].permute(4, 0, 2, 1, 3, 5, 6).reshape(2, rows, heads, -1, dim)
    i = torch.arange(new, device=DEV)
    source = (s.starts[:-1, None] + i).clamp(max=s.total - 1)                 # [rows, new]
    y = q[source].view(rows, new, heads, group, dim).permute(0, 2, 1, 3, 4).reshape(rows, heads, new * group, dim)
    scores = (y.float() @ x[0].transpose(-1, -2)) / dim ** 0.5
    place = (lengths - s.add)[:, None] + i                                    # [rows, new]
    token = torch.arange(x.shape[3], device=DEV)
    seen = token <= place[:, :, None]
    if window:
        seen &= token > place[:, :, None] - window
    seen = seen.repeat_interleave(group, 1)[:, None]
    scores = torch.where(seen, scores, -math.inf)
    p = (scores - scores.amax(-1, keepdim=True)).exp()
    y = (p @ x[1]) / p.sum(-1, keepdim=True)
    y = y.view(rows, heads, new, group, dim).permute(0, 2, 1, 3, 4).reshape(rows, new, heads * group, dim)
    return y[(i < s.add[:, None])].to(q.dtype)


def _fork(s, parents):
    s.tables.copy_(s.tables[parents.long()])
    s.lengths.copy_(s.lengths[parents.long()])
    held = s.tables.view(-1)
    s.refs.copy_(torch.zeros(s.refs.numel() + 1, dtype=torch.int32, device=DEV).index_add_(0, torch.where(held < 0, s.refs.numel(), held).long(),
                                                                                          torch.ones_like(held))[:-1])


def _reserve(s):
    """A place for one more token in every row: a new page where the last one is full, a copy of a last page that others hold too."""
    page, (rows, places), pool = s.case["page"], s.tables.shape, s.refs.numel()
    at = (s.lengths // page).long().clamp(max=places - 1)
    r = torch.arange(rows, device=DEV)
    last = s.tables[r, at]
    full = s.lengths % page == 0
    copy = ~full & (s.refs[last.long().clamp(min=0)] > 1)
    need = (full | copy).int()
    free = torch.sort((s.refs > 0).int(), stable=True).indices                # free pages first, in order
    count = (s.refs == 0).sum()
    mine = need.cumsum(0) - need
    granted = ((need == 0) | (mine < count)) & (s.lengths // page < places)
    got = (granted & (need > 0))
    new = free[mine.clamp(max=pool - 1)]
    s.tables[r, at] = torch.where(got, new.int(), last)
    r = (got & copy).nonzero().view(-1)
    filled = torch.arange(page // BLOCK, device=DEV) * BLOCK < (s.lengths % page)[r, None]      # blocks that hold tokens
    for x in (s.codes.view(torch.uint8), s.scales):
        keep = filled.view(1, -1, 1, page // BLOCK, 1, *[1] * (x.dim() - 5))
        x[:, new[r]] = torch.where(keep, x[:, last[r].long()], x[:, new[r]])
    s.refs.index_add_(0, new, got.int())
    s.refs.index_add_(0, last.long().clamp(min=0), -(got & copy).int())
    s.lengths += granted.int()
    return granted.int()


def _compact(s):
    used = s.refs > 0
    count = used.sum()
    page = torch.arange(s.refs.numel(), device=DEV)
    src, dst = (used & (page >= count)).nonzero().view(-1), (~used & (page < count)).nonzero().view(-1)
    to = page.clone()
    to[src] = dst
    s.codes.view(torch.uint8)[:, dst] = s.codes.view(torch.uint8)[:, src]
    s.scales[:, dst] = s.scales[:, src]
    s.tables.copy_(torch.where(s.tables >= 0, to[s.tables.long().clamp(min=0)].int(), -1))
    s.refs[dst] = s.refs[src]
    s.refs[src] = 0
    return count.int().view(1)


def _book(s):
    return dict(tables=s.tables, lengths=s.lengths, refs=s.refs)


def _whole(s):
    """What the pages in use hold (pages that a table names; what the others held is nobody's)."""
    return dict(codes=s.codes, scales=s.scales)


def run(s):
    case, kind = s.case, s.case["kind"]
    if own:
        return _run_own(s, case, kind)
    if kind == "rotate":
        return [_rotate(x, s.positions, s.frequencies, case["inter"], s.factor) for x in (s.q, s.k)]
    if kind == "attend":
        return _attend(s, 0, s.q, s.lengths)
    if kind == "append":
        # the rows hold the new tokens from now on; their pages are there
        s.book.copy_(s.start)
        granted = _grow(s)
        _append(s, 0, s.k, s.v, s.lengths)
        return dict(_whole(s), **_book(s), granted=granted)
    s.book.copy_(s.start)
    if kind == "compact":
        used = _compact(s)
        return dict(_whole(s), **_book(s), used=used)
    _fork(s, s.parents)
    granted = _reserve(s)
    if kind == "fork":
        return dict(_whole(s), **_book(s), granted=granted)
    out = []
    for layer in range(case["layers"]):
        q, k = (_rotate(x, s.positions, s.frequencies, False) for x in (s.q[layer], s.k[layer]))
        _append(s, layer, k, s.v[layer], s.lengths)
        out.append(_attend(s, layer, q, s.lengths))
    return dict(_whole(s), **_book(s), granted=granted, out=out)


def _grow(s):
    """Places for all new tokens of rows that share no page: free pages in order, row by row."""
    page, (rows, places) = s.case["page"], s.tables.shape
    had, has = -(-s.lengths // page), -(-(s.lengths + s.add) // page)
    mine = (has - had).cumsum(0) - (has - had)
    free = torch.sort((s.refs > 0).int(), stable=True).indices.int()
    j = torch.arange(places, device=DEV)
    gets = (j >= had[:, None]) & (j < has[:, None])
    new = free[(mine[:, None] + j - had[:, None]).clamp(0, free.numel() - 1)]
    s.tables.copy_(torch.where(gets, new, s.tables))
    s.refs.index_add_(0, new.view(-1), gets.view(-1).int())
    s.lengths += s.add
    return s.add


def _run_own(s, case, kind):
    if kind == "rotate":
        return s.cache.rotate_positions((s.q, s.k), s.positions, s.frequencies, interleaved=case["inter"], factor=s.factor)
    p = s.pages
    if kind == "attend":
        if case["new"] == 1:
            return p.attend(0, s.q, window=case["window"])
        return p.attend(0, s.q, starts=s.starts, most=s.most, window=case["window"])
    p.book.copy_(s.start)
    if kind == "append":
        granted = p.reserve(s.add)
        if case["new"] == 1:
            p.append(0, s.k, s.v)
        else:
            p.append(0, s.k, s.v, starts=s.starts, most=s.most)
        return dict(_whole(s), **_book(s), granted=granted)
    if kind == "compact":
        used = p.compact()
        return dict(_whole(s), **_book(s), used=used)
    p.fork(s.parents)
    granted = p.reserve()
    if kind == "fork":
        return dict(_whole(s), **_book(s), granted=granted)
    out = []
    for layer in range(case["layers"]):
        q, k = s.cache.rotate_positions((s.q[layer], s.k[layer]), s.positions, s.frequencies)
        p.append(layer, k, s.v[layer])
        out.append(p.attend(layer, q))
    return dict(_whole(s), **_book(s), granted=granted, out=out)


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    kind, dim = case["kind"], case["dim"]
    if kind == "rotate":
        n = case["tokens"] * (case["q_heads"] + case["heads"])
        return {"bytes": n * dim * (4 if case["bf16"] else 8) + 4 * case["tokens"], "flops": 3 * n * case["rot"]}
    past, new = _lengths(case)
    heads, size = case["heads"], 2 if case.get("bf16", True) else 4
    token = 2 * heads * (dim + 1 / BLOCK)               # bytes of a token's keys and values in a layer
    append = sum(new) * (2 * heads * dim * size + token)
    if kind == "append":
        return {"bytes": append, "flops": 6 * sum(new) * heads * dim}
    pages = sum(_pages(n, case["page"]) for n in past)
    if kind == "compact":
        most, pool = _pool(case)
        moved = pages * (1 - pages / pool)              # the pages in use lie evenly over the pool
        return {"bytes": 2 * moved * case["page"] * token * case["layers"] + 8 * pages + 4 * pool, "flops": 0}
    fork = 8 * pages + 0.5 * sum(2 * (n % case["page"]) for n in past) * token * case.get("layers", 1)   # half of the last pages are shared
    if kind == "fork":
        return {"bytes": fork, "flops": 0}
    seen = read = 0                                     # pairs of a query and a token; tokens read by a row
    for p, n in zip(past, new):
        w = case.get("window", 0) or p + n
        read += min(p + n, w + n - 1)
        full = max(0, min(n, p + n - w + 1))            # queries that see a whole window
        seen += full * w + sum(p + 1 + i for i in range(n - full))
    queries = sum(new) * heads * case["group"] * dim
    attend = {"bytes": read * token + 2 * queries * size, "flops": 4 * seen * heads * case["group"] * dim}
    if kind == "attend":
        return attend
    one = attend["bytes"] + append + 2 * (queries + sum(new) * heads * dim) * size
    return {"bytes": case["layers"] * one + fork, "flops": case["layers"] * attend["flops"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _places(dims):
    """Where token t, dim c of a block's keys and values lie among its bytes: [2, 32, dims]."""
    t = torch.arange(32, device=DEV)[:, None]
    c = torch.arange(dims, device=DEV)[None, :]
    keys = (c // 32) * 1024 + ((c % 32 // 8) * 16 + t % 16) * 16 + (t // 16) * 8 + c % 8
    values = (c // 32) * 1024 + ((t % 16 // 4) * 16 + c % 16) * 16 + (c % 32 // 16) * 8 + (t // 16) * 4 + t % 4
    return torch.stack([keys, values])


def _read(s, layer, r, n, table):
    """The first n tokens' keys and values of a row in 64 bits, [2, heads, n, dim]."""
    case = s.case
    per, dims = case["page"] // BLOCK, _padded(case)
    ids = torch.tensor(table, device=DEV)[: _pages(n, case["page"])]
    x = s.codes[layer].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double()   # [pages, heads, blocks, 2, bytes]
    at = _places(dims).view(2, -1)
    x = torch.stack([x[..., 0, :][..., at[0]], x[..., 1, :][..., at[1]]], 3).view(*x.shape[:4], 32, dims)
    x = x * torch.exp2(s.scales[layer, ids].double() - 127)[..., None, None]
    return x.permute(3, 1, 0, 2, 4, 5).reshape(2, case["heads"], -1, dims)[:, :, :n, : case["dim"]]


def _exact_attend(s):
    case = s.case
    group, dim, window = case["group"], case["dim"], case["window"]
    starts, lengths, tables, out = s.starts.tolist(), s.lengths.tolist(), s.tables.tolist(), []
    for r, n in enumerate(lengths):
        q = s.q[starts[r]:starts[r + 1]].double()
        kv = _read(s, 0, r, n, tables[r])
        rows = []
        for h in range(case["heads"]):
            for at in range(0, q.shape[0], 1024):
                piece = q[at:at + 1024, h * group:(h + 1) * group].reshape(-1, dim)
                x = torch.matmul(piece, kv[0, h].t().contiguous()) / math.sqrt(dim)
                place = (n - q.shape[0] + at + torch.arange(piece.shape[0], device=DEV) // group)[:, None]
                token = torch.arange(n, device=DEV)[None, :]
                hidden = (token > place) | (token <= place - window if window else token < 0)
                rows.append((h, at, torch.matmul(torch.softmax(x.masked_fill(hidden, -math.inf), 1), kv[1, h]).view(-1, group, dim)))
        y = torch.empty(q.shape, dtype=torch.float64, device=DEV)
        for h, at, part in rows:
            y[at:at + part.shape[0], h * group:(h + 1) * group] = part
        out.append(y)
    return torch.cat(out)


def _nearest(t):
    """The nearest number of 1 + 4 + 3 bits, halfway cases to the even one."""
    step = torch.exp2(torch.frexp(t).exponent.double().clamp(min=-5) - 4)
    return torch.round(t / step) * step


def _exact_append(s):
    """Codes after the new tokens, block by block (the pages are those of the plain form's bookkeeping)."""
    case = s.case
    dims, page, dim = _padded(case), case["page"], case["dim"]
    _grow(s)
    codes = s.codes[0].double()
    starts, lengths, tables, add = s.starts.tolist(), s.lengths.tolist(), s.tables.tolist(), s.add.tolist()
    at = _places(dims)
    x64 = torch.stack([s.k, s.v]).double()              # [2, total, heads, dim]
    for r, n in enumerate(lengths):
        first = n - add[r]
        for b in range(first // BLOCK, _pages(n, BLOCK)):
            p, i, kept = tables[r][b * BLOCK // page], b * BLOCK % page // BLOCK, max(0, first - b * BLOCK)
            new = x64[:, starts[r] + max(0, b * BLOCK - first): starts[r] + min(n, (b + 1) * BLOCK) - first].movedim(2, 0)   # [heads, 2, m, dim]
            e = torch.ceil(torch.log2(new.abs().amax((-1, -2)) / 448)).clamp(min=-126)
            block = torch.zeros(case["heads"], 2, 32, dims, dtype=torch.float64, device=DEV)
            if kept:
                was = s.scales[0, p, :, i].double() - 127
                e = torch.maximum(e, was)
                held = torch.stack([codes[p, :, i, kv][:, at[kv]] for kv in (0, 1)], 1)
                block[:, :, :kept] = _nearest(held[:, :, :kept] * torch.exp2(was - e)[..., None, None])
            block[:, :, kept:kept + new.shape[2], :dim] = _nearest(new / torch.exp2(e)[..., None, None])
            for kv in (0, 1):
                codes[p, :, i, kv, at[kv].reshape(-1)] = block[:, kv].reshape(case["heads"], -1)
    return dict(codes=codes.unsqueeze(0), scales=None, tables=None, lengths=None, refs=None, granted=None)


def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "compact", "step"):
        return None                                     # copies and whole numbers; a step's parts are other cases
    if kind == "append" and sum(_lengths(case)[1]) > 20000:
        return None
    s = _prepare(case, seed)
    if kind == "append":
        return _exact_append(s)
    if kind == "attend":
        return _exact_attend(s)
    got = []
    for x in (s.q, s.k):
        y, rot = x.double(), case["rot"]
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if case["inter"] else (i, i + rot // 2)
            angle = (s.positions.double() * s.frequencies[i])[:, None]
            u, w = x[..., a].double(), x[..., b].double()
            y[..., a] = s.factor * (u * torch.cos(angle) - w * torch.sin(angle))
            y[..., b] = s.factor * (w * torch.cos(angle) + u * torch.sin(angle))
        got.append(y)
    return got
