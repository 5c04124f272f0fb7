"""The operators behind the caches of a generating model, as cases for timing and comparison: what no layer freezes goes
through the model's output layer in 8 bits, the next tokens of a request's beams are chosen, and the batch's states follow
the beams that were kept.

Every case is a dict of plain values; its "kind" says which public entry points a pass goes through:

  quantise  rows into 8-bit codes (e4m3) with a power of two for each block of 128 values
  project   the dense layer on such codes: rows are quantised within the call, or handed over as codes ("given")
  select    the k best continuations of every group of beams over beams and vocabulary
  reorder   states of the rows of a batch, taken from the rows' parents
  step      project, select and reorder one after the other, as a step of decoding does

Sizes are those of the repository's benchmark configurations (8,192, 16,384 and 65,536 values a row, 1,024 outputs of a
dimension-reducing layer, batches of 10,000), generic ones for vocabularies, and odd sizes between them.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 128


def listed():
    return [
        # one step's rows of a serving batch before several products share them: launches and latencies count
        dict(name="quantise_rows_16", kind="quantise", b=16, d=4096, bf16=True),
        # an evaluation batch of a block's outputs
        dict(name="quantise_batch", kind="quantise", b=10000, d=8192, bf16=False),
        # the output layer for one request: the weights are read once for one row
        dict(name="project_token", kind="project", b=1, d=4096, m=32768, bf16=True, out16=False, relu=False, bias=False, given=False),
        # the output layer for the beams of a serving batch, the largest vocabulary
        dict(name="project_beams", kind="project", b=32, d=8192, m=131072, bf16=True, out16=False, relu=False, bias=False, given=False),
        # the dimension-reducing layer in front of a look-up, a whole evaluation batch
        dict(name="project_block", kind="project", b=10000, d=8192, m=1024, bf16=False, out16=False, relu=True, bias=True, given=False),
        # a prompt's rows through a square layer: bound by the matrix pipes
        dict(name="project_square", kind="project", b=4096, d=8192, m=8192, bf16=True, out16=True, relu=False, bias=False, given=False),
        # odd sizes, a middling batch whose codes several products share
        dict(name="project_odd", kind="project", b=301, d=16391, m=1501, bf16=False, out16=False, relu=False, bias=True, given=True),
        # one request, four beams
        dict(name="select_one", kind="select", groups=1, beams=4, vocab=32000, k=4, bf16=False, masked=0.0, done=0.0, first=False),
        # a serving batch, twice as many continuations as beams, some tokens forbidden, some beams at their end
        dict(name="select_batch", kind="select", groups=64, beams=8, vocab=131072, k=16, bf16=True, masked=0.02, done=0.1, first=False),
        # keys and values of a small model, one request: latency counts
        dict(name="reorder_one", kind="reorder", states=8, rows=4, heads=4, most=256, used=77, width=64),
        # keys and values of 16 layers for 32 beams, 1,021 of 1,280 places used
        dict(name="reorder_batch", kind="reorder", states=32, rows=32, heads=8, most=1280, used=1021, width=128),
        # a step of decoding: output layer, choice, states
        dict(name="step_batch", kind="step", groups=8, beams=4, d=4096, vocab=50021, states=16, heads=8, most=512, used=300, width=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantise", "project", "project", "project", "project", "select", "select", "reorder", "step"])
    if kind == "quantise":
        d = rng.choice([512, 8192, _log(rng, 100, 65536), _log(rng, 100, 65536) // 8 * 8])
        return dict(kind=kind, b=_log(rng, 1, max(2, min(10000, 8e7 / d))), d=d, bf16=rng.random() < 0.5)
    if kind == "project":
        d = rng.choice([1024, 4096, 8192, _log(rng, 100, 65536), _log(rng, 100, 65536) // 16 * 16])
        m = rng.choice([1024, 32768, _log(rng, 64, 131072), _log(rng, 64, 131072) // 8 * 8])
        m = int(max(64, min(m, 1.0e9 // d)))
        b = _log(rng, 1, max(2, min(10000, 2.7e11 / d / m)))
        return dict(kind=kind, b=b, d=d, m=m, bf16=rng.random() < 0.6, out16=rng.random() < 0.4, relu=rng.random() < 0.3,
                    bias=rng.random() < 0.5, given=rng.random() < 0.25)
    if kind == "select":
        beams = rng.choice([1, 2, 4, 5, 8, 16])
        vocab = rng.choice([32000, 131072, _log(rng, 500, 131072)])
        groups = _log(rng, 1, max(2, min(128, 6.7e7 / beams / vocab)))
        return dict(kind=kind, groups=groups, beams=beams, vocab=vocab, k=min(rng.choice([beams, 2 * beams]), vocab),
                    bf16=rng.random() < 0.5, masked=rng.choice([0.0, 0.02, 0.5]), done=rng.choice([0.0, 0.1, 0.4]),
                    first=rng.random() < 0.2)
    if kind == "reorder":
        rows, heads, width = _log(rng, 2, 64), rng.choice([1, 4, 8]), rng.choice([64, 80, 128, rng.randint(3, 200)])
        states = rng.choice([2, 8, 24, 48])
        most = _log(rng, 16, max(32, min(4096, 1.3e9 / (rows * heads * width * states))))
        return dict(kind=kind, states=states, rows=rows, heads=heads, most=most, used=rng.randint(1, most), width=width)
    d, vocab = rng.choice([1024, 4096, _log(rng, 300, 8192)]), _log(rng, 2000, 65536)
    most = _log(rng, 32, 512)
    return dict(kind=kind, groups=_log(rng, 1, 16), beams=rng.choice([1, 3, 4, 8]), d=d, vocab=vocab, states=rng.choice([4, 16]),
                heads=rng.choice([2, 8]), most=most, used=rng.randint(1, most), width=rng.choice([64, 128]))


class State:
    pass


def _rows(b, d, g, half):
    """Activations: rows of different size, values of a normal distribution, a few channels far larger."""
    x = torch.randn(b, d, generator=g, device=DEV)
    x *= torch.exp(torch.randn(b, 1, generator=g, device=DEV))
    x *= torch.where(torch.rand(1, d, generator=g, device=DEV) < 0.01, 20.0, 1.0)
    return x.to(torch.bfloat16) if half else x


def _codes(x):
    """Plain form of the quantisation: codes [rows, columns padded to 128], scale bytes [rows, blocks padded to 4]."""
    b, d = x.shape
    nb = -(-d // BLOCK)
    t = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - d)).view(b, nb, BLOCK)
    bits = t.abs().amax(2).view(torch.int32)
    # the largest value is 1.f 2^E: at most 448 = 1.75 2^8 after the division by 2^e
    e = ((bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp_(min=-126)
    codes = (t * ((127 - e) << 23).view(torch.float32).unsqueeze(2)).to(torch.float8_e4m3fn).view(b, nb * BLOCK)
    return codes, torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -nb % 4), value=1)


def _values(codes, scales):
    """The values that codes and scale bytes stand for (an exponent of -126 at least: the scale is a normal number)."""
    nb = codes.shape[1] // BLOCK
    s = (scales[:, :nb].to(torch.int32) << 23).view(torch.float32)
    return (codes.float().view(-1, nb, BLOCK) * s.unsqueeze(2)).view(codes.shape)


def _weights(s, m, d, g, bias):
    w = torch.empty(m, d, device=DEV, dtype=torch.bfloat16).normal_(generator=g)
    parts = [_codes(p) for p in (w / d ** 0.5).split(8192)]
    s.w_codes, s.w_scales = (torch.cat([p[i] for p in parts]) for i in (0, 1))
    s.bias = torch.randn(m, generator=g, device=DEV) * 0.1 if bias else None


def _states(s, case, rows, g):
    shape = (case["states"], rows, case["heads"], case["most"], case["width"])
    s.src = torch.empty(shape, device=DEV, dtype=torch.bfloat16).normal_(generator=g)
    s.dst = torch.zeros(shape, device=DEV, dtype=torch.bfloat16)
    s.used = case["used"]


def _prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(1000003 * seed + 17)
    s = State()
    s.case, kind = case, case["kind"]
    if kind == "quantise":
        s.x = _rows(case["b"], case["d"], g, case["bf16"])
    elif kind == "project":
        s.x = _rows(case["b"], case["d"], g, case["bf16"])
        _weights(s, case["m"], case["d"], g, case["bias"])
        s.given = _codes(s.x) if case["given"] else None
    elif kind == "select":
        rows, v = case["groups"] * case["beams"], case["vocab"]
        x = torch.randn(rows, v, generator=g, device=DEV) * 2.5
        if case["masked"]:
            x.masked_fill_(torch.rand(rows, v, generator=g, device=DEV) < case["masked"], -math.inf)
        s.logits = x.to(torch.bfloat16) if case["bf16"] else x
        s.scores = -10 * torch.rand(rows, generator=g, device=DEV)
        if case["first"]:   # the first step: all beams but one of a group are empty
            s.scores.view(-1, case["beams"])[:, 1:] = -math.inf
        s.done = (torch.rand(rows, generator=g, device=DEV) < case["done"]).to(torch.uint8)
    elif kind == "reorder":
        _states(s, case, case["rows"], g)
        s.parents = torch.randint(0, case["rows"], (case["rows"],), generator=g, device=DEV, dtype=torch.int32)
    else:
        rows = case["groups"] * case["beams"]
        s.x = _rows(rows, case["d"], g, True)
        s.x = (s.x.float() / s.x.float().square().mean(1, keepdim=True).sqrt() * 2.5).to(torch.bfloat16)   # a last norm's output
        _weights(s, case["vocab"], case["d"], g, False)
        s.scores = -10 * torch.rand(rows, generator=g, device=DEV)
        s.done = torch.zeros(rows, dtype=torch.uint8, device=DEV)
        _states(s, case, rows, g)
    return s


END = 2   # the end token


def prepare(case, seed):
    s = _prepare(case, seed)
    if own:
        from paper_2002_02645_amd import binding

        s.cache = binding.FreezeCache(1, DEV)
        if case["kind"] in ("project", "step"):
            s.cache.build_quantised(0, s.w_codes, s.bias, scales=s.w_scales, d=case["d"])
    return s


# ---- plain forms ------------------------------------------------------------------------------------

def _project(codes, scales, s, relu, half):
    y = _values(codes, scales) @ _values(s.w_codes, s.w_scales).t()
    if s.bias is not None:
        y = y + s.bias
    if relu:
        y = y.clamp(min=0)
    return y.to(torch.bfloat16) if half else y


def _select(logits, scores, done, groups, beams, k):
    x = logits.double()   # sums over the vocabulary, and totals that lie close together
    top = x.amax(1, keepdim=True).clamp(min=-1e300)
    total = scores.double().unsqueeze(1) + (x - top - (x - top).exp().sum(1, keepdim=True).log())
    total = torch.where(torch.isnan(total), -math.inf, total)   # nothing left in the row
    last = torch.full_like(total, -math.inf)
    last[:, END] = scores.double()
    total = torch.where(done.bool().unsqueeze(1), last, total).view(groups, -1)
    best, at = total.sort(dim=1, descending=True, stable=True)
    best, at = best[:, :k], at[:, :k]
    vocab = logits.shape[1]
    some = best > -math.inf
    tokens = torch.where(some, at % vocab, END).int()
    first = beams * torch.arange(groups, device=at.device).unsqueeze(1)
    parents = (first + torch.where(some, at // vocab, 0)).int()
    return dict(score=best.float(), token=tokens, parent=parents, finished=(tokens == END).to(torch.uint8))


def _reorder(s, parents):
    s.dst[:, :, :, : s.used] = s.src[:, parents.long(), :, : s.used]
    return s.dst


def run(s):
    case, kind = s.case, s.case["kind"]
    if own:
        return _run_own(s, case, kind)
    if kind == "quantise":
        return _codes(s.x)
    if kind == "project":
        codes, scales = s.given or _codes(s.x)
        return _project(codes, scales, s, case["relu"], case["out16"])
    if kind == "select":
        return _select(s.logits, s.scores, s.done, case["groups"], case["beams"], case["k"])
    if kind == "reorder":
        return _reorder(s, s.parents)
    logits = _project(*_codes(s.x), s, False, False)
    out = _select(logits, s.scores, s.done, case["groups"], case["beams"], case["beams"])
    return dict(out, logits=logits, states=_reorder(s, out["parent"].view(-1)))


def _run_own(s, case, kind):
    c = s.cache
    if kind == "quantise":
        return c.quantise_rows(s.x)
    if kind == "project":
        out_dtype = torch.bfloat16 if case["out16"] else torch.float32
        if s.given:
            return c.quantised_project(0, s.given[0], scales=s.given[1], relu=case["relu"], out_dtype=out_dtype)
        return c.quantised_project(0, s.x, relu=case["relu"], out_dtype=out_dtype)
    if kind == "select":
        return c.beam_select(s.logits, s.scores, case["beams"], case["k"], finished=s.done, end_token=END)
    if kind == "reorder":
        c.reorder_states(s.src, s.dst, s.parents, used=s.used, row_dim=1)
        return s.dst
    logits = c.quantised_project(0, s.x)
    out = c.beam_select(logits, s.scores, case["beams"], case["beams"], finished=s.done, end_token=END)
    c.reorder_states(s.src, s.dst, out["parent"].view(-1), used=s.used, row_dim=1)
    return dict(out, logits=logits, states=s.dst)


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "quantise":
        n = case["b"] * case["d"]
        return {"bytes": n * ((2 if case["bf16"] else 4) + 1 + 1 / BLOCK), "flops": 3 * n}
    if kind in ("project", "step"):
        b = case["b"] if kind == "project" else case["groups"] * case["beams"]
        m, d = case["m"] if kind == "project" else case["vocab"], case["d"]
        x = (1 + 1 / BLOCK) if case.get("given") else (2 if case.get("bf16", True) else 4)
        size = m * d * (1 + 1 / BLOCK) + b * d * x + b * m * (2 if case.get("out16") else 4) + (4 * m if case.get("bias") else 0)
        more = 4 * _moved(case, b) if kind == "step" else 0
        return {"bytes": size + more, "flops": 2 * b * m * d}
    if kind == "select":
        n = case["groups"] * case["beams"] * case["vocab"]
        return {"bytes": n * (2 if case["bf16"] else 4) * (1 - case["done"]) + 13 * case["groups"] * case["k"], "flops": 5 * n}
    return {"bytes": 4 * _moved(case, case["rows"]), "flops": 0}


def _moved(case, rows):
    return case["states"] * rows * case["heads"] * case["used"] * case["width"]


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def _exact_codes(x):
    """(codes as the numbers they are, exponents) of rows in 64 bits, from the definition: the smallest exponent >= -126 with
    max|x| <= 448 2^e, then the nearest number of 1 + 4 + 3 bits, halfway cases to the even one."""
    x = x.double()
    b, d = x.shape
    nb = (d + BLOCK - 1) // BLOCK
    t = torch.zeros(b, nb * BLOCK, dtype=torch.float64, device=x.device)
    t[:, :d] = x
    t = t.reshape(b, nb, BLOCK)
    e = torch.ceil(torch.log2(t.abs().max(2).values / 448)).clamp(-126, 127)   # log2(0): -inf, clamped
    t = t / torch.exp2(e).unsqueeze(2)
    step = torch.exp2(torch.frexp(t).exponent.double().clamp(min=-5) - 4)   # subnormal codes: steps of 2^-9
    return (torch.round(t / step) * step).reshape(b, nb * BLOCK), e


def _exact_values(codes, e):
    return (codes.reshape(codes.shape[0], -1, BLOCK) * torch.exp2(e).unsqueeze(2)).reshape(codes.shape)


def _exact_project(x, s, relu):
    xv = _exact_values(*_exact_codes(x))
    out = []
    for at in range(0, s.w_codes.shape[0], 16384):
        codes = s.w_codes[at:at + 16384].double()
        nb = codes.shape[1] // BLOCK
        w = _exact_values(codes, s.w_scales[at:at + 16384, :nb].double() - 127)
        y = xv @ w.t().contiguous()
        if s.bias is not None:
            y += s.bias[at:at + 16384].double()
        out.append(y)
    y = torch.cat(out, 1)
    return torch.relu(y) if relu else y


def _exact_select(logits, scores, done, beams, k):
    rows, vocab = logits.shape
    found = []
    for g in range(rows // beams):
        total = []
        for r in range(g * beams, (g + 1) * beams):
            row = torch.full((vocab,), -math.inf, dtype=torch.float64, device=logits.device)
            if done[r]:
                row[END] = scores[r].double()
            elif scores[r] > -math.inf and (logits[r] > -math.inf).any():
                x = logits[r].double()
                row = scores[r].double() + x - torch.logsumexp(x, 0)
            total.append(row)
        order = torch.sort(torch.cat(total), descending=True, stable=True)
        found.append(order.values[:k])
    # which tokens and parents: whole numbers, held to the plain form's
    return dict(score=torch.stack(found), token=None, parent=None, finished=None)


def exact(case, seed):
    s, kind = _prepare(case, seed), case["kind"]
    if kind == "quantise":
        return _exact_codes(s.x)[0], None
    if kind == "project":
        return _exact_project(s.x, s, case["relu"])
    if kind == "select":
        return _exact_select(s.logits, s.scores, s.done, case["beams"], case["k"])
    if kind == "reorder":
        out = s.dst.clone()
        for r, p in enumerate(s.parents.tolist()):
            out[:, r, :, : s.used] = s.src[:, p, :, : s.used]
        return out
    logits = _exact_project(s.x, s, False)
    return dict(_exact_select(logits, s.scores, s.done, case["beams"], case["beams"]), logits=logits, states=None)
