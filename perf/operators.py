"""Performance cases of the latent-cache operators: appending rotated rows to a
paged cache, attention over the rows that a step selected, 4-bit microscaled
quantisation and the product of two such matrices.

A row of the cache is one position's latent key (512 values, which are also its
value) and its rotated part (64 values): 1152 bytes in bfloat16, or 400 bytes
with the latent part in 4 bits (256 bytes of e2m1 codes, even column in the low
half of a byte, then 16 power-of-two scales, one per 32 columns) and the rotated
part in bfloat16.  A pass of a case is one call as a decode step or a prefill
makes it.
"""
import math

import torch

own = False         # the framework's kernels in place of the plain forms

LATENT, ROPE = 512, 64
BLOCK = 32          # values per scale
SHARED = 0.95       # of a later query token's rows are the first token's
SCALE = 192 ** -0.5  # of the scores: heads of 128 + 64 dimensions before the latent projection

# Fields of a case, by operator:
# append: requests, tokens of the longest one (ragged: the others have fewer), heads whose queries
#   are rotated, rows of a page, positions per request, row format
# attend: requests, query tokens, heads, selected rows per token (sparse) or longest context (dense:
#   every row of the context, through a page table), slots or context rows per request, row format,
#   whether part of the selected rows is masked
# quantize: rows, columns
# project: products, rows, columns and inner size of each; heads: whether the products are heads that
#   interleave in the activations' and the outputs' rows


def _append(name=None, **kw):
    return _named(dict(dict(op="append", requests=1, tokens=1, ragged=False, heads=16, page=64, context=512, mx4=True,
                            halves=False), **kw), name)


def _attend(name=None, **kw):
    return _named(dict(dict(op="attend", requests=1, tokens=1, heads=16, rows=2048, slots=8192, page=0, mx4=True,
                            masked=False), **kw), name)


def _quantize(name=None, **kw):
    return _named(dict(dict(op="quantize", rows=1, cols=512), **kw), name)


def _project(name=None, **kw):
    return _named(dict(dict(op="project", batch=1, m=1, n=512, k=512, heads=False), **kw), name)


def _named(case, name):
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # the new rows of a decode step: 64 requests with one draft token each, all heads' queries
        _append("append_step64", requests=64, tokens=2, heads=128, mx4=False),
        # a prefill of four prompts of different lengths into a cache of 4-bit rows
        _append("append_prefill", requests=4, tokens=8191, ragged=True, context=8192, halves=True),
        # one request of a small model: the smallest call, all latency
        _attend("attend_tiny", rows=256, slots=1024),
        # sizes off every power of two, two draft tokens, short contexts and a token without rows
        _attend("attend_odd11", requests=11, tokens=3, heads=40, rows=1000, slots=4096, masked=True),
        # the serving batch of the headline benchmark: one draft token, every head on this GPU
        _attend("attend_step64", requests=64, tokens=2, heads=128),
        # an ordinary batch over the rows as they are today, heads split over two GPUs
        _attend("attend_step16_bf16", requests=16, heads=64, mx4=False),
        # layers that attend over the whole of four long contexts, heads split over eight GPUs
        _attend("attend_long", requests=4, rows=131072, slots=131072, page=64),
        # one layer's activations of few tokens
        _quantize("quantize_odd", rows=33, cols=1184),
        # the attention's outputs of a step: 128 tokens of 128 heads
        _quantize("quantize_step64", rows=16384, cols=512),
        # one token through a weight matrix: the weights' bytes count
        _project("project_one", n=4096, k=4096),
        # the step's queries into the latent space, head by head
        _project("project_heads", batch=128, m=128, n=512, k=128, heads=True),
        # a prefill's tokens through a weight matrix
        _project("project_prefill", m=8192, n=4096, k=4096),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "quantize", "project"))
    if op == "append":
        if rng.random() < 0.5:
            tokens, requests = rng.choice((1, 2, 3, 4)), _log_between(rng, 1, 128)
        else:
            requests = rng.randint(1, 8)
            tokens = _log_between(rng, 16, 16384 // requests)
        heads = rng.choice((0, 8, 16, 20, 64, 128) if requests * tokens <= 1024 else (0, 8, 16))
        return _append(requests=requests, tokens=tokens, ragged=rng.random() < 0.5, heads=heads,
                       page=rng.choice((16, 64, 256)), context=tokens + rng.randint(1, 256),
                       mx4=rng.random() < 0.6, halves=rng.random() < 0.5)
    if op == "attend":
        heads = rng.choice((1, 8, 16, 16, 20, 32, 40, 64, 128))
        if rng.random() < 0.3:   # the whole context
            requests, tokens = rng.randint(1, 8), rng.choice((1, 1, 2))
            mx4 = rng.random() < 0.7
            most = min(131072, 4 * 131072 // (requests * tokens) * 16 // max(16, heads)) // (1 if mx4 else 3)
            rows = _log_between(rng, 1000, max(1001, most))
            return _attend(requests=requests, tokens=tokens, heads=heads, rows=rows, slots=rows,
                           page=rng.choice((16, 64, 256)), mx4=mx4, masked=rng.random() < 0.5)
        requests, tokens = _log_between(rng, 1, 64), rng.choice((1, 1, 2, 2, 3, 4))
        rows = rng.choice((256, 512, 1024, 2048, 2048, _log_between(rng, 100, 2048)))
        slots = min(8192, max(1024, 2 << (tokens * rows - 1).bit_length()))
        requests = max(1, min(requests, 128 // tokens))
        return _attend(requests=requests, tokens=tokens, heads=heads, rows=rows, slots=slots,
                       mx4=rng.random() < 0.7, masked=rng.random() < 0.4)
    if op == "quantize":
        cols = BLOCK * rng.choice((4, 16, 16, 37, 128, rng.randint(1, 256)))
        return _quantize(rows=_log_between(rng, 1, 16384 * 512 // cols), cols=cols)
    if rng.random() < 0.3:
        n, k = rng.choice(((512, 128), (128, 512), (256, 192)))
        return _project(batch=rng.choice((16, 20, 64, 128)), m=_log_between(rng, 1, 256), n=n, k=k, heads=True)
    return _project(m=_log_between(rng, 1, 4096), n=rng.choice((512, 1000, 1536, 2048, 4096)),
                    k=BLOCK * rng.choice((16, 37, 64, 128, 128)))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _marks(dev):
    """The values of the sixteen e2m1 codes."""
    return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6],
                        dtype=torch.float32, device=dev)


def _values(codes, scales, marks):
    """float32 values of e2m1 codes [..., K/2] with scales [..., K/32]."""
    v = torch.stack((marks[(codes & 15).long()], marks[(codes >> 4).long()]), -1).flatten(-2)
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    return (v.unflatten(-1, (-1, BLOCK)) * s.unsqueeze(-1)).flatten(-2)


def _quantized(x):
    """(codes, scales) of x [..., K]: per 32 values the power of two that leaves the largest one below 7
    (which rounds to at most 6), values rounded to the nearest of e2m1, ties to the even code."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1)
    e = (((top.contiguous().view(torch.int32) + 0x200000) >> 23) - 2).clamp(min=2)
    a = x.abs() / (e << 23).view(torch.float32).unsqueeze(-1)
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    c = (c + 8 * (x < 0)).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 2))
    return c[..., 0] | (c[..., 1] << 4), e.to(torch.uint8)


def _rows_of(latent, rope, mx4):
    """Bytes of the cache rows of latent [..., 512] and rope [..., 64], both bfloat16."""
    if not mx4:
        return torch.cat((latent, rope), -1).contiguous().view(torch.uint8)
    codes, scales = _quantized(latent)
    return torch.cat((codes, scales, rope.contiguous().view(torch.uint8)), -1)


def _row_bytes(mx4):
    return 400 if mx4 else 1152


def _lengths(case):
    n, r = case["tokens"], case["requests"]
    return [max(1, n - i * (n // r)) if case["ragged"] else n for i in range(r)]


def _pages_of(case):
    return -(-case["context"] // case["page"])


def _attend_lengths(case):
    """Verified length per request and token; in masked cases some positions lie at or past it."""
    far = 4 * case["rows"] if not case["page"] else case["rows"]
    out = []
    for r in range(case["requests"]):
        for g in range(case["tokens"]):
            if not case["masked"]:
                out.append(far)
            else:
                out.append(0 if (r + g) % 11 == 1 else max(1, far * (1 + (5 * r + 3 * g) % 7) // 7))
    return out


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(dev).manual_seed(seed)

    def normal(*shape, by=1.0):
        x = torch.randn(shape, generator=gen, device=dev)
        return (x * by).to(torch.bfloat16)

    s = dict(case, marks=_marks(dev))
    if case["op"] == "append":
        lengths, pages = _lengths(case), _pages_of(case)
        starts = [int(torch.randint(0, case["context"] - n + 1, (1,), generator=gen, device=dev)) for n in lengths]
        total = sum(lengths)
        s["request"] = torch.repeat_interleave(torch.arange(case["requests"], device=dev, dtype=torch.int32),
                                               torch.tensor(lengths, device=dev))
        s["position"] = torch.cat([torch.arange(a, a + n, device=dev) for a, n in zip(starts, lengths)])
        s["latent"], s["rope"] = normal(total, LATENT), normal(total, ROPE)
        s["q_rope"] = normal(total, case["heads"], ROPE) if case["heads"] else None
        s["q"] = torch.zeros(total, case["heads"], LATENT + ROPE, dtype=torch.bfloat16, device=dev) if case["heads"] else None
        turn = torch.arange(case["context"], device=dev, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, ROPE, 2, device=dev, dtype=torch.float64) / ROPE)
        s["angles"] = torch.stack((turn.cos(), turn.sin()), -1).float()
        s["table"] = torch.randperm(case["requests"] * pages, generator=gen, device=dev).to(torch.int32).view(-1, pages)
        s["pool"] = torch.zeros(case["requests"] * pages, case["page"], _row_bytes(case["mx4"]), dtype=torch.uint8, device=dev)
        return s
    if case["op"] == "attend":
        b, t, k, n = case["requests"], case["tokens"], case["rows"], case["slots"]
        per = case["page"] or n
        pages = -(-n // per)
        pool = torch.empty(b * pages, per, _row_bytes(case["mx4"]), dtype=torch.uint8, device=dev)
        for i in range(0, b * pages * per, 1 << 16):
            rows = pool.view(-1, pool.shape[-1])[i:i + (1 << 16)]
            rows.copy_(_rows_of(normal(rows.shape[0], LATENT), normal(rows.shape[0], ROPE), case["mx4"]))
        s["pool"] = pool
        s["q"] = normal(b, t, case["heads"], LATENT + ROPE)
        s["lens"] = torch.tensor(_attend_lengths(case), device=dev).view(b, t)
        if case["page"]:
            s["table"] = torch.randperm(b * pages, generator=gen, device=dev).to(torch.int32).view(b, pages)
            return s
        # a later token shares most of the first one's rows and has some of its own
        free = torch.rand(b, n, generator=gen, device=dev).argsort(-1).to(torch.int32)
        fresh = k - int(SHARED * k)
        s["picked"] = torch.stack([torch.cat((free[:, :k - fresh], torch.roll(free, -(g + 1) * fresh, 1)[:, k - fresh:k]), 1)
                                 if g else free[:, :k] for g in range(t)], 1).contiguous()
        s["index"] = torch.rand(b, t, 4 * k, generator=gen, device=dev).argsort(-1)[..., :k].to(torch.int32)
        return s
    if case["op"] == "quantize":
        # activations: a few columns are much larger than the others
        x = normal(case["rows"], case["cols"])
        s["x"] = x * torch.where(torch.rand(case["cols"], generator=gen, device=dev) < 0.02, 20.0, 1.0).to(torch.bfloat16)
        return s
    b, m, n, k = (case[f] for f in ("batch", "m", "n", "k"))
    s["x"] = normal(m, b, k)
    w = normal(b, n, k, by=k ** -0.5)
    s["w"] = _quantized(w)
    # the queries' buffer, whose last columns are the rotated part
    s["out"] = torch.zeros(m, b, n + (ROPE if case["heads"] else 0), dtype=torch.bfloat16, device=dev)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _rotated(x, angles, halves):
    """x [..., 64] turned by angles [..., 32, (cos, sin)]; pairs are neighbours, or columns i and i + 32."""
    x = x.float().unflatten(-1, (2, -1) if halves else (-1, 2))
    a, b = (x[..., 0, :], x[..., 1, :]) if halves else (x[..., 0], x[..., 1])
    c, s = angles[..., 0], angles[..., 1]
    return torch.stack((a * c - b * s, a * s + b * c), -2 if halves else -1).flatten(-2).to(torch.bfloat16)


def _keys(rows, mx4, marks):
    """float32 [..., 576] of cache rows in bytes."""
    if not mx4:
        return rows.view(torch.bfloat16).float()
    return torch.cat((_values(rows[..., :256], rows[..., 256:272], marks),
                      rows[..., 272:].contiguous().view(torch.bfloat16).float()), -1)


def _plain_append(s):
    turn = s["angles"][s["position"]]
    rows = _rows_of(s["latent"], _rotated(s["rope"], turn, s["halves"]), s["mx4"])
    page = s["table"][s["request"].long(), s["position"] // s["page"]].long()
    s["pool"][page, s["position"] % s["page"]] = rows
    out = {}
    if s["heads"]:
        s["q"][..., LATENT:] = _rotated(s["q_rope"], turn[:, None], s["halves"])
        out["q"] = s["q"]
    out["cache"] = _keys(s["pool"][page, s["position"] % s["page"]], True, s["marks"]).to(torch.bfloat16) if s["mx4"] \
        else s["pool"].view(torch.bfloat16)
    return out


def _plain_attend(s):
    b, t, k = s["requests"], s["tokens"], s["rows"]
    at = torch.arange(k, device=s["q"].device)
    if s["page"]:
        flat = (s["table"][:, at // s["page"]].long() * s["page"] + at % s["page"])[:, None]
        where = at
    else:
        flat = s["picked"].long() + (torch.arange(b, device=at.device) * s["slots"])[:, None, None]
        where = s["index"]
    keys = _keys(s["pool"].view(-1, s["pool"].shape[-1])[flat], s["mx4"], s["marks"])
    scores = torch.matmul(s["q"].float(), keys.transpose(-1, -2)) * SCALE
    seen = (where < s["lens"][..., None])[..., None, :]
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, keys[..., :LATENT]) / torch.where(total > 0, total, 1.0)
    return {"out": out.to(torch.bfloat16), "lse": (top + torch.log(total)).squeeze(-1)}


def _plain_project(s):
    x = _values(*_quantized(s["x"]), s["marks"]).transpose(0, 1)
    s["out"][..., :s["n"]] = torch.matmul(x, _values(*s["w"], s["marks"]).transpose(-1, -2)).transpose(0, 1)
    return s["out"]


def run(state):
    s = state
    if not own:
        if s["op"] == "append":
            return _plain_append(s)
        if s["op"] == "attend":
            return _plain_attend(s)
        if s["op"] == "quantize":
            return _values(*_quantized(s["x"]), s["marks"]).to(torch.bfloat16)
        return _plain_project(s)
    from paper_2609_37538_amd import latent as L
    if "pool" in s and "cache" not in s:   # a program makes this once
        s["cache"] = L.LatentCache(s["pool"], s["requests"], L.AVSG_ROWS_MX4 if s["mx4"] else L.AVSG_ROWS_BF16,
                                   page_table=s.get("table"))
    cache = s.get("cache")
    if s["op"] == "append":
        cache.append(s["latent"], s["rope"], s["request"], s["position"], s["angles"],
                     style=L.AVSG_ROPE_HALVES if s["halves"] else L.AVSG_ROPE_PAIRS,
                     q_rope=s["q_rope"], q_out=None if s["q"] is None else s["q"][..., LATENT:])
        out = {} if s["q"] is None else {"q": s["q"]}
        out["cache"] = cache.read(s["request"], s["position"]) if s["mx4"] else s["pool"].view(torch.bfloat16)
        return out
    if s["op"] == "attend":
        if s["page"]:
            o, lse = cache.attend(s["q"], lens=s["lens"], longest=s["rows"], scale=SCALE)
        else:
            o, lse = cache.attend(s["q"], rows=s["picked"], index=s["index"], lens=s["lens"], scale=SCALE)
        return {"out": o, "lse": lse}
    if s["op"] == "quantize":
        return L.mx4_dequantize(L.mx4_quantize(s["x"]))
    L.mx4_matmul(L.mx4_quantize(s["x"]).transpose(0, 1), L.Mx4(*s["w"]), out=s["out"][..., :s["n"]].transpose(0, 1))
    return s["out"]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["op"] == "append":
        t, h = sum(_lengths(case)), case["heads"]
        moved = t * (2 * (LATENT + ROPE) + _row_bytes(case["mx4"]) + 4 * ROPE + 12 + h * 4 * ROPE)
        if case["mx4"]:
            moved += t * 2 * (LATENT + ROPE)
        return {"bytes": moved, "flops": t * ((h + 1) * 3 * ROPE + (4 * LATENT if case["mx4"] else 0))}
    if case["op"] == "attend":
        b, t, h, k = case["requests"], case["tokens"], case["heads"], case["rows"]
        seen = _attend_lengths(case)
        if case["page"]:
            used = [min(n, k) for n in seen]
            read = sum(max(used[r * t:(r + 1) * t]) for r in range(b)) * _row_bytes(case["mx4"])
            listed_ = 4 * -(-k // case["page"]) * b
        else:
            used = [k * min(n, 4 * k) // (4 * k) for n in seen]
            read = sum(max(used[r * t:(r + 1) * t]) * (1 + (t - 1) * (1 - SHARED)) for r in range(b)) * _row_bytes(case["mx4"])
            listed_ = 8 * b * t * k
        return {"bytes": read + listed_ + b * t * h * (2 * (2 * LATENT + ROPE) + 4),
                "flops": sum(used) * h * 2 * (2 * LATENT + ROPE)}
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * 4, "flops": 4 * n}
    b, m, n, k = (case[f] for f in ("batch", "m", "n", "k"))
    return {"bytes": b * (2 * m * k + n * k * 17 / 32 + 2 * m * n), "flops": 2 * b * m * n * k}


# ---------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_quantized(x):
    """Values that the 4-bit form of x stands for: the nearest multiple of the block's power of two among
    the eight magnitudes, of two equally near ones that with the even place in their list."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    marks = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    top = x.abs().amax(-1, keepdim=True)
    part, power = torch.frexp(top)
    power = power.double() - 3 + (part >= 0.875)
    unit = torch.exp2(torch.where(top > 0, power, 0.0).clamp(min=-125).round())
    a = x.abs() / unit
    place = torch.searchsorted(marks, a).clamp(1, 7)
    below, above = a - marks[place - 1], marks[place] - a
    pick = torch.where((below < above) | ((below == above) & (place % 2 == 1)), place - 1, place)
    return (torch.sign(x) * marks[pick] * unit).flatten(-2)


def _exact_codes(codes, scales):
    both = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
    size, sign = both % 8, 1 - 2 * (both // 8)
    value = torch.where(size < 2, size * 0.5, (1 + (size % 2) * 0.5) * torch.exp2((size // 2 - 1).double()))
    unit = torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1)
    return sign * value * unit


def _exact_rows(rows, mx4):
    if not mx4:
        return rows.contiguous().view(torch.bfloat16).double()
    return torch.cat((_exact_codes(rows[..., :256], rows[..., 256:272]),
                      rows[..., 272:].contiguous().view(torch.bfloat16).double()), -1)


def _exact_turned(x, angles, halves):
    pair = torch.view_as_complex(angles.double().contiguous())
    x = x.double()
    z = torch.complex(x[..., :32], x[..., 32:]) if halves else torch.view_as_complex(x.unflatten(-1, (32, 2)).contiguous())
    z = z * pair
    return torch.cat((z.real, z.imag), -1) if halves else torch.view_as_real(z).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        turn = s["angles"][s["position"]]
        row = torch.cat((_exact_quantized(s["latent"]) if case["mx4"] else s["latent"].double(),
                         _exact_turned(s["rope"], turn, case["halves"])), -1)
        out = {}
        if case["heads"]:
            out["q"] = s["q"].double()
            out["q"][..., LATENT:] = _exact_turned(s["q_rope"], turn[:, None], case["halves"])
        if case["mx4"]:
            out["cache"] = row
        else:
            out["cache"] = torch.zeros(*s["pool"].shape[:2], LATENT + ROPE, dtype=torch.float64, device=row.device)
            for r in range(case["requests"]):
                mine = s["request"] == r
                for p in (s["position"][mine] // case["page"]).unique().tolist():
                    here = mine & (s["position"] // case["page"] == p)
                    out["cache"][int(s["table"][r, p])][s["position"][here] % case["page"]] = row[here]
        return out
    if case["op"] == "attend":
        outs, lses = [], []
        for r in range(case["requests"]):
            if case["page"]:
                keys_all = _exact_rows(s["pool"][s["table"][r].long()].flatten(0, 1)[:case["rows"]], case["mx4"])
            for g in range(case["tokens"]):
                n = int(s["lens"][r, g])
                if case["page"]:
                    keys = keys_all[:n]
                else:
                    keys = _exact_rows(s["pool"][r][s["picked"][r, g][s["index"][r, g] < n].long()], case["mx4"])
                x = s["q"][r, g].double() @ keys.T * SCALE
                if keys.shape[0] == 0:
                    outs.append(torch.zeros(case["heads"], LATENT, dtype=torch.float64, device=x.device))
                    lses.append(torch.full((case["heads"],), -math.inf, dtype=torch.float64, device=x.device))
                else:
                    outs.append(torch.softmax(x, -1) @ keys[:, :LATENT])
                    lses.append(torch.logsumexp(x, -1))
        lead = (case["requests"], case["tokens"])
        return {"out": torch.stack(outs).unflatten(0, lead), "lse": torch.stack(lses).unflatten(0, lead)}
    if case["op"] == "quantize":
        return _exact_quantized(s["x"])
    x, w = _exact_quantized(s["x"]), _exact_codes(*s["w"])
    out = s["out"].double()
    for i in range(case["batch"]):
        out[:, i, :case["n"]] = x[:, i] @ w[i].T
    return out
