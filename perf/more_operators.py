"""Performance cases of what makes a step's selection, and of 8-bit products: the cache
of 8-bit index keys, the scores over it with the positions that they select, attention
over the selected rows, and the product of matrices in 8-bit floating point.

A row of the key cache is one position's index key: 128 codes of 8 bits and a float32
scale, 132 bytes.  A query token has several index queries of 128 codes, each with a
weight (which holds the query's scale); the score of a position is

    scale * sum over queries of weight * max(0, query . key)

rounded to float32.  The positions (or blocks of neighbouring ones, by their best score)
with the largest scores are selected, ties go to the lowest.  Matrices in 8-bit floating
point (e4m3) have a float32 scale for each 128 columns of a row (activations) or for each
block of 128 x 128 (weights).  A pass of a case is one call as a decode step or a prefill
makes it.
"""
import math

import torch

own = False         # the framework's kernels in place of the plain forms

DIM = 128           # of index keys and queries
ROPE = 64           # of them turned by the position
LATENT = 512        # of the rows that the attention reads, which end in ROPE rotated values
BLOCK = 128         # columns (and rows) per scale of an 8-bit matrix
SCALE = 192 ** -0.5  # of the attention's scores

# Fields of a case, by operator:
# keys: requests, tokens of the longest one (ragged: the others have fewer), index queries per token (heads),
#   rows of a page, positions per request, whether the rotated columns are the last ones and pairs are halves
# select: requests, query tokens, index queries per token, positions per request (context; a multiple of the
#   page), selected positions per token (topk), positions per block, masked: tokens see less than the context
#   (a prefill's tokens see all up to themselves), first and recent positions that are always selected
# sparse: the same, then attention of `wide` heads over the selected rows of a paged cache in bfloat16
# product: products, rows, columns and inner size; heads: whether the products are heads that interleave in
#   the activations' and the outputs' rows


def _keys(name=None, **kw):
    return _named(dict(dict(op="keys", requests=1, tokens=1, ragged=False, heads=64, page=64, context=512, halves=False), **kw), name)


def _select(name=None, **kw):
    return _named(dict(dict(op="select", requests=1, tokens=1, heads=64, context=1024, topk=256, block=1, page=64, masked=False,
                            first=0, recent=0), **kw), name)


def _sparse(name=None, **kw):
    return _named(dict(_select(**kw), op="sparse", wide=kw.get("wide", 16)), name)


def _product(name=None, **kw):
    return _named(dict(dict(op="product", batch=1, m=1, n=512, k=512, heads=False), **kw), name)


def _named(case, name):
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # the new keys of a decode step, 64 requests with one draft token each, and all index queries
        _keys("keys_step64", requests=64, tokens=2),
        # a prefill of four prompts of different lengths
        _keys("keys_prefill", requests=4, tokens=2047, ragged=True, context=2048, halves=True),
        # one request of a small model: the smallest call, all latency
        _select("select_tiny", heads=16, context=1024, topk=256),
        # sizes off every power of two, two draft tokens, a token that sees nothing, positions that are always taken
        _select("select_odd7", requests=7, tokens=3, heads=40, context=5008, topk=600, page=16, masked=True, first=3, recent=70),
        # the serving batch: one draft token, contexts of 32768
        _select("select_step64", requests=64, tokens=2, context=32768, topk=2048),
        # four long contexts, one token each: few rows, long ones
        _select("select_long", requests=4, context=131072, topk=2048),
        # a prefill's chunk of tokens, each of which sees what stands before it
        _select("select_prefill", tokens=2048, context=16384, topk=2048, masked=True),
        # blocks of 64 positions selected and attended over, eight requests with one draft token
        _sparse("sparse_blocks8", requests=8, tokens=2, heads=32, context=16384, topk=2048, block=64, recent=64, masked=True),
        # a short chunk of a prompt, each token with its own rows
        _sparse("sparse_chunk", tokens=192, heads=64, context=8192, topk=1024, masked=True, wide=64),
        # one token through a weight matrix: the weights' bytes count
        _product("product_one", n=4096, k=4096),
        # sizes off every tile and block
        _product("product_odd", m=333, n=1000, k=1184),
        # a prefill's tokens through a weight matrix
        _product("product_prefill", m=8192, n=4096, k=4096),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("keys", "select", "select", "sparse", "product", "product"))
    if op == "keys":
        requests = _log_between(rng, 1, 128)
        tokens = rng.choice((1, 2, 3, 4)) if rng.random() < 0.5 else _log_between(rng, 1, max(1, 5000 // requests))
        return _keys(requests=requests, tokens=tokens, ragged=rng.random() < 0.5, heads=rng.choice((0, 1, 8, 16, 40, 64, 64)),
                     page=rng.choice((16, 64, 256)), context=tokens + rng.randint(1, 256), halves=rng.random() < 0.5)
    if op == "product":
        if rng.random() < 0.3:
            n, k = rng.choice(((512, 128), (128, 512), (256, 192)))
            return _product(batch=rng.choice((16, 20, 64, 128)), m=_log_between(rng, 1, 256), n=n, k=k, heads=True)
        return _product(m=_log_between(rng, 1, 4096), n=rng.choice((512, 1000, 1536, 2048, 4096)),
                        k=16 * rng.choice((8, 37, 74, 128, 256, 256)))
    page, heads, block = rng.choice((16, 64, 256)), rng.choice((1, 8, 16, 32, 40, 64, 64)), rng.choice((1, 1, 2, 16, 64, 128))
    step = max(page, block)
    if rng.random() < 0.3:
        requests, tokens = 1, _log_between(rng, 16, 1024)
    else:
        requests, tokens = _log_between(rng, 1, 64), rng.choice((1, 1, 2, 3, 4))
    most = 131072 if op == "select" else 16384
    context = -(-_log_between(rng, max(512, 16 * block), min(most, max(4096, (1 << 22) // (requests * max(2, tokens))))) // step) * step
    topk = _log_between(rng, max(80, 4 * block), max(256, min(2048, context // 2))) // block * block
    case = dict(requests=requests, tokens=tokens, heads=heads, context=context, topk=min(topk, context), block=block, page=page,
                masked=rng.random() < 0.7, first=rng.choice((0, 0, 1, 4)), recent=rng.choice((0, 0, 1, 64)))
    if op == "select":
        return _select(**case)
    if requests * tokens > 256:
        case["tokens"] = max(1, 256 // requests)
    return _sparse(**case, wide=rng.choice((1, 16, 16, 40, 64)))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _eighths(y):
    """(codes, scale) of y [..., 128] in float32: 127 steps to the largest magnitude, none for vectors of zeros."""
    top = y.abs().amax(-1, keepdim=True)
    codes = torch.round(y * torch.where(top > 0, 127 / top, 0.0)).to(torch.int8)
    return codes, (top / 127).squeeze(-1)


def _key_rows(y):
    codes, scale = _eighths(y)
    return torch.cat((codes.view(torch.uint8), scale.unsqueeze(-1).contiguous().view(torch.uint8)), -1)


def _fp8(x):
    """(codes, scales) of x [..., K], a scale for each 128 columns of a row."""
    k = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, -k % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    codes = (x * torch.where(top > 0, 448 / top, 0.0)).to(torch.float8_e4m3fn)
    return codes.flatten(-2)[..., :k].contiguous(), (top / 448).squeeze(-1)


def _fp8_blocks(w):
    """(codes, scales) of w [batch][N][K], a scale for each block of 128 x 128."""
    n, k = w.shape[-2:]
    w = torch.nn.functional.pad(w.float(), (0, -k % BLOCK, 0, -n % BLOCK)).unflatten(-1, (-1, BLOCK)).unflatten(1, (-1, BLOCK))
    top = w.abs().amax((2, 4), keepdim=True)
    codes = (w * torch.where(top > 0, 448 / top, 0.0)).to(torch.float8_e4m3fn)
    return codes.flatten(-2).flatten(1, 2)[:, :n, :k].contiguous(), (top / 448).squeeze(4).squeeze(2).contiguous()


def _lengths(case):
    n, r = case["tokens"], case["requests"]
    return [max(1, n - i * (n // r)) if case["ragged"] else n for i in range(r)]


def _seen(case):
    """Positions that each token of each request sees: a chunk's tokens stand at the end of the context."""
    n, t = case["context"], case["tokens"]
    out = []
    for r in range(case["requests"]):
        for g in range(t):
            if not case["masked"]:
                out.append(n)
            elif t > 4:
                out.append(max(0, n - t + 1 + g))
            else:
                out.append(0 if (r + g) % 11 == 5 else n * (3 + (5 * r + 3 * g) % 5) // 7)
    return out


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(dev).manual_seed(seed)

    def normal(*shape, by=1.0):
        return torch.randn(shape, generator=gen, device=dev) * by

    s = dict(case)
    if case["op"] == "keys":
        lengths, pages, heads = _lengths(case), -(-case["context"] // case["page"]), case["heads"]
        starts = [int(torch.randint(0, case["context"] - n + 1, (1,), generator=gen, device=dev)) for n in lengths]
        total = sum(lengths)
        s["request"] = torch.repeat_interleave(torch.arange(case["requests"], device=dev, dtype=torch.int32),
                                               torch.tensor(lengths, device=dev))
        s["position"] = torch.cat([torch.arange(a, a + n, device=dev) for a, n in zip(starts, lengths)])
        s["key"] = normal(total, DIM).to(torch.bfloat16)
        s["q"] = normal(total, heads, DIM).to(torch.bfloat16) if heads else None
        s["weights"] = normal(total, heads, by=heads ** -0.5) if heads else None
        s["q_codes"] = torch.zeros(total, heads, DIM, dtype=torch.int8, device=dev) if heads else None
        s["q_weights"] = torch.zeros(total, heads, device=dev) if heads else None
        turn = torch.arange(case["context"], device=dev, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, ROPE, 2, device=dev, dtype=torch.float64) / ROPE)
        s["angles"] = torch.stack((turn.cos(), turn.sin()), -1).float()
        s["table"] = torch.randperm(case["requests"] * pages, generator=gen, device=dev).to(torch.int32).view(-1, pages)
        s["pool"] = torch.zeros(case["requests"] * pages, case["page"], DIM + 4, dtype=torch.uint8, device=dev)
        return s
    if case["op"] in ("select", "sparse"):
        b, t, h, n, page = (case[f] for f in ("requests", "tokens", "heads", "context", "page"))
        pages = n // page
        pool = torch.empty(b * pages, page, DIM + 4, dtype=torch.uint8, device=dev)
        for i in range(0, b * n, 1 << 20):
            rows = pool.view(-1, DIM + 4)[i:i + (1 << 20)]
            rows.copy_(_key_rows(normal(rows.shape[0], DIM)))
        s["pool"] = pool
        s["table"] = torch.randperm(b * pages, generator=gen, device=dev).to(torch.int32).view(b, pages)
        s["q"], scale = _eighths(normal(b, t, h, DIM))
        s["weights"] = normal(b, t, h, by=h ** -0.5) * scale
        s["lens"] = torch.tensor(_seen(case), device=dev).view(b, t)
        if case["op"] == "sparse":
            s["rows"] = normal(b * pages, page, LATENT + ROPE).to(torch.bfloat16).view(torch.uint8)
            s["wide_q"] = normal(b, t, case["wide"], LATENT + ROPE).to(torch.bfloat16)
        return s
    b, m, n, k = (case[f] for f in ("batch", "m", "n", "k"))
    # activations: a few columns are much larger than the others
    s["x"] = (normal(m, b, k) * torch.where(torch.rand(k, generator=gen, device=dev) < 0.02, 20.0, 1.0)).to(torch.bfloat16)
    s["w"] = _fp8_blocks(normal(b, n, k, by=k ** -0.5))
    # the queries' buffer, whose last columns are the rotated part
    s["out"] = torch.zeros(m, b, n + (ROPE if case["heads"] else 0), dtype=torch.bfloat16, device=dev)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _turned(x, angles, halves):
    """x [..., 128] in float32 with 64 columns turned by angles [..., 32, (cos, sin)]: the first ones in
    neighbouring pairs, or the last ones in pairs of columns i and i + 32."""
    x = x.float()
    part, rest = (x[..., ROPE:], x[..., :ROPE]) if halves else (x[..., :ROPE], x[..., ROPE:])
    part = part.unflatten(-1, (2, -1) if halves else (-1, 2))
    a, b = (part[..., 0, :], part[..., 1, :]) if halves else (part[..., 0], part[..., 1])
    c, s = angles[..., 0], angles[..., 1]
    part = torch.stack((a * c - b * s, a * s + b * c), -2 if halves else -1).flatten(-2)
    return torch.cat((rest, part) if halves else (part, rest), -1)


def _plain_keys(s):
    turn = s["angles"][s["position"]]
    page = s["table"][s["request"].long(), s["position"] // s["page"]].long()
    s["pool"][page, s["position"] % s["page"]] = _key_rows(_turned(s["key"], turn, s["halves"]))
    rows = s["pool"][page, s["position"] % s["page"]]
    scale = rows[..., DIM:].contiguous().view(torch.float32)
    out = {"keys": (rows[..., :DIM].view(torch.int8).float() * scale).to(torch.bfloat16)}
    if s["heads"]:
        codes, scale = _eighths(_turned(s["q"], turn[:, None], s["halves"]))
        s["q_codes"].copy_(codes)
        s["q_weights"].copy_(s["weights"] * scale)
        out["q"], out["weights"] = s["q_codes"].to(torch.bfloat16), s["q_weights"]
    return out


def _plain_scores(s):
    """float32 scores [B][n_q][context]; the products of codes are whole numbers that float32 holds."""
    rows = s["pool"][s["table"].long()].flatten(1, 2)
    keys, scale = rows[..., :DIM].view(torch.int8).float(), rows[..., DIM:].contiguous().view(torch.float32).squeeze(-1)
    each = torch.matmul(s["q"].flatten(1, 2).float(), keys.transpose(1, 2).contiguous()).clamp_(min=0)
    each = each.unflatten(1, (s["tokens"], s["heads"])).double()
    total = torch.matmul(s["weights"].double().unsqueeze(2), each).squeeze(2)
    return (total * scale.double().unsqueeze(1)).float()


def _plain_select(s):
    scores = _plain_scores(s)
    at, seen = torch.arange(s["context"], device=scores.device), s["lens"].unsqueeze(-1)
    scores = torch.where((at < s["first"]) | (at >= seen - s["recent"]), math.inf, scores)
    scores = torch.where(at < seen, scores, -math.inf).unflatten(-1, (-1, s["block"])).amax(-1)
    count = s["topk"] // s["block"]
    best = torch.sort(scores, dim=-1, descending=True, stable=True).indices[..., :count].sort(-1).values
    index = (best.unsqueeze(-1) * s["block"] + torch.arange(s["block"], device=best.device)).flatten(-2)
    return {"index": index.to(torch.int32), "scores": scores.gather(-1, best)}


def _plain_sparse(s):
    picked = _plain_select(s)
    index = picked["index"].long()
    flat = torch.gather(s["table"].long().unsqueeze(1).expand(-1, s["tokens"], -1), 2, index // s["page"]) * s["page"] + index % s["page"]
    keys = s["rows"].view(torch.bfloat16).flatten(0, 1)[flat].float()
    scores = torch.matmul(s["wide_q"].float(), keys.transpose(-1, -2)) * SCALE
    scores = scores.masked_fill((index >= s["lens"].unsqueeze(-1)).unsqueeze(2), -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, keys[..., :LATENT]) / torch.where(total > 0, total, 1.0)
    return dict(picked, out=out.to(torch.bfloat16), lse=(top + torch.log(total)).squeeze(-1))


def _plain_product(s):
    (codes, scales), (w, w_scales), k, n = _fp8(s["x"]), s["w"], s["k"], s["n"]
    x = codes.float() * scales.repeat_interleave(BLOCK, -1)[..., :k]
    w = w.float() * w_scales.repeat_interleave(BLOCK, 1)[:, :n].repeat_interleave(BLOCK, 2)[..., :k]
    s["out"][..., :n] = torch.matmul(x.transpose(0, 1), w.transpose(1, 2)).transpose(0, 1)
    return s["out"]


def run(state):
    s = state
    if not own:
        return {"keys": _plain_keys, "select": _plain_select, "sparse": _plain_sparse, "product": _plain_product}[s["op"]](s)
    from paper_2609_37538_amd import fp8 as F
    from paper_2609_37538_amd import latent as L
    from paper_2609_37538_amd import selection as S
    if s["op"] == "product":
        if "weight" not in s:   # a program makes this once
            s["weight"] = F.Fp8(s["w"][0], s["w"][1], rows=BLOCK)
        F.fp8_matmul(F.fp8_quantize(s["x"]).transpose(0, 1), s["weight"], out=s["out"][..., :s["n"]].transpose(0, 1))
        return s["out"]
    if "cache" not in s:        # likewise
        s["cache"] = S.KeyCache(s["pool"], s["requests"], page_table=s["table"])
        if s["op"] == "sparse":
            s["latents"] = L.LatentCache(s["rows"], s["requests"], L.AVSG_ROWS_BF16, page_table=s["table"])
    if s["op"] == "keys":
        style, at = (L.AVSG_ROPE_HALVES, ROPE) if s["halves"] else (L.AVSG_ROPE_PAIRS, 0)
        s["cache"].append(s["key"], s["request"], s["position"], s["angles"], style=style, rope_at=at, q=s["q"],
                          weights=s["weights"], q_out=s["q_codes"], weights_out=s["q_weights"])
        out = {"keys": s["cache"].read(s["request"], s["position"])}
        if s["heads"]:
            out["q"], out["weights"] = s["q_codes"].to(torch.bfloat16), s["q_weights"]
        return out
    index, scores = s["cache"].select(s["q"], s["weights"], topk=s["topk"], block=s["block"], lens=s["lens"],
                                      longest=s["context"], first=s["first"], recent=s["recent"])
    if s["op"] == "select":
        return {"index": index, "scores": scores}
    out, lse = s["latents"].attend(s["wide_q"], rows=index, index=index, lens=s["lens"], scale=SCALE)
    return {"index": index, "scores": scores, "out": out, "lse": lse}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["op"] == "keys":
        t, h = sum(_lengths(case)), case["heads"]
        return {"bytes": t * (2 * DIM + 8 * ROPE // 2 + 12 + 2 * (DIM + 4) + 2 * DIM + h * (3 * DIM + 8)),
                "flops": t * (h + 1) * (3 * ROPE + 3 * DIM)}
    if case["op"] in ("select", "sparse"):
        b, t, h, k = (case[f] for f in ("requests", "tokens", "heads", "topk"))
        seen = _seen(case)
        keys = sum(max(seen[r * t:(r + 1) * t]) for r in range(b))
        w = {"bytes": keys * (DIM + 4) + b * t * (h * (DIM + 4) + 8 + 4 * k + 4 * k // case["block"]), "flops": sum(seen) * h * 2 * DIM}
        if case["op"] == "sparse":
            rows = [min(k, n) for n in seen]
            most = sum(min(sum(rows[r * t:(r + 1) * t]), max(seen[r * t:(r + 1) * t])) for r in range(b))
            w["bytes"] += most * 2 * (LATENT + ROPE) + b * t * case["wide"] * (2 * (2 * LATENT + ROPE) + 4)
            w["flops"] += sum(rows) * case["wide"] * 2 * (2 * LATENT + ROPE)
        return w
    b, m, n, k = (case[f] for f in ("batch", "m", "n", "k"))
    return {"bytes": b * (2 * m * k + n * k + 2 * m * n), "flops": 2 * b * m * n * k}


# ---------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_turned(x, angles, halves):
    x, pair = x.double().clone(), torch.view_as_complex(angles.double().contiguous())
    if halves:
        z = torch.complex(x[..., 64:96], x[..., 96:]) * pair
        x[..., 64:96], x[..., 96:] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :64].unflatten(-1, (32, 2)).contiguous()) * pair
        x[..., :64] = torch.view_as_real(z).flatten(-2)
    return x


def _exact_codes(y):
    step = y.abs().amax(-1, keepdim=True) / 127
    return torch.round(y / torch.where(step > 0, step, 1.0)), step


def _exact_best(s, r):
    """(positions, block scores) that request r's tokens select, scores rounded to float32 before they are ranked."""
    t, n, size = s["tokens"], s["context"], s["block"]
    rows = s["pool"][s["table"][r].long()].flatten(0, 1)
    keys, scale = rows[:, :DIM].view(torch.int8).double(), rows[:, DIM:].contiguous().view(torch.float32).double()[:, 0]
    values = torch.empty(t, n, dtype=torch.float64, device=keys.device)
    for g in range(t):
        values[g] = (s["weights"][r, g].double()[:, None] * torch.relu(s["q"][r, g].double() @ keys.T)).sum(0) * scale
    for g in range(t):
        seen = int(s["lens"][r, g])
        values[g, max(0, seen - s["recent"]):] = math.inf
        values[g, :s["first"]] = math.inf
        values[g, seen:] = -math.inf
    values = values.view(t, n // size, size).max(-1).values
    place = torch.arange(n // size, device=keys.device).expand(t, -1)
    order = values.float().argsort(dim=-1, descending=True, stable=True)
    chosen = torch.zeros_like(place, dtype=torch.bool).scatter_(1, order[:, :s["topk"] // size], True)
    blocks = place[chosen].view(t, -1)
    index = (blocks[..., None] * size + torch.arange(size, device=keys.device)).flatten(1)
    return index, values.gather(1, blocks)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "keys":
        turn = s["angles"][s["position"]]
        codes, step = _exact_codes(_exact_turned(s["key"], turn, case["halves"]))
        out = {"keys": codes * step}
        if case["heads"]:
            out["q"], step = _exact_codes(_exact_turned(s["q"], turn[:, None], case["halves"]))
            out["weights"] = s["weights"].double() * step.squeeze(-1)
        return out
    if case["op"] in ("select", "sparse"):
        found = [_exact_best(s, r) for r in range(case["requests"])]
        out = {"index": torch.stack([i for i, _ in found]).to(torch.int32), "scores": torch.stack([v for _, v in found])}
        if case["op"] == "select":
            return out
        outs, lses = [], []
        for r, (index, _) in enumerate(found):
            rows = s["rows"][s["table"][r].long()].flatten(0, 1)
            for g in range(case["tokens"]):
                mine = rows[index[g][index[g] < s["lens"][r, g]]].contiguous().view(torch.bfloat16).double()
                x = s["wide_q"][r, g].double() @ mine.T * SCALE
                if mine.shape[0] == 0:
                    outs.append(torch.zeros(case["wide"], LATENT, dtype=torch.float64, device=x.device))
                    lses.append(torch.full((case["wide"],), -math.inf, dtype=torch.float64, device=x.device))
                else:
                    outs.append(torch.softmax(x, -1) @ mine[:, :LATENT])
                    lses.append(torch.logsumexp(x, -1))
        lead = (case["requests"], case["tokens"])
        return dict(out, out=torch.stack(outs).unflatten(0, lead), lse=torch.stack(lses).unflatten(0, lead))
    m, n, k = case["m"], case["n"], case["k"]
    out = s["out"].double()
    for i in range(case["batch"]):
        x, total = s["x"][:, i].double(), torch.zeros(m, n, dtype=torch.float64, device=s["x"].device)
        for at in range(0, k, BLOCK):
            part = x[:, at:at + BLOCK]
            step = part.abs().amax(1, keepdim=True) / 448
            codes = (part / torch.where(step > 0, step, 1.0)).float().to(torch.float8_e4m3fn).double()
            scale = s["w"][1][i, :, at // BLOCK].double().repeat_interleave(BLOCK)[:n]
            total += (codes * step) @ (s["w"][0][i, :, at:at + BLOCK].double().T * scale)
        out[:, i, :n] = total
    return out
