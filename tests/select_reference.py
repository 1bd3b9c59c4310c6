"""Plain forms on the CPU of the key cache and the selection: the quantisation in
float32 step by step as it is stated, everything else in 64 bits."""
import math

import torch

DIM, ROPE, ROW = 128, 64, 132


def turned(x, angles, halves, at):
    """float32 [..., 128] with 64 columns from `at` turned; every product and sum rounded."""
    x = x.cpu().float().clone()
    if angles is None:
        return x
    part = x[..., at:at + ROPE]
    a, b = (part[..., :32], part[..., 32:]) if halves else (part[..., 0::2], part[..., 1::2])
    c, s = angles.cpu()[..., 0], angles.cpu()[..., 1]
    u, v = a * c - b * s, a * s + b * c
    x[..., at:at + ROPE] = torch.cat((u, v), -1) if halves else torch.stack((u, v), -1).flatten(-2)
    return x


def eighths(y):
    """(codes int8, scale float32) of y [..., 128] in float32."""
    top = y.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(y).all(-1, keepdim=True)
    some = (top >= 2.0 ** -119) & ~bad
    steps = torch.where(some, torch.tensor(127.0) / torch.where(some, top, 1.0), 0.0)
    codes = torch.round(torch.where(bad, 0.0, y) * steps).to(torch.int8)
    scale = torch.where(some, top / torch.full_like(top, 127.0), 0.0)
    return codes, torch.where(bad, math.nan, scale).squeeze(-1)


def rows_of(y):
    """Bytes [..., 132] of the rows of y."""
    codes, scale = eighths(y)
    return torch.cat((codes.view(torch.uint8), scale.unsqueeze(-1).contiguous().view(torch.uint8)), -1)


def scores(q, weights, rows):
    """float32 [H-summed] scores [n] of one token: q [H][128] int8, weights [H], rows [n][132]."""
    keys, scale = rows[:, :DIM].contiguous().view(torch.int8).double(), rows[:, DIM:].contiguous().view(torch.float32)[:, 0].double()
    dots = (q.double() @ keys.T).clamp(min=0)
    return ((weights.double()[:, None] * dots).sum(0) * scale).float()


def best(s, seen, topk, block, first=0, recent=0):
    """(positions, block scores) that a token with scores s [longest] selects."""
    s = torch.where(torch.isnan(s), -math.inf, s)
    at = torch.arange(len(s))
    seen = max(0, min(seen, len(s)))
    s = torch.where((at < first) | (at >= seen - recent), math.inf, s)
    s = torch.where(at < seen, s, -math.inf).view(-1, block).amax(-1) + 0.0
    picked = torch.sort(s, descending=True, stable=True).indices[:topk // block].sort().values
    index = (picked[:, None] * block + torch.arange(block)).flatten()
    return index.to(torch.int32), s[picked]


def request_rows(pool, table, r, per):
    """Rows [per * page_rows][132] of request r on the CPU; those of pages that do not exist have scale NaN."""
    pool = pool.cpu()
    pages = table[r].tolist() if table is not None else list(range(r * per, (r + 1) * per))
    none = torch.cat((torch.zeros(pool.shape[1], DIM, dtype=torch.uint8),
                      torch.full((pool.shape[1], 1), math.nan).view(torch.uint8)), -1)
    return torch.cat([pool[i] if 0 <= i < pool.shape[0] else none for i in pages])


def select(q, weights, pool, table, lens, *, topk, block=1, longest=None, first=0, recent=0):
    """(index, scores) on the CPU of a whole call."""
    b, n_q = q.shape[:2]
    q, weights = q.cpu(), weights.cpu()
    per = table.shape[1] if table is not None else pool.shape[0] // b
    table = None if table is None else table.cpu()
    index, values = [], []
    for r in range(b):
        rows = request_rows(pool, table, r, per)
        rows = rows[:len(rows) if longest is None else longest]
        for g in range(n_q):
            seen = len(rows) if lens is None else int(lens[r, g])
            i, v = best(scores(q[r, g], weights[r, g], rows), seen, topk, block, first, recent)
            index.append(i)
            values.append(v)
    return torch.stack(index).view(b, n_q, -1), torch.stack(values).view(b, n_q, -1)
