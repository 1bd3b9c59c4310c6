"""Every way to carry out a call of attention: each kernel in each row format, with every kind of join, on cases
that the choice gives it now."""
import ctypes

import pytest
import torch

from paper_2609_37538_amd import latent as L

KERNELS = ("16 heads", "16 heads alone", "64 heads")
JOINS = ("one part", "few parts", "more parts", "many parts of few results", "many parts")


def path(fmt, tokens, heads, k):
    """(kernel, join, parts) of a call."""
    f = L.load().avsg_internal_attend_plan
    f.restype, f.argtypes = ctypes.c_int64, [ctypes.c_int32] * 5
    plan = f(fmt, tokens, 1, heads, k)
    parts = plan >> 32
    join = 0 if parts == 1 else 1 if parts <= 4 else 2 if parts <= 16 else 3 if tokens * heads <= 128 else 4
    return KERNELS[plan & 0xffffffff], JOINS[join], parts


# by tokens * rows: small ones first
CASES = sorted(((t, h, k) for t in (1, 2, 3, 4, 6, 8, 11, 16, 24, 33, 48, 66, 96, 130, 200, 256) for h in (5, 16, 17, 33, 40, 64, 70, 128)
                for k in (61, 100, 150, 257, 500, 777, 1060, 1720, 2000, 2047, 4100, 8200, 16500, 33000, 66000)),
               key=lambda c: (c[0] * c[2], c[0] * c[1] * c[2]))
# ways that no case takes: in bfloat16, 128-row tiles are chosen for a few calls of one part alone
NEVER = {(0, "16 heads alone", join) for join in JOINS[1:]}


def case_of(fmt, kernel, join):
    """The smallest case whose parts go over several tiles, or the smallest."""
    cases = [c for c in CASES if path(fmt, *c)[:2] == (kernel, join)]
    return next((c for c in cases if c[2] / path(fmt, *c)[2] > 200), cases[0] if cases else None)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("join", JOINS)
def test_a_case_for_every_path(join, kernel, fmt):
    """The choice gives each way some case of the list, so that the test below runs it."""
    assert (case_of(fmt, kernel, join) is None) == ((fmt, kernel, join) in NEVER)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("join", JOINS)
def test_every_path(join, kernel, fmt):
    """Scores that rise along the entries, of which some do not count and hold NaN, in tokens that see all, some
    and none of them; in a workspace of exactly the size asked for, full of NaN."""
    from test_latent import check_attend, gen, normal, row_bytes
    if (fmt, kernel, join) in NEVER:
        assert case_of(fmt, kernel, join) is None
        return
    tokens, heads, k = case_of(fmt, kernel, join)
    print(f"{kernel}, {join}: {tokens} tokens, {heads} heads, {k} rows, {path(fmt, tokens, heads, k)[2]} parts", flush=True)
    g, slots = gen(tokens + heads + k), k + 50
    latent, rope = normal(g, slots, 512, by=0.1), normal(g, slots, 64, by=0.1)
    latent[:, :32] = torch.linspace(-6, 6, slots, device="cuda")[:, None].to(torch.bfloat16)
    pool = row_bytes(latent, rope, fmt == 1).unsqueeze(0).expand(tokens, -1, -1).contiguous()
    pool[:, 3::11] = 0xff
    cache = L.LatentCache(pool, tokens, fmt)
    first = torch.arange(tokens, device="cuda") % 50
    rows = (first[:, None] + torch.arange(k, device="cuda")).to(torch.int32).view(tokens, 1, k).contiguous()
    index = torch.where(rows % 11 == 3, -1, rows).contiguous()
    lens = torch.randint(1, slots + 1, (tokens, 1), generator=g, device="cuda")
    lens[0] = slots
    if tokens > 1:
        lens[tokens // 2], lens[-1] = 0, 1 + k // 2
    q = normal(g, tokens, 1, heads, 576)
    q[..., :32] = 1.0 + torch.arange(heads, device="cuda")[:, None] / heads
    out, lse = cache.attend(q, rows=rows, index=index, lens=lens, scale=1.5)
    assert torch.isfinite(out).all()
    some = torch.tensor(sorted({0, tokens // 2, tokens - 1}), device="cuda")
    few, pick = L.LatentCache(pool[some].contiguous(), len(some), fmt), lambda x: x[some].contiguous()  # noqa: E731
    check_attend(few, pick(q), pick(out), pick(lse), pick(rows), pick(index), pick(lens), scale=1.5)

    need, guard = L.avsg_attend_workspace_bytes(tokens, 1, heads, k), 4096
    room = torch.full((need + guard,), 0xff, dtype=torch.uint8, device="cuda")     # float32 of such bytes are NaN
    again, lse_again = torch.empty_like(out), torch.empty_like(lse)
    a = L.AvsgAttention(1, heads, k, 1.5, q.data_ptr(), heads * 576, 576, rows.data_ptr(), index.data_ptr(), lens.data_ptr(),
                        again.data_ptr(), heads * 512, 512, lse_again.data_ptr())
    L.avsg_attend(cache.c, a, room.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(again, out) and torch.equal(lse_again, lse)
    assert (room[need:] == 0xff).all(), "written outside the workspace"
