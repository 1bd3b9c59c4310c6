"""Latent-cache operators on the GPU against plain forms in 64 bits: rows
appended, read back and attended over, in both row formats."""
import math

import pytest
import torch

import latent_reference as R

pytestmark = pytest.mark.gpu

SCALE = 192 ** -0.5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2609_37538_amd import latent as L
    L.load()            # fails loudly when the HIP library is missing


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def normal(g, *shape, by=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * by).to(torch.bfloat16)


def row_bytes(latent, rope, mx4):
    """Rows in bytes, made on the CPU by the plain form."""
    latent, rope = latent.cpu(), rope.cpu().contiguous()
    if not mx4:
        return torch.cat((latent, rope), -1).contiguous().view(torch.uint8).cuda()
    codes, scales = R.quantize(latent)
    return torch.cat((codes, scales, rope.view(torch.uint8)), -1).cuda()


def pool_of(g, pages, page_rows, mx4, pad=0):
    n = pages * page_rows
    raw = row_bytes(normal(g, n, 512), normal(g, n, 64), mx4)
    room = torch.full((pages, page_rows, raw.shape[-1] + pad), 0xff, dtype=torch.uint8, device="cuda")
    view = room[..., :raw.shape[-1]]
    view.copy_(raw.view(pages, page_rows, -1))
    return view


def close(got, want, bound, what):
    got = got.cpu().double()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).eq(torch.isfinite(want)).all(), f"{what}: infinities or NaN"
    fine = torch.isfinite(want)
    assert got[~fine].eq(want[~fine]).all(), f"{what}: infinities differ"
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: {over.max()} over its bound"


def check_attend(cache, q, out, lse, rows=None, index=None, lens=None, longest=None, scale=SCALE, what=""):
    """out and lse against the plain form over the rows that count."""
    mx4 = cache.row_format == 1
    pool, table = cache.pool, cache.page_table
    per = pool.shape[0] // cache.batch
    ids = torch.arange(cache.batch * per).view(cache.batch, per) if table is None else table.cpu().long()
    for b in range(q.shape[0]):
        at = ids[b].clamp(0, pool.shape[0] - 1)
        keys = R.row_values(pool[at.cuda()].flatten(0, 1), mx4)
        exists = ((ids[b] >= 0) & (ids[b] < pool.shape[0])).repeat_interleave(pool.shape[1])
        for g in range(q.shape[1]):
            k = rows.shape[-1] if rows is not None else (longest if longest is not None else keys.shape[0])
            row = rows[b, g].cpu().long() if rows is not None else torch.arange(k)
            pos = index[b, g].cpu().long() if index is not None else torch.arange(k)
            n = int(lens[b, g]) if lens is not None else 1 << 40
            counts = (row >= 0) & (row < keys.shape[0]) & (pos >= 0) & (pos < n)
            row = row.clamp(0, keys.shape[0] - 1)
            counts &= exists[row]
            o, s, eo, es = R.attend(q[b, g], keys[row], counts, scale)
            close(out[b, g], o, eo, f"{what} request {b} token {g}: out")
            close(lse[b, g], s, es, f"{what} request {b} token {g}: lse")


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("batch,n_q,heads,k,slots", [
    (1, 1, 1, 1, 2), (1, 1, 16, 1, 64), (2, 1, 16, 63, 64), (1, 3, 17, 64, 128), (3, 2, 33, 65, 256),
    (1, 1, 64, 127, 128), (2, 2, 65, 129, 512), (1, 1, 128, 300, 512), (9, 1, 20, 257, 512), (1, 1, 16, 2048, 4096),
    (1, 4, 128, 513, 4096), (5, 1, 8, 1000, 1024), (17, 2, 48, 96, 256), (1, 2, 130, 700, 1024)])
def test_attend_sparse(batch, n_q, heads, k, slots, mx4):
    from paper_2609_37538_amd import latent as L
    g = gen(batch * 1000 + heads * 10 + k)
    cache = L.LatentCache(pool_of(g, batch, slots, mx4), batch, int(mx4))
    q = normal(g, batch, n_q, heads, 576)
    rows = torch.rand(batch, n_q, slots, generator=g, device="cuda").argsort(-1)[..., :k].to(torch.int32).contiguous()
    index = torch.rand(batch, n_q, 4 * k, generator=g, device="cuda").argsort(-1)[..., :k].to(torch.int32).contiguous()
    lens = torch.randint(1, 4 * k + 1, (batch, n_q), generator=g, device="cuda")
    out, lse = cache.attend(q, rows=rows, scale=SCALE)
    check_attend(cache, q, out, lse, rows, what="no mask")
    out, lse = cache.attend(q, rows=rows, index=index, lens=lens, scale=SCALE)
    check_attend(cache, q, out, lse, rows, index, lens, what="by position")
    lens = torch.randint(0, k + 1, (batch, n_q), generator=g, device="cuda")
    out, lse = cache.attend(q, rows=rows, lens=lens, scale=SCALE)
    check_attend(cache, q, out, lse, rows, None, lens, what="first entries")


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("batch,n_q,heads,page,pages,longest", [
    (1, 1, 16, 16, 5, 80), (2, 1, 64, 64, 3, 150), (3, 2, 8, 16, 20, 320), (1, 1, 128, 256, 9, 2200),
    (2, 3, 40, 1, 70, 70), (1, 1, 16, 64, 80, 5000)])
def test_attend_whole_context(batch, n_q, heads, page, pages, longest, mx4):
    """Every row up to a length that ends inside a page, through a page table."""
    from paper_2609_37538_amd import latent as L
    g = gen(heads + page + longest)
    pool = pool_of(g, batch * pages + 3, page, mx4, pad=16)
    table = torch.randperm(batch * pages + 3, generator=g, device="cuda")[:batch * pages].to(torch.int32).view(batch, pages)
    cache = L.LatentCache(pool, batch, int(mx4), page_table=table.contiguous())
    q = normal(g, batch, n_q, heads, 576)
    lens = torch.randint(longest // 2, longest + 1, (batch, n_q), generator=g, device="cuda")
    lens.view(-1)[0] = longest - page // 2
    out, lse = cache.attend(q, lens=lens, longest=longest, scale=SCALE)
    check_attend(cache, q, out, lse, lens=lens, longest=longest)
    out, lse = cache.attend(q, scale=SCALE)
    check_attend(cache, q, out, lse)


@pytest.mark.parametrize("mx4", [False, True])
def test_attend_masks(mx4):
    """Tokens without rows, whole tiles that are masked, rows and pages that do not exist, and NaN and
    infinities in every row that must not be read."""
    from paper_2609_37538_amd import latent as L
    g = gen(5)
    batch, n_q, heads, k, slots = 3, 4, 24, 400, 512
    pool = pool_of(g, batch, slots, mx4)
    used = torch.arange(slots, device="cuda") % 3 != 1
    # 0xff bytes are NaN in bfloat16 and a NaN scale in 4 bits; 0x7f80 words are infinities in bfloat16
    pool[:, ~used] = 0xff
    if not mx4:
        pool[:, 1::6] = torch.tensor([0x80, 0x7f], dtype=torch.uint8, device="cuda").repeat(576)
    cache = L.LatentCache(pool, batch, int(mx4))
    q = normal(g, batch, n_q, heads, 576)
    rows = torch.randint(0, slots, (batch, n_q, k), generator=g, device="cuda").to(torch.int32)
    index = torch.where(used[rows.long()], torch.arange(k, device="cuda", dtype=torch.int32),
                        torch.where(rows % 2 == 1, -1, 10 ** 6).to(torch.int32)).contiguous()
    lens = torch.tensor([[0, 400, 399, 1], [2, 64, 65, 200], [0, 0, 300, 128]], device="cuda")
    index[1, 3, :150] = 10 ** 6        # the first tiles have nothing
    index[2, 2, 64:256] = -5
    rows[0, 1, 7], rows[0, 1, 9], rows[0, 2, :60] = -1, slots, 2 ** 31 - 1
    rows[1, 3, 160] = -2 ** 31
    out, lse = cache.attend(q, rows=rows, index=index, lens=lens, scale=SCALE)
    check_attend(cache, q, out, lse, rows, index, lens)
    assert (out[0, 0] == 0).all() and (lse[0, 0] == -math.inf).all()


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("batch,n_q,heads,k,slots", [
    (33, 2, 64, 700, 1024), (65, 2, 64, 300, 512), (50, 2, 33, 1500, 2048), (150, 2, 70, 100, 128),
    (9, 1, 16, 4096, 4096), (64, 1, 128, 33, 64), (16, 1, 130, 900, 1024)])
def test_attend_many_tokens(batch, n_q, heads, k, slots, mx4):
    """Enough tokens that 64 heads share a workgroup, with and without parts to join, and more parts
    than one thread takes; tokens without rows, tiles without rows, and NaN in rows that do not count."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch + heads + k)
    pool = pool_of(g, batch, slots, mx4)
    pool[:, 5::7] = 0xff
    cache = L.LatentCache(pool, batch, int(mx4))
    q = normal(g, batch, n_q, heads, 576)
    rows = torch.randint(0, slots, (batch, n_q, k), generator=g, device="cuda").to(torch.int32)
    index = torch.where(rows % 7 == 5, -1, torch.randint(0, 2 * k, rows.shape, generator=g, device="cuda")).to(torch.int32)
    index[batch // 2, 0, :k // 2] = 2 ** 31 - 1
    lens = torch.randint(0, 2 * k + 1, (batch, n_q), generator=g, device="cuda")
    lens[0, 0], lens[-1, -1] = 0, 2 * k
    out, lse = cache.attend(q, rows=rows, index=index, lens=lens, scale=SCALE)
    assert (out[0, 0] == 0).all() and (lse[0, 0] == -math.inf).all()
    some = torch.tensor(sorted({0, 1, batch // 2, batch - 1}), device="cuda")
    few = L.LatentCache(pool[some].contiguous(), len(some), int(mx4))
    pick = lambda x: x[some].contiguous()  # noqa: E731
    check_attend(few, pick(q), pick(out), pick(lse), pick(rows), pick(index), pick(lens))
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("order", ["rising", "falling", "one far above", "far below zero"])
def test_attend_score_ranges_many_tokens(order, mx4):
    """The same ranges as below, with every token of a large batch at another place of the ramp."""
    from paper_2609_37538_amd import latent as L
    g = gen(17)
    batch, k, heads = 66, 700, 64
    latent, rope = normal(g, k, 512, by=0.1), normal(g, k, 64, by=0.1)
    ramp = torch.linspace(-6, 6, k, device="cuda")
    if order == "falling":
        ramp = -ramp
    elif order == "one far above":
        ramp = torch.where(torch.arange(k, device="cuda") == 500, 6.0, -6.0)
    elif order == "far below zero":
        ramp = ramp - 30
    latent[:, :32] = ramp[:, None].to(torch.bfloat16)
    pool = row_bytes(latent, rope, mx4).unsqueeze(0).expand(batch, -1, -1).contiguous()
    cache = L.LatentCache(pool, batch, int(mx4))
    rows = ((torch.arange(k, device="cuda")[None] + 10 * torch.arange(batch, device="cuda")[:, None]) % k).to(torch.int32)
    rows = rows.view(batch, 1, k).contiguous()
    q = normal(g, batch, 1, heads, 576)
    q[..., :32] = 1.0 + torch.arange(heads, device="cuda")[:, None] / heads
    out, lse = cache.attend(q, rows=rows, scale=1.5)
    some = torch.tensor([0, 1, 30, batch - 1], device="cuda")
    few = L.LatentCache(pool[some].contiguous(), len(some), int(mx4))
    check_attend(few, q[some].contiguous(), out[some].contiguous(), lse[some].contiguous(), rows[some].contiguous(), scale=1.5)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("order", ["rising", "falling", "one far above", "far below zero"])
def test_attend_score_ranges(order, mx4):
    """Scores that grow over hundreds along the entries, so that every later row outweighs all before
    it, and the other way round; sums are relative to maxima that move."""
    from paper_2609_37538_amd import latent as L
    g = gen(7)
    k, heads = 777, 32
    latent, rope = normal(g, k, 512, by=0.1), normal(g, k, 64, by=0.1)
    ramp = torch.linspace(-6, 6, k, device="cuda")
    if order == "falling":
        ramp = -ramp
    elif order == "one far above":
        ramp = torch.where(torch.arange(k, device="cuda") == 500, 6.0, -6.0)
    elif order == "far below zero":
        ramp = ramp - 30
    latent[:, :32] = ramp[:, None].to(torch.bfloat16)
    cache = L.LatentCache(row_bytes(latent, rope, mx4).unsqueeze(0), 1, int(mx4))
    q = normal(g, 1, 1, heads, 576)
    q[..., :32] = 1.0 + torch.arange(heads, device="cuda")[:, None] / heads
    out, lse = cache.attend(q, scale=1.5)
    check_attend(cache, q, out, lse, scale=1.5)


@pytest.mark.parametrize("batch,heads,k,mx4", [(132, 64, 700, True), (33, 40, 1000, True), (66, 32, 600, True),
                                               (130, 16, 500, False), (128, 16, 600, False), (40, 40, 1000, False)])
@pytest.mark.parametrize("order", ["rising", "falling"])
def test_attend_rising_and_masked(order, batch, heads, k, mx4):
    """Scores that grow or fall along the entries, of which some do not count and hold NaN, in batches of
    the sizes between few tokens and many: tiles of every kind, whole and in parts."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch + heads)
    slots = k + 50
    latent, rope = normal(g, slots, 512, by=0.1), normal(g, slots, 64, by=0.1)
    ramp = torch.linspace(-6, 6, slots, device="cuda")
    latent[:, :32] = (ramp if order == "rising" else -ramp)[:, None].to(torch.bfloat16)
    pool = row_bytes(latent, rope, mx4).unsqueeze(0).expand(batch, -1, -1).contiguous()
    pool[:, 3::11] = 0xff
    cache = L.LatentCache(pool, batch, int(mx4))
    first = torch.arange(batch, device="cuda") % 50
    rows = (first[:, None] + torch.arange(k, device="cuda")).to(torch.int32).view(batch, 1, k).contiguous()
    index = torch.where(rows % 11 == 3, -1, rows).contiguous()
    lens = torch.randint(0, slots + 1, (batch, 1), generator=g, device="cuda")
    lens[0], lens[1], lens[batch - 1] = 0, 1, slots
    q = normal(g, batch, 1, heads, 576)
    q[..., :32] = 1.0 + torch.arange(heads, device="cuda")[:, None] / heads
    out, lse = cache.attend(q, rows=rows, index=index, lens=lens, scale=1.5)
    assert torch.isfinite(out).all() and (out[0] == 0).all() and (lse[0] == -math.inf).all()
    some = torch.tensor([0, 1, 2, batch // 2, batch - 1], device="cuda")
    few, pick = L.LatentCache(pool[some].contiguous(), len(some), int(mx4)), lambda x: x[some].contiguous()
    check_attend(few, pick(q), pick(out), pick(lse), pick(rows), pick(index), pick(lens), scale=1.5)


def test_attend_scale_extremes():
    """Scales of zero and below zero."""
    from paper_2609_37538_amd import latent as L
    g = gen(8)
    cache = L.LatentCache(pool_of(g, 1, 200, True), 1, 1)
    q = normal(g, 1, 2, 16, 576)
    for scale in (0.0, -0.2):
        out, lse = cache.attend(q, scale=scale)
        check_attend(cache, q, out, lse, scale=scale)


@pytest.mark.parametrize("mx4", [False, True])
def test_attend_row_of_infinity(mx4):
    """A row that counts and holds what no sum survives makes NaN, in its query tokens alone."""
    from paper_2609_37538_amd import latent as L
    g = gen(9)
    pool = pool_of(g, 1, 256, mx4)
    pool[0, 100] = 0xff
    cache = L.LatentCache(pool, 1, int(mx4))
    q = normal(g, 1, 2, 16, 576)
    lens = torch.tensor([[100, 101]], device="cuda")
    out, lse = cache.attend(q, lens=lens, scale=SCALE)
    check_attend(cache, q[:, :1], out[:, :1], lse[:, :1], lens=lens[:, :1])
    assert out[0, 1].isnan().all() and lse[0, 1].isnan().all()


def test_attend_strides_and_streams():
    """Queries and outputs inside wider tensors, a stream of its own, and results that do not change
    from call to call."""
    from paper_2609_37538_amd import latent as L
    g = gen(11)
    cache = L.LatentCache(pool_of(g, 2, 512, True, pad=32), 2, 1)
    wide = normal(g, 2, 3, 40, 640)
    q = wide[:, :, 3:23, 16:592]
    room = torch.zeros(2, 3, 30, 576, dtype=torch.bfloat16, device="cuda")
    out = room[:, :, 5:25, 64:]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, lse = cache.attend(q, scale=SCALE, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert got is out
    check_attend(cache, q, out, lse, what="strided")
    again, lse2 = cache.attend(q.contiguous(), scale=SCALE)
    assert torch.equal(again, out) and torch.equal(lse, lse2)
    room[:, :, 5:25, 64:] = 0
    assert not room.any(), "written outside the output"


@pytest.mark.parametrize("mx4", [False, True])
def test_attend_long_offsets(mx4):
    """Rows whose byte offsets pass 32 bits."""
    from paper_2609_37538_amd import latent as L
    g = gen(12)
    row = L.avsg_row_bytes(int(mx4))
    page = 2304 * 1024 * 1024 // row // 16 * 16       # rows of a page: over 2 GiB
    room = torch.zeros((3, page, row), dtype=torch.uint8, device="cuda")
    k = 200
    for p in range(3):
        room[p, page - k:] = row_bytes(normal(g, k, 512), normal(g, k, 64), mx4)
    cache = L.LatentCache(room, 3, int(mx4))
    rows = (page - 1 - torch.randperm(k, generator=g, device="cuda")).to(torch.int32).view(1, 1, k).repeat(3, 1, 1)
    q = normal(g, 3, 1, 16, 576)
    out, lse = cache.attend(q, rows=rows, scale=SCALE)
    for b in range(3):
        keys = R.row_values(room[b][rows[b, 0].long()], mx4)
        o, s, eo, es = R.attend(q[b, 0], keys, torch.ones(k, dtype=torch.bool), SCALE)
        close(out[b, 0], o, eo, f"request {b}: out")
        close(lse[b, 0], s, es, f"request {b}: lse")


def test_attend_graph():
    """Captured once and replayed on new queries, with other work between the replays."""
    from paper_2609_37538_amd import latent as L
    g = gen(13)
    cache = L.LatentCache(pool_of(g, 2, 1024, True), 2, 1)
    q = normal(g, 2, 2, 32, 576)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.attend(q, scale=SCALE)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = cache.attend(q, scale=SCALE)
    for _ in range(4):
        q.copy_(normal(g, 2, 2, 32, 576))
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse = cache.attend(q, scale=SCALE)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


# ---------------------------------------------------------------------------
# append and read
# ---------------------------------------------------------------------------
def angles_of(n):
    t = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    return torch.stack((t.cos(), t.sin()), -1).float().cuda()


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("tokens,heads,page,batch", [(1, 0, 64, 1), (1, 1, 16, 1), (5, 16, 16, 2), (130, 20, 64, 3),
                                                     (1000, 8, 256, 2)])
def test_append_and_read(tokens, heads, page, batch, mx4, halves):
    from paper_2609_37538_amd import latent as L
    g = gen(tokens + heads)
    pages = -(-tokens // page) + 1
    room = torch.full((batch * pages + 1, page, L.avsg_row_bytes(int(mx4)) + 16), 0x55, dtype=torch.uint8, device="cuda")
    pool = room[..., :-16]
    table = torch.randperm(batch * pages + 1, generator=g, device="cuda")[:-1].to(torch.int32).view(batch, pages).contiguous()
    cache = L.LatentCache(pool, batch, int(mx4), page_table=table)
    total = pages * page
    spots = torch.randperm(batch * total, generator=g, device="cuda")[:tokens]
    request, position = (spots // total).to(torch.int32), (spots % total).contiguous()
    latent = normal(g, tokens, 520)[:, :512]
    latent[0, :32] = 0.0
    rope = normal(g, tokens, 64)
    q = normal(g, tokens, heads, 64) if heads else None
    wide = torch.full((tokens, heads, 576), 7.0, dtype=torch.bfloat16, device="cuda") if heads else None
    angles = angles_of(total)
    cache.append(latent, rope, request, position, angles, style=int(halves), q_rope=q,
                 q_out=wide[..., 512:] if heads else None)
    where = table.cpu()[request.cpu().long(), position.cpu() // page].long()
    raw = pool.cpu()[where, position.cpu() % page]
    turn = angles[position]
    want, bound = R.rotate(rope, turn, halves)
    if mx4:
        codes, scales = R.quantize(latent.cpu())
        assert torch.equal(raw[:, :256], codes) and torch.equal(raw[:, 256:272], scales)
        kept = R.values(codes, scales)
    else:
        kept = latent.cpu().double()
        assert torch.equal(raw[:, :1024].contiguous().view(torch.bfloat16), latent.cpu())
    got = R.row_values(raw, mx4)
    close(got[:, 512:], want, bound, "rotated part")
    # no other byte changed
    room.cpu()
    rest = room.clone()
    rest[where.cuda(), position % page, :-16] = 0x55
    assert (rest == 0x55).all()
    if heads:
        want, bound = R.rotate(q, turn[:, None], halves)
        close(wide[..., 512:], want, bound, "queries")
        assert (wide[..., :512] == 7.0).all()
        # in place
        cache.append(latent, rope, request, position, angles, style=int(halves), q_rope=q, q_out=q)
        assert torch.equal(q, wide[..., 512:])
    back = cache.read(request, position)
    close(back[:, :512], kept, torch.zeros(1), "read latent")
    assert torch.equal(back[:, 512:].cpu().double(), got[:, 512:])


@pytest.mark.parametrize("mx4", [False, True])
def test_append_skips_what_does_not_exist(mx4):
    """Padding tokens, requests and positions out of range, and pages that are not there."""
    from paper_2609_37538_amd import latent as L
    g = gen(21)
    pool = torch.zeros((6, 16, L.avsg_row_bytes(int(mx4))), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[0, 1, -1], [6, 4, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    cache = L.LatentCache(pool, 2, int(mx4), page_table=table)
    request = torch.tensor([0, 0, 0, 2, -1, 0, 1, 1, 1, 0, 1], dtype=torch.int32, device="cuda")
    position = torch.tensor([3, -1, 48, 1, 1, 40, 2, 20, 33, 2 ** 40, 47], device="cuda")
    n = request.shape[0]
    latent, rope, q = normal(g, n, 512), normal(g, n, 64), normal(g, n, 4, 64)
    out = torch.full_like(q, 9.0)
    cache.append(latent, rope, request, position, angles_of(45), q_rope=q, q_out=out)
    written = pool.view(96, -1).any(-1).nonzero().flatten().tolist()
    assert written == [3, 4 * 16 + 4]
    zero = [i for i in range(n) if not 0 <= int(position[i]) < 45]
    assert (out[zero] == 0).all()
    rest = [i for i in range(n) if i not in zero]
    want, bound = R.rotate(q[rest], angles_of(45)[position[rest]][:, None], False)
    close(out[rest], want, bound, "queries")
    back = cache.read(request, position)
    for i in range(n):
        assert bool(back[i].any()) == (i in (0, 7)), i


def test_append_of_infinities():
    """A block with an infinity or a NaN reads back as NaN, its neighbours as they were."""
    from paper_2609_37538_amd import latent as L
    g = gen(22)
    pool = torch.zeros((1, 16, 400), dtype=torch.uint8, device="cuda")
    cache = L.LatentCache(pool, 1, 1)
    latent, rope = normal(g, 2, 512), normal(g, 2, 64)
    plain = latent.clone()
    latent[0, 40], latent[1, 511], latent[1, 0] = math.inf, math.nan, -math.inf
    at = torch.tensor([0, 1], device="cuda")
    cache.append(latent, rope, at.int() * 0, at, angles_of(16))
    back = cache.read(at.int() * 0, at)[:, :512].cpu().double()
    codes, scales = R.quantize(plain.cpu())
    want = R.values(codes, scales)
    want[0, 32:64], want[1, 480:], want[1, :32] = math.nan, math.nan, math.nan
    assert torch.equal(back.isnan(), want.isnan())
    assert torch.equal(back.nan_to_num(), want.nan_to_num())


def test_append_nothing():
    from paper_2609_37538_amd import latent as L
    cache = L.LatentCache(torch.zeros((1, 16, 400), dtype=torch.uint8, device="cuda"), 1, 1)
    e = torch.empty(0, 512, dtype=torch.bfloat16, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    cache.append(e, e[:, :64].contiguous(), none.int(), none, angles_of(1))
    assert cache.read(none.int(), none).shape == (0, 576)


def test_append_to_host_rows():
    """Rows appended to pinned host memory are there for a host that reads them."""
    import numpy as np
    from paper_2609_37538_amd import avsg as A, latent as L
    g = gen(23)
    rows = 40
    region = A.HostRegion(2 * rows * 400)
    view = region.view()
    view[:] = 0x55
    cache = L.LatentCache(None, 2, 1, base=region.ptr, pages=2, page_rows=rows, device="cuda")
    latent, rope = normal(g, 3, 512), normal(g, 3, 64)
    request = torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda")
    position = torch.tensor([39, 0, 17], device="cuda")
    cache.append(latent, rope, request, position, angles_of(rows))
    torch.cuda.synchronize()
    codes, scales = R.quantize(latent.cpu())
    at = np.array([39, 40, 57])
    raw = torch.from_numpy(view.reshape(-1, 400)[at].copy())
    assert torch.equal(raw[:, :256], codes) and torch.equal(raw[:, 256:272], scales)
    assert (np.delete(view.reshape(-1, 400), at, 0) == 0x55).all()
    back = cache.read(request, position)
    assert torch.equal(back[:, :512].cpu().double(), R.values(codes, scales))
    del view
    region.free()


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def test_wrapper_refusals():
    from paper_2609_37538_amd import latent as L
    pool = torch.zeros((2, 64, 400), dtype=torch.uint8, device="cuda")
    cache = L.LatentCache(pool, 2, 1)
    q = torch.zeros((2, 1, 16, 576), dtype=torch.bfloat16, device="cuda")
    rows = torch.zeros((2, 1, 8), dtype=torch.int32, device="cuda")
    lens = torch.ones((2, 1), dtype=torch.int64, device="cuda")
    bad = [
        lambda: L.LatentCache(pool, 2, 0), lambda: L.LatentCache(pool, 2, 5), lambda: L.LatentCache(pool, 3, 1),
        lambda: L.LatentCache(pool.cpu(), 2, 1), lambda: L.LatentCache(pool, 0, 1),
        lambda: L.LatentCache(pool, 2, 1, page_table=torch.zeros((2, 1), dtype=torch.int64, device="cuda")),
        lambda: L.LatentCache(None, 2, 1),
        lambda: cache.attend(q.float(), rows=rows, scale=1.0), lambda: cache.attend(q[:1], rows=rows[:1], scale=1.0),
        lambda: cache.attend(q[..., :512], rows=rows, scale=1.0), lambda: cache.attend(q, rows=rows.long(), scale=1.0),
        lambda: cache.attend(q, rows=rows[..., ::2], scale=1.0), lambda: cache.attend(q, rows=rows, index=rows[..., :4], scale=1.0),
        lambda: cache.attend(q, rows=rows, lens=lens.int(), scale=1.0), lambda: cache.attend(q, rows=rows, longest=8, scale=1.0),
        lambda: cache.attend(q, rows=rows.cpu(), scale=1.0), lambda: cache.attend(q, scale=1.0, out=q),
        lambda: cache.attend(torch.zeros((2, 1, 16, 577), dtype=torch.bfloat16, device="cuda")[..., 1:], rows=rows, scale=1.0),
        lambda: cache.read(rows[:, 0, 0].contiguous(), rows[:, 0, 0].contiguous()),
        lambda: cache.read(rows[:, 0, 0].contiguous(), lens[:, 0].contiguous(), out=q[:, 0, 0, :512]),
        lambda: cache.append(q[:, 0, 0], q[:, 0, 0], rows[:, 0, 0].contiguous(), lens[:, 0].contiguous(), angles_of(4)),
        lambda: cache.append(q[:, 0, 0, :512], q[:, 0, 0, 512:], rows[:, 0, 0].contiguous(), lens[:, 0].contiguous(),
                             angles_of(4), q_rope=q[:, 0, :, 512:]),
        lambda: cache.append(q[:, 0, 0, :512], q[:, 0, 0, 512:], rows[:, 0, 0].contiguous(), lens[:, 0].contiguous(),
                             angles_of(4).double()),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"refusal {i} did not happen")
    # too many pages in a row for one that is no power of two
    with pytest.raises(L.AvsgError, match="power of two"):
        L.LatentCache(torch.zeros((4, 48, 400), dtype=torch.uint8, device="cuda"), 2, 1).attend(q, rows=rows, scale=1.0)
