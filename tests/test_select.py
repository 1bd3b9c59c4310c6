"""The key cache and the selection against plain forms on the CPU: quantisation step
by step in float32, scores in whole numbers and 64 bits.  Codes, scales and positions
have to be equal; scores may be off by one rounding to float32 where 64-bit sums of
another order round differently."""
import math

import pytest
import torch

import select_reference as R
from paper_2609_37538_amd import avsg as A
from paper_2609_37538_amd import latent as L
from paper_2609_37538_amd import selection as S

gpu = pytest.mark.gpu
ULP = 2.0 ** -23


def noise(g, *shape, by=1.0):
    return torch.randn(shape, generator=g) * by


def turns(positions):
    a = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    return torch.stack((a.cos(), a.sin()), -1).float()


def made(g, batch, n_q, heads, pages, page, *, stride=132, table=True, keys=None):
    """(q, weights, pool, table) on the CPU; rows `stride` bytes apart."""
    keys = noise(g, pages * page, 128) if keys is None else keys
    pool = torch.zeros(pages, page, stride, dtype=torch.uint8)
    pool[..., :132] = R.rows_of(keys).view(pages, page, 132)
    q, scale = R.eighths(noise(g, batch, n_q, heads, 128))
    weights = noise(g, batch, n_q, heads) * scale
    table = torch.randperm(pages, generator=g)[:batch * (pages // batch)].view(batch, -1).to(torch.int32) if table else None
    return q, weights, pool, table


def check(got, want, block=1):
    index, scores = got[0].cpu(), got[1].cpu()
    assert torch.equal(index, want[0])
    both = torch.isfinite(want[1])
    assert torch.equal(torch.where(both, 0.0, scores), torch.where(both, 0.0, want[1]))
    off = (scores - want[1])[both].abs()
    assert (off <= ULP * want[1][both].abs()).all()


def run(q, weights, pool, table, lens, **kw):
    pool = pool.cuda()
    cache = S.KeyCache(pool[..., :132], q.shape[0], page_table=None if table is None else table.cuda())
    return cache.select(q.cuda(), weights.cuda(), lens=None if lens is None else lens.cuda(), **kw)


# batch, n_q, heads, pages, page rows, topk, block, kind of lengths
CASES = [
    (1, 1, 1, 1, 1, 1, 1, None), (1, 1, 1, 2, 16, 32, 1, "all"), (1, 1, 16, 8, 64, 100, 1, "all"),
    (2, 1, 3, 6, 16, 17, 1, "mixed"), (3, 2, 17, 9, 64, 40, 1, "mixed"), (2, 3, 40, 8, 32, 64, 2, "mixed"),
    (1, 5, 33, 10, 64, 128, 4, "causal"), (2, 2, 64, 16, 64, 256, 8, "mixed"), (1, 4, 64, 16, 64, 160, 16, "causal"),
    (2, 1, 65, 16, 64, 192, 32, "mixed"), (1, 2, 128, 32, 64, 512, 64, "mixed"), (2, 3, 100, 16, 256, 384, 128, "mixed"),
    (1, 19, 8, 40, 64, 500, 1, "causal"), (5, 1, 32, 20, 256, 1024, 1, "mixed"), (1, 1, 64, 80, 256, 2048, 1, "mixed"),
    (4, 9, 20, 8, 64, 1, 1, "mixed"), (1, 1, 4, 300, 256, 2048, 1, "all"), (1, 2, 1, 300, 256, 70000, 1, "mixed"),
    (2, 2, 12, 34, 64, 0, 1, "mixed"),
]


def lengths(kind, g, batch, n_q, n):
    if kind is None or kind == "all":
        return None if kind is None else torch.full((batch, n_q), n)
    if kind == "causal":
        return (n - n_q + 1 + torch.arange(n_q)).clamp(min=0).expand(batch, -1).contiguous()
    lens = torch.randint(1, n + 1, (batch, n_q), generator=g)
    lens.view(-1)[::5] = torch.tensor([0, -3, 1, n + 7, n])[torch.arange(len(lens.view(-1)[::5])) % 5]
    return lens


@gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_selection(case):
    batch, n_q, heads, pages, page, topk, block, kind = case
    g = torch.Generator().manual_seed(sum(case[:7]))
    q, weights, pool, table = made(g, batch, n_q, heads, pages, page)
    n = pages // batch * page
    lens = lengths(kind, g, batch, n_q, n)
    check(run(q, weights, pool, table, lens, topk=topk, block=block),
          R.select(q, weights, pool, table, lens, topk=topk, block=block))


@gpu
@pytest.mark.parametrize("first,recent,block", [(1, 0, 1), (0, 1, 1), (5, 70, 1), (3, 40, 16), (0, 64, 64), (500, 500, 2), (2 ** 31 - 1, 0, 1),
                                                (0, 2 ** 31 - 1, 128)])
def test_positions_always_taken(first, recent, block):
    g = torch.Generator().manual_seed(first % 1000 + recent % 1000)
    q, weights, pool, table = made(g, 2, 4, 16, 16, 64)
    lens = torch.tensor([[512, 130, 7, 0], [511, 64, 65, 300]])
    kw = dict(topk=256, block=block, first=first, recent=recent)
    check(run(q, weights, pool, table, lens, **kw), R.select(q, weights, pool, table, lens, **kw))


@gpu
@pytest.mark.parametrize("n,topk", [(512, 100), (512, 500), (8192, 3000), (40000, 2048), (66048, 2048)])
def test_equal_scores_go_to_the_lowest(n, topk):
    """Few different keys, keys of zeros, and scores that are all zero (weights and products of either sign)."""
    g = torch.Generator().manual_seed(n)
    keys = noise(g, 7, 128)[torch.randint(0, 7, (n,), generator=g)]
    keys[torch.randint(0, n, (n // 3,), generator=g)] = 0.0
    q, weights, pool, _ = made(g, 1, 3, 4, n // 256 if n % 256 == 0 else 1, 256 if n % 256 == 0 else n, keys=keys, table=False)
    weights[0, 1] = 0.0
    weights[0, 2] = -weights[0, 2].abs()
    q[0, 1, 0] = 0
    check(run(q, weights, pool, None, None, topk=topk), R.select(q, weights, pool, None, None, topk=topk))


@gpu
def test_missing_pages_nan_and_infinities():
    """Pages that do not exist, rows whose scale is NaN, and weights that are not finite."""
    g = torch.Generator().manual_seed(3)
    keys = noise(g, 16 * 64, 128)
    keys[5] = math.nan
    keys[700, 3] = math.inf
    keys[9] = 1e-38
    q, weights, pool, table = made(g, 2, 3, 8, 16, 64, keys=keys)
    table[0, 2], table[1, 0], table[1, 3] = -1, 16, 2 ** 31 - 1
    weights[0, 1, 2], weights[1, 0, 1], weights[1, 2, 3] = math.inf, -math.inf, math.nan
    for topk, block in ((60, 1), (500, 1), (512, 16)):
        kw = dict(topk=topk, block=block)
        check(run(q, weights, pool, table, None, **kw), R.select(q, weights, pool, table, None, **kw))


@gpu
def test_largest_products_and_scales():
    """Codes of +-127 everywhere: the largest sums that the products have; and scales that overflow to infinity."""
    n = 256
    pool = torch.zeros(1, n, 132, dtype=torch.uint8)
    pool[..., :128] = 127
    pool[0, 1::2, :128] = 129                        # -127
    scale = torch.full((n,), 3e38)
    scale[::3] = 1.0
    pool[0, :, 128:] = scale[:, None].view(torch.uint8).view(n, 4)
    q = torch.full((1, 1, 128, 128), 127, dtype=torch.int8)
    q[0, 0, ::2] = -127
    weights = torch.linspace(-1, 1.5, 128).view(1, 1, 128)
    check(run(q, weights, pool, None, None, topk=200), R.select(q, weights, pool, None, None, topk=200))


@gpu
@pytest.mark.parametrize("turn", [1, 2, 5, 7, 30])
def test_small_workspaces_take_turns(turn):
    g = torch.Generator().manual_seed(turn)
    q, weights, pool, table = made(g, 3, 5, 16, 12, 64)
    lens = lengths("mixed", g, 3, 5, 256)
    want = R.select(q, weights, pool, table, lens, topk=50)
    ws = torch.empty(S.avsg_select_workspace_least(256, 1) * turn + 12, dtype=torch.uint8, device="cuda")
    check(run(q, weights, pool, table, lens, topk=50, workspace=ws), want)


@gpu
@pytest.mark.parametrize("stride", [136, 144, 1284])
def test_strides(stride):
    """Rows further apart, pages too; queries and weights as parts of wider tensors; results into given tensors."""
    g = torch.Generator().manual_seed(stride)
    q, weights, pool, table = made(g, 2, 3, 8, 8, 32, stride=stride)
    wide = torch.full((8, 40, stride), 255, dtype=torch.uint8)
    wide[:, :32] = pool
    dev = wide.cuda()
    cache = S.KeyCache(dev[:, :32, :132], 2, page_table=table.cuda())
    wq = torch.full((2, 3, 11, 144), -1, dtype=torch.int8)
    wq[:, :, 2:10, 16:] = q
    ww = torch.full((2, 3, 13), math.nan)
    ww[..., 4:12] = weights
    index = torch.full((2, 3, 20), -1, dtype=torch.int32, device="cuda")
    scores = torch.empty((2, 3, 20), device="cuda")
    got = cache.select(wq.cuda()[:, :, 2:10, 16:], ww.cuda()[..., 4:12], topk=20, index=index, scores=scores)
    assert got[0] is index and got[1] is scores
    check(got, R.select(q, weights, pool[..., :132], table, None, topk=20))


@gpu
@pytest.mark.parametrize("longest", [1, 100, 333, 384])
def test_part_of_the_rows(longest):
    g = torch.Generator().manual_seed(longest)
    q, weights, pool, table = made(g, 2, 2, 16, 12, 64)
    lens = torch.tensor([[384, 50], [longest, 1]])
    kw = dict(topk=min(longest, 64), longest=longest)
    check(run(q, weights, pool, table, lens, **kw), R.select(q, weights, pool, table, lens, **kw))


@gpu
@pytest.mark.parametrize("page", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("n_q,heads,block", [(1, 16, 1), (2, 40, 1), (3, 100, 32), (9, 8, 1), (6, 64, 128)])
def test_small_pages(page, n_q, heads, block):
    """Pages that end inside a tile of keys, some of which do not exist."""
    g = torch.Generator().manual_seed(page + n_q)
    pages = 2 * 640 // page
    q, weights, pool, table = made(g, 2, n_q, heads, pages, page)
    table[:, ::7] = torch.tensor([[-1], [pages]], dtype=torch.int32)
    lens = torch.randint(1, 641, (2, n_q), generator=g)
    kw = dict(topk=256, block=block)
    check(run(q, weights, pool, table, lens, **kw), R.select(q, weights, pool, table, lens, **kw))


@gpu
@pytest.mark.parametrize("n", [1, 15, 17, 100, 1001])
def test_one_page_of_any_rows(n):
    """Rows of one page per request whose number is no multiple of a tile, up to the pool's last byte."""
    g = torch.Generator().manual_seed(n)
    q, weights, pool, _ = made(g, 3, 2, 20, 3, n, table=False)
    check(run(q, weights, pool, None, None, topk=min(n, 50)), R.select(q, weights, pool, None, None, topk=min(n, 50)))
    q, weights, pool, _ = made(g, 2, 7, 20, 2, n, table=False)
    check(run(q, weights, pool, None, None, topk=min(n, 50)), R.select(q, weights, pool, None, None, topk=min(n, 50)))


@gpu
def test_rows_that_no_token_sees_are_not_read():
    """What lies past the lengths does not matter: NaN scales there, and pages that do not exist."""
    g = torch.Generator().manual_seed(11)
    q, weights, pool, table = made(g, 1, 2, 16, 8, 64)
    lens = torch.tensor([[100, 65]])
    a = run(q, weights, pool, table, lens, topk=128)
    pool[table[0, 2:].long()] = 255
    table[0, 2:] = -1
    b = run(q, weights, pool, table, lens, topk=128)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(a[0][0, 0].cpu(), torch.arange(128, dtype=torch.int32))


@gpu
def test_a_chunk_selects_what_its_tokens_select_alone():
    """Bit for bit, whatever kernels and turns take them."""
    g = torch.Generator().manual_seed(21)
    q, weights, pool, table = made(g, 1, 37, 64, 24, 64)
    lens = lengths("causal", g, 1, 37, 24 * 64)
    all_ = run(q, weights, pool, table, lens, topk=200)
    for t in (0, 1, 17, 36):
        one = run(q[:, t:t + 1], weights[:, t:t + 1], pool, table, lens[:, t:t + 1].contiguous(), topk=200)
        assert torch.equal(one[0][0, 0], all_[0][0, t]) and torch.equal(one[1][0, 0], all_[1][0, t])


# ---------------------------------------------------------------------------
# append and read
# ---------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("at", [0, 64, None])
@pytest.mark.parametrize("tokens,heads", [(1, 0), (1, 1), (3, 5), (70, 64)])
def test_append(tokens, heads, at, halves):
    g = torch.Generator().manual_seed(tokens * 100 + heads)
    key, q = noise(g, tokens, 128).bfloat16(), noise(g, tokens, heads, 128).bfloat16()
    weights = noise(g, tokens, heads)
    angles = None if at is None else turns(300)
    batch, page, per = 3, 32, 10
    table = torch.randperm(batch * per, generator=g).view(batch, per).to(torch.int32)
    request = torch.randint(0, batch, (tokens,), generator=g).to(torch.int32)
    position = torch.randperm(batch * 100, generator=g)[:tokens] % 300
    pool = torch.randint(0, 256, (batch * per, page, 132), generator=g).to(torch.uint8)
    dev = pool.cuda()
    cache = S.KeyCache(dev, batch, page_table=table.cuda())
    kw = {}
    if heads:
        kw = dict(q=q.cuda(), weights=weights.cuda(), q_out=torch.empty(tokens, heads, 128, dtype=torch.int8, device="cuda"),
                  weights_out=torch.empty(tokens, heads, device="cuda"))
    cache.append(key.cuda(), request.cuda(), position.cuda(), None if angles is None else angles.cuda(),
                 style=L.AVSG_ROPE_HALVES if halves else L.AVSG_ROPE_PAIRS, rope_at=at or 0, **kw)
    turn = None if angles is None else angles[position]
    y = R.turned(key, turn, halves, at)
    for t in range(tokens):
        pool[table[request[t], position[t] // page], position[t] % page] = R.rows_of(y[t])
    assert torch.equal(dev.cpu(), pool)
    got = cache.read(request.cuda(), position.cuda()).cpu()
    codes, scale = R.eighths(y)
    assert torch.equal(got, (codes.float() * scale[:, None]).bfloat16())
    # by the definition in 64 bits: half a step, the products' and sums' roundings in it, and the result's
    assert ((got.double() - y.double()).abs() <= scale[:, None].double() * (0.5 + 2.0 ** -14) + 2.0 ** -8 * y.abs()).all()
    if heads:
        codes, scale = R.eighths(R.turned(q, None if turn is None else turn[:, None], halves, at))
        assert torch.equal(kw["q_out"].cpu(), codes) and torch.equal(kw["weights_out"].cpu(), weights * scale)


@gpu
def test_append_values_and_padding():
    """Zeros, infinities, NaN, the least and the largest numbers; tokens out of range write nothing and get zeros."""
    key = torch.zeros(10, 128).bfloat16()
    key[1, 5], key[2, 7], key[3, 100] = math.inf, math.nan, -math.inf
    key[4] = torch.linspace(-1, 1, 128).bfloat16() * 2.0 ** -126
    key[5] = torch.linspace(-1, 1, 128).bfloat16() * 3e38
    key[6] = torch.linspace(-1, 1, 128).bfloat16() * 2.0 ** -119
    key[7:] = 1.0
    request = torch.tensor([0, 0, 0, 1, 1, 1, 1, -1, 2, 0], dtype=torch.int32)
    position = torch.tensor([0, 1, 2, 3, 4, 5, 6, 0, 0, -1])
    pool = torch.full((2, 8, 132), 77, dtype=torch.uint8)
    dev = pool.cuda()
    q_out = torch.full((10, 1, 128), 9, dtype=torch.int8, device="cuda")
    w_out = torch.full((10, 1), 9.0, device="cuda")
    S.KeyCache(dev, 2).append(key.cuda(), request.cuda(), position.cuda(), q=key.cuda()[:, None], q_out=q_out, weights_out=w_out)
    for t in range(7):
        pool[request[t], position[t]] = R.rows_of(key[t].float())
    got = dev.cpu()
    scale = pool[..., 128:].contiguous().view(torch.float32)
    assert torch.equal(got[..., :128], pool[..., :128])
    assert torch.equal(torch.nan_to_num(got[..., 128:].contiguous().view(torch.float32), -1.0), torch.nan_to_num(scale, -1.0))
    codes, scale = R.eighths(key.float())
    assert torch.equal(q_out[:9, 0].cpu(), codes[:9]) and not q_out[9].any()
    assert torch.equal(torch.nan_to_num(w_out[:9, 0].cpu(), -1.0), torch.nan_to_num(scale[:9], -1.0)) and w_out[9] == 0
    # positions past the angles, with rotation: likewise
    before = dev.clone()
    S.KeyCache(dev, 2).append(key.cuda()[:1], request.cuda()[:1], torch.tensor([5], device="cuda"), turns(5).cuda(),
                              q=key.cuda()[:1, None], q_out=q_out[:1], weights_out=w_out[:1])
    assert torch.equal(before, dev) and not q_out[0].any() and w_out[0] == 0


@gpu
def test_read_of_rows_that_do_not_exist():
    dev = torch.full((4, 16, 132), 1, dtype=torch.uint8, device="cuda")
    cache = S.KeyCache(dev, 2, page_table=torch.tensor([[0, -1], [3, 9]], dtype=torch.int32, device="cuda"))
    request = torch.tensor([0, 0, 1, 1, 2, -1, 0, 0], dtype=torch.int32, device="cuda")
    position = torch.tensor([3, 16, 15, 20, 0, 0, -1, 32], device="cuda")
    got = cache.read(request, position).cpu()
    some = got.any(-1).tolist()
    assert some == [True, False, True, False, False, False, False, False]


@gpu
def test_host_rows():
    """Keys in pinned host memory, rows 132 bytes apart."""
    region = A.HostRegion(2 * 64 * 132)
    cache = S.KeyCache(None, 2, base=region.ptr, pages=2, page_rows=64, device="cuda")
    g = torch.Generator().manual_seed(1)
    key = noise(g, 128, 128).bfloat16()
    request = torch.arange(2, dtype=torch.int32).repeat_interleave(64)
    position = torch.arange(64).repeat(2)
    cache.append(key.cuda(), request.cuda(), position.cuda())
    q, scale = R.eighths(noise(g, 2, 1, 8, 128))
    got = cache.select(q.cuda(), scale.cuda(), topk=10)
    pool = R.rows_of(key.float()).view(2, 64, 132)
    check(got, R.select(q, scale, pool, None, None, topk=10))
    torch.cuda.synchronize()
    region.free()


# ---------------------------------------------------------------------------
# as a program runs them
# ---------------------------------------------------------------------------
@gpu
def test_streams_and_graphs():
    """Two captured selections with workspaces of their own, replayed with eager calls between; every replay is the
    eager result on what the inputs hold by then."""
    g = torch.Generator().manual_seed(5)
    q, weights, pool, table = made(g, 2, 2, 16, 16, 64)
    other = made(g, 2, 2, 16, 16, 64)
    dq, dw, dp = q.cuda(), weights.cuda(), pool.cuda()
    cache = S.KeyCache(dp, 2, page_table=table.cuda())
    lens = torch.tensor([[512, 300], [64, 0]], device="cuda")
    cache.select(dq, dw, topk=64, lens=lens)
    outs, graphs = [], []
    for block in (1, 16):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(cache.select(dq, dw, topk=64, lens=lens, block=block))
        graphs.append(graph)
    for q_now, w_now, p_now in ((q, weights, pool), other[:3], (q, weights, other[2])):
        dq.copy_(q_now)
        dw.copy_(w_now)
        dp.copy_(p_now)
        for i in (0, 1, 0):
            graphs[i].replay()
            eager = cache.select(dq, dw, topk=32)
            torch.cuda.synchronize()
            check(outs[i], R.select(q_now, w_now, p_now, table, lens, topk=64, block=(1, 16)[i]))
            check(eager, R.select(q_now, w_now, p_now, table, None, topk=32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cache.select(dq, dw, topk=64, lens=lens)
    side.synchronize()
    check(got, R.select(q, weights, other[2], table, lens, topk=64))


@gpu
@pytest.mark.parametrize("block", [1, 16])
def test_append_select_step_attend(block):
    """A decode step as a program runs it: new keys and rows, the selection, the step that brings the selected
    rows into the slots, attention over them; against the plain selection and attention over the host's rows."""
    batch, n_q, heads, wide, context, topk, slots = 3, 2, 8, 16, 512, 64, 256
    g = torch.Generator(device="cuda").manual_seed(block)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    region = A.HostRegion(batch * context * 1152)
    host = L.LatentCache(None, batch, L.AVSG_ROWS_BF16, base=region.ptr, pages=batch, page_rows=context, device="cuda")
    pool = torch.zeros(batch, context, 132, dtype=torch.uint8, device="cuda")
    keys = S.KeyCache(pool, batch)
    angles = turns(context).cuda()
    everyone = torch.arange(batch, dtype=torch.int32, device="cuda").repeat_interleave(context)
    places = torch.arange(context, device="cuda").repeat(batch)
    keys.append(rand(batch * context, 128), everyone, places, angles)
    host.append(rand(batch * context, 512), rand(batch * context, 64), everyone, places, angles)
    cfg = A.make_config(batch, topk, n_q, slots, row_bytes=(1152,), gather_mode=A.AVSG_GATHER_RESIDENT)
    op = A.Operator(cfg, [region.ptr + r * context * 1152 for r in range(batch)], [context] * batch)
    slot_rows = L.LatentCache.of_slots(op)
    verified = torch.tensor([200, 33, 500], device="cuda")
    for _ in range(3):
        position = (verified[:, None] - 1 + torch.arange(n_q, device="cuda")).reshape(-1)
        request = torch.arange(batch, dtype=torch.int32, device="cuda").repeat_interleave(n_q)
        q_codes = torch.empty(batch * n_q, heads, 128, dtype=torch.int8, device="cuda")
        q_weights = torch.empty(batch * n_q, heads, device="cuda")
        keys.append(rand(batch * n_q, 128), request, position, angles, q=rand(batch * n_q, heads, 128), q_out=q_codes,
                    weights_out=q_weights)
        host.append(rand(batch * n_q, 512), rand(batch * n_q, 64), request, position, angles)
        lens = (position + 1).view(batch, n_q)
        q_codes, q_weights = q_codes.view(batch, n_q, heads, 128), q_weights.view(batch, n_q, heads)
        index, scores = keys.select(q_codes, q_weights, topk=topk, block=block, lens=lens, recent=1)
        check((index, scores), R.select(q_codes, q_weights, pool, None, lens, topk=topk, block=block, recent=1))
        placed, _ = op.step(index, verified)
        q = rand(batch, n_q, wide, 576)
        out, lse = slot_rows.attend(q, rows=placed, index=index, lens=lens, scale=0.1)
        want, want_lse = host.attend(q, rows=index, index=index, lens=lens, scale=0.1)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert torch.isfinite(lse).all()
        verified = verified + 1
    torch.cuda.synchronize()
    op.close()
    region.free()


@gpu
def test_refusals():
    dev = "cuda"
    pool = torch.zeros(4, 64, 132, dtype=torch.uint8, device=dev)
    cache = S.KeyCache(pool, 2)
    q, w = torch.zeros(2, 1, 4, 128, dtype=torch.int8, device=dev), torch.ones(2, 1, 4, device=dev)
    cache.select(q, w, topk=4)
    bad = [
        lambda: cache.select(q.float(), w, topk=4), lambda: cache.select(q[:1], w, topk=4), lambda: cache.select(q[..., :64], w, topk=4),
        lambda: cache.select(q.transpose(2, 3).contiguous().transpose(2, 3), w, topk=4), lambda: cache.select(q, w.double(), topk=4),
        lambda: cache.select(q, w[..., :3], topk=4), lambda: cache.select(q, w.clone().requires_grad_(), topk=4),
        lambda: cache.select(q, w, topk=-1), lambda: cache.select(q, w, topk=6, block=4), lambda: cache.select(q, w, topk=4, block=0),
        lambda: cache.select(q, w, topk=4, lens=torch.zeros(2, 1, dtype=torch.int32, device=dev)),
        lambda: cache.select(q, w, topk=4, lens=torch.zeros(2, 1, dtype=torch.int64)),
        lambda: cache.select(q, w, topk=4, index=torch.zeros(2, 1, 5, dtype=torch.int32, device=dev)),
        lambda: cache.select(q, w, topk=4, workspace=torch.zeros(4096, device=dev)), lambda: cache.select(q.cpu(), w, topk=4),
        lambda: S.KeyCache(pool[..., :131], 2), lambda: S.KeyCache(pool, 3), lambda: S.KeyCache(pool.cpu(), 2), lambda: S.KeyCache(None, 2),
        lambda: cache.append(torch.zeros(1, 128, device=dev), None, None),
        lambda: cache.append(torch.zeros(1, 128, dtype=torch.bfloat16, device=dev), torch.zeros(1, dtype=torch.int64, device=dev),
                             torch.zeros(1, dtype=torch.int64, device=dev)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for kw in (dict(topk=129), dict(topk=4, longest=200), dict(topk=6, block=3), dict(topk=4, workspace=torch.zeros(256, dtype=torch.uint8, device=dev))):
        with pytest.raises(A.AvsgError):
            cache.select(q, w, **kw)


# ---------------------------------------------------------------------------
# any scores: one head, one column, so that a row's scale is its score
# ---------------------------------------------------------------------------
def with_scores(scores):
    n = len(scores)
    pool = torch.zeros(1, n, 132, dtype=torch.uint8)
    pool[..., 0] = 1
    pool[0, :, 128:] = scores.float().contiguous().view(n, 1).view(torch.uint8).view(n, 4)
    q = torch.zeros(1, 1, 1, 128, dtype=torch.int8)
    q[..., 0] = 1
    return q, torch.ones(1, 1, 1), pool


def shapes(kind, n, g):
    x = torch.randn(n, generator=g)
    at = torch.arange(n)
    return {
        "normal": lambda: x,
        "ascending": lambda: x.sort().values, "descending": lambda: x.sort(descending=True).values,
        "periodic": lambda: torch.where(at % 4 == 0, x + 10, x), "rare": lambda: torch.where(at % 4 == 1, x + 10, x),
        "outliers": lambda: torch.where(at % 997 == 5, x * 1e38, x), "wide": lambda: x.sign() * torch.exp2(x * 40),
        "tiny": lambda: x * 1e-44, "few": lambda: (x * 2).round(), "one": lambda: torch.zeros(n), "two": lambda: (at % 3 == 0).float(),
        "neighbours": lambda: (1.0 + 2.0 ** -23 * torch.randint(0, 50, (n,), generator=g).double()).float(),
        "infinite": lambda: torch.where(x > 1, math.inf, torch.where(x < -1, -math.inf, x)),
        "nothing": lambda: torch.where(x > 2, x, math.nan), "late": lambda: torch.where(at > n - 50, x, -math.inf),
        "close": lambda: 1000.0 + x * 1e-3,
    }[kind]()


@gpu
@pytest.mark.parametrize("n", [300, 4096, 4097, 9000, 16384, 20001, 70000, 140000])
@pytest.mark.parametrize("kind", ["normal", "ascending", "descending", "periodic", "rare", "outliers", "wide", "tiny", "few", "one", "two",
                                  "neighbours", "infinite", "nothing", "late", "close"])
def test_any_scores(kind, n):
    g = torch.Generator().manual_seed(n)
    s = shapes(kind, n, g)
    q, weights, pool = with_scores(s)
    cache = S.KeyCache(pool.cuda(), 1)
    for topk in sorted({1, 63, n // 3, min(2048, n - 1), min(2561, n - 1), min(7000, n - 1), n - 1, n}):
        for lens in (None, torch.tensor([[n - 17]])):
            got = cache.select(q.cuda(), weights.cuda(), topk=topk, lens=None if lens is None else lens.cuda())
            want = R.best(s, n if lens is None else n - 17, topk, 1)
            assert torch.equal(got[0][0, 0].cpu(), want[0]), (topk, lens)
            assert torch.equal(got[1][0, 0].cpu(), want[1]), (topk, lens)
