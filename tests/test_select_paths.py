"""Every kernel of a selection's scores, through runs of keys as long as large calls have them, on cases that the
choice gives it now; which rows they read; and what the positions that are always taken have precedence over."""
import ctypes
import math

import pytest
import torch

import select_reference as R
from paper_2609_37538_amd import selection as S
from test_select import check, made

gpu = pytest.mark.gpu


def path(batch, n_q, heads, longest):
    """(kernel, tiles or stages of a run): 100 times the heads' tiles, and for waves on their own 10 times the waves of
    a workgroup on different tokens and the tokens of each."""
    f = S.load().avsg_internal_score_plan
    f.restype, f.argtypes = ctypes.c_int64, [ctypes.c_int32] * 4
    plan = f(batch, n_q, heads, longest)
    return plan & 0xffffffff, plan >> 32


# kernel, run, batch, query tokens, heads, pages of a request, rows of a page, block
CASES = [
    # workgroups that share their keys
    (100, 16, 1, 1030, 16, 128, 64, 1), (100, 16, 1, 1030, 9, 512, 16, 32), (200, 16, 2, 520, 30, 32, 256, 128), (200, 4, 1, 200, 20, 1024, 8, 1),
    (400, 16, 1, 1030, 64, 128, 64, 2), (400, 4, 1, 192, 64, 128, 64, 64), (400, 10, 1, 700, 40, 1, 7001, 1), (800, 16, 1, 1100, 100, 64, 128, 1),
    (800, 2, 1, 9, 100, 128, 64, 16), (800, 16, 3, 400, 128, 33, 256, 128),
    # waves on their own
    (111, 64, 300, 1, 16, 513, 16, 1), (112, 64, 300, 2, 16, 33, 256, 64), (112, 64, 120, 3, 9, 2052, 4, 1), (211, 64, 300, 1, 30, 1, 8207, 1),
    (212, 64, 300, 2, 30, 129, 64, 32), (411, 64, 300, 1, 64, 33, 256, 128), (412, 32, 120, 2, 64, 129, 64, 1), (412, 32, 40, 5, 64, 513, 16, 16),
    (811, 64, 300, 1, 100, 129, 64, 4), (811, 64, 120, 3, 128, 1026, 8, 8), (841, 64, 200, 5, 100, 130, 64, 128), (841, 8, 1, 5, 70, 129, 64, 1),
    (841, 64, 60, 4, 128, 2, 4096, 1), (412, 40, 64, 2, 64, 1025, 16, 1),
]


def test_kernel_of_a_case():
    for kernel, run, batch, n_q, heads, pages, page, block in CASES:
        assert path(batch, n_q, heads, pages * page) == (kernel, run) and pages * page % block == 0, (batch, n_q, heads)
    assert {c[0] for c in CASES} == {100, 200, 400, 800, 111, 112, 211, 212, 411, 412, 811, 841}


@gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_long_runs(case):
    """Requests whose tables hold the same pages in other orders, some of them missing, with NaN between the rows; lengths
    that end anywhere in a run.  Some tokens are compared, the first, the last and one that sees nothing among them."""
    kernel, run, batch, n_q, heads, pages, page, block = case
    n = pages * page
    assert path(batch, n_q, heads, n) == (kernel, run)
    print(f"kernel {kernel}, runs of {run}", flush=True)
    g = torch.Generator().manual_seed(n + n_q + heads)
    _, _, pool, _ = made(g, 1, 1, 1, pages, page, stride=136)
    pool[..., 132:] = 255
    q = torch.randint(-127, 128, (batch, n_q, heads, 128), generator=g).to(torch.int8)
    weights = torch.randn(batch, n_q, heads, generator=g) * torch.rand(batch, n_q, heads, generator=g)
    table = torch.stack([torch.randperm(pages, generator=g) for _ in range(batch)]).to(torch.int32)
    if pages > 8:
        table[torch.rand(batch, pages, generator=g) < 0.03] = -1
        table[torch.rand(batch, pages, generator=g) < 0.01] = pages
    lens = torch.randint(1, n + 1, (batch, n_q), generator=g)
    lens[-1, -1], lens[0, 0], lens[batch // 2, n_q // 2] = n, n - 1, 0
    kw = dict(topk=512, block=block, first=3, recent=70 if block < 64 else 1)
    cache = S.KeyCache(pool.cuda()[..., :132], batch, page_table=table.cuda())
    index, scores = cache.select(q.cuda(), weights.cuda(), lens=lens.cuda(), **kw)
    tokens = torch.randint(0, batch * n_q, (14,), generator=g).tolist() + [0, batch * n_q - 1, batch // 2 * n_q + n_q // 2]
    rows = {}
    for t in sorted(tokens):
        r, i = divmod(t, n_q)
        if r not in rows:
            rows = {r: R.request_rows(pool[..., :132], table, r, pages)}
        want = R.best(R.scores(q[r, i], weights[r, i], rows[r]), int(lens[r, i]), **kw)
        check((index[r, i], scores[r, i]), want)


@pytest.mark.parametrize("page", [16, 32, 64, 256, 4096])
def test_rows_that_no_token_sees_are_not_addressed(page):
    """Every row that a run's loads go to, those of the tiles after its last among them, is one that some token sees,
    and those that count are the keys' own: for pages that end in each other's place relative to the run."""
    f = S.load().avsg_internal_score_row
    f.restype, f.argtypes = ctypes.c_int32, [ctypes.c_int32] * 6
    shift = page.bit_length() - 1
    for run in (8, 24, 64):
        for most in (1, 15, 16, 17, 100, 127, 128, 129, 500, 1024, 1025, 1500, 4096, 4100):
            for first in range(0, most, run * 16):
                tiles = min(run, (most - first + 15) // 16)
                for tile in range(tiles + 8):
                    for lane in (0, 1, 7, 14, 15):
                        key, row = first + tile * 16 + lane, f(first, tiles, tile, lane, most, shift)
                        assert 0 <= row < most, (run, most, first, tile, lane)
                        if tile < tiles:
                            assert row == min(key, most - 1)
                        assert f(first, tiles, tile, lane, most, 2) == f(first, tiles, tile, lane, most, 31) == min(key, most - 1)


@gpu
@pytest.mark.parametrize("n_q", [1, 2, 7])
@pytest.mark.parametrize("block", [1, 16])
def test_always_taken_whatever_the_row_is(n_q, block):
    """Positions of `first` and `recent` that a token sees are taken, also where the row does not exist or its score is
    NaN; those that it does not see are not ranked by them."""
    g = torch.Generator().manual_seed(n_q)
    q, weights, pool, table = made(g, 1, n_q, 8, 8, 64)
    table[0, 0], table[0, 4] = -1, 8
    pool[table[0, 3].long(), 40, 128:] = 255          # a scale of NaN at position 232
    lens = torch.full((1, n_q), 300)
    kw = dict(topk=128, block=block, first=5, recent=70)
    cache = S.KeyCache(pool.cuda(), 1, page_table=table.cuda())
    got = cache.select(q.cuda(), weights.cuda(), lens=lens.cuda(), **kw)
    check(got, R.select(q, weights, pool, table, lens, **kw))
    for t in range(n_q):
        picked = set(got[0][0, t].tolist())
        assert set(range(5)) <= picked and set(range(230, 300)) <= picked
        best = got[1][0, t]
        assert int((best == math.inf).sum()) == (75 if block == 1 else 6)
