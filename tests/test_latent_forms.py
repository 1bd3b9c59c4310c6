"""Forms of the latent-cache operators that a user has besides the ones of a decode step: contiguous results of
products, prompts of many tokens, whole contexts in bfloat16."""
import pytest
import torch

from test_latent import SCALE, _gpu, check_attend, gen, normal, pool_of  # noqa: F401
from test_mx4 import product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(1, 16, 64), (3, 8, 96), (17, 36, 160), (1, 1000, 1184), (2, 4096, 512), (31, 72, 2048),
                                   (64, 64, 256), (100, 512, 128), (129, 260, 544), (300, 132, 4096), (513, 772, 1024),
                                   (700, 1536, 4128), (2100, 1100, 1056)])
@pytest.mark.parametrize("f32", [False, True])
def test_product_into_rows_of_its_own(m, n, k, f32):
    """New contiguous results, whose columns are stored four and eight at a time, and the same into rows that
    are not aligned."""
    from paper_2609_37538_amd import latent as L
    g = gen(m + n + k)
    a = L.mx4_quantize(torch.randn(m, k, generator=g, device="cuda"))
    b = L.mx4_quantize(torch.randn(n, k, generator=g, device="cuda") * torch.exp2(torch.randint(-8, 9, (n, 1), generator=g, device="cuda").float()))
    dtype = torch.float32 if f32 else torch.bfloat16
    out = L.mx4_matmul(a, b, dtype=dtype)
    assert out.is_contiguous()
    product(a, b, out, f32)
    room = torch.full((m, n + 3), 5.0, dtype=dtype, device="cuda")
    assert torch.equal(L.mx4_matmul(a, b, out=room[:, 1:n + 1]), out)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("batch,n_q,heads,page,context", [(1, 70, 16, 16, 70), (2, 33, 40, 64, 300), (1, 300, 64, 64, 300),
                                                          (3, 9, 128, 256, 700), (1, 513, 8, 64, 1025)])
def test_attend_prompts(batch, n_q, heads, page, context, mx4):
    """The last n_q tokens of a context, of which each sees those up to itself, over pages of either format."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch + n_q + heads)
    pages = -(-context // page)
    table = torch.randperm(batch * pages + 2, generator=g, device="cuda")[:batch * pages].to(torch.int32).view(batch, pages).contiguous()
    cache = L.LatentCache(pool_of(g, batch * pages + 2, page, mx4), batch, int(mx4), page_table=table)
    q = normal(g, batch, n_q, heads, 576)
    lens = (context - n_q + 1 + torch.arange(n_q, device="cuda")).expand(batch, n_q).contiguous()
    out, lse = cache.attend(q, lens=lens, longest=context, scale=SCALE)
    some = torch.tensor(sorted({0, 1, n_q // 2, n_q - 1}), device="cuda")
    pick = lambda x: x[:, some].contiguous()  # noqa: E731
    check_attend(cache, pick(q), pick(out), pick(lse), lens=pick(lens), longest=context)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("batch,heads,page,context", [(1, 16, 64, 20000), (4, 64, 256, 5000), (2, 128, 16, 3001)])
def test_attend_whole_contexts_in_bfloat16(batch, heads, page, context):
    from paper_2609_37538_amd import latent as L
    g = gen(batch + heads + context)
    pages = -(-context // page)
    table = torch.randperm(batch * pages, generator=g, device="cuda").to(torch.int32).view(batch, pages).contiguous()
    cache = L.LatentCache(pool_of(g, batch * pages, page, False), batch, 0, page_table=table)
    q = normal(g, batch, 1, heads, 576)
    lens = torch.randint(context // 2, context + 1, (batch, 1), generator=g, device="cuda")
    out, lse = cache.attend(q, lens=lens, longest=context, scale=SCALE)
    check_attend(cache, q, out, lse, lens=lens, longest=context)
