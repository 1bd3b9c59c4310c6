"""The latent-cache operators at the ends of what their arguments can say."""
import random

import pytest
import torch

from paper_2609_37538_amd import avsg as A
from paper_2609_37538_amd import latent as L

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("batch,n_q,heads", [(1, 1, 16), (4, 1, 16), (1, 1, 64), (2, 3, 40), (16, 1, 128)])
def test_plans_of_the_longest_contexts(batch, n_q, heads):
    """The last counts of entries that 32 bits hold are shared by as many workgroups as those before them."""
    want = L.avsg_attend_workspace_bytes(batch, n_q, heads, 2 ** 31 - 4096)
    assert want > 0
    for k in [MOST - i for i in (0, 1, 30, 31, 62, 63, 64, 126, 127, 128, 200)]:
        assert L.avsg_attend_workspace_bytes(batch, n_q, heads, k) == want, k


@pytest.mark.gpu
@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("batch,n_q,heads", [(1, 1, 16), (2, 2, 64), (3, 1, 40)])
@pytest.mark.parametrize("longest", [MOST, MOST - 63])
def test_attend_without_a_limit(longest, batch, n_q, heads, mx4):
    """Contexts bounded by their lengths alone, and by the rows that exist."""
    from test_latent import SCALE, check_attend, gen, normal, pool_of
    g = gen(batch + heads)
    cache = L.LatentCache(pool_of(g, batch, 500, mx4), batch, int(mx4))
    q = normal(g, batch, n_q, heads, 576)
    lens = torch.randint(1, 501, (batch, n_q), generator=g, device="cuda")
    lens[0, 0] = 700       # 200 of them are not there
    out, lse = cache.attend(q, lens=lens, longest=longest, scale=SCALE)
    check_attend(cache, q, out, lse, lens=lens, longest=700)


def test_more_than_a_launch_takes():
    """Counts that no launch takes are refused by the checks, with the status that says so."""
    from test_latent_abi import append, attention, cache, status
    rng, rows = A.AVSG_E_RANGE, 67108860
    for heads, per in ((0, 1), (8, 2), (9, 3), (128, 17)):
        q = dict(heads=heads, d_q=4096, q_token_stride=64 * heads, q_head_stride=64, d_q_out=4096, q_out_token_stride=64 * heads,
                 q_out_head_stride=64)
        assert status(L.avsg_kv_append, cache(), append(tokens=rows // per + 1, **q)) == rng
    assert status(L.avsg_kv_read, cache(), rows + 1, 4096, 4096, 4096, 576) == rng
    many = cache(batch=2 ** 19, pages=2 ** 19, pages_per_request=1)
    assert status(L.avsg_attend, many, attention(heads=4096, topk=0), None, 0) == rng
    assert status(L.avsg_mx4_quantize, 4096, 0, 2 ** 30, 32, 32, 4096, 4096) == rng
    assert status(L.avsg_mx4_quantize, 4096, 1, 2 ** 20, 2 ** 15, 2 ** 15, 4096, 4096) == rng
    x = L.AvsgMx4(4096, 4096, 16, 16, 1, 1)
    assert status(L.avsg_mx4_dequantize, x, 2 ** 30, 32, 4096, 0, 32) == rng
    assert status(L.avsg_mx4_matmul, x, x, 1, 2 ** 19, 2 ** 19, 32, 4096, 0, 2 ** 19, 0) == rng
    assert status(L.avsg_mx4_matmul, x, x, 1, 129, 2 ** 30 - 1, 32, 4096, 0, 2 ** 30, 0) == rng


@pytest.mark.gpu
def test_cache_keeps_nothing_of_past_calls():
    """Contexts that grow by a position per step, as a decode over whole contexts has them."""
    from test_latent import SCALE, check_attend, gen, normal, pool_of
    g = gen(31)
    cache = L.LatentCache(pool_of(g, 1, 400, True), 1, 1)
    q = normal(g, 1, 1, 16, 576)

    def held():
        return sum(len(x) for x in vars(cache).values() if isinstance(x, (dict, list, set, tuple)))

    cache.attend(q, longest=300, scale=SCALE)
    before = held()
    for longest in (301, 302, 40, 303, 40, 399, 400, 1):
        out, lse = cache.attend(q, longest=longest, scale=SCALE)
        check_attend(cache, q, out, lse, longest=longest)
    assert held() == before


@pytest.mark.gpu
def test_gradients_are_not_lost_silently():
    """Tensors that require a gradient are refused where gradients are enabled, as torch refuses them for `out`."""
    from test_latent import angles_of, gen, normal, pool_of
    g = gen(32)
    cache = L.LatentCache(pool_of(g, 1, 64, True), 1, 1)
    q, latent, rope, turn = normal(g, 1, 1, 16, 576), normal(g, 1, 512), normal(g, 1, 64), normal(g, 1, 2, 64)
    at, angles, w = torch.zeros(1, dtype=torch.int64, device="cuda"), angles_of(64), normal(g, 32, 64)
    out, plain = torch.empty(1, 1, 16, 512, dtype=torch.bfloat16, device="cuda"), torch.randn(8, 64, device="cuda")
    lse, rows = torch.empty(1, 1, 16, device="cuda"), torch.empty(1, 576, dtype=torch.bfloat16, device="cuda")
    product = torch.empty(32, 32, dtype=torch.bfloat16, device="cuda")

    def calls():
        return [(q, lambda: cache.attend(q, scale=1.0)), (out, lambda: cache.attend(q, scale=1.0, out=out)),
                (lse, lambda: cache.attend(q, scale=1.0, lse=lse)), (rows, lambda: cache.read(at.int(), at, out=rows))] + [
            (x, lambda: cache.append(latent, rope, at.int(), at, angles, q_rope=turn, q_out=turn[:, :]))
            for x in (latent, rope, angles, turn)] + [
            (w, lambda: L.mx4_quantize(w)), (plain, lambda: L.mx4_quantize(plain)),
            (product, lambda: L.mx4_matmul(L.mx4_quantize(w), L.mx4_quantize(w), out=product))]

    for i, (x, call) in enumerate(calls()):
        call()
        x.requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            call()
            pytest.fail(f"call {i} lost a gradient")
        with torch.no_grad():
            call()
        x.requires_grad_(False)
        call()


def test_workspace_enough_for_any_call():
    """A smaller call may need more workspace than a larger one; there is a size that is enough for all."""
    rng, needs = random.Random(5), {}
    sizes = [(batch, n_q, heads, k) for batch in (1, 4, 16, 32, 48, 64) for n_q in (1, 2, 4) for heads in (1, 16, 17, 64, 128, 4096)
             for k in (1, 64, 65, 128, 700, 2048, 4096, 131072, MOST)]
    sizes += [(rng.randint(1, 300), rng.randint(1, 4), rng.randint(1, 300), int(2 ** rng.uniform(0, 24))) for _ in range(5000)]
    for s in sizes:
        needs[s] = L.avsg_attend_workspace_bytes(*s)
    assert any(needs[batch, 2, 128, 2048] > needs[64, 2, 128, 2048] for batch in (1, 4, 16, 32, 48))
    assert 0.9 * L.AVSG_ATTEND_WORKSPACE_MOST < max(needs.values()) <= L.AVSG_ATTEND_WORKSPACE_MOST


def test_workspaces_are_checked():
    """A long context of one request is shared by several workgroups, so a workspace is asked for, and one that is
    missing, too small or misaligned is refused."""
    from test_latent_abi import attention, cache, status
    need = L.avsg_attend_workspace_bytes(1, 1, 16, 100000)
    assert need > 0
    big = cache(batch=1, pages=2000, pages_per_request=2000)
    for at, size in ((None, need), (None, 0), (4096, need - 1), (4097, need), (4096 + 128, need)):
        assert status(L.avsg_attend, big, attention(topk=100000), at, size) == A.AVSG_E_INVAL
