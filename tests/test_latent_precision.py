"""Attention over latent rows against plain forms in 64 bits, to the accuracy
that the output's own rounding leaves."""
import pytest
import torch

import latent_reference as R
from test_latent import _gpu, close, gen, normal, pool_of, row_bytes  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("batch,heads,k", [(1, 8, 40), (2, 16, 300), (3, 128, 100), (8, 128, 100), (130, 17, 40), (66, 64, 700),
                                           (24, 8, 2048), (128, 16, 1720), (33, 40, 1000)])
def test_attend_weights_keep_their_bits(batch, heads, k, mx4):
    """A result is off by its own rounding to bfloat16 and little else: weights keep 12 bits at least.
    Head h's query is 1 in one rotated column, so scores are that column's values, exactly."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch + heads + k)
    cache = L.LatentCache(pool_of(g, batch, k, mx4), batch, int(mx4))
    q = torch.zeros(batch, 1, heads, 576, dtype=torch.bfloat16, device="cuda")
    q[..., torch.arange(heads), 512 + torch.arange(heads) % 64] = 1.0
    out, lse = cache.attend(q, scale=1.5)
    for b in sorted({0, batch // 2, batch - 1}):
        keys = R.row_values(cache.pool[b], mx4)
        s = q[b, 0].cpu().double() @ keys.T * 1.5
        p, v = torch.softmax(s, -1), keys[:, :512]
        want, size = p @ v, p @ v.abs()
        # every weight to 2^-12 of itself, or, where it lies far below the largest, to 2^-19 of that;
        # and float32 sums, exponentials and their arguments
        weights = 2.0 ** -12 * size + 2.0 ** -19 * p.amax(-1, keepdim=True) * v.abs().sum(0)
        f32 = (k + 64) * R.F32 + 4 * R.F32 * s.abs().amax(-1, keepdim=True)
        close(out[b, 0], want, R.HALF_ULP * want.abs() + weights + f32 * size, f"request {b}")
        close(lse[b, 0], torch.logsumexp(s, -1), f32[:, 0] + 4 * R.F32 * torch.logsumexp(s, -1).abs(), f"request {b}: lse")


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("order", ["flat", "low first", "rising"])
@pytest.mark.parametrize("batch,heads,k", [(1, 8, 40), (2, 16, 300), (1, 8, 3000), (3, 128, 100), (8, 128, 100), (130, 17, 40),
                                           (66, 64, 700), (24, 8, 2048), (128, 16, 1720), (33, 40, 1000)])
def test_attend_largest_values(batch, heads, k, order, mx4):
    """Values at the end of the row format's range, whose plain sum over the rows is infinite: a mean of them is
    not.  Scores are equal, or the first 150 rows' lie a little less than 8 powers of two below the
    others', or they grow from row to row by 80 powers of two in all."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch + heads + k)
    latent, rope = normal(g, k, 512), torch.zeros(k, 64, dtype=torch.bfloat16, device="cuda")
    most = 6 * 2.0 ** 125 if mx4 else torch.finfo(torch.bfloat16).max
    latent[:, 32:64], latent[:, 64:96] = most, -most
    at = torch.arange(k, device="cuda")
    rope[:, 0] = {"flat": at * 0.0, "low first": (at >= 150) * 7.75, "rising": at * (80 / k)}[order].to(torch.bfloat16)
    rope[:, 1] = torch.randn(k, generator=g, device="cuda").to(torch.bfloat16)
    pool = row_bytes(latent, rope, mx4).expand(batch, -1, -1).contiguous()
    cache = L.LatentCache(pool, batch, int(mx4))
    q = torch.zeros(batch, 1, heads, 576, dtype=torch.bfloat16, device="cuda")
    q[..., 512] = 1.0
    q[..., 1::2, 513] = 2.0 ** -6      # every second head's scores differ a little
    ln2 = 0.6931471805599453
    out, lse = cache.attend(q, scale=ln2)
    for b in sorted({0, batch // 2, batch - 1}):
        keys = R.row_values(pool[b], mx4)
        s = q[b, 0].cpu().double() @ keys.T * ln2
        p, v = torch.softmax(s, -1), keys[:, :512]
        want, size = p @ v, p @ v.abs()
        weights = 2.0 ** -12 * size + 2.0 ** -19 * p.amax(-1, keepdim=True) * v.abs().sum(0)
        f32 = (k + 64) * R.F32 + 4 * R.F32 * s.abs().amax(-1, keepdim=True)
        close(out[b, 0], want, R.HALF_ULP * want.abs() + weights + f32 * size, f"request {b}")
        close(lse[b, 0], torch.logsumexp(s, -1), f32[:, 0] + 4 * R.F32 * torch.logsumexp(s, -1).abs(), f"request {b}: lse")


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("batch,heads,k", [(1, 8, 2000), (3, 128, 100), (130, 64, 2000), (24, 8, 2048)])
def test_attend_small_values(batch, heads, k, mx4):
    """Values near 2^-110, whose products with the weights are less than the least normal float32."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch + heads + k)
    latent = (torch.randint(2, 7, (k, 512), generator=g, device="cuda") * 2.0 ** -111).to(torch.bfloat16)
    pool = row_bytes(latent, normal(g, k, 64), mx4).expand(batch, -1, -1).contiguous()
    cache = L.LatentCache(pool, batch, int(mx4))
    q = torch.zeros(batch, 1, heads, 576, dtype=torch.bfloat16, device="cuda")
    q[..., 512] = 1.0
    out, lse = cache.attend(q, scale=1.0)
    for b in sorted({0, batch // 2, batch - 1}):
        keys = R.row_values(pool[b], mx4)
        s = q[b, 0].cpu().double() @ keys.T
        p, v = torch.softmax(s, -1), keys[:, :512]
        want, size = p @ v, p @ v.abs()
        weights = 2.0 ** -12 * size + 2.0 ** -19 * p.amax(-1, keepdim=True) * v.abs().sum(0)
        f32 = (k + 64) * R.F32 + 4 * R.F32 * s.abs().amax(-1, keepdim=True)
        # two products and additions per row, off by half of 2^-149 each, relative to weights of 2^-19 at least
        least = 4 * k * 2.0 ** -150 * 2.0 ** 19
        close(out[b, 0], want, R.HALF_ULP * want.abs() + weights + f32 * size + least, f"request {b}")
        assert (out[b, 0] != 0).all()
