"""Attention over latent rows against plain forms in 64 bits, to the accuracy
that the output's own rounding leaves."""
import pytest
import torch

import latent_reference as R
from test_latent import _gpu, close, gen, normal, pool_of  # noqa: F401

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
