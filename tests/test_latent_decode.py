"""The latent-cache operators with the sparse-gather step, as a decode step of the example runs them."""
import importlib.util
import os

import pytest
import torch

import test_latent as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "latent_decode.py")
    spec = importlib.util.spec_from_file_location("latent_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("batch,n_q,heads,prompt", [(3, 2, 20, 100), (1, 1, 16, 300), (2, 3, 64, 250)])
def test_decode(example, batch, n_q, heads, prompt):
    """Attention over the slots is attention over the host's rows, also of tokens that the same
    step appended, of drafts that were replaced, and of contexts shorter than the selection."""
    from paper_2609_37538_amd import latent as L
    hidden, topk, context = 256, 128, 400
    layer = example.Layer(batch, n_q, heads, hidden, topk, 512, context)
    g = layer.random
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    for request in range(batch):
        layer.prefill(request, normal(prompt, hidden))
    verified = torch.full((batch,), prompt, dtype=torch.int64, device="cuda")
    taste = torch.rand(batch, context, generator=g, device="cuda")
    for step in range(12):
        verified = verified + 1 + torch.randint(0, n_q if step else 1, (batch,), generator=g, device="cuda")
        taste = torch.where(torch.rand(taste.shape, generator=g, device="cuda") < 0.8, taste,
                            torch.rand(taste.shape, generator=g, device="cuda"))
        selected = layer.select(verified, taste)
        y = layer.step(normal(batch, n_q, hidden), verified, selected)
        torch.cuda.synchronize()
        lens = verified[:, None] + torch.arange(n_q, device="cuda")
        out, lse = layer.host.attend(layer.query, rows=selected, index=selected, lens=lens, scale=layer.scale)
        assert torch.equal(out, layer.attended) and torch.equal(lse, layer.lse), step
        assert torch.isfinite(y).all() and y.abs().max() > 0
        if step in (0, 11):
            seen = torch.from_numpy(layer.region.view().copy()).view(batch, context, -1)     # the rows as the host sees them
            copy = L.LatentCache(seen.cuda(), batch, L.AVSG_ROWS_MX4)
            T.check_attend(copy, layer.query, layer.attended, layer.lse, selected, selected, lens, scale=layer.scale)
    stats = layer.op.stats()
    assert stats["hits"] > 0 and stats["misses"] > 0, stats
    layer.close()
