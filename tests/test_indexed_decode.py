"""The example's decode step with its own indexer: every step selects what the plain form selects from the keys
in the cache, and attends over exactly these rows."""
import os
import sys

import pytest
import torch

import select_reference as R

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
def test_steps_with_an_indexer():
    import latent_decode as D
    batch, n_q, context, topk = 3, 2, 1024, 128
    layer = D.Layer(batch, n_q, 16, 512, topk, 512, context, index_heads=20)
    g = layer.random
    for r in range(batch):
        layer.prefill(r, torch.randn(300 + r, 512, generator=g, device="cuda", dtype=torch.bfloat16))
    verified = torch.full((batch,), 300, dtype=torch.int64, device="cuda")
    seen = []
    select = layer.keys.select
    layer.keys.select = lambda q, w, **kw: seen.append((q, w, kw)) or select(q, w, **kw)
    for _ in range(4):
        verified = verified + 1
        x = torch.randn(batch, n_q, 512, generator=g, device="cuda", dtype=torch.bfloat16)
        selected = layer.index(x, verified)
        q, w, kw = seen[-1]
        want = R.select(q, w, layer.keys.pool, None, kw["lens"].cpu(), topk=topk, recent=1)
        assert torch.equal(selected.cpu(), want[0])
        out = layer.step(x, verified, selected)
        assert torch.isfinite(out).all() and out.any()
        lens = kw["lens"]
        assert (selected == (lens - 1)[..., None]).any(-1).all()       # a token's own row
        again, lse = layer.host.attend(layer.query, rows=selected, index=selected, lens=lens, scale=layer.scale)
        assert torch.equal(layer.attended, again) and torch.equal(layer.lse, lse)
    layer.close()
