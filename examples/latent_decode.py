#!/usr/bin/env python3
"""Decode steps of one sparse-attention layer whose cache rows live in pinned
host memory in 4-bit form, on one GPU:

    tokens --quantise--> queries, latent and rope parts   (products of 4-bit matrices)
    append      the new rows to the host's rows, positions rotated in
    step        bring the selected rows that are missing into the device's slots
    attend      all heads over the slots, 4-bit rows read as they are
    outputs --quantise--> per-head values, output projection

Weights are random.  The selection is that of an indexer over 8-bit keys on the device, whose
projections are products of 8-bit matrices (--index-heads), or a stand-in for one (recent rows
and a slowly changing random set).  With draft tokens (n_q > 1) the verified length
goes to the step, which drops the drafts' rows when it is done.

    python examples/latent_decode.py [--batch 16] [--heads 64] [--steps 32] [--index-heads 64]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_37538_amd import avsg as A  # noqa: E402
from paper_2609_37538_amd import fp8 as F  # noqa: E402
from paper_2609_37538_amd import latent as L  # noqa: E402
from paper_2609_37538_amd import selection as S  # noqa: E402

NOPE, ROPE, LATENT, VALUE = 128, L.AVSG_ROPE_DIM, L.AVSG_LATENT_DIM, 128


class Layer:
    """Weights, the host's rows and the slots of one layer."""

    def __init__(self, batch, n_q, heads, hidden, topk, slots, context, seed=0, device="cuda", index_heads=0):
        self.batch, self.n_q, self.heads, self.topk, self.context = batch, n_q, heads, topk, context
        self.device = torch.device(device, torch.cuda.current_device())
        self.random = g = torch.Generator(self.device).manual_seed(seed)

        def weight(*shape):
            w = torch.randn(*shape, generator=g, device=self.device) * shape[-1] ** -0.5
            return L.mx4_quantize(w.to(torch.bfloat16))

        self.w_query = weight(heads * (NOPE + ROPE), hidden)
        self.w_row = weight(LATENT + ROPE, hidden)
        self.w_key = weight(heads, LATENT, NOPE)        # queries into the latent space, head by head
        self.w_value = weight(heads, VALUE, LATENT)
        self.w_out = weight(hidden, heads * VALUE)
        place = torch.arange(context, device=self.device)[:, None] * 10000.0 ** (-torch.arange(ROPE // 2, device=self.device) / (ROPE // 2))
        self.angles = torch.stack((place.cos(), place.sin()), -1).float().contiguous()

        row = L.avsg_row_bytes(L.AVSG_ROWS_MX4)
        self.region = A.HostRegion(batch * context * row)
        self.host = L.LatentCache(None, batch, L.AVSG_ROWS_MX4, base=self.region.ptr, pages=batch, page_rows=context,
                                  device=self.device)
        cfg = A.make_config(batch, topk, n_q, slots, row_bytes=(row,), gather_mode=A.AVSG_GATHER_RESIDENT)
        self.op = A.Operator(cfg, [self.region.ptr + r * context * row for r in range(batch)], [context] * batch)
        self.slots = L.LatentCache.of_slots(self.op)
        self.request = torch.arange(batch, dtype=torch.int32, device=self.device).repeat_interleave(n_q)
        self.scale = (NOPE + ROPE) ** -0.5
        self.index_heads = index_heads
        if index_heads:
            def weight8(*shape):
                w = torch.randn(*shape, generator=g, device=self.device) * shape[-1] ** -0.5
                return F.fp8_quantize(w.to(torch.bfloat16), rows=F.AVSG_FP8_BLOCK)

            self.w_index_query = weight8(index_heads * S.AVSG_KEY_DIM, hidden)
            self.w_index_key = weight8(S.AVSG_KEY_DIM, hidden)
            self.w_index_weight = weight8(index_heads, hidden)
            self.keys = S.KeyCache(torch.zeros(batch, context, S.AVSG_KEY_ROW_BYTES, dtype=torch.uint8, device=self.device), batch)

    def index(self, hidden_states, verified):
        """Keys of hidden_states [batch][n_q][hidden] into the key cache, and the topk positions that each token selects."""
        batch, n_q, hidden = hidden_states.shape
        tokens, heads = batch * n_q, self.index_heads
        position = (verified[:, None] - 1 + torch.arange(n_q, device=self.device)).reshape(-1)
        x = F.fp8_quantize(hidden_states.reshape(tokens, hidden))
        query = F.fp8_matmul(x, self.w_index_query).view(tokens, heads, S.AVSG_KEY_DIM)
        weights = F.fp8_matmul(x, self.w_index_weight, dtype=torch.float32)
        codes = torch.empty(tokens, heads, S.AVSG_KEY_DIM, dtype=torch.int8, device=self.device)
        scaled = torch.empty(tokens, heads, device=self.device)
        self.keys.append(F.fp8_matmul(x, self.w_index_key), self.request, position, self.angles, q=query, weights=weights,
                         q_out=codes, weights_out=scaled)
        selected, _ = self.keys.select(codes.view(batch, n_q, heads, -1), scaled.view(batch, n_q, heads), topk=self.topk,
                                       lens=(position + 1).view(batch, n_q), recent=1)
        return selected

    def prefill(self, request, hidden_states):
        """Rows of one request's hidden_states [length][hidden] into the host's rows from position 0."""
        length = len(hidden_states)
        rows = L.mx4_matmul(L.mx4_quantize(hidden_states), self.w_row)
        requests = torch.full((length,), request, dtype=torch.int32, device=self.device)
        places = torch.arange(length, device=self.device)
        self.host.append(rows[:, :LATENT], rows[:, LATENT:], requests, places, self.angles)
        if self.index_heads:
            self.keys.append(F.fp8_matmul(F.fp8_quantize(hidden_states), self.w_index_key), requests, places, self.angles)

    def step(self, hidden_states, verified, selected):
        """Outputs [batch][n_q][hidden] of hidden_states [batch][n_q][hidden], whose tokens stand at
        positions verified - 1 ..; selected: int32 [batch][n_q][topk] positions to attend over."""
        batch, n_q, hidden = hidden_states.shape
        tokens, heads = batch * n_q, self.heads
        x = L.mx4_quantize(hidden_states.reshape(tokens, hidden))
        query = L.mx4_matmul(x, self.w_query).view(tokens, heads, NOPE + ROPE)
        row = L.mx4_matmul(x, self.w_row)
        position = (verified[:, None] - 1 + torch.arange(n_q, device=self.device)).reshape(-1)

        q = torch.empty(tokens, heads, L.KEY_DIM, dtype=torch.bfloat16, device=self.device)
        nope = L.mx4_quantize(query[..., :NOPE].contiguous()).transpose(0, 1)
        L.mx4_matmul(nope, self.w_key, out=q[..., :LATENT].transpose(0, 1))
        self.host.append(row[:, :LATENT], row[:, LATENT:], self.request, position, self.angles,
                         q_rope=query[..., NOPE:], q_out=q[..., LATENT:])

        slots, _ = self.op.step(selected, verified)
        lens = (position + 1).view(batch, n_q)
        self.query = q.view(batch, n_q, heads, L.KEY_DIM)
        self.attended, self.lse = self.slots.attend(self.query, rows=slots, index=selected, lens=lens, scale=self.scale)

        latent = L.mx4_quantize(self.attended.view(tokens, heads, LATENT)).transpose(0, 1)
        value = torch.empty(tokens, heads, VALUE, dtype=torch.bfloat16, device=self.device)
        L.mx4_matmul(latent, self.w_value, out=value.transpose(0, 1))
        return L.mx4_matmul(L.mx4_quantize(value.view(tokens, heads * VALUE)), self.w_out).view(batch, n_q, hidden)

    def select(self, verified, taste):
        """Distinct positions that each token may see: its last ones and, of the others, those that
        `taste` [batch][context] ranks first (a token of a context shorter than topk takes
        positions past its own, which the attention masks)."""
        seen = verified[:, None] + torch.arange(self.n_q, device=self.device)          # lengths
        at = torch.arange(self.context, device=self.device)
        rank = taste[:, None].expand(-1, self.n_q, -1).clone()
        rank[(at >= seen[..., None] - self.topk // 8) & (at < seen[..., None])] += 2.0
        rank[at.expand_as(rank) >= seen[..., None]] -= 4.0
        return rank.topk(self.topk, dim=-1).indices.to(torch.int32)

    def close(self):
        torch.cuda.synchronize()
        self.op.close()
        self.region.free()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("batch", 16), ("n-q", 2), ("heads", 64), ("hidden", 2048), ("topk", 2048), ("slots", 8192),
                        ("context", 16384), ("prompt", 8192), ("steps", 32), ("index-heads", 0)):
        ap.add_argument(f"--{name}", type=int, default=value)
    args = ap.parse_args()
    layer = Layer(args.batch, args.n_q, args.heads, args.hidden, args.topk, args.slots, args.context, index_heads=args.index_heads)
    g = layer.random
    for request in range(args.batch):
        layer.prefill(request, torch.randn(args.prompt, args.hidden, generator=g, device=layer.device, dtype=torch.bfloat16))
    verified = torch.full((args.batch,), args.prompt, dtype=torch.int64, device=layer.device)
    taste = torch.rand(args.batch, args.context, generator=g, device=layer.device)
    times = []
    for step in range(args.steps):
        x = torch.randn(args.batch, args.n_q, args.hidden, generator=g, device=layer.device, dtype=torch.bfloat16)
        accepted = torch.randint(0, args.n_q if step else 1, (args.batch,), generator=g, device=layer.device)
        verified = verified + 1 + accepted     # the last step's drafts that were right, and a new token
        fresh = torch.rand(taste.shape, generator=g, device=layer.device)
        taste = torch.where(torch.rand(taste.shape, generator=g, device=layer.device) < 0.9, taste, fresh)
        selected = None if args.index_heads else layer.select(verified, taste)
        torch.cuda.synchronize()
        start = time.perf_counter()
        layer.step(x, verified, layer.index(x, verified) if args.index_heads else selected)
        torch.cuda.synchronize()
        times.append((time.perf_counter() - start) * 1e6)
    stats = layer.op.stats()
    warm = sorted(times[len(times) // 2:])
    print(f"{args.batch} requests x {args.n_q} tokens, {args.heads} heads, {args.topk} of {args.context} rows of "
          f"{L.avsg_row_bytes(L.AVSG_ROWS_MX4)} bytes: {warm[len(warm) // 2]:.0f} us per layer and step, "
          f"first step {times[0]:.0f} us, {stats['hits'] / stats['lookups']:.3f} of the lookups hits")
    layer.close()


if __name__ == "__main__":
    main()
