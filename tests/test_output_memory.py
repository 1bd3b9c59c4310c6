"""Outputs that a program brings: vectors may lie anywhere and between each other, but several entries in one
place of memory, whose value would be left to chance, are refused."""
import itertools

import pytest
import torch

from paper_2609_37538_amd import avsg as A
from paper_2609_37538_amd import fp8 as F
from paper_2609_37538_amd import latent as L
from paper_2609_37538_amd import selection as S


def test_vectors_that_share_memory():
    """Against all their entries, for every small count, distance and length."""
    for n0, n1, run in itertools.product(range(5), range(5), (0, 1, 2, 3)):
        for s0, s1 in itertools.product(range(14), repeat=2):
            at = [i * s0 + j * s1 + e for i in range(n0) for j in range(n1) for e in range(run)]
            assert L._apart(n0, s0, n1, s1, run) == (len(set(at)) == len(at)), (n0, s0, n1, s1, run)


def test_many_vectors_take_no_time():
    assert L._apart(1 << 19, 64 * 512, 64, 512, 512) and L._apart(64, 512, 1 << 19, 64 * 512, 512)
    assert not L._apart(1 << 19, 0, 64, 512, 512) and not L._apart(1 << 19, 511, 1, 0, 512) and L._apart(1 << 19, 0, 0, 0, 512)
    assert L._apart(1 << 19, 1 << 40, 1, 0, 512) and not L._apart(2, 1024, 3, 512, 512)


def shared(*shape, dtype=torch.bfloat16):
    """Tensors whose first, or second, entries are one place, and whose vectors overlap by a half."""
    vectors = shape[:-1] if dtype != torch.float32 else shape[:1]
    row = torch.zeros(*shape, dtype=dtype, device="cuda")
    for i in range(len(vectors)):
        if shape[i] > 1:
            yield row.narrow(i, 0, 1).expand(*shape)
    strides = list(row.stride())
    near = [(st // 2 if i < len(vectors) else st) for i, st in enumerate(strides)]
    yield row.as_strided(shape, near)


@pytest.mark.gpu
def test_shared_outputs_are_refused():
    dev = "cuda"
    bf16 = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    pool = torch.zeros(4, 64, 132, dtype=torch.uint8, device=dev)
    keys = S.KeyCache(pool, 2)
    request, position = torch.zeros(3, dtype=torch.int32, device=dev), torch.arange(3, device=dev)
    codes, weights = torch.zeros(3, 8, 128, dtype=torch.int8, device=dev), torch.zeros(3, 8, device=dev)
    append = lambda **kw: keys.append(bf16(3, 128), request, position, q=bf16(3, 8, 128), **kw)  # noqa: E731
    append(q_out=codes, weights_out=weights)
    for x in shared(3, 8, 128, dtype=torch.int8):
        with pytest.raises(ValueError, match="share"):
            append(q_out=x, weights_out=weights)
    for x in shared(3, 8, dtype=torch.float32):
        with pytest.raises(ValueError, match="share"):
            append(q_out=codes, weights_out=x)
    for x in shared(3, 128):
        with pytest.raises(ValueError, match="share"):
            keys.read(request, position, out=x)

    rows = torch.zeros(4, 64, 1152, dtype=torch.uint8, device=dev)
    cache, angles = L.LatentCache(rows, 2, L.AVSG_ROWS_BF16), torch.zeros(8, 32, 2, device=dev)
    for x in shared(3, 8, 64):
        with pytest.raises(ValueError, match="share"):
            cache.append(bf16(3, 512), bf16(3, 64), request, position, angles, q_rope=bf16(3, 8, 64), q_out=x)
    for x in shared(3, 576):
        with pytest.raises(ValueError, match="share"):
            cache.read(request, position, out=x)
    for x in (bf16(2, 1, 1, 512).expand(2, 1, 16, 512), bf16(1, 1, 16, 512).expand(2, 1, 16, 512)):
        with pytest.raises(ValueError, match="share"):
            cache.attend(bf16(2, 1, 16, 576), scale=0.1, out=x)

    for quantize, matmul, rows_of in ((L.mx4_quantize, L.mx4_matmul, {}), (F.fp8_quantize, F.fp8_matmul, dict(rows=128))):
        a, b = quantize(bf16(2, 5, 128)), quantize(bf16(2, 16, 128), **rows_of)
        for dtype in (torch.bfloat16, torch.float32):
            x = torch.zeros(2, 5, 16, dtype=dtype, device=dev)
            for out in (x[:1].expand(2, 5, 16), x[:, :1].expand(2, 5, 16), x.as_strided((2, 5, 16), (80, 8, 1))):
                with pytest.raises(ValueError, match="share"):
                    matmul(a, b, out=out)


@pytest.mark.gpu
def test_outputs_between_each_other():
    """Rows that interleave, as heads do, and whose distances nest in no order."""
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(2, 5, 128, generator=g).cuda(), torch.randn(2, 16, 128, generator=g).cuda()
    for quantize, matmul, rows in ((L.mx4_quantize, L.mx4_matmul, {}), (F.fp8_quantize, F.fp8_matmul, dict(rows=128))):
        a, b = quantize(x), quantize(w, **rows)
        want = matmul(a, b)
        for strides in ((16, 32, 1), (16, 48, 1), (80, 16, 1), (60, 40, 1)):
            room = torch.full((400,), 7.0, dtype=torch.bfloat16, device="cuda")
            out = room.as_strided((2, 5, 16), strides)
            assert matmul(a, b, out=out) is out and torch.equal(out, want)
            assert int((room == 7).sum()) >= 400 - out.numel()
    # (with the last of these, rows of 16 from 0, 40, .., 160 and from 60, 100, .., 220)
    key = torch.randn(4, 128, generator=g).bfloat16().cuda()
    q = torch.randn(4, 6, 128, generator=g).bfloat16().cuda()
    cache = S.KeyCache(torch.zeros(1, 8, 132, dtype=torch.uint8, device="cuda"), 1)
    request, position = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.arange(4, device="cuda")
    got = []
    for codes, weights in ((torch.zeros(4, 6, 128, dtype=torch.int8, device="cuda"), torch.zeros(4, 6, device="cuda")),
                           (torch.zeros(6, 4, 144, dtype=torch.int8, device="cuda")[..., :128].transpose(0, 1),
                            torch.zeros(4, 9, device="cuda")[:, 2:8])):
        cache.append(key, request, position, q=q, q_out=codes, weights_out=weights)
        got.append((codes, weights))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and got[0][0].any()
