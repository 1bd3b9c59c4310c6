"""Scales that a program brings for a matrix in 8-bit floating point: the kernels step through a row's scales one
by one, so they have to lie next to each other; rows of scales may lie anywhere, or be one row for all."""
import pytest
import torch

from paper_2609_37538_amd import fp8 as F
from paper_2609_37538_amd import latent as L


def matrix(codes, scales, rows):
    """An Fp8 of tensors on the CPU, for its description of them (no kernel runs)."""
    L._torch()
    m = F.Fp8.__new__(F.Fp8)
    m.device, m.rows, m._shape = codes.device, rows, tuple(codes.shape)
    m._codes, m._scales, m._base, m._view = codes, scales, None, None
    return m


def codes(*shape):
    return torch.zeros(*shape, dtype=torch.uint8).view(torch.float8_e4m3fn)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("lead", [(), (3,)])
def test_scales_that_stand_for_several_blocks_are_refused(rows, lead):
    """One scale for all blocks of a row, or for all of a matrix: their addresses do not go on with the blocks."""
    r, k = 130, 400
    down = -(-r // rows)
    for base in (torch.ones(*lead, down, 1), torch.ones(()), torch.ones(*lead, 1, 1)):
        with pytest.raises(ValueError):
            matrix(codes(*lead, r, k), base.expand(*lead, down, 4), rows)._c()
    for other in (torch.ones(*lead, 4, down).transpose(-1, -2), torch.ones(*lead, down, 8)[..., ::2]):
        with pytest.raises(ValueError):
            matrix(codes(*lead, r, k), other, rows)._c()


@pytest.mark.parametrize("rows", [1, 128])
def test_rows_of_scales_lie_anywhere(rows):
    r, k = 300, 400
    down = -(-r // rows)
    wide = torch.ones(down, 9)
    c = matrix(codes(r, k), wide[:, 2:6], rows)._c()
    assert (c.d_scales, c.scale_stride) == (wide.data_ptr() + 8, 9)
    c = matrix(codes(r, k), torch.ones(1, 4).expand(down, 4), rows)._c()
    assert c.scale_stride == 0
    # one block across: what its stride is does not matter
    for one in (torch.ones(down, 1), torch.ones(down, 8)[:, ::8], torch.ones(()).expand(down, 1)):
        c = matrix(codes(r, 112), one, rows)._c()
        assert c.scale_stride == one.stride(0)


@pytest.mark.gpu
def test_expanded_scales_on_the_gpu():
    """One scale for a whole matrix is refused by a product and by the way back, and taken once it is laid out."""
    g = torch.Generator().manual_seed(4)
    byte = torch.randint(0, 120, (130, 400), generator=g).to(torch.uint8).cuda()
    a, one = byte.view(torch.float8_e4m3fn), torch.full((), 0.5, device="cuda")
    w = F.fp8_quantize(torch.eye(400, device="cuda"), rows=128)
    for call in (lambda m: F.fp8_matmul(m, w), F.fp8_dequantize):
        with pytest.raises(ValueError):
            call(F.Fp8(a, one.expand(130, 4)))
    same_rows = one.expand(4).contiguous().expand(130, 4)
    want = a.float() * 0.5
    assert torch.equal(F.fp8_dequantize(F.Fp8(a, same_rows), torch.float32), want)
    assert torch.equal(F.fp8_dequantize(F.Fp8(a, one.expand(130, 4).contiguous()), torch.float32), want)
