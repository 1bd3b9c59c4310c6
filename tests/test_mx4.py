"""4-bit microscaled form on the GPU: quantisation, its inverse, and products."""
import math

import pytest
import torch

import latent_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2609_37538_amd import latent as L
    L.load()


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_bfloat16(dtype):
    """Every bfloat16 value, in blocks with others near it and in blocks with a much larger one."""
    from paper_2609_37538_amd import latent as L
    bits = torch.arange(65536, dtype=torch.int32)
    x = (bits << 16).view(torch.float32)
    mixed = x[torch.randperm(65536, generator=torch.Generator().manual_seed(1))]
    both = torch.stack((x, mixed)).reshape(-1, 256)
    m = L.mx4_quantize(both.to(dtype).cuda())
    codes, scales = R.quantize(both)
    assert torch.equal(m.scales.cpu(), scales)
    finite = (scales != 255).repeat_interleave(16, -1)     # a NaN scale says it all
    assert torch.equal(m.codes.cpu()[finite], codes[finite])
    for out in (torch.bfloat16, torch.float32):
        assert same(L.mx4_dequantize(m, out).cpu().double(), R.values(codes, scales))


def test_ties_and_edges():
    """Midpoints between codes go to the even code, for every block exponent; float32 values next to them do not."""
    from paper_2609_37538_amd import latent as L
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    e = torch.arange(-120, 121, 8).double()
    near = torch.cat((mid, -mid, mid * (1 + 2.0 ** -23), mid * (1 - 2.0 ** -24), torch.tensor([4.0, 6.0, 6.9999995, 0.0])))
    x = (near.double()[None] * torch.exp2(e)[:, None]).float()
    assert x.shape[1] == 32
    m = L.mx4_quantize(x.cuda())
    codes, scales = R.quantize(x)
    assert torch.equal(m.codes.cpu(), codes) and torch.equal(m.scales.cpu(), scales)


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (33, 1184), (257, 512), (1000, 96), (5, 8192)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_shapes(rows, cols, dtype):
    from paper_2609_37538_amd import latent as L
    wide = torch.randn(rows, cols + 40, generator=gen(rows), device="cuda").to(dtype)
    x = wide[:, 8:8 + cols]
    m = L.mx4_quantize(x)
    codes, scales = R.quantize(x.float().cpu())
    assert torch.equal(m.codes.cpu(), codes) and torch.equal(m.scales.cpu(), scales)
    three = L.mx4_quantize(x.unsqueeze(1).contiguous())
    assert three.shape == (rows, 1, cols) and torch.equal(three.codes[:, 0], m.codes)
    assert same(L.mx4_dequantize(m).cpu().double(), R.values(codes, scales))


def product(a, b, out, f32):
    """out against the float64 product of the values of a and b."""
    av, bv = R.values(a.codes, a.scales), R.values(b.codes, b.scales)
    want, size = av @ bv.transpose(-1, -2), av.abs() @ bv.abs().transpose(-1, -2)
    # products are exact; additions in float32 in some order, then one rounding
    bound = (av.shape[-1] + 8) * R.F32 * size + (0 if f32 else R.HALF_ULP) * want.abs()
    over = (out.cpu().double() - want).abs() - bound
    assert torch.isfinite(out).all() and (over.numel() == 0 or over.max() <= 0), over.max()


@pytest.mark.parametrize("m,n,k", [(1, 1, 32), (1, 16, 64), (3, 5, 96), (16, 16, 128), (17, 33, 160), (1, 1000, 1184),
                                   (2, 4096, 512), (31, 70, 2048), (64, 64, 256), (100, 512, 128), (128, 128, 32),
                                   (129, 257, 544), (300, 130, 4096), (256, 256, 256), (513, 770, 1024),
                                   (1024, 512, 512), (700, 1536, 4128)])
@pytest.mark.parametrize("f32", [False, True])
def test_product(m, n, k, f32):
    from paper_2609_37538_amd import latent as L
    g = gen(m + n + k)
    a = L.mx4_quantize(torch.randn(m, k, generator=g, device="cuda"))
    b = L.mx4_quantize(torch.randn(n, k, generator=g, device="cuda") * torch.exp2(torch.randint(-8, 9, (n, 1), generator=g, device="cuda").float()))
    room = torch.full((m + 2, n + 3), 5.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    out = L.mx4_matmul(a, b, out=room[1:m + 1, 1:n + 1])
    product(a, b, out, f32)
    out.fill_(5.0)
    assert (room == 5.0).all(), "written outside the output"
    assert torch.equal(L.mx4_matmul(a, b, dtype=room.dtype), L.mx4_matmul(a, b, dtype=room.dtype))


@pytest.mark.parametrize("batch,m,n,k", [(3, 1, 512, 128), (16, 4, 512, 128), (20, 37, 128, 512), (5, 130, 256, 192),
                                         (128, 128, 512, 128), (2, 300, 300, 1024)])
def test_product_of_heads(batch, m, n, k):
    """Heads that interleave in the rows of the activations and of the output, as projections of a
    decode step have them."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch)
    x = L.mx4_quantize(torch.randn(m, batch, k, generator=g, device="cuda")).transpose(0, 1)
    w = L.mx4_quantize(torch.randn(batch, n, k, generator=g, device="cuda"))
    room = torch.full((m, batch, n + 64), 3.0, dtype=torch.bfloat16, device="cuda")
    out = L.mx4_matmul(x, w, out=room[..., :n].transpose(0, 1))
    product(x, w, out, False)
    assert (room[..., n:] == 3.0).all()


@pytest.mark.parametrize("batch,m,n,k,f32", [(1, 2100, 1100, 1056, False), (1, 1100, 2100, 544, True), (20, 300, 300, 800, False),
                                             (1, 4200, 4100, 544, False), (1, 4097, 4096, 1120, True), (70, 300, 500, 576, False)])
def test_product_of_many_tiles(batch, m, n, k, f32):
    """Tiles through LDS, small and large: columns that end inside a step, rows and columns that end
    inside a tile, heads that interleave, an output whose rows are not aligned, and a NaN scale in the last block."""
    from paper_2609_37538_amd import latent as L
    g = gen(batch + m + k)
    x = L.mx4_quantize(torch.randn(m, batch, k, generator=g, device="cuda") * torch.exp2(torch.randint(-8, 9, (m, 1, 1), generator=g, device="cuda").float()))
    x, w = x.transpose(0, 1), L.mx4_quantize(torch.randn(batch, n, k, generator=g, device="cuda"))
    room = torch.full((m, batch, n + 3), 3.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    out = L.mx4_matmul(x, w, out=room[..., 1:n + 1].transpose(0, 1))
    for i in sorted({0, batch // 2, batch - 1}):
        product(L.Mx4(x.codes[i], x.scales[i]), L.Mx4(w.codes[i], w.scales[i]), out[i], f32)
    assert (room[..., 0] == 3.0).all() and (room[..., n + 1:] == 3.0).all()
    aligned = L.mx4_matmul(x, w, dtype=out.dtype)
    assert torch.equal(aligned, out)
    x.scales[batch - 1, m - 1, -1] = 255
    out = L.mx4_matmul(x, w, dtype=out.dtype)
    assert out[batch - 1, m - 1].isnan().all()
    out[batch - 1, m - 1] = aligned[batch - 1, m - 1]
    assert torch.equal(out, aligned)


def test_product_of_extreme_scales():
    """Block scales across the whole range, and a block that is NaN in one row."""
    from paper_2609_37538_amd import latent as L
    g = gen(3)
    a = L.mx4_quantize(torch.randn(40, 256, generator=g, device="cuda"))
    b = L.mx4_quantize(torch.randn(48, 256, generator=g, device="cuda"))
    a.scales.copy_(torch.randint(40, 120, a.scales.shape, generator=g, device="cuda").to(torch.uint8))
    b.scales.copy_(torch.randint(100, 200, b.scales.shape, generator=g, device="cuda").to(torch.uint8))
    product(a, b, L.mx4_matmul(a, b, dtype=torch.float32), True)
    clean = L.mx4_matmul(a, b)
    a.scales[7, 3] = 255
    out = L.mx4_matmul(a, b)
    assert out[7].isnan().all()
    keep = torch.arange(40, device="cuda") != 7
    assert torch.equal(out[keep], clean[keep])


def test_nothing():
    from paper_2609_37538_amd import latent as L
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    assert L.mx4_quantize(e(0, 64)).shape == (0, 64)
    assert L.mx4_dequantize(L.mx4_quantize(e(4, 0))).shape == (4, 0)
    assert L.mx4_matmul(L.mx4_quantize(e(0, 64)), L.mx4_quantize(e(5, 64).zero_())).shape == (0, 5)
    assert (L.mx4_matmul(L.mx4_quantize(e(3, 0)), L.mx4_quantize(e(5, 0))) == 0).all()


def test_graph_and_stream():
    """Captured, replayed on new inputs, with eager work between the replays."""
    from paper_2609_37538_amd import latent as L
    g = gen(4)
    x, w = torch.randn(40, 512, generator=g, device="cuda"), L.mx4_quantize(torch.randn(96, 512, generator=g, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = L.mx4_matmul(L.mx4_quantize(x), w)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, L.mx4_matmul(L.mx4_quantize(x), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = L.mx4_matmul(L.mx4_quantize(x), w)
    for _ in range(4):
        x.copy_(torch.randn(40, 512, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, L.mx4_matmul(L.mx4_quantize(x), w))


def test_refusals():
    from paper_2609_37538_amd import latent as L
    x = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    m = L.mx4_quantize(x)
    bad = [
        lambda: L.mx4_quantize(x.half()), lambda: L.mx4_quantize(x[:, :40]), lambda: L.mx4_quantize(x[0]),
        lambda: L.mx4_quantize(x.cpu()), lambda: L.mx4_quantize(torch.zeros(8, 65, dtype=torch.bfloat16, device="cuda")[:, 1:]),
        lambda: L.mx4_quantize(x.t().contiguous().t()[:, :32]),
        lambda: L.Mx4(m.codes, m.scales[:, :1]), lambda: L.Mx4(m.codes[:4], m.scales), lambda: L.Mx4(m.codes.cpu(), m.scales.cpu()),
        lambda: m.transpose(0, 1), lambda: L.mx4_dequantize(m, torch.half), lambda: L.mx4_dequantize(L.Mx4(m.codes[::2], m.scales[::2])),
        lambda: L.mx4_matmul(m, L.mx4_quantize(x[:, :32])), lambda: L.mx4_matmul(m, m, out=torch.zeros(8, 9, device="cuda")),
        lambda: L.mx4_matmul(m, m, out=torch.zeros(8, 8, device="cuda").t()), lambda: L.mx4_matmul(m, m, dtype=torch.half),
        lambda: L.mx4_matmul(m, L.mx4_quantize(x[None])),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"refusal {i} did not happen")
    assert not math.isnan(float(L.mx4_matmul(m, m).sum()))
