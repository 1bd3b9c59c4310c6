"""Every kernel of the product of 8-bit matrices, on sizes that the choice gives it now and that end off its tiles:
rows, columns, blocks of 128 columns, steps that two groups of waves share unevenly, batches, and strides too
long for 32-bit offsets."""
import ctypes

import pytest
import torch

from paper_2609_37538_amd import fp8 as F
from test_fp8 import BLOCK, activations, check

KERNELS = ("16 rows", "32 rows", "64 rows", "64, two groups", "128, two groups", "128", "256")
LONG = 2 ** 23      # bytes between rows that 32-bit offsets within 256 rows do not take


def path(batch, m, n, k, a_stride=None, b_stride=None):
    f = F.load().avsg_internal_fp8_plan
    f.restype, f.argtypes = ctypes.c_int32, [ctypes.c_int32] * 4 + [ctypes.c_int64] * 2
    return KERNELS[f(batch, m, n, k, a_stride or k, b_stride or k)]


# kernel, batch, rows, columns, inner size
CASES = [
    ("16 rows", 1, 1, 1, 16), ("16 rows", 1, 16, 1000, 1040), ("16 rows", 3, 7, 130, 272), ("16 rows", 128, 9, 129, 128),
    ("32 rows", 1, 17, 129, 400), ("32 rows", 2, 32, 300, 1184), ("32 rows", 30, 25, 500, 144),
    ("64, two groups", 1, 33, 65, 16), ("64, two groups", 1, 333, 1000, 272), ("64, two groups", 5, 70, 190, 400),
    ("64, two groups", 3, 17, 4096, 656),
    ("128, two groups", 1, 1000, 3000, 400), ("128, two groups", 1, 1030, 2050, 272), ("128, two groups", 1, 1025, 2040, 16),
    ("128, two groups", 6, 330, 1290, 144), ("128, two groups", 1, 700, 5000, 656), ("128, two groups", 1, 1000, 3008, 1424),
    ("128", 1, 2049, 2560, 400), ("128", 1, 2050, 2570, 16), ("128", 5, 1025, 1000, 144), ("128", 12, 300, 1800, 272), ("128", 1, 100, 70000, 128),
    ("256", 1, 2300, 4090, 400), ("256", 1, 2305, 4097, 144), ("256", 1, 3000, 4100, 16), ("256", 6, 1100, 1300, 272), ("256", 3, 1030, 3500, 128),
    ("256", 40, 200, 900, 272), ("256", 1, 129, 70000, 128), ("256", 1, 2310, 4090, 1424),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_kernel_of_a_case(case):
    assert path(*case[1:]) == case[0]


def test_kernel_of_long_strides():
    assert path(1, 300, 400, 256, LONG, 256) == path(1, 300, 400, 256, 256, LONG) == "64 rows"
    assert path(1, 16, 400, 256, LONG, 256) == "16 rows" and path(1, 17, 400, 256, 256, LONG) == "32 rows"
    assert path(1, 300, 400, 256, (2 ** 31 - 1 - 256) // 256) == "64, two groups"
    assert path(1, 300, 400, 256, 2 ** 63 - 16) == path(1, 300, 400, 256, -256) == path(1, 300, 400, 0) == "64 rows"
    assert {c[0] for c in CASES} | {"64 rows"} == set(KERNELS)


def codes(g, *shape):
    """Any codes but NaN."""
    return torch.randint(0, 127, shape, generator=g).to(torch.uint8) | torch.randint(0, 2, shape, generator=g).to(torch.uint8) << 7


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_every_kernel(case, dtype):
    """Normal values, results as the kernels store them at once."""
    kernel, batch, m, n, k = case
    assert path(batch, m, n, k) == kernel
    print(kernel, flush=True)
    g = torch.Generator().manual_seed(m + n + k)
    x = activations(g, batch * m, k).view(batch, m, k)
    a, b = F.fp8_quantize(x.cuda()), F.fp8_quantize(torch.randn(batch, n, k, generator=g).cuda() * k ** -0.5, rows=BLOCK)
    out = F.fp8_matmul(a, b, dtype=dtype)
    for i in {0, batch // 2, batch - 1}:
        check(out[i], (a.codes[i].cpu(), a.scales[i].cpu()), (b.codes[i].cpu(), b.scales[i].cpu()))


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_every_kernel_between_other_memory(case):
    """All codes, scales from 2^-40 to 2^40, as parts of wider tensors whose other entries are NaN; results at odd
    addresses with room between their rows, which stays as it was; then a code of NaN on either side."""
    kernel, batch, m, n, k = case
    assert path(batch, m, n, k, k + 16, k + 48) == kernel
    print(kernel, flush=True)
    g = torch.Generator().manual_seed(m + n + k)
    ca, cb, across, down = codes(g, batch, m, k), codes(g, batch, n, k), -(-k // BLOCK), -(-n // BLOCK)
    sa = torch.exp2(torch.randint(-40, 40, (batch, m, across), generator=g).float()) * 1.3
    sb = torch.exp2(torch.randint(-40, 40, (batch, down, across), generator=g).float()) * 0.7

    def between(x, pad, nan):
        wide = torch.full((*x.shape[:-1], x.shape[-1] + pad), nan, dtype=x.dtype, device="cuda")
        wide[..., :x.shape[-1]] = x.cuda()
        return wide[..., :x.shape[-1]]

    fa = F.Fp8(between(ca, 16, 0x7f).view(torch.float8_e4m3fn), between(sa, 3, torch.nan))
    fb = F.Fp8(between(cb, 48, 0xff).view(torch.float8_e4m3fn), between(sb, 1, torch.nan), rows=BLOCK)
    room = torch.full((batch * m * (n + 3) + 1,), 7.0, device="cuda")
    out = room[1:].view(batch, m, n + 3)[..., :n]
    F.fp8_matmul(fa, fb, out=out)
    for i in {0, batch - 1}:
        check(out[i], (ca[i].view(torch.float8_e4m3fn), sa[i]), (cb[i].view(torch.float8_e4m3fn), sb[i]))
    assert room[0] == 7 and (room[1:].view(batch, m, n + 3)[..., n:] == 7).all()
    fa.codes.view(torch.uint8)[batch // 2, m // 2, k - 1] = 0x7f
    fb.codes.view(torch.uint8)[batch // 2, n // 2, 0] = 0xff
    got = F.fp8_matmul(fa, fb).isnan()
    want = torch.zeros(batch, m, n, dtype=torch.bool, device="cuda")
    want[batch // 2, m // 2], want[batch // 2, :, n // 2] = True, True
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,far", [(5, 40, 400, "a"), (20, 33, 144, "b"), (35, 20, 272, "a"), (70, 20, 400, "b"), (65, 17, 1040, "b")])
def test_rows_far_apart(m, n, k, far):
    """Rows of one operand 8 MiB apart: the kernels with 64-bit offsets."""
    g = torch.Generator().manual_seed(m)
    ca, cb, across = codes(g, m, k), codes(g, n, k), -(-k // BLOCK)
    sa, sb = torch.rand(m, across, generator=g) + 0.5, torch.rand(1, across, generator=g) + 0.5
    stride = {"a": (LONG, k), "b": (k, LONG)}[far]
    assert path(1, m, n, k, *stride) == ("16 rows" if m <= 16 else "32 rows" if m <= 32 else "64 rows")
    rows = m if far == "a" else n
    room = torch.empty((rows - 1) * LONG + k, dtype=torch.uint8, device="cuda")
    wide = room.as_strided((rows, k), (LONG, 1))
    wide.copy_(ca if far == "a" else cb)
    fa = F.Fp8((wide if far == "a" else ca.cuda()).view(torch.float8_e4m3fn), sa.cuda())
    fb = F.Fp8((wide if far == "b" else cb.cuda()).view(torch.float8_e4m3fn), sb.cuda(), rows=BLOCK)
    check(F.fp8_matmul(fa, fb, dtype=torch.float32), (ca.view(torch.float8_e4m3fn), sa), (cb.view(torch.float8_e4m3fn), sb))
