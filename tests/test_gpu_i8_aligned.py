"""8-bit layers on rows that start and end on 16 bytes, which the kernels take in whole groups: the quantiser that keeps rows in registers (one, two and
four pieces of 8 values a thread, and more rows than its grid), and the one token that the product quantises itself.

Codes and scales are compared for equality.  So are the 32-bit outputs: an exact integer, rounded to fp32 and multiplied twice."""
import numpy as np
import pytest
import torch

from test_gpu_i8_layers import TYPES, random_codes, reference_codes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    assert c.fq_status() == 0
    c.fq_destroy()


def check(fq, x, pitch):
    """x [rows][cols] with cols a multiple of 8 -> copied to rows `pitch` elements apart; what lies behind them is larger."""
    rows, cols = x.shape
    full = torch.full((rows, pitch), 1e4, dtype=x.dtype, device="cuda")
    full[:, :cols] = x
    codes = torch.full((rows, cols + 24), 55, dtype=torch.int8, device="cuda")
    assert cols % 8 == 0 and pitch * x.element_size() % 16 == 0 and full.data_ptr() % 16 == 0 and codes.data_ptr() % 8 == 0
    c, s = fq.fq_quantize_rows(full[:, :cols], codes[:, :cols])
    q, ref = reference_codes(x)
    q[~np.isfinite(ref)] = 0
    assert np.array_equal(s.cpu().numpy(), ref, equal_nan=True)
    assert np.array_equal(c.cpu().numpy(), q)
    assert bool((codes[:, cols:] == 55).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 8), (5, 264), (148, 4096), (3, 8192), (2, 8200), (2, 11008), (100, 16384), (2, 20000), (2, 32768), (2, 32776), (149, 8),
                                       (300, 4096), (300, 64), (5000, 512), (9600, 520), (2000, 4096), (700, 16384), (320, 32768)])
def test_aligned_rows(fq, dtype, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols)
    x = torch.randn((rows, cols), device="cuda", generator=g) * torch.rand((rows, 1), device="cuda", generator=g)
    x[:, cols // 3] *= 5                                      # rows of different ranges next to one another
    check(fq, x.to(dtype), cols + (8 if cols % 16 else 0))


def border_rows(dtype):
    """Rows whose quotients are on the borders k + 1/2 between codes, or next to them in fp32."""
    a = torch.arange(128, 256, dtype=torch.float32)
    x = torch.cat([torch.arange(-256, 257) / 2, torch.arange(-256, 257) / 256]).repeat(128, 1)
    x = torch.cat([a[:, None], torch.where(x.abs() > a[:, None], torch.zeros(()), x)], 1)
    k = torch.arange(-127, 127).double() + 0.5
    top = torch.rand(64, 1, generator=torch.Generator().manual_seed(1)).double() * 3 + 0.1
    top = top.to(dtype).double()
    mid = (k[None, :] * top / 127).to(dtype).float()
    step = mid.abs() * torch.finfo(dtype).eps
    near = torch.cat([top.float(), mid, mid + step, mid - step], 1).to(dtype).float()
    near = torch.where(near.abs() > near[:, :1], torch.zeros(()), near)
    width = -(-max(x.shape[1], near.shape[1]) // 8) * 8
    return torch.cat([torch.nn.functional.pad(v, (0, width - v.shape[1])) for v in (x, near)]).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
def test_borders_in_aligned_rows(fq, dtype):
    x = border_rows(dtype)
    rows, cols = x.shape
    check(fq, x[64:192], cols)                                # one piece a thread
    wide = torch.zeros((128, 8192 + cols), dtype=dtype, device="cuda")
    wide[:, 8192:] = x[64:192]
    check(fq, wide, wide.shape[1])                            # two
    check(fq, x.repeat(16, 1), cols + 16)                     # four, and rows that a CTA takes after its first


@pytest.mark.parametrize("dtype", TYPES)
def test_aligned_rows_without_a_range(fq, dtype):
    """Zeros, the type's smallest and largest values, infinities and NaN, among a CTA's first rows and its later ones."""
    fi = torch.finfo(dtype)
    x = torch.zeros((9, 304), dtype=dtype)
    x[1, 17] = -0.0
    x[2, :3] = torch.tensor([fi.smallest_normal, -fi.smallest_normal / 2, 0.0]).to(dtype)
    x[3, 5] = float(np.float32(fi.smallest_normal)) * float(fi.eps)               # the smallest subnormal
    x[4, :3] = torch.tensor([fi.max, -fi.max, fi.max / 2], dtype=torch.float64).to(dtype)
    x[5:] = torch.randn((4, 304), generator=torch.Generator().manual_seed(3)).to(dtype)
    x[5, 100], x[6, 303], x[7, 0] = float("inf"), float("nan"), float("-inf")
    for times in (1, 20, 700):
        check(fq, x.repeat(times, 1).cuda(), 304)


def expected(xq, xs, wc, sw):
    """fl(fl(fl(sum) sx) sw): the sum is exact in 64 bits."""
    total = torch.from_numpy(xq).cuda().double() @ wc.double().T
    return total.float() * torch.from_numpy(xs).cuda()[:, None] * sw[None, :]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 33, 8), (1, 300, 16), (1, 1000, 2000), (1, 513, 4088), (1, 4096, 4096), (1, 64, 4104), (1, 100, 11008), (2, 640, 2000), (4, 96, 4096),
                                   (5, 200, 1000), (40, 100, 2048), (300, 260, 512)])
@pytest.mark.parametrize("kind", ["normal", "borders", "zeros", "inf", "nan"])
def test_linear_on_aligned_tokens(fq, dtype, m, n, k, kind):
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    wc, sw = random_codes(n, k, 2)
    x = torch.randn((m, k), device="cuda", generator=g).to(dtype)
    if kind == "borders":
        b = border_rows(dtype)
        x = b[[(37 * i + 130) % len(b) for i in range(m)]].repeat(1, -(-k // b.shape[1]))[:, :k].contiguous()
    elif kind == "zeros":
        x[0] = 0.0
    elif kind == "inf":
        x[0, k - 1] = float("-inf")
    elif kind == "nan":
        x[0, k // 2] = float("nan")
    assert x.data_ptr() % 16 == 0
    q, s = reference_codes(x)
    q[~np.isfinite(s)] = 0
    ref = expected(q, s, wc, sw)
    for shifted in (x, torch.nn.functional.pad(x, (1, 7))[:, 1:k + 1]):         # in whole groups, and not
        y = torch.full((m, -(-n // 8) * 8 + 8), 7.0, dtype=torch.float32, device="cuda")
        fq.fq_linear_i8(shifted, wc, sw, y[:, :n])
        got = y[:, :n]
        assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.nan_to_num(), ref.nan_to_num())
        assert bool((y[:, n:] == 7.0).all()) and bool(got[0].isnan().all()) == (kind in ("inf", "nan"))
