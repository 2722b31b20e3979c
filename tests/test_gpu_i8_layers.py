"""8-bit layers: the row quantiser and the int8 product against the definitions in 64 bits.

Tolerances.  Codes are exact and a scale is one fp32 division, so both are compared for equality.  An output is
fl(fl(fl(sum) sx) sw), three fp32 roundings of at most 2^-24 each, and one rounding to the output type of at most eps / 2, or half of
its smallest subnormal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}     # half of the smallest subnormal


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    assert c.fq_status() == 0
    c.fq_destroy()


def pitched(rows, cols, dtype, multiple, fill=None):
    t = torch.empty((rows, -(-cols // multiple) * multiple), dtype=dtype, device="cuda")
    if fill is not None:
        t.fill_(fill)
    return t[:, :cols]


def reference_codes(x):
    """(codes, scales) of the rows, in 64 bits; the quotient of two 24-bit numbers that is not on a border is off it in 64 bits."""
    x = x.detach().cpu().double().numpy()
    a = np.abs(x).max(axis=1)
    with np.errstate(all="ignore"):
        q = np.rint(127.0 * x / np.where(a > 0, a, 1.0)[:, None])
    q[~np.isfinite(a)] = 0
    s = np.where(np.isfinite(a), (a.astype(np.float32) / np.float32(127)), np.float32(np.nan))
    return q, s.astype(np.float32)


def reference_product(xc, sx, wc, sw):
    return (xc.double() @ wc.double().T) * sx.double()[:, None] * sw.double()[None, :]


def close(y, ref):
    tol = ref.abs() * (torch.finfo(y.dtype).eps / 2 + 4 * 2.0 ** -24) + TINY[y.dtype]
    bad = (y.double() - ref).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((y.double() - ref).abs() / tol).max()))


def random_codes(rows, cols, seed, multiple=16, fill=77):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = pitched(rows, cols, torch.int8, multiple, fill)
    t.copy_(torch.randint(-127, 128, (rows, cols), device="cuda", generator=g))
    return t, torch.rand(rows, device="cuda", generator=g) * 0.01 + 1e-4


# ---------------------------------------------------------------------------------------------------------------- quantiser
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 100), (2, 255), (4, 256), (7, 1000), (1, 4096), (3, 4097), (2, 11008), (2, 40001), (300, 64)])
def test_codes_and_scales(fq, dtype, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols)
    for shift, extra in ((0, 0), (3, 5)):                     # rows that start anywhere
        x = torch.full((rows, cols + extra), 1e4, dtype=dtype, device="cuda")[:, shift:shift + cols]
        x.copy_(torch.randn((rows, cols), device="cuda", generator=g) * torch.rand((rows, 1), device="cuda", generator=g))
        codes = torch.full((rows, cols + 9), 55, dtype=torch.int8, device="cuda")
        c, s = fq.fq_quantize_rows(x, codes[:, :cols])
        q, ref = reference_codes(x)
        assert np.array_equal(c.cpu().numpy(), q) and np.array_equal(s.cpu().numpy(), ref)
        assert bool((codes[:, cols:] == 55).all())            # columns behind the row stay


@pytest.mark.parametrize("dtype", TYPES)
def test_borders_between_codes(fq, dtype):
    """Every quotient of two 8-bit significands, a / 2 (63.5) among them, and in fp32 neighbours of the borders k + 1/2."""
    a = torch.arange(128, 256, dtype=torch.float32)
    x = torch.cat([torch.arange(-256, 257) / 2, torch.arange(-256, 257) / 256]).repeat(128, 1)
    x = torch.where(x.abs() > a[:, None], torch.zeros(()), x)
    x = torch.cat([a[:, None], x], 1)
    if dtype == torch.float32:
        k = torch.arange(-127, 127).double() + 0.5
        top = torch.rand(64, 1, generator=torch.Generator().manual_seed(1)).double() * 3 + 0.1
        mid = (k[None, :] * top.float().double() / 127).float()
        near = torch.cat([top.float(), mid, torch.nextafter(mid, torch.tensor(9.0)), torch.nextafter(mid, torch.tensor(-9.0))], 1)
        x = torch.nn.functional.pad(x, (0, max(0, near.shape[1] - x.shape[1])))
        x = torch.cat([x, torch.nn.functional.pad(near, (0, x.shape[1] - near.shape[1]))])
    x = x.to(dtype).cuda()
    c, s = fq.fq_quantize_rows(x)
    q, ref = reference_codes(x)
    assert np.array_equal(c.cpu().numpy(), q) and np.array_equal(s.cpu().numpy(), ref)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_a_range(fq, dtype):
    """Zeros, the type's smallest and largest values, infinities and NaN."""
    fi = torch.finfo(dtype)
    x = torch.zeros((8, 300), dtype=dtype)
    x[1, 17] = -0.0
    x[2, :3] = torch.tensor([fi.smallest_normal, -fi.smallest_normal / 2, 0.0]).to(dtype)
    x[3, 5] = float(np.float32(fi.smallest_normal)) * float(fi.eps)               # the smallest subnormal
    x[4, :3] = torch.tensor([fi.max, -fi.max, fi.max / 2], dtype=torch.float64).to(dtype)
    x[5] = torch.randn(300, generator=torch.Generator().manual_seed(3)).to(dtype)
    x[5, 100] = float("inf")
    x[6, 299] = float("nan")
    x[7, 0] = float("-inf")
    c, s = fq.fq_quantize_rows(x.cuda())
    q, ref = reference_codes(x)
    q[~np.isfinite(ref)] = 0
    assert np.array_equal(c.cpu().numpy(), np.nan_to_num(q)) and np.array_equal(s.cpu().numpy(), ref, equal_nan=True)
    assert np.isnan(ref[5:]).all() and (ref[:2] == 0).all()


# ---------------------------------------------------------------------------------------------------------------- product
SHAPES = [(1, 1, 1), (1, 16, 16), (2, 40, 33), (5, 1000, 127), (8, 129, 128), (9, 257, 129), (1, 4096, 4096), (16, 300, 1000), (17, 64, 5000),
          (33, 513, 640), (64, 96, 14336), (77, 4096, 1100), (128, 128, 128), (129, 640, 257), (130, 5120, 300), (255, 31, 999), (300, 13824, 260),
          (600, 1000, 4224), (2047, 300, 512), (2, 20000, 64), (4, 8, 40000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(fq, dtype, m, n, k):
    xc, sx = random_codes(m, k, 1)
    wc, sw = random_codes(n, k, 2)
    full = torch.full((m + 1, -(-n // 8) * 8 + 8), 7.0, dtype=dtype, device="cuda")       # row and columns behind the outputs
    y = full[:m, :n]
    fq.fq_gemm_i8(xc, sx, wc, sw, y)
    close(y, reference_product(xc, sx, wc, sw))
    assert bool((full[m:] == 7.0).all()) and bool((full[:, n:] == 7.0).all())


def test_longest_sum_is_exact(fq):
    """131071 products of the same sign: the largest sum there is, and one that fp32 alone would lose."""
    k = 131071
    xc, wc = pitched(3, k, torch.int8, 16), pitched(40, k, torch.int8, 16)
    xc[0], xc[1], xc[2] = 127, -128, -127
    wc[:] = 127
    wc[3] = -128
    wc[7, 5] = 126
    one = torch.ones(40, device="cuda")
    y = torch.empty((3, 40), dtype=torch.float32, device="cuda")
    fq.fq_gemm_i8(xc, one[:3], wc, one, y)
    ref = (xc.double() @ wc.double().T).float()
    assert torch.equal(y, ref)


def test_scales_that_are_not_numbers(fq):
    """A token or a channel whose scale is NaN (it held an infinity or a NaN), or 0: only its own outputs tell."""
    xc, sx = random_codes(20, 500, 3)
    wc, sw = random_codes(50, 500, 4)
    sx[3], sw[7], sx[5] = float("nan"), float("nan"), 0.0
    for rows in (20, 6):
        y = torch.empty((rows, 56), dtype=torch.bfloat16, device="cuda")[:, :50]
        fq.fq_gemm_i8(xc[:rows], sx[:rows], wc, sw, y)
        nan = torch.zeros((rows, 50), dtype=torch.bool, device="cuda")
        nan[3], nan[:, 7] = True, True
        assert torch.equal(torch.isnan(y), nan)
        assert bool((y[5, :7] == 0).all())
        close(y[nan.logical_not()], reference_product(xc[:rows], sx[:rows], wc, sw)[nan.logical_not()])


# ---------------------------------------------------------------------------------------------------------------- both
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (1, 33, 100), (1, 1000, 14336), (2, 640, 1000), (3, 96, 257), (4, 11008, 512), (7, 64, 4224), (8, 4096, 300),
                                   (9, 100, 1111), (16, 2000, 640), (40, 100, 1000), (77, 512, 11008), (300, 300, 300)])
def test_linear_is_quantiser_and_product(fq, dtype, m, n, k):
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    x = torch.empty((m, k + 3), dtype=dtype, device="cuda")[:, 1:k + 1]
    x.copy_(torch.randn((m, k), device="cuda", generator=g))
    if m > 2:
        x[1], x[2, k // 2] = 0.0, float("nan")
    w = torch.randn((n, k), device="cuda", generator=g) * 0.02
    wc, sw = fq.fq_quantize_rows(w)
    y, y2 = pitched(m, n, dtype, 8), pitched(m, n, dtype, 8)
    fq.fq_linear_i8(x, wc, sw, y)
    xc, sx = fq.fq_quantize_rows(x)
    fq.fq_gemm_i8(xc, sx, wc, sw, y2)
    assert torch.equal(y.isnan(), y2.isnan()) and torch.equal(y.nan_to_num(), y2.nan_to_num())
    q, s = reference_codes(x)
    ref = reference_product(torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), wc, sw)
    there = ~torch.isnan(ref)
    assert torch.equal(there, ~torch.isnan(y)) and (m <= 2 or bool(y[2].isnan().all()) and bool((y[1] == 0).all()))
    close(y[there], ref[there])


@pytest.mark.parametrize("m", [1, 6, 50, 300])
def test_two_streams_and_a_graph(fq, m):
    """Calls that overlap on two streams, and a captured one that is replayed on new activations, in a context that is used meanwhile."""
    n, k = 1000, 2000
    g = torch.Generator(device="cuda").manual_seed(m)
    wc, sw = fq.fq_quantize_rows(torch.randn((n, k), device="cuda", generator=g))
    xs = [torch.randn((m, k), device="cuda", generator=g).half() for _ in range(4)]
    want = [fq.fq_linear_i8(x, wc, sw, pitched(m, n, torch.float16, 8)).clone() for x in xs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [pitched(m, n, torch.float16, 8) for _ in xs]
    torch.cuda.synchronize()
    for i, x in enumerate(xs):
        with torch.cuda.stream(streams[i & 1]):
            fq.fq_linear_i8(x, wc, sw, got[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x, y = xs[0].clone(), pitched(m, n, torch.float16, 8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.fq_linear_i8(x, wc, sw, y)
    for i in (1, 2, 3, 0):
        x.copy_(xs[i])
        graph.replay()
        other = fq.fq_linear_i8(xs[3 - i], wc, sw, pitched(m, n, torch.float16, 8))
        torch.cuda.synchronize()
        assert torch.equal(y, want[i]) and torch.equal(other, want[3 - i])
    del graph
