"""The largest sizes that the 8-bit layers and the calls on logits take: 2^20 rows, columns, tokens or outputs.  Codes, 32-bit products (two roundings, done
here as well) and empty or certain answers are compared for equality, the others as in the tests of their kind."""
import pytest
import torch

from test_gpu_logits import check_distill, check_logprobs, rows_of, tokens_of

pytestmark = pytest.mark.gpu
MOST = 1 << 20


@pytest.fixture(scope="module")
def fq():
    import paper_2501_07139_b200 as P
    c = P.FlexQ(1)
    yield c
    assert c.fq_status() == 0
    c.fq_destroy()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols,pitch", [(MOST, 8, 8), (MOST, 3, 3), (3, MOST, MOST), (2, MOST - 1, MOST + 1)])
def test_quantiser(fq, dtype, rows, cols, pitch):
    """Values that are whole numbers up to 127, one of them 127: their codes are themselves and the scale is 1."""
    x = torch.randint(-127, 128, (rows, pitch), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[:, cols // 2] = 127
    c, s = fq.fq_quantize_rows(x.to(dtype)[:, :cols])
    assert torch.equal(c, x[:, :cols].to(torch.int8)) and bool((s == 1).all())


@pytest.mark.parametrize("m,n,k", [(MOST, 8, 16), (MOST, 24, 40), (1, MOST, 32), (4, MOST, 48), (5, MOST, 32), (200, MOST, 16), (300, MOST - 3, 16)])
def test_product(fq, m, n, k):
    g = torch.Generator(device="cuda").manual_seed(2)
    pitch = -(-k // 16) * 16
    xc = torch.randint(-127, 128, (m, pitch), device="cuda", generator=g).to(torch.int8)[:, :k]
    wc = torch.randint(-127, 128, (n, pitch), device="cuda", generator=g).to(torch.int8)[:, :k]
    sx, sw = torch.rand(m, device="cuda", generator=g), torch.rand(n, device="cuda", generator=g)
    y = torch.empty((m, -(-n // 4) * 4), dtype=torch.float32, device="cuda")[:, :n]
    fq.fq_gemm_i8(xc, sx, wc, sw, y)
    for r in range(0, m, 1 << 17):                            # sums below 2^24: exact in fp32 as well
        part = slice(r, r + (1 << 17))
        ref = (xc[part].double() @ wc.double().T).float() if n < 1000 else xc[part].float() @ wc.float().T
        ref *= sx[part, None]
        ref *= sw[None, :]
        assert torch.equal(y[part], ref)
        del ref


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_logits(fq, dtype):
    z = rows_of("normal", MOST, 6, dtype, 3)
    check_logprobs(fq, z, tokens_of(MOST, 6, 3), 2, 0.7)
    g = torch.Generator(device="cuda").manual_seed(4)
    ids = torch.randint(-1, 6, (MOST, 3), device="cuda", generator=g).int()
    check_distill(fq, z, ids, torch.randn((MOST, 3), device="cuda", generator=g), 0.7, torch.rand(MOST, device="cuda", generator=g))
