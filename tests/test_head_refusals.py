"""Arguments that the 8-bit layers and the calls on logits refuse.  Every check comes before the context or a pointer is looked into, so
that a refused call needs no GPU: the context here is a page of zeros and the buffers are addresses."""
import ctypes as C

import pytest

import paper_2501_07139_b200 as P

ARG, SHAPE, ALIGN = -1, -3, -4
PAGE = C.create_string_buffer(1 << 16)
CTX = C.addressof(PAGE)
BUF = 0x10000                # aligned to anything asked for; never read
F16, BF16, F32 = 0, 1, 2

QUANT = dict(ctx=CTX, x=BUF, dtype=BF16, rows=4, cols=40, ldx=40, codes=BUF, ldc=48, scales=BUF, stream=None)
GEMM = dict(ctx=CTX, xc=BUF, sx=BUF, m=4, ldx=48, wc=BUF, sw=BUF, n=24, k=40, ldw=48, y=BUF, y_dtype=BF16, ldy=24, stream=None)
LINEAR = dict(ctx=CTX, x=BUF, x_dtype=F16, m=4, ldx=40, wc=BUF, sw=BUF, n=24, k=40, ldw=48, codes=BUF, ldc=48, scales=BUF, y=BUF,
              y_dtype=BF16, ldy=24, stream=None)
LOGPROBS = dict(ctx=CTX, z=BUF, dtype=BF16, rows=4, vocab=100, ld=100, tokens=BUF, id_bytes=8, t=1.0, logprob=BUF, entropy=BUF, n_top=5,
                ids=BUF, tops=BUF, stream=None)
DISTILL = dict(ctx=CTX, z=BUF, dtype=BF16, rows=4, vocab=100, ld=100, ids=BUF, id_bytes=4, teacher=BUF, n_top=5, t=1.0, g=BUF, loss=BUF,
               lse=BUF, grad=BUF, ldg=100, stream=None)
GRAD = dict(ctx=CTX, z=BUF, dtype=BF16, rows=4, vocab=100, ld=100, ids=BUF, id_bytes=4, teacher=BUF, n_top=5, t=1.0, g=BUF, lse=BUF, grad=BUF,
            ldg=100, stream=None)

ROWS = [("rows", 0, SHAPE), ("rows", -1, SHAPE), ("rows", (1 << 20) + 1, SHAPE), ("vocab", 0, SHAPE), ("vocab", P.FQ_MAX_VOCAB + 1, SHAPE),
        ("ld", 99, SHAPE), ("z", 0, ARG), ("z", BUF + 1, ALIGN), ("dtype", 3, ARG), ("dtype", -1, ARG), ("id_bytes", 2, ARG), ("t", 0.0, ARG),
        ("t", -1.0, ARG), ("t", float("inf"), ARG), ("t", float("nan"), ARG), ("t", 1e-31, ARG), ("t", 1e31, ARG), ("n_top", 129, SHAPE), ("ctx", None, ARG)]
SLOTS = [("ids", 0, ARG), ("ids", BUF + 2, ALIGN), ("teacher", 0, ARG), ("teacher", BUF + 2, ALIGN), ("n_top", 0, SHAPE), ("lse", 0, ARG),
         ("lse", BUF + 4, ALIGN), ("grad", BUF + 1, ALIGN), ("ldg", 99, SHAPE), ("g", 0, ARG), ("g", BUF + 1, ALIGN)]
WEIGHTS = [("m", 0, SHAPE), ("m", (1 << 20) + 1, SHAPE), ("n", 0, SHAPE), ("k", 0, SHAPE), ("k", 131072, SHAPE), ("ldw", 32, SHAPE),
           ("ldw", 40, SHAPE), ("ldy", 16, SHAPE), ("ldy", 28, SHAPE), ("wc", BUF + 8, ALIGN), ("y", BUF + 8, ALIGN), ("sw", BUF + 2, ALIGN),
           ("wc", 0, ARG), ("sw", 0, ARG), ("y", 0, ARG), ("y_dtype", 5, ARG), ("ctx", None, ARG)]
BAD = {
    "fq_quantize_rows": (QUANT, [("ctx", None, ARG), ("x", 0, ARG), ("codes", 0, ARG), ("scales", 0, ARG), ("dtype", 7, ARG), ("rows", 0, SHAPE),
                                 ("cols", 0, SHAPE), ("rows", (1 << 20) + 1, SHAPE), ("cols", (1 << 20) + 1, SHAPE), ("ldx", 39, SHAPE),
                                 ("ldc", 39, SHAPE), ("x", BUF + 1, ALIGN), ("scales", BUF + 2, ALIGN)]),
    "fq_gemm_i8": (GEMM, WEIGHTS + [("xc", 0, ARG), ("sx", 0, ARG), ("xc", BUF + 4, ALIGN), ("sx", BUF + 1, ALIGN), ("ldx", 32, SHAPE),
                                    ("ldx", 41, SHAPE)]),
    "fq_linear_i8": (LINEAR, WEIGHTS + [("x", 0, ARG), ("codes", 0, ARG), ("scales", 0, ARG), ("x_dtype", 3, ARG), ("ldx", 39, SHAPE),
                                        ("ldc", 40, SHAPE), ("x", BUF + 1, ALIGN), ("codes", BUF + 8, ALIGN), ("scales", BUF + 2, ALIGN)]),
    "fq_token_logprobs": (LOGPROBS, ROWS + [("tokens", 0, ARG), ("tokens", BUF + 4, ALIGN), ("logprob", 0, ARG), ("entropy", 0, ARG), ("ids", 0, ARG),
                                            ("tops", 0, ARG), ("n_top", -1, SHAPE), ("logprob", BUF + 1, ALIGN)]),
    "fq_distill_topk": (DISTILL, ROWS + SLOTS + [("loss", 0, ARG), ("loss", BUF + 2, ALIGN)]),
    "fq_distill_topk_grad": (GRAD, ROWS + SLOTS + [("grad", 0, ARG)]),
}


@pytest.mark.parametrize("name,field,value,code", [(n, f, v, c) for n, (_, bad) in BAD.items() for f, v, c in bad])
def test_refused(name, field, value, code):
    args = {**BAD[name][0], field: value}
    assert getattr(P.lib(), name)(*args.values()) == code
    assert PAGE.raw == bytes(1 << 16)


def test_methods_name_what_does_not_fit():
    """The binding's own checks, on CPU tensors: a context without a device refuses them all."""
    import torch
    fq = P.FlexQ.__new__(P.FlexQ)
    fq._h, fq.device, fq._index = C.c_void_p(), torch.device("cuda", 0), 0
    x = torch.zeros((2, 8), dtype=torch.float16)
    for call in (lambda: fq.fq_quantize_rows(x), lambda: fq.fq_token_logprobs(x, torch.zeros(2, dtype=torch.int64)),
                 lambda: fq.fq_distill_topk(x, torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3))),
                 lambda: fq.fq_gemm_i8(x, x, x, x, x), lambda: fq.fq_linear_i8(x, x, x, x)):
        with pytest.raises(ValueError, match="cuda:0"):
            call()
