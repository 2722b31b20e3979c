"""Calls of the 8-bit layers and on logits whose first launch in the process is a captured one, and calls from several threads at a time."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

pytestmark = pytest.mark.gpu


def calls(fq, m, v, seed):
    """Inputs made from a seed, and what runs on them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, k, rows, top = 640, 512, m + 3, 7
    x = torch.randn((m, k), device="cuda", generator=g).half()
    wc = torch.randint(-127, 128, (n, k), device="cuda", generator=g).to(torch.int8)
    sw = torch.rand(n, device="cuda", generator=g) * 0.01
    z = torch.randn((rows, v), device="cuda", generator=g).bfloat16()
    tokens = torch.randint(0, v, (rows,), device="cuda", generator=g)
    ids = torch.randint(0, v, (rows, top), device="cuda", generator=g)
    teacher, up = torch.randn((rows, top), device="cuda", generator=g), torch.rand(rows, device="cuda", generator=g)

    def run():
        y = fq.fq_linear_i8(x, wc, sw, torch.empty((m, n), dtype=torch.float16, device="cuda"))
        codes, scales = fq.fq_quantize_rows(x)
        y2 = fq.fq_gemm_i8(codes, scales, wc, sw, torch.empty((m, n), dtype=torch.float32, device="cuda"))
        a = fq.fq_token_logprobs(z, tokens, top)
        loss, lse, grad = fq.fq_distill_topk(z, ids, teacher, 1.0, up)
        alone = fq.fq_distill_topk(z, ids, teacher)[0]
        return [y, codes, scales, y2, *a, loss, lse, grad, alone, fq.fq_distill_topk_grad(z, ids, teacher, lse, up)]

    return run


CASES = [(1, 5000), (3, 900), (40, 40000), (300, 3000)]


def child():
    import paper_2501_07139_b200 as P
    fq = P.FlexQ(1)
    for m, v in CASES:
        run = calls(fq, m, v, m)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, run())), (m, v)
        del graph
    assert fq.fq_status() == 0
    fq.fq_destroy()


def test_a_first_call_may_be_captured():
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]


def test_several_threads():
    import paper_2501_07139_b200 as P
    fq = P.FlexQ(1)
    runs = [calls(fq, m, v, 10 * m + i) for i in range(2) for m, v in CASES]
    want = [[t.clone() for t in run()] for run in runs]
    torch.cuda.synchronize()

    def work(run):
        with torch.cuda.stream(torch.cuda.Stream()):
            outs = [run() for _ in range(5)]
            torch.cuda.current_stream().synchronize()
        return outs

    with ThreadPoolExecutor(len(runs)) as pool:
        for outs, ref in zip(pool.map(work, runs), want):
            assert all(torch.equal(a, b) for out in outs for a, b in zip(out, ref))
    assert fq.fq_status() == 0
    fq.fq_destroy()


if __name__ == "__main__":
    child()
