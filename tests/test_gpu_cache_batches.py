"""Steps of batches around the sizes at which the bookkeeping's shared memory grows, each as the first call of a process."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for path in (ROOT, os.path.join(ROOT, "tests")):
    if path not in sys.path:
        sys.path.insert(0, path)

pytestmark = pytest.mark.gpu


def child(sizes):
    import torch

    import fq_paged as O
    import paper_2501_07139_b200 as P
    fq = P.FlexQ(1)
    for n in sizes:
        for tokens in (n + 5, 2 * n + 4000):                # rows by the same kernel where there are few, by one of their own
            g = torch.Generator().manual_seed(n)
            lens = torch.randint(0, 20, (n,), generator=g).tolist()
            keep = [v if b % 3 else v // 2 for b, v in enumerate(lens)]
            new = torch.randint(0, 2, (n,), generator=g).tolist()
            blocks = sum(O.ceil_div(v, 8) for v in lens) + n + 1
            table, rest = O.make_table(lens, 8, 4, blocks, g)
            free = rest + [-7] * (blocks - len(rest))
            d = [torch.tensor(t, dtype=torch.int32, device="cuda") for t in (lens, keep, new)]
            dt, df, dc = table.cuda(), torch.tensor(free, dtype=torch.int32, device="cuda"), torch.tensor([len(rest)], dtype=torch.int32, device="cuda")
            got = fq.fq_cache_step(*d, dt, df, dc, 8, tokens)
            rows = table.tolist()
            starts, slots, positions, _, count = O.step(lens, keep, new, rows, free, len(rest), 8, tokens)
            assert fq.fq_status() == 0
            assert got[0].tolist() == starts and got[1].tolist() == slots and got[2].tolist() == positions
            assert d[0].tolist() == lens and dt.tolist() == rows and int(dc) == count and df.tolist()[:count] == free[:count]
    fq.fq_destroy()


@pytest.mark.parametrize("sizes", [[4096], [4079, 4080, 4095, 4097], [1365, 12288, 12289, 16384]])
def test_first_calls(sizes):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), *map(str, sizes)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]


if __name__ == "__main__":
    child([int(v) for v in sys.argv[1:]])
