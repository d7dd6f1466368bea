"""Searches whose shared memory is near what a launch may have without asking, and searches of different sizes from
several threads."""
import os
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

# a kernel's first call in its process, of a row length and a number of candidates for which the tables take the last of
# 48 KB and the kernel's own variables more than that
_FIRST = """
import torch
from paper_2002_00104_b200 import pwlq
x = torch.randn(600, {n}, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
ratios = (torch.arange({K}, device="cuda") + 1.0) / {K}
if {two}:
    pwlq.search2(x, 4, ratios, m=x.abs().amax(1))
else:
    pwlq.search(x, 4, ratios)
torch.cuda.synchronize()
"""


@pytest.mark.parametrize("n,K,two", [(5408, 64, False), (5424, 64, False), (4816, 256, False), (2004, 1000, False),
                                     (8164, 2048, False), (8192, 2048, False), (3600, 64, True), (3612, 64, True)])
def test_first_calls_at_the_limit(n, K, two):
    done = subprocess.run([sys.executable, "-c", _FIRST.format(n=n, K=K, two=two)], cwd=ROOT, capture_output=True,
                          text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-500:]


def test_searches_of_different_sizes_from_several_threads():
    from paper_2002_00104_b200 import pwlq
    cases = []
    for n, K in ((8192, 1024), (6000, 64), (5000, 512), (8192, 4096), (8000, 2048)):
        x = torch.randn(600, n, generator=torch.Generator("cuda").manual_seed(n + K), device="cuda")
        ratios = ((torch.arange(K, device="cuda") + 1.0) / K)
        m = x.abs().amax(1)
        want = pwlq.search(x, 4, ratios, m=m)
        out = {k: torch.empty_like(v) for k, v in want.items() if k in ("p", "err", "idx")}
        cases.append((x, ratios, m, torch.empty_like(want["workspace"]), out, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    failed = [0] * len(cases)

    def work(i):
        x, ratios, m, workspace, out, _, stream = cases[i]
        torch.cuda.set_device(0)
        for n in range(300):
            try:
                pwlq.search(x, 4, ratios, m=m, workspace=workspace, out=out, stream=stream)
            except pwlq.PwlqError:
                failed[i] += 1
            if n % 100 == 99:
                stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert failed == [0] * len(cases)
    for *_, out, want, _ in cases:
        for k, v in out.items():
            assert np.array_equal(v.cpu().numpy(), want[k].cpu().numpy())
