"""The learner's operators called by several host threads at once, each on its own stream, with sizes that need different amounts of shared
memory; in a process of its own, so that the first calls of all kernels are among them."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
import threading
import torch
from paper_2205_05248_b200 import binding

g = torch.Generator().manual_seed(0)
rand = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
mats = [[rand(16, 9)], [rand(128, 1024)], [rand(3, 64, 102), rand(3, 192, 64)], [rand(384, 128)], [rand(40, 17, 5)], [rand(64, 1000)]]
scans = [(rand(2, L, C), rand(2, L, C)) for L, C in ((40, 64), (100, 64), (300, 96), (64, 128), (1000, 64), (33, 48))]
rows = [rand(5, 70000), rand(300, 14), rand(9, 500)]
torch.cuda.synchronize()
start = threading.Barrier(6)
got, errors = [None] * 6, []

def scan(k):
    gate, x = scans[k]
    r = binding.marl_linear_scan(gate, x, keep=True)
    d = binding.marl_linear_scan_backward(gate, x, r["states"], x)
    return [r["y"], r["last"], d["dgate"], d["dx"], d["dh0"]]

def logprob(k):
    x = rows[k % 3]
    r = binding.marl_policy_logprob(x, torch.zeros(x.shape[0], dtype=torch.int32, device="cuda"), top=3)
    return [r["logp"], r["top_index"]]

def work(k):
    try:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            start.wait()
            for _ in range(20):
                out = binding.marl_orthogonalise(mats[k]) + scan(k) + logprob(k)
        s.synchronize()
        got[k] = out
    except Exception as e:
        errors.append("%d: %s" % (k, e))

threads = [threading.Thread(target=work, args=(k,)) for k in range(6)]
for t in threads:
    t.start()
for t in threads:
    t.join()
assert not errors, errors
for k in range(6):
    want = binding.marl_orthogonalise(mats[k]) + scan(k) + logprob(k)
    assert len(want) == len(got[k]) and all(torch.equal(a, b) for a, b in zip(want, got[k])), k
print("same results")
"""


def test_threads_with_different_sizes():
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same results" in r.stdout, r.stderr[-2000:]
