"""The library's first calls made by several host threads at once, in a process
of their own: what a call finds out once and keeps (the driver's entry points,
a kernel's sizes and limits) must not depend on which thread comes first."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import threading
import torch
import paper_2607_25852_gb300 as spec
from paper_2607_25852_gb300 import _native

N, B, ps, Hkv, p = 8, 3, 16, 2, 200
_native.load()
torch.cuda.init()
results, failures = {}, []
g = torch.Generator(device="cuda").manual_seed(1)
shapes = [(D, K, G) for D in (64, 128) for K, G in ((0, 8), (3, 8), (7, 8), (16, 8), (40, 8))]
inputs = []
for D, K, G in shapes:
    k, v = (torch.randn((40, ps, Hkv, D), device="cuda", generator=g).bfloat16() for _ in range(2))
    q = torch.randn((B * (K + 1), Hkv * G, D), device="cuda", generator=g).bfloat16()
    table = torch.arange(39, dtype=torch.int32, device="cuda").view(B, 13) % 40
    table = torch.cat([table, table], 1).contiguous()
    inputs.append((q, k, v, table, torch.full((B,), p, dtype=torch.int64, device="cuda"), K))
torch.cuda.synchronize()
gate = threading.Barrier(N)

def work(n):
    try:
        stream = torch.cuda.Stream()
        gate.wait()
        with torch.cuda.stream(stream):
            outs = []
            for q, k, v, table, pos, K in inputs:
                ws = spec.attend_workspace(B, K, q.shape[1], Hkv, q.shape[2])
                out = torch.empty_like(q)
                spec.spec_attend(q, k, v, table, pos, B, K, out, ws)
                outs.append((out, ws))
        stream.synchronize()
        results[n] = outs
    except Exception as e:
        failures.append(repr(e))

threads = [threading.Thread(target=work, args=(n,)) for n in range(N)]
for t in threads:
    t.start()
for t in threads:
    t.join()
assert not failures, failures
for n in range(1, N):
    for a, b in zip(results[0], results[n]):
        assert torch.equal(a[0], b[0]) and bool(a[0].float().isfinite().all())
print("the same in all threads")
"""


def test_first_calls_from_several_threads():
    run = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "the same in all threads" in run.stdout, run.stderr[-2000:]
