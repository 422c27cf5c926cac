"""spec_attend inside its workspace where every CTA has parts of items, in every
form, and in one workspace that shapes of several forms use in turn."""
import pytest
import torch

import paper_2607_25852_gb300 as spec
from test_gpu_attend import BF16, F32, Case

pytestmark = pytest.mark.gpu

SHAPES = [  # dtype, D, page size, K, query heads over 2: the CUDA cores, the tensor cores for few columns and for many
    (F32, 64, 16, 0, 4), (F32, 128, 16, 16, 16), (F32, 8, 16, 3, 4), (BF16, 256, 16, 40, 8), (BF16, 96, 16, 7, 16),
    (BF16, 64, 10, 16, 16), (BF16, 64, 16, 0, 16), (BF16, 64, 16, 2, 8), (BF16, 128, 16, 11, 16), (BF16, 128, 16, 16, 16),
    (BF16, 64, 16, 16, 16), (BF16, 128, 16, 31, 16), (BF16, 64, 16, 32, 16),
]


def case(dtype, D, ps, K, Hq):
    return Case([500 + 31 * (i % 9) for i in range(100)], [K] * 100, K, Hq, 2, D, ps, dtype, seed=D + K)


@pytest.mark.parametrize("dtype,D,ps,K,Hq", SHAPES)
def test_writes_stay_inside(dtype, D, ps, K, Hq):
    from test_gpu_canaries import Guarded, assert_intact, guarded_workspace
    c = case(dtype, D, ps, K, Hq)
    want = c.call()
    ws = guarded_workspace(spec.spec_attend_workspace(c.B, K, Hq, 2, D, dtype))
    out, lse = Guarded(c.q.shape, dtype, 7.0), Guarded(c.q.shape[:2], F32, 7.0)
    c.call(ws=ws.t, out=out.t, lse=lse.t)
    assert_intact(ws=ws, out=out, lse=lse)
    assert torch.equal(out.t, want[0]) and torch.equal(lse.t, want[1]) and int(c.status.item()) == 0


def test_one_workspace_for_several_shapes():
    cases = [case(*s) for s in SHAPES]
    want = [c.call() for c in cases]
    ws = torch.zeros(max(c.ws.numel() for c in cases), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        for c, (out, lse) in zip(cases, want):
            got = c.call(ws=ws)
            assert torch.equal(got[0], out) and torch.equal(got[1], lse)
