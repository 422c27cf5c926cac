"""Idle requests of a round: all rows before position 0.  And pos_base = -1 with
drafts, which is not idle: its rows 1.. lie at positions 0.."""
import math

import pytest
import torch

from paper_2607_25852_gb300.paged import PagedCache

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("K", [0, 2, 40])
def test_idle_requests_take_nothing_and_get_zeros(K, dtype, D):
    B, ps, Hq, Hkv = 3, 8, 4, 2
    c = PagedCache(1, 40, ps, Hq, Hkv, D, B, 64, K, dtype)
    c.k.fill_(math.nan)
    c.v.fill_(math.nan)
    g = torch.Generator().manual_seed(K)
    pos = torch.tensor([0, -(K + 1), -(K + 9)], device=DEV)
    k, v = (torch.randn((B * (K + 1), Hkv, D), generator=g).to(dtype).to(DEV) for _ in range(2))
    q = torch.randn((B * (K + 1), Hq, D), generator=g).to(dtype).to(DEV)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    assert c.reserve(pos).tolist() == [1, 1, 1]
    c.append(0, k, v, pos)
    c.attend(0, q, pos, out, lse_out=lse)
    assert (c.page_table[1:] == -1).all() and int(c.page_refs.sum()) == K // ps + 1
    assert int(c.k[0, :, :, 0, 0].isfinite().sum()) == K + 1
    assert (out[K + 1:] == 0).all() and (lse[K + 1:] == -math.inf).all()
    assert out[:K + 1].float().isfinite().all() and lse[:K + 1].isfinite().all() and int(c.status) == 0
    c.commit(pos, torch.tensor([K, 0, K], dtype=torch.int32, device=DEV))
    assert (c.page_table[1:] == -1).all() and int(c.page_refs.sum()) == K // ps + 1 and int(c.status) == 0


def test_minus_one_is_idle_without_drafts_alone():
    B, K, ps, D = 2, 2, 8, 64
    c = PagedCache(1, 8, ps, 1, 1, D, B, 64, K)
    new = torch.ones((B * (K + 1), 1, D), dtype=torch.bfloat16, device=DEV)
    pos = torch.tensor([-1, -1], device=DEV)
    depth = torch.tensor([2, 0], dtype=torch.int32, device=DEV)
    c.k.zero_()
    c.reserve(pos, depth)
    c.append(0, new, new, pos, depth)
    assert c.page_table[:, 0].tolist() == [0, -1]
    assert c.k[0, 0, :, 0, 0].tolist() == [1, 1] + [0] * 6   # rows 1 and 2 of request 0, at positions 0 and 1
    assert int(c.status) == 0
