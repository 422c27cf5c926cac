"""spec_attend over long runs of tiles by one CTA: requests that share one long
prefix, page by page, so that the cache itself stays small."""
import math

import pytest
import torch

import paper_2607_25852_gb300 as spec

pytestmark = pytest.mark.gpu

DEV = "cuda"


def shared_prefix(B, K, G, D, p, ps, seed=1):
    """B requests with the same pages up to position p - 1 and pages of their own for p .. p + K (one key-value head)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    common, own = p // ps, (p + K) // ps - p // ps + 1
    pages = common + B * own
    k, v = (torch.randn((pages, ps, 1, D), device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    table = torch.empty((B, common + own), dtype=torch.int32, device=DEV)
    table[:, :common] = torch.arange(common, dtype=torch.int32, device=DEV)
    table[:, common:] = torch.arange(common, pages, dtype=torch.int32, device=DEV).view(B, own)
    q = torch.randn((B * (K + 1), G, D), device=DEV, generator=g).to(torch.bfloat16)
    return q, k, v, table, torch.full((B,), p, dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("D,K,G", [(64, 3, 4), (64, 16, 8), (128, 16, 8), (64, 63, 4), (128, 63, 4)])
@pytest.mark.parametrize("window", [0, 40000])
def test_a_value_that_is_not_finite_costs_no_walk_over_the_context(D, K, G, window):
    """The rows that see an infinite value get it back in the epilogue: whatever the context's length, from the few
    positions that some rows see and some do not.  (A walk over all of them took 100 times the call itself.)"""
    B, p, ps, at = 160, 65536, 64, K // 2
    q, k, v, table, pos = shared_prefix(B, K, G, D, p, ps)
    ws = spec.attend_workspace(B, K, G, 1, D)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)

    def call():
        out = torch.empty_like(q)
        spec.spec_attend(q, k, v, table, pos, B, K, out, ws, window=window, status=st)
        torch.cuda.synchronize()
        best = math.inf
        for _ in range(3):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            spec.spec_attend(q, k, v, table, pos, B, K, out, ws, window=window, status=st)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        assert int(st) == 0
        return out.view(B, K + 1, G, D), best
    clean, clean_ms = call()
    t = p + at                                            # rows at .. K see it
    v[table[:, t // ps].long(), t % ps, 0, 5] = math.inf
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[:, at:, :, 5] = True
    if window:
        u = p - window + 1 + at                           # rows 0 .. at see it
        v[table[0, u // ps].long(), u % ps, 0, 3] = -math.inf
        hit[:, :at + 1, :, 3] = True
    out, ms = call()
    assert (~out[hit].isfinite()).all() and torch.equal(out[~hit], clean[~hit])
    assert ms < 10 * clean_ms, (ms, clean_ms)


@pytest.mark.parametrize("D,K,G,B,p", [(64, 0, 4, 320, 150_000_000), (128, 63, 4, 160, 80_000_000)])
def test_a_segment_may_take_longer_than_a_wait(D, K, G, B, p):
    """Items of more than a second each, parts of two or more per CTA (the waits are bounded to about a second).  All positions
    hold the same few pages over and over, so that the keys come from the L2, and every request the same queries."""
    ps, pages = 1 << 16, 8
    g = torch.Generator(device=DEV).manual_seed(2)
    k, v = (torch.randn((pages, ps, 1, D), device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    slots = (p + K) // ps + 1
    table = (torch.arange(slots, dtype=torch.int32, device=DEV) % pages).repeat(B, 1)
    q = torch.randn((K + 1, G, D), device=DEV, generator=g).to(torch.bfloat16).repeat(B, 1, 1)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    ws = spec.attend_workspace(B, K, G, 1, D)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    spec.spec_attend(q, k, v, table, torch.full((B,), p, dtype=torch.int64, device=DEV), B, K, out, ws, lse_out=lse, status=st)
    b.record()
    torch.cuda.synchronize()
    print(f"{a.elapsed_time(b):.0f} ms")
    assert int(st) == 0
    # Every position is there as often as every other, give or take one of the p / (8 * 65,536) rounds of the pages.
    # A thread's sum has a term per tile of 128 positions, with many rows one per 8 positions: as many roundings of 2^-24.
    tol = pages * ps / p + (p / 128 if K == 0 else p / 8) * 2.0 ** -24 + 1e-4
    x = torch.einsum("jhd,td->jht", q[:K + 1].double(), k.view(-1, D).double()) * D ** -0.5
    want = torch.logsumexp(x, 2) + math.log(p / (pages * ps))
    assert ((lse.view(B, K + 1, G).double() - want).abs() < tol).all()
