"""spec_attend for requests of many rows (more than 144 columns of row and query
head per key-value head: the tensor cores' other form), and the division of few
items, against attention in 64 bits."""
import pytest
import torch

import paged_ref as ref
import paper_2607_25852_gb300 as spec
from test_gpu_attend import BF16, DEV, F32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,ps,K", [(8, 1, 128, 16, 18), (8, 1, 64, 64, 31), (16, 2, 128, 8, 32), (4, 2, 64, 48, 80),
                                           (2, 2, 128, 128, 255), (3, 1, 64, 24, 100), (64, 1, 128, 32, 3),
                                           (64, 1, 64, 16, 4), (5, 1, 128, 40, 57)])
def test_ragged_rows(Hq, Hkv, D, ps, K):
    """One set of 128 columns, two, several items of 256, and a last item of few."""
    pos = [0, 1, 127, 128, 700, 65, -1, 300]
    depth = [0, K, K // 2, 0, K, K // 3, 0, K - 1]
    c = Case(pos, depth, K, Hq, Hkv, D, ps, BF16, seed=Hq + D + ps)
    c.check(*c.call())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (100, 0), (128, 128), (129, 130), (300, 64), (5000, 4),
                                          (37, 1000)])
def test_window_and_sinks(window, sinks, D):
    pos, depth = [0, 130, 511, 1300], [40, 3, 39, 40]
    c = Case(pos, depth, 40, 8, 2, D, 16, BF16, window=window, sinks=sinks, seed=window + sinks)
    c.check(*c.call())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D,ps", [(64, 16), (128, 64)])
def test_what_masked_places_hold_does_not_matter(D, ps, bad):
    for window, sinks in ((0, 0), (90, 3)):
        c = Case([333, 0, 95], [40, 0, 21], 40, 8, 2, D, ps, BF16, window=window, sinks=sinks, seed=11)
        seen = torch.zeros(c.k.shape[:2], dtype=torch.bool)
        for i, p in enumerate(c.pos):
            for j in range(c.rows.depth[i] + 1):
                for t in ref.visible(p + j, window, sinks):
                    seen[c.table[i, t // ps], t % ps] = True
        for x in (c.k, c.v):
            x[~seen.to(DEV)] = bad
        c.check(*c.call())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (128, 50)])
def test_a_later_row_does_not_reach_an_earlier_one(D, window, bad):
    """A value that is not finite reaches the rows that see it and no other, also
    across the two sets of an item."""
    K = n = 63
    for p in (60, 300):
        c = Case([p], [n], K, 8, 2, D, 16, BF16, window=window, seed=p)
        want, want_lse, mass, big = ref.attend(c.q, c.k, c.v, c.table, c.pos, c.rows, ref.sqrt_scale(D), window)
        hit = torch.zeros(want.shape, dtype=torch.bool)
        for first in (20, 50):  # visible from this row on, with a window for its length
            t = p + first
            c.v[c.table[0, t // 16].long(), t % 16, 1, first] = bad
            hit[first:min(K + 1, first + window) if window else K + 1, 4:, first] = True
        out, lse = c.call()
        tol, tol_lse = ref.bounds(want, mass, big, p + K + 1, D, True)
        got = out.cpu().double()
        assert (~got[hit].isfinite()).all()
        assert ((got - want).abs() <= tol)[~hit].all()
        assert ((lse.cpu().double() - want_lse).abs() <= tol_lse).all()


def test_scores_of_every_size():
    """Maxima that move by much along the cache, up and down, and equal scores."""
    for ramp in (0.0, 0.02, -0.02):
        c = Case([1500], [39], 39, 8, 2, 64, 16, BF16, seed=5, q_scale=4.0)
        if ramp:
            t = torch.arange(1540)
            add = (ramp * t).to(BF16).to(DEV)
            c.k[c.table[0, t // 16].long().to(DEV), (t % 16).to(DEV)] += add[:, None, None]
            c.q[:] = c.q.abs()
            c.q[20:] *= 0.01  # rows whose maxima hardly move beside rows whose do
        else:
            c.q.zero_()
        c.check(*c.call())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pos,K,Hq,Hkv", [
    ([9000], 31, 8, 1),             # one item: few of the CTAs, a join of several parts
    ([5000], 2, 4, 1),              # the same with few columns
    ([5000], 16, 8, 1),
    ([400] * 30, 31, 8, 1),         # an item per CTA
    ([400] * 30, 3, 8, 1),
    ([4000] + [90, 31] * 6, 31, 8, 2),  # one long item among short ones
    ([4000] + [90, 31] * 6, 3, 8, 2),
    ([2000, 2100, -1, 1900], 40, 8, 2),
    ([700, 650], 255, 8, 2),
    ([300] * 45, 40, 8, 2),         # more items than CTAs
])
def test_every_division_of_the_work(pos, K, Hq, Hkv, D):
    depth = [K if p >= 0 else 0 for p in pos]
    c = Case(pos, depth, K, Hq, Hkv, D, 64, BF16, seed=len(pos) + K)
    first = c.call()
    c.check(*first)
    again = c.call()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_every_division_in_fp32():
    for pos, K in (([5000], 3), ([300] * 20, 4), ([4000] + [90, 31] * 6, 3)):
        c = Case(pos, [K] * len(pos), K, 8, 2, 64, 16, F32, seed=len(pos) + K)
        c.check(*c.call())


@pytest.mark.parametrize("D", [64, 128])
def test_long_runs(D):
    """Many tiles per CTA; equal requests get equal results whatever share of the work they fall into."""
    B, p, K, Hkv, G = 40, 2900, 63, 2, 8
    g = torch.Generator().manual_seed(K)
    slots = (p + K) // 64 + 1
    k = torch.randn((slots, 64, Hkv, D), generator=g).to(BF16).to(DEV)
    v = torch.randn((slots, 64, Hkv, D), generator=g).to(BF16).to(DEV)
    q1 = torch.randn((K + 1, Hkv * G, D), generator=g).to(BF16)
    table = torch.arange(slots, dtype=torch.int32, device=DEV).repeat(B, 1)
    q = q1.repeat(B, 1, 1).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    ws = spec.attend_workspace(B, K, Hkv * G, Hkv, D, BF16, DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    pos = torch.full((B,), p, dtype=torch.int64, device=DEV)
    want, want_lse, mass, big = ref.attend(q1, k, v, table, [p], ref.Rows([K], K), ref.sqrt_scale(D))
    tol, tol_lse = ref.bounds(want, mass, big, p + K + 1, D, True)
    for _ in range(5):
        out.fill_(7.0)
        spec.spec_attend(q, k, v, table, pos, B, K, out, ws, lse_out=lse, status=st)
        assert int(st.item()) == 0
        got = out.view(B, K + 1, -1, D).cpu().double()
        assert ((got - want).abs() <= tol).all()
        assert ((lse.view(B, K + 1, -1).cpu().double() - want_lse).abs() <= tol_lse).all()


@pytest.mark.parametrize("D,ps", [(128, 16), (64, 64)])
def test_bad_pages_and_writes(D, ps):
    from test_gpu_canaries import Guarded, assert_intact, guarded_workspace
    c = Case([1000, 0, 129, 64], [40, 0, 40, 2], 40, 8, 2, D, ps, BF16, seed=31)
    want = c.call()
    n = spec.spec_attend_workspace(c.B, c.K, c.Hq, c.Hkv, D, BF16)
    ws = guarded_workspace(n)
    out, lse = Guarded(c.q.shape, BF16, 7.0), Guarded(c.q.shape[:2], F32, 7.0)
    c.call(ws=ws.t, out=out.t, lse=lse.t)
    assert_intact(ws=ws, out=out, lse=lse)
    assert torch.equal(out.t, want[0]) and torch.equal(lse.t, want[1])
    # a visible slot without a page: its keys are left out, as if they were masked
    r = c.rows.offsets
    for entry in (-1, 10 ** 6):
        c.table[2, 1] = entry
        got, _ = c.call()
        assert int(c.status.item()) == spec.ERR_BAD_INPUT
        c.status.zero_()
        assert torch.equal(got[:r[2]], want[0][:r[2]]) and torch.equal(got[r[3]:], want[0][r[3]:])
        assert got[r[2]:r[3]].float().isfinite().all() and not torch.equal(got[r[2]:r[3]], want[0][r[2]:r[3]])
