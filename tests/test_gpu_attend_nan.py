"""spec_attend where scores are NaN: a row with a NaN query, and rows that see a
long run of NaN keys, get NaN however the work is divided, and no other row
does.  Tolerances of the others: the kernel's error bounds (paged_ref.bounds)."""
import pytest
import torch

import paged_ref as ref
import paper_2607_25852_gb300 as spec
from test_gpu_attend import BF16, DEV, F32, Case

pytestmark = pytest.mark.gpu

# the CUDA cores in both types, the tensor cores for few columns and for many
FORMS = [(F32, 128, 64, 0), (F32, 64, 16, 3), (BF16, 96, 16, 0), (BF16, 128, 10, 3), (BF16, 256, 16, 2), (BF16, 128, 64, 0),
         (BF16, 64, 16, 5), (BF16, 128, 16, 40), (BF16, 64, 64, 80)]


def check(c, out, lse, want, spoiled):
    """NaN where `spoiled` [R, Hq], within the bounds of `want` elsewhere."""
    exact, exact_lse, mass, big = want
    tol, tol_lse = ref.bounds(exact, mass, big, c.pos[0] + c.K + 1, c.D, c.dtype == BF16)
    got, got_lse = out.cpu().double(), lse.cpu().double()
    assert got[spoiled].isnan().all() and got_lse[spoiled].isnan().all()
    assert ((got - exact).abs() <= tol)[~spoiled].all()
    assert ((got_lse - exact_lse).abs() <= tol_lse)[~spoiled].all()
    assert int(c.status.item()) == 0
    assert int(c.ws.view(torch.uint8)[:768].sum()) == 0


@pytest.mark.parametrize("dtype,D,ps,K", FORMS)
@pytest.mark.parametrize("p", [40, 3000])
def test_a_nan_query_spoils_its_row_and_no_other(p, dtype, D, ps, K):
    c = Case([p], [K], K, 8, 2, D, ps, dtype, seed=p + D + K)
    want = ref.attend(c.q, c.k, c.v, c.table, c.pos, c.rows, ref.sqrt_scale(D))
    spoiled = torch.zeros((K + 1, 8), dtype=torch.bool)
    spoiled[K // 2, 3] = spoiled[0, 6] = True
    c.q[spoiled.to(DEV)] = float("nan")
    check(c, *c.call(), want, spoiled)


@pytest.mark.parametrize("dtype,D,ps,K", FORMS)
@pytest.mark.parametrize("first,last", [(0, 1500), (700, 2200), (1500, 3001), (2999, 3000)])
def test_a_run_of_nan_keys_spoils_the_heads_that_see_it(first, last, dtype, D, ps, K):
    c = Case([3000], [K], K, 8, 2, D, ps, dtype, seed=first + D + K)
    want = ref.attend(c.q, c.k, c.v, c.table, c.pos, c.rows, ref.sqrt_scale(D))
    t = torch.arange(first, last)
    c.k[c.table[0, t // ps].long().to(DEV), (t % ps).to(DEV), 1] = float("nan")
    spoiled = torch.zeros((K + 1, 8), dtype=torch.bool)
    spoiled[:, 4:] = True
    check(c, *c.call(), want, spoiled)


@pytest.mark.parametrize("dtype,D,ps,K", FORMS)
def test_parts_that_see_nan_keys_alone(dtype, D, ps, K):
    """The run ends at a tile's end, so that for some of its lengths a part of a
    divided item holds nothing else."""
    for tiles in range(1, 24):
        n = 64 * tiles
        c = Case([3000], [K], K, 8, 2, D, ps, dtype, seed=D + K)
        t = torch.arange(n)
        c.k[c.table[0, t // ps].long().to(DEV), (t % ps).to(DEV), 1] = float("nan")
        out, lse = c.call()
        assert out[:, 4:].isnan().all() and lse[:, 4:].isnan().all(), n
        assert out[:, :4].float().isfinite().all() and lse[:, :4].isfinite().all()


@pytest.mark.parametrize("dtype,D,ps,K", FORMS)
def test_a_window_hides_nan_keys(dtype, D, ps, K):
    c = Case([3000], [K], K, 8, 2, D, ps, dtype, window=900, sinks=4, seed=D + K)
    want = ref.attend(c.q, c.k, c.v, c.table, c.pos, c.rows, ref.sqrt_scale(D), 900, 4)
    t = torch.arange(4, 3000 - 900 + 1)
    c.k[c.table[0, t // ps].long().to(DEV), (t % ps).to(DEV)] = float("nan")
    check(c, *c.call(), want, torch.zeros((K + 1, 8), dtype=torch.bool))


@pytest.mark.parametrize("dtype,D,ps,K", FORMS)
@pytest.mark.parametrize("window,sinks", [(2, 0), (2, (1 << 31) - 1), (1, 1), (3, 2)])
def test_infinite_values_beside_rows_before_the_first_position(window, sinks, dtype, D, ps, K):
    """Some rows lie before position 0 and see nothing; an infinite value of position 1 reaches the rows that see it."""
    if K < 3:
        K = 3
    c = Case([-2], [K], K, 8, 2, D, ps, dtype, window=window, sinks=sinks, seed=D + K)
    want, want_lse, mass, big = ref.attend(c.q, c.k, c.v, c.table, c.pos, c.rows, ref.sqrt_scale(D), window, sinks)
    c.v[int(c.table[0, 1 // ps]), 1 % ps, 1, 5] = float("inf")
    hit = torch.zeros(want.shape, dtype=torch.bool)
    for j in range(K + 1):
        hit[j, 4:, 5] = 1 in ref.visible(j - 2, window, sinks)
    out, lse = c.call()
    tol, tol_lse = ref.bounds(want, mass, big, K + 1, D, dtype == BF16)
    got, got_lse = out.cpu().double(), lse.cpu().double()
    assert (~got[hit].isfinite()).all() and ((got - want).abs() <= tol)[~hit].all()
    assert torch.equal(got_lse == -float("inf"), want_lse == -float("inf")) and (got_lse[:2] == -float("inf")).all()
    assert ((got_lse - want_lse).abs() <= tol_lse)[2:].all() and int(c.status.item()) == 0
