"""spec_attend's weights, by values that show them (paged_precision): their two
bf16 halves on the tensor cores, and every tile of a long context in its place.
The bounds are relative to each element."""
import pytest
import torch

import paged_precision as pp
import paged_ref as ref
from test_gpu_attend import BF16, DEV, F32, Case

pytestmark = pytest.mark.gpu

FORMS = [(BF16, 128, 64, 0), (BF16, 64, 16, 3), (BF16, 128, 16, 8), (BF16, 128, 16, 16), (BF16, 64, 64, 16), (BF16, 128, 64, 40),
         (BF16, 64, 16, 63), (F32, 64, 16, 2), (F32, 128, 64, 0), (BF16, 96, 16, 4)]


def check(c, values, adds):
    t = torch.arange(values.shape[0])
    for i in range(c.B):
        c.v[c.table[i, t // c.ps].long().to(DEV), (t % c.ps).to(DEV)] = values.to(c.dtype).to(DEV)
    out, lse = c.call()
    want, want_lse, _, big = ref.attend(c.q, c.k, c.v, c.table, c.pos, c.rows, ref.sqrt_scale(c.D))
    split = c.dtype == BF16 and c.D in (64, 128)
    tol, tol_lse = pp.bounds(want, want_lse, big, c.pos[0] + c.K + 1, adds, c.D, c.dtype == BF16, split)
    err = (out.cpu().double() - want).abs()
    assert (err <= tol).all(), (err / tol).nan_to_num().max()
    err = (lse.cpu().double() - want_lse).abs()
    assert (err <= tol_lse).all(), (err / tol_lse).max()
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("dtype,D,ps,K", FORMS)
@pytest.mark.parametrize("p,B", [(1500, 1), (5000, 1), (2900, 40)])
def test_every_tile_in_its_place(p, B, dtype, D, ps, K):
    """Every block of positions at a d of its own (or, of more blocks than D, of two); one divided item, and many."""
    if B > 1:
        K = min(K, 8)
    c = Case([p] * B, [K] * B, K, 8, 2, D, ps, dtype, seed=p + D + K, q_scale=0.25)
    values = pp.block_values(p + K + 1, 2, D)
    check(c, values, pp.BLOCK * -(-(p + K + 1) // (pp.BLOCK * D)))


@pytest.mark.parametrize("D,p,K", [(128, 20000, 0), (128, 20000, 5), (64, 16000, 16)])
def test_every_tile_of_a_long_context(D, p, K):
    c = Case([p], [K], K, 8, 2, D, 64, BF16, seed=p, q_scale=0.25)
    check(c, pp.block_values(p + K + 1, 2, D), pp.BLOCK * -(-(p + K + 1) // (pp.BLOCK * D)))


@pytest.mark.parametrize("dtype,D,ps,K", FORMS)
def test_single_weights(dtype, D, ps, K):
    """One position per d, in the first tile, across tiles and at the end."""
    p = 1000
    for base in (0, 100, 127, 500, p + 1 - D):
        c = Case([p], [K], K, 8, 2, D, ps, dtype, seed=base + D + K, q_scale=0.25)
        check(c, pp.single_values(p + K + 1, 2, D, base), 1)
