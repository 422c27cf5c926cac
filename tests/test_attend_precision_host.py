"""The bounds of paged_precision on the CPU: the arithmetic that spec.h promises
lies inside them, and the mistakes that they are there to find lie outside."""
import pytest
import torch

import paged_precision as pp


def bf16(x):
    return x.to(torch.bfloat16).float()


def upper(x):
    return (x.view(torch.int32) & -65536).view(torch.float32)


def test_a_weight_in_two_numbers_is_off_by_at_most_2_to_the_minus_16():
    g = torch.Generator().manual_seed(1)
    x = torch.exp2(torch.rand(1 << 22, generator=g) * 30 - 20)
    x = torch.cat([x, torch.tensor([1.0 + 2.0 ** -8 + 2.0 ** -16])])
    two = upper(x).double() + bf16(x - upper(x)).double()
    err = ((two - x.double()).abs() / x.double())
    assert float(err.max()) <= 2.0 ** -16 and float(err[-1]) > 2.0 ** -17


# name: a weight as the second product takes it, and whether the bound has to find that out from blocks, from singles
# (None: the result's own rounding may hide it)
FORMS = {
    "as promised": (lambda w: upper(w) + bf16(w - upper(w)), False, False),
    "upper numbers alone": (upper, True, True),
    "one rounded number": (bf16, None, True),
}


def setting(p, D, heads, seed):
    g = torch.Generator().manual_seed(seed)
    q, k = torch.randn((heads, D), generator=g) * 0.25, bf16(torch.randn((p, heads, D), generator=g))
    q = bf16(q)
    scale = D ** -0.5
    x64 = torch.einsum("hd,thd->ht", q.double(), k.double()) * scale
    big = (torch.einsum("hd,thd->ht", q.double().abs(), k.double().abs()) * scale).amax(1)
    x = torch.einsum("hd,thd->ht", q, k) * scale
    return x64, big, torch.exp(x - x.amax(1, keepdim=True))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("p,D", [(128, 128), (3000, 64), (20000, 128)])
def test_forms_of_the_weights(p, D, form):
    heads = 8
    split, seen_in_blocks, seen_in_singles = FORMS[form]
    x64, big, w = setting(p, D, heads, p + D)
    lse = torch.logsumexp(x64, 1)
    exact = torch.exp(x64 - lse[:, None])
    total = w.double().sum(1)
    for values, adds, seen in ((pp.block_values(p, heads, D), pp.BLOCK * (-(-p // (pp.BLOCK * D))), seen_in_blocks),
                               (pp.single_values(p, heads, D, p // 2), 1, seen_in_singles)):
        want = torch.einsum("ht,thd->hd", exact, values.double())
        got = torch.einsum("ht,thd->hd", split(w).double(), values.double()) / total[:, None]
        tol, _ = pp.bounds(want, lse, big, p, adds, D, True, True)
        err = (bf16(got.float()).double() - want).abs()
        assert seen is None or bool((err > tol).any()) == seen


@pytest.mark.parametrize("p,D", [(3000, 64), (20000, 128)])
def test_a_lost_or_exchanged_block_is_found(p, D):
    heads = 8
    x64, big, _ = setting(p, D, heads, p)
    lse = torch.logsumexp(x64, 1)
    exact = torch.exp(x64 - lse[:, None])
    values = pp.block_values(p, heads, D).double()
    want = torch.einsum("ht,thd->hd", exact, values)
    tol, _ = pp.bounds(want, lse, big, p, 2 * pp.BLOCK, D, True, True)
    for b in range(p // pp.BLOCK):
        lost = values.clone()
        lost[b * pp.BLOCK:(b + 1) * pp.BLOCK] = 0
        moved = values.clone()
        a = (b + 1) % (p // pp.BLOCK)
        moved[b * pp.BLOCK:(b + 1) * pp.BLOCK] = values[a * pp.BLOCK:(a + 1) * pp.BLOCK]
        for wrong in (lost, moved):
            err = (torch.einsum("ht,thd->hd", exact, wrong) - want).abs()
            assert ((err > 20 * tol).sum(1) >= 1).all(), b
