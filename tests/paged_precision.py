"""Values that show what spec_attend does with its weights: each position, or
each block of positions, has a d of its own, where its values are 1 (or another
number that bf16 holds) and all others 0.  So an element of the output is the
weight of one position or block, nothing cancels, and adding the others' zeros
rounds nothing: an error bound can be relative to the element itself."""
import torch

BLOCK = 128


def block_values(positions, heads, D):
    """[positions, heads, D]: block b of 128 positions at d = b mod D, with a number of its own per head and block."""
    t = torch.arange(positions)
    b = t // BLOCK
    v = torch.zeros((positions, heads, D))
    for h in range(heads):
        v[t, h, b % D] = 1.0 + ((b + 3 * h) % 8).float() / 8
    return v


def single_values(positions, heads, D, base):
    """[positions, heads, D]: 1 at d = t - base for the D positions from base, 0 elsewhere."""
    v = torch.zeros((positions, heads, D))
    t = torch.arange(base, min(base + D, positions))
    v[t, :, t - base] = 1.0
    return v


def bounds(want, want_lse, big, terms, adds, D, bf16, split):
    """Bounds of out and lse for such values; `big` as in paged_ref.attend, `terms` positions, of which an element of
    the output adds up to `adds`.

    A score is a sum of D products in fp32, off by at most (D + 4) 2^-23 big with truncating adders and its scaling, and
    a weight relatively by as much, and by 2^-22 for its exponential; a part's weight in a join by 2^-22 again.  `split`
    (the second product on the tensor cores): the weight's upper bf16 number and its rest, rounded to 8 bits: the rest is
    below 2^-7 of the weight, so 2^-16.  An element adds `adds` products (2^-23 each, truncating), and its two halves; it
    is scaled once a tile where the maximum moves (2^-24 each), and once a part.  The sum of the weights is added up by
    threads with no more than one in eight of the terms each, by lanes and warps, and by parts (fewer than 400).  All of
    this for numerator and denominator alike.  Rounding the result: half of the last of 8 bits, 2^-8, in bf16, else 2^-24."""
    score = (D + 4) * 2.0 ** -23 * big
    sums = (2 * adds + terms / 8 + terms / 64 + 1000) * 2.0 ** -24
    rel = 2 * score + 2.0 ** -20 + sums + (2.0 ** -16 if split else 0.0)
    rounding = 2.0 ** -8 if bf16 else 2.0 ** -24
    tol = want * (rel[..., None] * 1.01 + rounding)
    return tol, score + 2.0 ** -21 + sums + want_lse.abs() * 2.0 ** -22
