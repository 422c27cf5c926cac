"""Plain implementations in 64 bits of rotary positions, linear attention and token
log probabilities, with the magnitudes that error bounds are made of.  Nothing here
comes from the library."""
import math

import torch

EPS = 2.0 ** -24  # fp32's rounding


def half_step(dtype):
    """The largest relative error of one rounding to dtype."""
    return torch.finfo(dtype).eps / 2


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------
def frequencies(rotary_dim, base=10000.0, scaling="plain", factor=1.0, original=0, low=1.0, high=32.0):
    if scaling == "base":
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    out = []
    for d in range(rotary_dim // 2):
        f = base ** (-2 * d / rotary_dim)
        if scaling == "linear":
            f /= factor
        if scaling == "ramp":
            keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low)))
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return out


def rotate(x, position, freq, interleaved, amplitude):
    """x [heads, D] of one row: its turned form and the error bound of an fp32 one, both fp64."""
    x = x.double()
    n = len(freq)
    angle = torch.tensor([math.remainder(position * f, 2 * math.pi) for f in freq], dtype=torch.float64)
    c, s = torch.cos(angle) * amplitude, torch.sin(angle) * amplitude
    i = torch.arange(n)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    y = x.clone()
    y[:, ia] = x[:, ia] * c - x[:, ib] * s
    y[:, ib] = x[:, ib] * c + x[:, ia] * s
    size = torch.zeros_like(x)
    size[:, ia] = size[:, ib] = (x[:, ia].abs() + x[:, ib].abs()) * abs(amplitude)
    # the angle: position * f rounded in the reference (2^-53 of it, and 2^-53 of the reduction) and f / 2 pi in
    # the kernel (2^-52); its fp32 form 2^-24 of at most pi.  cos and sin 2^-22, the amplitude's product 2^-24,
    # the two products and their sum 2^-23.
    far = torch.tensor([abs(position * f) * 2.0 ** -50 for f in freq], dtype=torch.float64)
    err = torch.zeros_like(x)
    err[:, ia] = err[:, ib] = far + math.pi * EPS + 4 * EPS + EPS + 2 * EPS
    return y, size * err


# ---------------------------------------------------------------------------
# Linear attention
# ---------------------------------------------------------------------------
def linear(q, k, v, log_decay, start, scale, take=None):
    """One request: q [n, Hq, Dk], k [n, H, Dk], v [n, H, Dv], log_decay [n, H], start [H, Dk, Dv]; the state after
    `take` rows (all if None).  Returns out [n, Hq, Dv], the state, and both from absolute values (the sums' sizes)."""
    q, k, v, s = q.double(), k.double(), v.double(), start.double().clone()
    n, Hq, Dk = q.shape
    H, Dv = k.shape[1], v.shape[2]
    G = Hq // H
    size = s.abs()
    out, out_size = torch.zeros((n, Hq, Dv), dtype=torch.float64), torch.zeros((n, Hq, Dv), dtype=torch.float64)
    after, after_size = s, size
    for j in range(n):
        f = torch.exp(log_decay[j].double())[:, None, None]
        s = torch.where(f == 0, 0.0, f * s) + k[j][:, :, None] * v[j][:, None, :]
        size = f * size + k[j].abs()[:, :, None] * v[j].abs()[:, None, :]
        out[j] = scale * torch.einsum("hd,hdv->hv", q[j], s.repeat_interleave(G, 0))
        out_size[j] = abs(scale) * torch.einsum("hd,hdv->hv", q[j].abs(), size.repeat_interleave(G, 0))
        if take is None or j < take:
            after, after_size = s, size
    return out, after, out_size, after_size


def linear_bounds(out, out_size, state, state_size, n, Dk, dtype):
    """Error bounds of out and state.  Sums of at most Dk + n terms and n rescalings in fp32, adders that truncate
    included: 2^-23 of the size each.  A weight is exp2 of a difference rounded in fp32: of 24 binary orders it is off
    by 24 * 2^-24, below that it is itself below 2^-24, and exp2 by 2^-22.  bf16 rows may go through products of split
    numbers: 2^-16 of the size for the scores and as much for the state in out, 2^-24 in the state."""
    sums = (Dk + 2 * n + 32) * 2 * EPS + 32 * EPS
    split = 2 * 2.0 ** -16 if dtype == torch.bfloat16 else 0.0
    return (out_size * (sums + split) + out.abs() * half_step(dtype) * 1.01 + 1e-37,
            state_size * sums + 1e-37)


# ---------------------------------------------------------------------------
# Log probabilities
# ---------------------------------------------------------------------------
def logprobs(row, token, t, n):
    """One row (1-d, its own dtype): logprob, rank, entropy, the n best tokens and their log probabilities."""
    x = row.double()
    lp = torch.log_softmax(x / t, 0)
    order = sorted(range(len(x)), key=lambda v: (-float(x[v]), v)) if len(x) < 5000 else torch.sort(
        x, descending=True, stable=True)[1].tolist()
    best = [v for v in order[:n] if x[v] > -math.inf]
    logprob, rank = -math.inf, 0
    if token >= 0:
        logprob = float(lp[token])
        rank = 1 + int(((x > x[token]) | ((x == x[token]) & (torch.arange(len(x)) < token))).sum())
    p = lp.exp()
    entropy = float(-(p * torch.where(p > 0, lp, 0.0)).sum())
    pad = n - len(best)
    return logprob, rank, entropy, best + [-1] * pad, [float(lp[v]) for v in best] + [-math.inf] * pad


def logprob_bound(row, t, logprob):
    """A term 2^d has d = l c2 - m c2 off by three roundings, c2's among them (|d| < 150, but weighted with 2^d: at
    most 2^-22 of its sum; m c2's own cancels in ln p), and ex2's 2^-22; a thread's running sum takes up to 33 steps a round of 16,384 entries and
    30 joins.  log2 and the products: 2^-22 of the result."""
    return (33 * (len(row) // 16384 + 1) + 46) * EPS + abs(logprob) * 8 * EPS
