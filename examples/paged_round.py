"""Speculative decoding of a small random-weight transformer over a paged
key-value cache: allocation, the target forward over the packed rows
(reserve, append and attend per layer), verification, commit and the release
of the rejected drafts' pages, round after round.

    python examples/paged_round.py

The drafter looks the last token up in the sequence so far and proposes what
followed it (a random-weight model decoded greedily soon repeats itself, so
many drafts are accepted).
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_25852_gb300 as spec
from paper_2607_25852_gb300.paged import PagedCache


class Target:
    """`layers` blocks of attention with a residual, random weights."""

    def __init__(self, layers, q_heads, kv_heads, head_dim, vocab, max_positions, dtype=torch.float32, seed=0,
                 device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.q_heads, self.kv_heads, self.head_dim, self.vocab = q_heads, kv_heads, head_dim, vocab
        width = q_heads * head_dim

        def rand(*shape, scale=1.0):
            return (torch.randn(shape, generator=g) * scale).to(dtype).to(device)
        self.embed, self.unembed = rand(vocab, width, scale=0.5), rand(width, vocab)
        self.position = rand(max_positions, width, scale=0.02)
        self.w_qkv = [rand(width, (q_heads + 2 * kv_heads) * head_dim, scale=0.7 * width ** -0.5) for _ in range(layers)]
        self.w_out = [rand(width, width, scale=width ** -0.5) for _ in range(layers)]

    def forward(self, tokens, positions, attention):
        """Logits of rows; attention(layer, q, k, v) returns the rows' attention outputs."""
        Hq, Hkv, D = self.q_heads, self.kv_heads, self.head_dim
        h = self.embed[tokens] + self.position[positions]
        for layer, (w, wo) in enumerate(zip(self.w_qkv, self.w_out)):
            rows = (torch.nn.functional.normalize(h, dim=-1) * h.shape[-1] ** 0.5 @ w).view(-1, Hq + 2 * Hkv, D)
            o = attention(layer, rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:])
            h = h + o.reshape(h.shape) @ wo
        return h @ self.unembed


def lookup_drafts(sequence, K):
    """What followed the last earlier occurrence of the last token, repeated to K tokens."""
    last = sequence[-1]
    for at in range(len(sequence) - 2, -1, -1):
        if sequence[at] == last:
            tail = sequence[at + 1:]
            return [tail[j % len(tail)] for j in range(K)]
    return [last] * K


def generate(target, prompts, new_tokens, K=4, page_size=16, pages=256, window=0, sinks=0, compact_every=3,
             device="cuda"):
    """Greedy continuations of the prompts (lists of token ids) and the rounds it took."""
    B, V, R = len(prompts), target.vocab, len(prompts) * (K + 1)
    Hq, Hkv, D = target.q_heads, target.kv_heads, target.head_dim
    dtype = target.embed.dtype
    chunk = 63  # prompt rows per forward, less one
    cache = PagedCache(len(target.w_qkv), pages, page_size, Hq, Hkv, D, B, target.position.shape[0], max(K, chunk),
                       dtype, window, sinks, device)
    i32 = dict(dtype=torch.int32, device=device)

    def forward(tokens, positions, pos_base, depth, row_offsets):
        cache.reserve(pos_base, depth, row_offsets)
        out = torch.zeros((tokens.numel(), Hq, D), dtype=dtype, device=device)

        def attention(layer, q, k, v):
            cache.append(layer, k, v, pos_base, depth, row_offsets)
            cache.attend(layer, q, pos_base, out, depth, row_offsets)
            return out
        return target.forward(tokens.clamp(min=0).long(), positions.clamp(min=0), attention)

    # ---- the prompts, all but their last tokens, in chunks; a request that is done idles at position -1 ----
    done = [0] * B
    while any(d < len(p) - 1 for d, p in zip(done, prompts)):
        take = [min(chunk + 1, len(p) - 1 - d) for d, p in zip(done, prompts)]
        depth = [max(t, 1) - 1 for t in take]
        base = [d if t > 0 else -1 for d, t in zip(done, take)]
        offsets = [0]
        for n in depth:
            offsets.append(offsets[-1] + n + 1)
        tokens = [p[d + j] if t > 0 else 0 for p, d, t, n in zip(prompts, done, take, depth) for j in range(n + 1)]
        positions = [max(b + j, 0) for b, n in zip(base, depth) for j in range(n + 1)]
        forward(torch.tensor(tokens, **i32), torch.tensor(positions, device=device), torch.tensor(base, device=device),
                torch.tensor(depth, **i32), torch.tensor(offsets, **i32))
        done = [d + max(t, 0) for d, t in zip(done, take)]

    # ---- rounds ----
    sequences = [list(p) for p in prompts]
    pos_base = torch.tensor([len(p) - 1 for p in prompts], device=device)
    last = torch.tensor([p[-1] for p in prompts], **i32)
    seeds = torch.zeros(B, dtype=torch.int64, device=device)
    ids = torch.arange(B, device=device)
    conf = torch.full((B, K), 0.8, device=device)
    budgets = spec.spec_budget_from_ratios(B, K, [1, 1], [2, 1])
    depth, offsets = torch.zeros(B, **i32), torch.zeros(B + 1, **i32)
    packed, chosen = torch.zeros(R, **i32), torch.zeros(1, **i32)
    positions = torch.zeros(R, dtype=torch.int64, device=device)
    accepted, tokens = torch.zeros(B, **i32), torch.zeros((B, K + 1), **i32)
    committed, commit_offsets = torch.zeros(R, **i32), torch.zeros(B + 1, **i32)
    ws = spec.verify_workspace(B, K, V, device)
    rounds = 0
    while min(len(s) - len(p) for s, p in zip(sequences, prompts)) < new_tokens:
        drafts = torch.tensor([lookup_drafts(s, K) for s in sequences], **i32)
        spec.spec_allocate(conf, budgets, [1.0, 1.5], last, drafts, pos_base, depth, offsets, packed, positions,
                           chosen, status=cache.status)
        logits = forward(packed, positions, pos_base, depth, offsets).contiguous()
        spec.spec_verify(logits, drafts, None, B, K, V, 0.0, seeds, ids, pos_base, accepted, tokens, ws,
                         row_offsets=offsets, depth=depth, status=cache.status)
        spec.spec_commit(accepted, tokens, None, B, K, committed, commit_offsets, row_offsets=offsets,
                         status=cache.status)
        cache.commit(pos_base, accepted)
        pos_base = pos_base + accepted + 1
        last = tokens.gather(1, accepted.long()[:, None]).squeeze(1).contiguous()
        rounds += 1
        if rounds % compact_every == 0:
            cache.compact()
        at, flat = commit_offsets.tolist(), committed.tolist()  # the tokens, for the next look-up
        for i in range(B):
            sequences[i] += flat[at[i]:at[i + 1]]
    assert int(cache.status) == 0, spec.spec_error_string(int(cache.status))
    cache.commit(torch.zeros_like(pos_base))  # every request is done
    assert int(cache.page_refs.sum()) == 0
    return [s[:len(p) + new_tokens] for s, p in zip(sequences, prompts)], rounds


def main():
    V = 48
    target = Target(layers=3, q_heads=8, kv_heads=2, head_dim=64, vocab=V, max_positions=1024)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, V, (n,), generator=g).tolist() for n in (5, 90, 33, 1, 200, 64)]
    out, rounds = generate(target, prompts, new_tokens=48)
    for p, s in zip(prompts, out):
        print(f"prompt of {len(p):3d} tokens -> ... {s[len(p):len(p) + 12]} ...")
    print(f"48 tokens for {len(prompts)} requests in {rounds} rounds: {48 / rounds:.2f} tokens a round and request")


if __name__ == "__main__":
    main()
