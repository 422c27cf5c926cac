"""Rounds of a small target with an attention layer and a linear-attention layer:
rotary positions, the paged cache, the states, verification, commit and the
tokens' log probabilities together, against a plain model in 64 bits."""
import math

import pytest
import torch

import paper_2607_25852_gb300 as spec
import rows_ref as ref
from paper_2607_25852_gb300.paged import PagedCache
from paper_2607_25852_gb300.states import LinearStates

pytestmark = pytest.mark.gpu

DEV = "cuda"
F32 = torch.float32
HQ, HKV, D, E, V = 4, 2, 64, 48, 500


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Weights:
    def __init__(self):
        g = torch.Generator().manual_seed(11)

        def w(a, b):
            return torch.randn((a, b), generator=g) * a ** -0.5
        self.embed, self.head = torch.randn((V, E), generator=g), w(E, V) * 3
        self.qkv = [w(E, (HQ + 2 * HKV) * D) for _ in range(2)]
        self.out = [w(HQ * D, E) for _ in range(2)]
        self.gate = w(E, HKV)
        self.freq = spec.spec_rotary_frequencies(D, 10000.0, device="cpu")

    def to(self, dtype, device):
        for name, value in vars(self).items():
            if name != "freq":
                move = lambda x: x.to(dtype).to(device)
                setattr(self, name, [move(x) for x in value] if isinstance(value, list) else move(value))
        self.freq = self.freq.to(device)
        return self


def split(x, w):
    rows = (x @ w).unflatten(1, (HQ + 2 * HKV, D))
    return rows[:, :HQ], rows[:, HQ:HQ + HKV], rows[:, HQ + HKV:]


def decay_of(x, w):
    return -torch.nn.functional.softplus(x @ w)


def plain_logits(tokens, w):
    """The whole sequence at once, fp64 on the CPU: logits of every position."""
    x = w.embed[torch.tensor(tokens)]
    n = len(tokens)
    q, k, v = split(x, w.qkv[0])
    q, k = (torch.stack([ref.rotate(t[i], i, w.freq.tolist(), False, 1.0)[0] for i in range(n)]) for t in (q, k))
    k, v = (t.repeat_interleave(HQ // HKV, 1) for t in (k, v))
    s = torch.einsum("jhd,thd->hjt", q, k) * D ** -0.5
    s = s.masked_fill(torch.ones((n, n), dtype=torch.bool).triu(1), -math.inf).softmax(-1)
    x = x + torch.einsum("hjt,thd->jhd", s, v).flatten(1) @ w.out[0]
    q, k, v = split(x, w.qkv[1])
    o, _, _, _ = ref.linear(q, k, v, decay_of(x, w.gate), torch.zeros((HKV, D, D)), D ** -0.5)
    return (x + o.flatten(1) @ w.out[1]) @ w.head


class Target:
    """B requests of rounds of up to K + 1 rows, all of one stride."""

    def __init__(self, w, B, K):
        self.w, self.B, self.K = w, B, K
        self.cache = PagedCache(1, 256, 8, HQ, HKV, D, B, 256, K, F32)
        self.states = LinearStates(1, HQ, HKV, D, D, B, K + 1, F32)

    def layers(self, x, pos, depth, offsets):
        at = dict(depth=depth, row_offsets=offsets)
        q, k, v = split(x, self.w.qkv[0])
        self.cache.reserve(pos, depth, offsets)
        turned, o = torch.zeros_like(q), torch.zeros((len(x), HQ, D), device=DEV)
        self.cache.append_rotary(0, q, k, v, pos, self.w.freq, turned, **at)
        self.cache.attend(0, turned, pos, o, **at)
        x = x + o.flatten(1) @ self.w.out[0]
        q, k, v = split(x, self.w.qkv[1])
        decay = decay_of(x, self.w.gate)
        o = torch.zeros((len(x), HQ, D), device=DEV)
        self.states.attend(0, q, k, v, decay, o, K=self.K, **at)
        return (x + o.flatten(1) @ self.w.out[1]) @ self.w.head, (k, v, decay)


@pytest.mark.parametrize("B,K", [(3, 4), (2, 20)])
@pytest.mark.parametrize("captured", [False, True])
def test_rounds(B, K, captured):
    """Every round: the last token and drafts, some of them right; what is accepted is the target's own greedy text,
    its log probabilities those of the plain model, and cache and states are those of the accepted tokens."""
    plain, w = Weights().to(torch.float64, "cpu"), Weights().to(F32, DEV)
    t = Target(w, B, K)
    texts = [[5 * i + 1] for i in range(B)]
    greedy = []
    for i in range(B):  # the target's own continuation
        text = list(texts[i])
        for _ in range(3 * (K + 1) + 2):
            text.append(int(plain_logits(text, plain)[-1].argmax()))
        greedy.append(text)
    n = K + 1
    tokens_in, drafts = torch.zeros(B * n, dtype=torch.int64, device=DEV), torch.zeros((B, K), dtype=torch.int32, device=DEV)
    pos, depth, offsets = torch.zeros(B, dtype=torch.int64, device=DEV), i32([K] * B), i32([i * n for i in range(B + 1)])
    accepted, status = i32([0] * B), i32([0])
    tokens = torch.zeros((B, n), dtype=torch.int32, device=DEV)
    lp, rank = torch.zeros((B, n), device=DEV), torch.zeros((B, n), dtype=torch.int32, device=DEV)
    logits = torch.zeros((B * n, V), device=DEV)
    seeds, ids = torch.zeros(B, dtype=torch.int64, device=DEV), torch.arange(B, device=DEV)
    vws, lws = spec.verify_workspace(B, K, V, DEV), spec.logprobs_workspace(B, K, V, 0, DEV)

    def round_():
        got, kept = t.layers(w.embed[tokens_in], pos, depth, offsets)
        logits.copy_(got)
        spec.spec_verify(logits, drafts, None, B, K, V, 0.0, seeds, ids, pos, accepted, tokens, vws, row_offsets=offsets,
                         depth=depth, status=status)
        t.states.commit(0, *kept, accepted_len=accepted, depth=depth, row_offsets=offsets, K=K)
        t.cache.commit(pos, accepted)
        spec.spec_logprobs(logits, tokens, B, K, V, lp, lws, row_offsets=offsets, depth=depth, accepted_len=accepted,
                           rank_out=rank, status=status)
        pos.add_(accepted + 1)
    graph = None
    for step in range(3):
        for i in range(B):
            at = len(texts[i])
            right = greedy[i][at:at + K]
            wrong = (step + i) % n  # the first draft that is not the target's choice; K of them right at the last
            d = [x if j < wrong else (x + 1) % V for j, x in enumerate(right)]
            drafts[i] = i32(d)
            tokens_in[i * n:(i + 1) * n] = torch.tensor(texts[i][-1:] + d)
        if captured and step == 1:
            side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(graph, stream=side):
                round_()
        graph.replay() if graph else round_()
        torch.cuda.synchronize()
        assert int(status) == 0 and int(t.cache.status) == 0 and int(t.states.status) == 0
        for i in range(B):
            a = (step + i) % n
            assert int(accepted[i]) == a
            new = tokens[i, :a + 1].tolist()
            assert new == greedy[i][len(texts[i]):][:a + 1]
            want = plain_logits(texts[i] + new[:-1], plain)[len(texts[i]) - 1:].log_softmax(1)
            for j, x in enumerate(new):
                # an element behind the two layers is off by at most 4e-4 (sums of 48, 64, 63 and 256 terms in fp32,
                # 2^-24 each of their sizes, at most 16); the head's 48 weights of 0.43 make at most 7e-3 of that
                assert abs(float(lp[i, j]) - float(want[j, x])) < 1e-2 and int(rank[i, j]) == 1
            assert bool((rank[i, a + 1:] == 0).all())
            texts[i] += new


def test_calls_at_once():
    """Calls on two streams, each with its own workspace, give what they give one after another."""
    g = torch.Generator().manual_seed(7)

    def make(B, K, H, dk, V, n, dtype):
        R = B * (K + 1)
        q, k, v = (torch.randn((R, H, dk), generator=g).to(dtype).to(DEV) for _ in range(3))
        decay = (-torch.rand((R, H), generator=g)).to(DEV)
        states = torch.randn((2 * B, H, dk, dk), generator=g).to(DEV)
        start, to = torch.arange(B, dtype=torch.int32, device=DEV), torch.arange(B, 2 * B, dtype=torch.int32, device=DEV)
        ws, lws = spec.linear_workspace(B, K, H, H, dk, dk, dtype, DEV), spec.logprobs_workspace(B, K, V, n, DEV)
        logits = torch.randn((R, V), generator=g).to(dtype).to(DEV)
        tokens = torch.randint(0, V, (B, K + 1), generator=g).to(torch.int32).to(DEV)
        freq, pos = spec.spec_rotary_frequencies(dk), torch.arange(B, device=DEV) * 37
        turned, out = torch.empty_like(q), torch.empty_like(v)
        lp, status = torch.empty((B, K + 1), device=DEV), i32([0])
        top = torch.empty((B, K + 1, n), dtype=torch.int32, device=DEV)

        def call():
            spec.spec_rotary(q, freq, pos, B, K, turned, status=status)
            spec.spec_linear_attend(turned, k, v, decay, states, start, to, B, K, out, ws, status=status)
            spec.spec_logprobs(logits, tokens, B, K, V, lp, lws, top_tokens_out=top, status=status)
        return call, (turned, out, states, lp, top, status)
    for sizes in [((40, 3, 8, 64, 3000, 4, torch.bfloat16), (2, 255, 8, 128, 500, 2, torch.bfloat16)),
                  ((3, 200, 4, 64, 900, 8, F32), (70, 0, 16, 128, 5000, 3, F32))]:
        calls = [make(*s) for s in sizes]
        want = []
        for call, result in calls:
            call()
            torch.cuda.synchronize()
            want.append([x.clone() for x in result])
        streams = [torch.cuda.Stream() for _ in calls]
        for _ in range(5):
            for stream, (call, result) in zip(streams, calls):
                with torch.cuda.stream(stream):
                    for x in result[:2]:
                        x.zero_()
                    call()
            torch.cuda.synchronize()
            for (_, result), w in zip(calls, want):
                assert all(torch.equal(a, b) for a, b in zip(result, w)) and int(result[-1]) == 0


def test_calls_at_once_write_everything():
    """As above, with every output of the calls, the new states among them, set to something else before."""
    g = torch.Generator().manual_seed(7)

    def make(B, K, H, dk, V, n, dtype):
        R = B * (K + 1)
        q, k, v = (torch.randn((R, H, dk), generator=g).to(dtype).to(DEV) for _ in range(3))
        decay = (-torch.rand((R, H), generator=g)).to(DEV)
        states = torch.randn((2 * B, H, dk, dk), generator=g).to(DEV)
        start, to = torch.arange(B, dtype=torch.int32, device=DEV), torch.arange(B, 2 * B, dtype=torch.int32, device=DEV)
        ws, lws = spec.linear_workspace(B, K, H, H, dk, dk, dtype, DEV), spec.logprobs_workspace(B, K, V, n, DEV)
        logits = torch.randn((R, V), generator=g).to(dtype).to(DEV)
        tokens = torch.randint(0, V, (B, K + 1), generator=g).to(torch.int32).to(DEV)
        freq, pos = spec.spec_rotary_frequencies(dk), torch.arange(B, device=DEV) * 37
        turned, out = torch.empty_like(q), torch.empty_like(v)
        lp, status = torch.empty((B, K + 1), device=DEV), i32([0])
        top = torch.empty((B, K + 1, n), dtype=torch.int32, device=DEV)

        def call():
            spec.spec_rotary(q, freq, pos, B, K, turned, status=status)
            spec.spec_linear_attend(turned, k, v, decay, states, start, to, B, K, out, ws, status=status)
            spec.spec_logprobs(logits, tokens, B, K, V, lp, lws, top_tokens_out=top, status=status)
        def spoil():
            for x in (turned, out, states[B:], lp):
                x.fill_(77.0)
            top.fill_(-9)
        return call, spoil, (turned, out, states, lp, top, status)
    for sizes in [((40, 3, 8, 64, 3000, 4, torch.bfloat16), (2, 255, 8, 128, 500, 2, torch.bfloat16)),
                  ((3, 200, 4, 64, 900, 8, F32), (70, 0, 16, 128, 5000, 3, F32))]:
        calls = [make(*s) for s in sizes]
        want = []
        for call, spoil, result in calls:
            spoil()
            call()
            torch.cuda.synchronize()
            want.append([x.clone() for x in result])
        streams = [torch.cuda.Stream() for _ in calls]
        for _ in range(5):
            for stream, (call, spoil, _) in zip(streams, calls):
                with torch.cuda.stream(stream):
                    spoil()
                    call()
            torch.cuda.synchronize()
            for (_, _, result), w in zip(calls, want):
                assert all(torch.equal(a, b) for a, b in zip(result, w)) and int(result[-1]) == 0
