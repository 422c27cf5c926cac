"""spec_logprobs against log-softmax in 64 bits; ranks and alternatives exactly."""
import math

import pytest
import torch

import paper_2607_25852_gb300 as spec
import rows_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Call:
    def __init__(self, logits, tokens, B, K, n, t=1.0, offsets=None, depth=None, accepted=None, ws=None, stream=None):
        V = logits.shape[1]
        self.ws = spec.logprobs_workspace(B, K, V, n, DEV) if ws is None else ws
        shape = (B, K + 1)
        self.lp, self.entropy = torch.full(shape, 9.0, device=DEV), torch.full(shape, 9.0, device=DEV)
        self.rank = torch.full(shape, 9, dtype=torch.int32, device=DEV)
        self.top = torch.full(shape + (n,), 9, dtype=torch.int32, device=DEV) if n else None
        self.top_lp = torch.full(shape + (n,), 9.0, device=DEV) if n else None
        self.status = i32([0])
        self.run = lambda: spec.spec_logprobs(
            logits, tokens, B, K, V, self.lp, self.ws, temperature=t, row_offsets=offsets, depth=depth,
            accepted_len=accepted, rank_out=self.rank, entropy_out=self.entropy, top_tokens_out=self.top,
            top_logprobs_out=self.top_lp, status=self.status, stream=stream)
        self.run()

    def check_row(self, i, j, row, token, t, n):
        lp, rank, entropy, best, best_lp = ref.logprobs(row, token, t, n)
        got = float(self.lp[i, j])
        assert got == lp or abs(got - lp) <= ref.logprob_bound(row, t, lp), (got, lp)
        assert int(self.rank[i, j]) == rank
        # each term of the entropy is of one sign, and off as the sums are
        assert abs(float(self.entropy[i, j]) - entropy) <= 2 * (1 + entropy) * ref.logprob_bound(row, t, entropy)
        if n:
            assert self.top[i, j].tolist() == best
            for a, b in zip(self.top_lp[i, j].tolist(), best_lp):
                assert a == b or abs(a - b) <= ref.logprob_bound(row, t, b)

    def nothing(self, i, j):
        assert float(self.lp[i, j]) == -math.inf and int(self.rank[i, j]) == 0 and float(self.entropy[i, j]) == 0
        if self.top is not None:
            assert bool((self.top[i, j] == -1).all()) and bool((self.top_lp[i, j] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,B,K,n,t", [
    (1, 2, 0, 3, 1.0), (7, 3, 2, 32, 1.0), (255, 2, 1, 1, 0.5), (1000, 3, 4, 5, 1.0), (4097, 1, 0, 20, 2.0),
    (32003, 1, 0, 5, 1.0), (50021, 2, 3, 32, 0.7), (201088, 2, 1, 8, 1.0), (100001, 1, 2, 0, 1.0)])
def test_values(V, B, K, n, t, dtype):
    g = torch.Generator().manual_seed(V + n)
    logits = (torch.randn((B * (K + 1), V), generator=g) * 3).to(dtype)
    tokens = torch.randint(0, V, (B, K + 1), generator=g)
    tokens[0, 0] = int(logits[0].float().argmax())
    call = Call(logits.to(DEV), tokens.to(torch.int32).to(DEV), B, K, n, t)
    assert int(call.status) == 0
    for i in range(B):
        for j in range(K + 1):
            call.check_row(i, j, logits[i * (K + 1) + j], int(tokens[i, j]), t, n)
    first = [x.clone() for x in (call.lp, call.entropy)]
    call.run()  # the workspace is ready again, and the result does not depend on the run
    assert torch.equal(first[0], call.lp) and torch.equal(first[1], call.entropy)


def test_packed_rows_and_accepted():
    """The arrays of a verified round: rows past the accepted ones and rows of no request are not asked for."""
    V, B, K, n = 3001, 4, 3, 4
    depth, accepted = [3, 0, 2, 1], [1, 0, 2, 0]
    offsets = [0, 4, 5, 8, 10]
    g = torch.Generator().manual_seed(3)
    logits = torch.randn((12, V), generator=g).to(BF16)
    tokens = torch.full((B, K + 1), -1)
    for i, a in enumerate(accepted):
        tokens[i, :a + 1] = torch.randint(0, V, (a + 1,), generator=g)
    tokens[2, 1] = -1  # asked for its alternatives alone
    call = Call(logits.to(DEV), tokens.to(torch.int32).to(DEV), B, K, n, 0.0, i32(offsets), i32(depth), i32(accepted))
    assert int(call.status) == 0
    for i in range(B):
        for j in range(K + 1):
            if j <= accepted[i]:
                call.check_row(i, j, logits[offsets[i] + j], int(tokens[i, j]), 1.0, n)
            else:
                call.nothing(i, j)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["equal", "few_levels", "zeros", "one_finite", "few_finite", "masked_blocks", "sorted",
                                  "reversed", "huge", "last"])
def test_ties_and_masks(kind, dtype):
    """Lists that many equal entries overflow, entries at -inf, both zeros, every order; 32 alternatives."""
    V, n = 40007, 32
    g = torch.Generator().manual_seed(5)
    x = torch.randn((1, V), generator=g)
    if kind == "equal":
        x.fill_(1.5)
    elif kind == "few_levels":
        x = torch.randint(0, 3, (1, V), generator=g).float()
    elif kind == "zeros":
        x = torch.where(x > 0, 0.0, -0.0)
    elif kind == "one_finite":
        x.fill_(-math.inf)
        x[0, 17001] = -3.0
    elif kind == "few_finite":
        x[0, torch.randperm(V, generator=g)[11:]] = -math.inf
    elif kind == "masked_blocks":
        x[0, :39000] = -math.inf
    elif kind == "sorted":
        x = x.sort(descending=True)[0]
    elif kind == "reversed":
        x = x.sort()[0]
    elif kind == "huge":
        x = x * 1e37
    elif kind == "last":
        x[0, -1] = 40.0
    row = x.to(dtype)
    for token in (0, V // 2, V - 1):
        call = Call(row.to(DEV), i32([[token]]), 1, 0, n)
        assert int(call.status) == 0
        call.check_row(0, 0, row[0], token, 1.0, n)


@pytest.mark.parametrize("V", [5, 20000])
def test_bad_rows(V):
    g = torch.Generator().manual_seed(6)
    good = torch.randn(V, generator=g)
    for bad in (math.nan, math.inf, None):
        rows = good.repeat(2, 1)
        if bad is None:
            rows[1] = -math.inf
        else:
            rows[1, V - 2] = bad
        call = Call(rows.to(DEV), i32([[1], [2]]), 2, 0, 3)
        assert int(call.status) == spec.ERR_BAD_INPUT
        call.nothing(1, 0)
        call.check_row(0, 0, rows[0], 1, 1.0, 3)
    # tokens and accepted lengths out of range
    rows = good.repeat(6, 1)
    call = Call(rows.to(DEV), i32([[V, 0], [0, 1], [3, 3]]), 3, 1, 2, accepted=i32([1, 2, 1]))
    assert int(call.status) == spec.ERR_BAD_INPUT
    call.check_row(0, 0, good, -1, 1.0, 2)
    call.check_row(0, 1, good, 0, 1.0, 2)
    call.check_row(2, 1, good, 3, 1.0, 2)
    call.nothing(1, 0), call.nothing(1, 1)


def test_unaligned_view_graph_and_stream():
    """Logits at an odd address, on a stream of their own, in a replayed graph."""
    V, B = 5003, 2
    flat = torch.randn(1 + B * V, device=DEV).to(BF16)
    logits = flat[1:].view(B, V)
    assert logits.data_ptr() % 4 == 2
    tokens = i32([[7], [5002]])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = Call(logits, tokens, B, 0, 6, 0.9, stream=side)
    side.synchronize()
    for i in range(B):
        call.check_row(i, 0, logits[i].cpu(), int(tokens[i, 0]), 0.9, 6)
    plain = Call(logits, tokens, B, 0, 6, 0.9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plain.run()
    for _ in range(2):
        flat.copy_(torch.randn(1 + B * V, device=DEV))
        graph.replay()
        for i in range(B):
            plain.check_row(i, 0, logits[i].cpu(), int(tokens[i, 0]), 0.9, 6)
    assert int(plain.status) == 0


@pytest.mark.parametrize("B,K,V,n", [(700, 2, 611, 3), (513, 0, 2500, 0), (1500, 1, 33, 32)])
def test_many_requests(B, K, V, n):
    """More requests than a CTA lists; bad ones among them, whose rows the others' places do not depend on."""
    g = torch.Generator().manual_seed(B)
    depth = torch.randint(0, K + 1, (B,), generator=g).tolist()
    offsets = [0]
    for d in depth:
        offsets.append(offsets[-1] + d + 1)
    logits = torch.randn((offsets[-1], V), generator=g).to(BF16)
    tokens = torch.randint(0, V, (B, K + 1), generator=g)
    accepted = [int(torch.randint(0, d + 1, (1,), generator=g)) for d in depth]
    given = list(accepted)
    bad = {2, B // 2, B - 1}
    for i in bad:
        given[i] = depth[i] + 1
    call = Call(logits.to(DEV), tokens.to(torch.int32).to(DEV), B, K, n, 0.8, i32(offsets), i32(depth), i32(given))
    assert int(call.status) == spec.ERR_BAD_INPUT
    for i in range(B):
        for j in range(K + 1):
            if i in bad or j > accepted[i]:
                call.nothing(i, j)
            elif i % 23 == 0 or i > B - 5:
                call.check_row(i, j, logits[offsets[i] + j], int(tokens[i, j]), 0.8, n)
    x = logits.double() / 0.8
    lse = torch.logsumexp(x, 1)
    got = call.lp.cpu().double()
    for i in range(B):
        if i not in bad:
            for j in range(accepted[i] + 1):
                r = offsets[i] + j
                want = float(x[r, tokens[i, j]] - lse[r])
                assert abs(float(got[i, j]) - want) <= ref.logprob_bound(logits[r], 0.8, want)


@pytest.mark.parametrize("V,B,K,n", [(40961, 12, 4, 32), (201088, 3, 0, 32), (201089, 1, 16, 20)])
def test_captured_rounds(V, B, K, n):
    """Rows in many pieces that end inside spans; other accepted lengths, other tokens, other logits at each replay."""
    g = torch.Generator().manual_seed(V)
    R = B * (K + 1)
    logits = (torch.randn((R, V), generator=g) * 2).to(BF16).to(DEV)
    tokens, accepted = i32([[0] * (K + 1)] * B), i32([0] * B)
    call = Call(logits, tokens, B, K, n, 1.0, accepted=accepted)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call.run()
    for step in range(3):
        kept = [(i + step * (K + 1) // 2) % (K + 1) for i in range(B)]
        accepted.copy_(i32(kept))
        tokens.copy_(torch.randint(0, V, (B, K + 1), generator=g))
        if step == 2:
            logits.copy_(logits.flip(0).roll(1234, 1))
        graph.replay()
        torch.cuda.synchronize()
        assert int(call.status) == 0
        rows, picked = logits.cpu(), tokens.tolist()
        for i in range(B):
            for j in range(K + 1):
                if j <= kept[i]:
                    if (i + j) % 3 == 0:
                        call.check_row(i, j, rows[i * (K + 1) + j], picked[i][j], 1.0, n)
                else:
                    call.nothing(i, j)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t", [2.0 ** -126, 1e-30, 1e-3, 1e30, 3e38])
def test_extreme_temperatures(t, dtype):
    """From a distribution that is one entry's to a flat one."""
    V = 5001
    g = torch.Generator().manual_seed(12)
    row = torch.randn((1, V), generator=g).to(dtype)
    best = int(row[0].float().argmax())
    for token in (best, 17):
        call = Call(row.to(DEV), i32([[token]]), 1, 0, 3, t)
        assert int(call.status) == 0
        want = float(torch.log_softmax(row[0].double() / t, 0)[token])
        got = float(call.lp[0, 0])
        # where its binary logarithm is beyond fp32's range a log probability is -inf
        assert (want / math.log(2) < -3.4e38 and got == -math.inf) or abs(got - want) <= ref.logprob_bound(row[0], t, want), (got, want)
        assert float(call.entropy[0, 0]) >= 0 and float(call.entropy[0, 0]) < 1.001 * math.log(V)
        assert int(call.top[0, 0, 0]) == best


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t", [2.0 ** -126, 1e-3, 1e30, 1e35, 4e35, 6e35, 1e37, 3.4028234e38])
@pytest.mark.parametrize("kind", ["finite", "masked", "wide"])
def test_entropy_at_extreme_temperatures(t, kind, dtype):
    """Also where 1,000 binary orders below the largest logit lie outside the type: entries at -inf, and what fills a
    row's last vector, are no part of the sum.  Logits of the whole range stay what they are beside such a temperature."""
    for V in (5001, 40003):
        g = torch.Generator().manual_seed(13)
        row = torch.randn(V, generator=g) if kind != "wide" else torch.empty(V).uniform_(-1.0, 1.0, generator=g) * 3e38
        if kind == "masked":
            row[torch.rand(V, generator=g) < 0.4] = -math.inf
        row = row.to(dtype)
        best = int(row.float().argmax())
        call = Call(row[None].to(DEV), i32([[best]]), 1, 0, 4, t)
        assert int(call.status) == 0
        _, _, entropy, top, _ = ref.logprobs(row, best, t, 4)
        # c2 = log2(e) / t below the smallest normal number is off by up to 2^-150, with logits of up to 2^128 on both
        # sides of a difference 2^-21 in all
        tol = 2 * (1 + entropy) * ref.logprob_bound(row, t, entropy) + (2.0 ** -21 if kind == "wide" else 0.0)
        assert abs(float(call.entropy[0, 0]) - entropy) <= tol, (float(call.entropy[0, 0]), entropy)
        assert call.top[0, 0].tolist() == top


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("t,V", [(1.0, 5001), (0.01, 5001), (0.01, 201088), (100.0, 40003)])
def test_sums_of_two_references(t, V, sign):
    """The largest logits around 8,192 binary orders on either side: below that a sum is relative to its largest logit's
    rounded product with log2(e) / t, beyond it to the exact one, and sums of both kinds meet in a row.  (In bf16 such
    logits are 32 binary orders apart, and only the largest counts.)"""
    n = 8
    g = torch.Generator().manual_seed(V)
    row = sign * 8192 * math.log(2) * t + t * torch.empty(V).uniform_(-1.0, 1.0, generator=g)
    # some have the border within a thread's own elements, some between threads, some between a row's pieces
    for r in (row, row.sort()[0], row.sort(descending=True)[0]):
        tokens = [0, int(r.argmax()), V - 1]
        call = Call(r.repeat(3, 1).to(DEV), i32([[x] for x in tokens]), 3, 0, n, t)
        assert int(call.status) == 0
        for i, token in enumerate(tokens):
            call.check_row(i, 0, r, token, t, n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t", [1.0, 1.3, 7.0, 1e5])
@pytest.mark.parametrize("kind", ["masked", "all_masked", "wide"])
def test_masks_of_the_lowest_value(kind, t, dtype):
    """Entries at the type's lowest value are entries like others: ln p of them is what it is, where it is in fp32's
    range, as a token's and among the alternatives; logits of the whole range likewise."""
    V, n = 3001, 32
    g = torch.Generator().manual_seed(14)
    row = torch.randn(V, generator=g)
    if kind == "wide":
        row = torch.empty(V).uniform_(-1.0, 1.0, generator=g) * 3.3e38
    row = row.to(dtype)
    if kind == "masked":
        row[torch.randperm(V, generator=g)[7:]] = torch.finfo(dtype).min
    elif kind == "all_masked":
        row.fill_(torch.finfo(dtype).min)
    for token in (0, int(row.argmin()), int(row.argmax()), V - 1):
        call = Call(row[None].to(DEV), i32([[token]]), 1, 0, n, t)
        assert int(call.status) == 0
        lp, rank, entropy, best, best_lp = ref.logprobs(row, token, t, n)

        def same(got, want):
            # fp32's largest number is 2^128 - 2^104: what is at -2^128 or below is -inf in it
            return got == -math.inf if want <= -2.0 ** 128 else abs(got - want) <= ref.logprob_bound(row, t, want)
        assert same(float(call.lp[0, 0]), lp) and int(call.rank[0, 0]) == rank
        assert abs(float(call.entropy[0, 0]) - entropy) <= 2 * (1 + entropy) * ref.logprob_bound(row, t, entropy)
        assert call.top[0, 0].tolist() == best
        assert all(same(a, b) for a, b in zip(call.top_lp[0, 0].tolist(), best_lp))
