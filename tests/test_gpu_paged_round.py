"""The paged cache in use: speculative decoding over it gives the tokens of
plain greedy decoding with attention over the whole sequence, and its pages
come and go as the requests do."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_round.py")
    s = importlib.util.spec_from_file_location("paged_round", path)
    m = importlib.util.module_from_spec(s)
    s.loader.exec_module(m)
    return m


def plain_greedy(target, prompt, new_tokens, window, sinks):
    """Token by token, every layer's attention over the whole sequence, in fp32."""
    seq = list(prompt)
    Hq, Hkv, D = target.q_heads, target.kv_heads, target.head_dim
    for _ in range(new_tokens):
        n = len(seq)
        t = torch.arange(n, device=DEV)
        seen = t[None] <= t[:, None]
        if window:
            seen &= (t[None] > t[:, None] - window) | (t[None] < sinks)

        def attention(layer, q, k, v):
            k, v = (x.repeat_interleave(Hq // Hkv, 1).transpose(0, 1) for x in (k, v))
            x = (q.transpose(0, 1) @ k.transpose(1, 2)) * D ** -0.5
            return (torch.softmax(x.masked_fill(~seen, float("-inf")), -1) @ v).transpose(0, 1)
        logits = target.forward(torch.tensor(seq, device=DEV), t, attention)
        seq.append(int(logits[-1].argmax()))
    return seq


@pytest.mark.parametrize("window,sinks,page_size", [(0, 0, 16), (24, 3, 8), (40, 0, 10)])
def test_speculative_decoding_over_the_paged_cache(example, window, sinks, page_size):
    V = 29
    target = example.Target(2, 4, 2, 32, V, 256, seed=3)
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, V, (n,), generator=g).tolist() for n in (1, 7, 130, 40)]
    out, rounds = example.generate(target, prompts, 20, K=3, page_size=page_size, pages=400 // page_size + 60,
                                   window=window, sinks=sinks)
    assert 20 / 4 <= rounds < 20     # some drafts are accepted
    for p, s in zip(prompts, out):
        assert s == plain_greedy(target, p, 20, window, sinks)


def test_forked_requests_write_their_own_pages():
    from paper_2607_25852_gb300.paged import PagedCache
    L, ps, Hq, Hkv, D, B = 2, 8, 4, 2, 64, 4
    c = PagedCache(L, 32, ps, Hq, Hkv, D, B, 64, 2, torch.bfloat16)
    g = torch.Generator().manual_seed(2)

    def rows():
        return torch.randn((B * 3, Hkv, D), generator=g).to(torch.bfloat16).to(DEV)
    pos = torch.tensor([0, -9, -9, -9], device=DEV)  # request 0 alone writes
    history = [[], []]
    for step in range(4):                            # positions 0 .. 11, the last page half full
        c.reserve(pos)
        k, v = rows(), rows()
        for layer in range(L):
            c.append(layer, k, v, pos)
        history[0].append(k[:3])
        history[1].append(v[:3])
        pos = pos + torch.tensor([3, 0, 0, 0], device=DEV)
    c.fork(torch.tensor([0, 0, -1, 0], dtype=torch.int32, device=DEV))
    table = c.page_table.tolist()
    assert table[0][:2] == table[1][:2] == table[3][:2] and table[2] == [-1] * 8
    assert sorted(c.page_refs.tolist())[-2:] == [3, 3]
    pos = torch.tensor([12, 12, -9, 12], device=DEV)
    assert c.reserve(pos).tolist() == [1, 1, 1, 1]
    table = c.page_table.tolist()
    assert len({table[i][1] for i in (0, 1, 3)}) == 3 and table[0][0] == table[1][0] == table[3][0]
    k, v = rows(), rows()
    q = torch.randn((B * 3, Hq, D), generator=g).to(torch.bfloat16).to(DEV)
    out = torch.empty_like(q)
    for layer in range(L):
        c.append(layer, k, v, pos)
    for i in range(2):                               # before and after the pages have moved
        c.attend(1, q, pos, out)
        for r in (0, 1, 3):
            kk = torch.cat(history[0] + [k[3 * r:3 * r + 3]]).float().repeat_interleave(2, 1)
            vv = torch.cat(history[1] + [v[3 * r:3 * r + 3]]).float().repeat_interleave(2, 1)
            x = torch.einsum("hd,thd->ht", q[3 * r + 2].float(), kk) * D ** -0.5
            want = torch.einsum("ht,thd->hd", torch.softmax(x, 1), vv)
            # the weights' and the result's roundings: 2^-9 of sum p |v| <= max |v|, and of the result
            assert ((out[3 * r + 2].float() - want).abs() <= 2.0 ** -8 * vv.abs().amax()).all()
        assert (out[6:9] == 0).all()                 # the idle request
        c.commit(torch.tensor([12, 12, 0, 12], device=DEV), torch.tensor([2, 2, 0, 2], dtype=torch.int32, device=DEV))
        c.commit(torch.tensor([15, 15, 0, 15], device=DEV))
        c.compact()
    live = int((c.page_refs > 0).sum())
    assert live == 1 + 3 and (c.page_refs[:live] > 0).all() and int(c.status) == 0
    c.commit(torch.zeros(B, dtype=torch.int64, device=DEV))
    assert int(c.page_refs.sum()) == 0


def test_a_full_cache_grants_in_order():
    from paper_2607_25852_gb300.paged import PagedCache
    import paper_2607_25852_gb300 as spec
    c = PagedCache(1, 3, 4, 2, 1, 64, 4, 16, 0)
    pos = torch.zeros(4, dtype=torch.int64, device=DEV)
    assert c.reserve(pos).tolist() == [1, 1, 1, 0] and int(c.status) == spec.ERR_CACHE_FULL
    c.commit(torch.tensor([1, 0, 1, 0], device=DEV))  # the second request gives its page back
    c.status.zero_()
    assert c.reserve(torch.tensor([1, -1, 1, 0], device=DEV)).tolist() == [1, 1, 1, 1] and int(c.status) == 0
