"""PagedCache in captured CUDA graphs: a graph goes on reading and writing the
cache's own table after a fork, and a captured fork acts at every replay."""
import pytest
import torch

import paged_ref as ref
from paper_2607_25852_gb300.paged import PagedCache

pytestmark = pytest.mark.gpu

DEV = "cuda"
L, PS, HQ, HKV, D, B, K = 1, 8, 4, 2, 64, 4, 2


def filled(seed):
    """A cache in which each request holds a few written pages, and its next positions."""
    c = PagedCache(L, 64, PS, HQ, HKV, D, B, 64, K, torch.bfloat16)
    g = torch.Generator().manual_seed(seed)
    pos = torch.zeros(B, dtype=torch.int64, device=DEV)
    for step in range(5):
        c.reserve(pos)
        k, v = (torch.randn((B * (K + 1), HKV, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
        c.append(0, k, v, pos)
        pos += K + 1
    return c, pos, g


def test_a_captured_round_follows_a_fork():
    c, pos, g = filled(1)
    q = torch.randn((B * (K + 1), HQ, D), generator=g).to(torch.bfloat16).to(DEV)
    k, v = (torch.randn((B * (K + 1), HKV, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    out = torch.empty_like(q)

    def step():
        c.reserve(pos)
        c.append(0, k, v, pos)
        c.attend(0, q, pos, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    c.fork(torch.tensor([2, 2, 3, 0], dtype=torch.int32, device=DEV))
    before = [x.clone() for x in (c.page_table, c.page_refs, c.k, c.v)]
    step()
    want = [x.clone() for x in (c.page_table, c.page_refs, out)]
    for x, y in zip((c.page_table, c.page_refs, c.k, c.v), before):
        x.copy_(y)
    out.zero_()
    graph.replay()
    for x, y in zip((c.page_table, c.page_refs, out), want):
        assert torch.equal(x, y)
    assert int(c.status) == 0


def test_a_captured_fork_acts_at_every_replay():
    c, pos, _ = filled(2)
    parent = torch.zeros(B, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.fork(parent)
    for children in ([1, 0, 3, 2], [0, 0, 2, -1], [3, 1, 1, 2], [0, 1, 2, 3]):
        want, want_refs = ref.fork(c.page_table.tolist(), c.page_refs.tolist(), children)
        parent.copy_(torch.tensor(children, dtype=torch.int32))
        graph.replay()
        assert c.page_table.tolist() == want and c.page_refs.tolist() == want_refs and int(c.status) == 0


def test_a_fork_on_a_side_stream():
    c, pos, _ = filled(3)
    want, want_refs = ref.fork(c.page_table.tolist(), c.page_refs.tolist(), [3, 3, 0, -1])
    parent = torch.tensor([3, 3, 0, -1], dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.fork(parent, stream=s)
    s.synchronize()
    assert c.page_table.tolist() == want and c.page_refs.tolist() == want_refs and int(c.status) == 0
