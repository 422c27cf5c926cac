"""The page operators against loops over lists (paged_ref): whole numbers, so
everything has to be equal."""
import pytest
import torch

import paged_ref as ref
import paper_2607_25852_gb300 as spec

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def i64(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


def new_status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def gen(seed):
    return torch.Generator().manual_seed(seed)


SIZES = [(1, 1, 1, 0), (3, 5, 64, 2), (7, 40, 300, 9), (33, 130, 5000, 50), (40, 1500, 70000, 1000)]


@pytest.mark.parametrize("B,M,P,extra", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
def test_fork(B, M, P, extra, in_place):
    g = gen(B + M)
    have = [int(torch.randint(0, min(M, P // B) + 1, (1,), generator=g)) for _ in range(B)]
    table, refs = ref.random_pages(B, M, P, have, g, extra=min(extra, P - sum(have)))
    for B2 in (1, B, 2 * B + 1):
        parent = torch.randint(-1, B, (B2,), generator=g).tolist()
        want, want_refs = ref.fork(table, refs, parent)
        t, r, st = i32(table), i32(refs), new_status()
        out = torch.full((B2, M), 99, dtype=torch.int32, device=DEV)
        r_out = r if in_place else torch.full((P,), 99, dtype=torch.int32, device=DEV)
        spec.spec_cache_fork(t, r, i32(parent), out, r_out, status=st)
        assert out.tolist() == want and r_out.tolist() == want_refs and int(st) == 0
        assert t.tolist() == table


def test_fork_reports_bad_parents_and_entries():
    st = new_status()
    out, refs = torch.zeros((3, 2), dtype=torch.int32, device=DEV), i32([1, 1, 0])
    spec.spec_cache_fork(i32([[0, -1], [1, -1]]), refs, i32([1, 5, 0]), out, refs, status=st)
    assert int(st) == spec.ERR_BAD_INPUT and out.tolist() == [[1, -1], [-1, -1], [0, -1]]
    assert refs.tolist() == [1, 1, 0]
    st, refs = new_status(), i32([1, 1, 0])
    spec.spec_cache_fork(i32([[0, 3], [1, -2]]), refs, i32([1, 0, 0]), out, refs, status=st)
    assert int(st) == spec.ERR_BAD_INPUT and out.tolist() == [[1, -1], [0, -1], [0, -1]]
    assert refs.tolist() == [2, 1, 0]


def run_reserve(table, refs, pos, depth, K, ps, packed=False):
    B = len(table)
    t, r, st = i32(table), i32(refs), new_status()
    cap = B * (K // ps + 2)
    src, dst = (torch.full((cap,), 99, dtype=torch.int32, device=DEV) for _ in range(2))
    counts, granted = torch.full((2,), 99, dtype=torch.int32, device=DEV), torch.full((B,), 99, dtype=torch.int32, device=DEV)
    ws = spec.cache_workspace(B, K, ps, DEV)
    offsets = i32(ref.Rows(depth, K).offsets) if packed else None
    spec.spec_cache_reserve(t, r, i64(pos), B, K, ps, src, dst, counts, granted, ws, row_offsets=offsets,
                            depth=i32(depth), status=st)
    return t.tolist(), r.tolist(), src.tolist(), dst.tolist(), counts.tolist(), granted.tolist(), int(st)


@pytest.mark.parametrize("B,M,P,extra", SIZES + [(1100, 8, 9000, 0)])
@pytest.mark.parametrize("K,ps", [(0, 16), (4, 1), (16, 16), (40, 10), (255, 24)])
def test_reserve(B, M, P, extra, K, ps):
    g = gen(B + M + K)
    span = K // ps + 2
    if M < span:
        M = span
    have = [int(torch.randint(0, min(M - span + 1, max(1, P // (2 * B))) + 1, (1,), generator=g)) for _ in range(B)]
    while sum(have) > P:
        have[have.index(max(have))] -= 1
    table, refs = ref.random_pages(B, M, P, have, g, extra=min(extra, P - sum(have)))
    depth = torch.randint(0, K + 1, (B,), generator=g).tolist()
    pos = []
    for i in range(B):
        top = have[i] * ps  # the next position: in the last page, at its end, or an idle request
        back = int(torch.randint(0, ps + 1, (1,), generator=g))
        pos.append(-1 if i % 7 == 6 else max(0, top - back))
    # shared last pages: half of the requests fork a neighbour
    for i in range(1, B, 2):
        if have[i - 1]:
            for e in table[i]:
                if e >= 0:
                    refs[e] -= 1
            table[i], pos[i] = list(table[i - 1]), pos[i - 1]
            for e in table[i]:
                if e >= 0:
                    refs[e] += 1
    want = ref.reserve(table, refs, pos, depth, ps)
    got = run_reserve(table, refs, pos, depth, K, ps, packed=B % 2 == 1)
    n = len(want[2])
    assert got[5] == want[5]
    assert got[0] == want[0] and got[1] == want[1]
    assert got[2][:n] == want[2] and got[3][:n] == want[3]
    assert set(got[2][n:]) <= {-1} and set(got[3][n:]) <= {-1}
    assert got[4] == [n, want[4]]
    assert got[6] == (spec.ERR_CACHE_FULL if want[6] else 0)


def test_reserve_when_the_cache_is_full():
    refs = [1, 0, 2, 1, 0, 1]
    table = [[0, -1, -1], [2, -1, -1], [2, 3, -1], [5, -1, -1]]
    pos, depth = [4, 2, 8, 1], [0, 3, 0, 1]       # page size 4: needs 1, 2, 1 and none
    want = ref.reserve(table, refs, pos, depth, 4)
    got = run_reserve(table, refs, pos, depth, 3, 4)
    assert want[5] == [1, 0, 0, 1] and got[5] == want[5]
    assert got[0] == want[0] and got[1] == want[1] and got[6] == spec.ERR_CACHE_FULL and got[4] == [0, 1]


def test_reserve_reports_bad_input():
    for table, pos, depth in ([[[0, -1]], [8], [0]], [[[9, -1]], [1], [0]], [[[-3, -1]], [1], [0]], [[[0, -1]], [0], [2]],
                              [[[0, -1]], [1 << 40], [0]]):
        t = table + [[1, -1]]
        got = run_reserve(t, [1, 1, 0, 0], pos + [4], depth + [0], 1, 4)
        assert got[6] == spec.ERR_BAD_INPUT and got[5] == [0, 1] and got[0] == [table[0], [1, 2]], got
        assert got[1] == [1, 1, 1, 0]


@pytest.mark.parametrize("B,M,P,extra", SIZES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (20, 4), (33, 40)])
def test_release(B, M, P, extra, window, sinks):
    g = gen(B + M + window)
    ps = 8
    have = [int(torch.randint(0, min(M, P // B) + 1, (1,), generator=g)) for _ in range(B)]
    table, refs = ref.random_pages(B, M, P, have, g)
    pos = [int(torch.randint(-1, max(1, h * ps), (1,), generator=g)) for h in have]
    acc = torch.randint(0, 5, (B,), generator=g).tolist()
    for accepted in (acc, None):
        keep = [max(0, p + a + 1) for p, a in zip(pos, acc)] if accepted else [max(0, p) for p in pos]
        want, want_refs = ref.release(table, refs, keep, ps, window, sinks)
        t, r, st = i32(table), i32(refs), new_status()
        spec.spec_cache_release(t, r, i64(pos), ps, accepted_len=None if accepted is None else i32(accepted),
                                window=window, sinks=sinks, status=st)
        assert t.tolist() == want and r.tolist() == want_refs and int(st) == 0


def test_release_reports_bad_input():
    for table, refs, acc in ([[[7]], [1], 0], [[[-2]], [1], 0], [[[0]], [0], 0], [[[-1]], [1], -1]):
        st, t, r = new_status(), i32(table), i32(refs)
        spec.spec_cache_release(t, r, i64([-1]), 4, accepted_len=i32([acc]), status=st)
        assert int(st) == spec.ERR_BAD_INPUT and t.tolist() == ([[0]] if acc < 0 and table == [[0]] else [[-1]])


@pytest.mark.parametrize("B,M,P,extra", SIZES + [(2, 3, 8192, 4000), (5, 9, 64, 0)])
def test_compact(B, M, P, extra):
    g = gen(B + P)
    have = [int(torch.randint(0, min(M, P // B) + 1, (1,), generator=g)) for _ in range(B)]
    table, refs = ref.random_pages(B, M, P, have, g, extra=min(extra, P - sum(have)))
    want, want_refs, src, dst, page_map, n = ref.compact(table, refs)
    cap = max(1, P // 2)
    t, r, st = i32(table), i32(refs), new_status()
    o = [torch.full((m,), 99, dtype=torch.int32, device=DEV) for m in (cap, cap, P, 2)]
    spec.spec_cache_compact(t, r, *o, status=st)
    assert o[3].tolist() == [len(src), n]
    assert o[0].tolist() == src + [-1] * (cap - len(src)) and o[1].tolist() == dst + [-1] * (cap - len(dst))
    assert o[2].tolist() == page_map
    assert t.tolist() == want and r.tolist() == want_refs and int(st) == 0


def test_compact_reports_dead_and_bad_entries():
    st, t, r = new_status(), i32([[3, 1, 9, -5]]), i32([0, 0, 0, 2])
    o = [torch.zeros(m, dtype=torch.int32, device=DEV) for m in (2, 2, 4, 2)]
    spec.spec_cache_compact(t, r, *o, status=st)
    assert int(st) == spec.ERR_BAD_INPUT and t.tolist() == [[0, -1, -1, -1]] and r.tolist() == [2, 0, 0, 0]


LAYOUTS = ["token", "head", "interleaved", "sliced"]


def cache(layout, L, P, ps, H, D, dtype, g):
    if layout == "token":
        return [torch.randn((L, P, ps, H, D), generator=g).to(dtype).to(DEV) for _ in range(2)]
    if layout == "head":
        return [torch.randn((L, P, H, ps, D), generator=g).to(dtype).to(DEV).transpose(2, 3) for _ in range(2)]
    if layout == "interleaved":
        both = torch.randn((P, L, ps, 2, H, D), generator=g).to(dtype).to(DEV).transpose(0, 1)
        return [both[..., 0, :, :], both[..., 1, :, :]]
    wide = torch.randn((2, L, P, ps, H + 1, D + 8), generator=g).to(dtype).to(DEV)  # heads with gaps between them
    return [wide[0, ..., :H, :D], wide[1, ..., :H, :D]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("L,ps,H,D", [(1, 16, 2, 64), (3, 10, 3, 8), (2, 1, 1, 96), (1, 128, 8, 128)])
def test_copy(L, ps, H, D, layout, dtype):
    g = gen(L + ps)
    P = 40
    k, v = cache(layout, L, P, ps, H, D, dtype, g)
    want = [k.clone(), v.clone()]
    perm = torch.randperm(P, generator=g).tolist()
    src, dst = perm[:15], perm[15:30]
    for w in want:
        w[:, dst] = w[:, src]
    st = new_status()
    spec.spec_cache_copy(k, v, i32(src + [0] * 5), i32(dst + [0] * 5), i32([15, 77]), status=st)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and int(st) == 0
    spec.spec_cache_copy(k, v, i32(src), i32(dst), i32([0]), status=st)  # nothing to copy
    assert torch.equal(k, want[0]) and int(st) == 0


def test_copy_reports_bad_pages_and_counts():
    k, v = (torch.randn((4, 2, 1, 8), device=DEV) for _ in range(2))
    for src, dst, n in ([[0, 4], [1, 2], 2], [[0, 1], [1, -1], 2], [[0], [1], 9], [[0], [1], -3]):
        st, kk, vv = new_status(), k.clone(), v.clone()
        spec.spec_cache_copy(kk, vv, i32(src), i32(dst), i32([n]), status=st)
        assert int(st) == spec.ERR_BAD_INPUT
        want = k.clone()
        if n > 0:
            want[1] = k[0]
        assert torch.equal(kk, want)


def test_copy_past_32_bits():
    P, ps, H, D = (1 << 32) // (64 * 2 * 128) + 9, 64, 2, 128
    k = torch.empty((P, ps, H, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty((P, ps, H, D), dtype=torch.bfloat16, device=DEV)
    for x in (k, v):
        x[P - 2:] = torch.randn((2, ps, H, D), device=DEV).to(torch.bfloat16)
    a, b = k[P - 1].clone(), v[P - 1].clone()
    st = new_status()
    spec.spec_cache_copy(k, v, i32([P - 1, P - 2]), i32([3, P - 3]), i32([2]), status=st)
    assert torch.equal(k[3], a) and torch.equal(v[3], b) and torch.equal(k[P - 3], k[P - 2]) and int(st) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("ps,H,D,K", [(16, 2, 64, 4), (10, 3, 8, 0), (1, 1, 96, 16), (64, 8, 128, 255)])
def test_append(ps, H, D, K, layout, dtype):
    g = gen(ps + K)
    depth = [K, 0, K // 2, K]
    pos = [0, 31, -1, 97]
    rows = ref.Rows(depth, K)
    need = [(p + n) // ps + 1 for p, n in zip(pos, depth)]
    P, M, layer = sum(need) + 2, max(need), 1
    table = ref.random_table(4, need, P, M, g)
    k, v = cache(layout, 2, P, ps, H, D, dtype, g)
    want = [k.clone(), v.clone()]
    fused = torch.randn((rows.R, 2 * H * D + 16), generator=g).to(dtype).to(DEV)
    k_new = fused[:, :H * D].view(rows.R, H, D)
    v_new = fused[:, H * D + 16:].view(rows.R, H, D)
    for i in range(4):
        for j in range(depth[i] + 1):
            p = pos[i] + j
            if p < 0:
                continue
            for w, n in zip(want, (k_new, v_new)):
                w[layer, int(table[i, p // ps]), p % ps] = n[rows.offsets[i] + j]
    st = new_status()
    spec.spec_cache_append(k_new, v_new, k, v, table.to(DEV), i64(pos), 4, K, row_offsets=i32(rows.offsets),
                           depth=i32(depth), layer=layer, status=st)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and int(st) == 0


def test_append_skips_and_reports_bad_rows():
    k, v = (torch.zeros((4, 2, 1, 8), device=DEV) for _ in range(2))
    new = torch.ones((4, 1, 8), device=DEV)
    table = i32([[0, -1], [1, 9]])
    for pos, depth, written in (([1, 0], [1, 1], [(0, 1), (1, 0), (1, 1)]),      # slot 1 of request 0 has no page
                                ([0, 2], [1, 0], [(0, 0), (0, 1)]),              # page 9 does not exist
                                ([0, 3], [1, 1], [(0, 0), (0, 1)]),              # position 4 is past the table too
                                ([0, 1 << 41], [0, 0], [(0, 0)]), ([0, 0], [0, 2], [(0, 0)])):
        st = new_status()
        k.zero_()
        spec.spec_cache_append(new, new, k, v, table, i64(pos), 2, 1, depth=i32(depth), status=st)
        assert int(st) == spec.ERR_BAD_INPUT
        got = {(int(a), int(b)) for a, b in k[:, :, 0, 0].nonzero().tolist()}
        assert got == set(written), (pos, got)


def test_page_operators_write_inside():
    from test_gpu_canaries import Guarded, assert_intact
    g = gen(5)
    B, M, P, K, ps = 6, 9, 61, 7, 4
    table, refs = ref.random_pages(B, M, P, [4, 0, 7, 2, 5, 3], g, extra=3)
    parent = [0, 0, 2, 2, 2, 5, -1]
    B2 = len(parent)
    t1, r1 = Guarded((B2, M), torch.int32, 99), Guarded((P,), torch.int32, 99)
    spec.spec_cache_fork(i32(table), i32(refs), i32(parent), t1.t, r1.t)
    pos, depth = [13, 14, 25, 26, 27, 9, 0], [7, 0, 7, 3, 1, 7, 7]
    cap = B2 * (K // ps + 2)
    o = {n: Guarded((m,), torch.int32, 99) for n, m in dict(src=cap, dst=cap, counts=2, granted=B2).items()}
    ws = Guarded((spec.spec_cache_workspace(B2, K, ps),), torch.uint8, 0)
    spec.spec_cache_reserve(t1.t, r1.t, i64(pos), B2, K, ps, o["src"].t, o["dst"].t, o["counts"].t, o["granted"].t,
                            ws.t, depth=i32(depth))
    f, fr = ref.fork(table, refs, parent)
    want = ref.reserve(f, fr, pos, depth, ps)
    assert t1.t.tolist() == want[0] and r1.t.tolist() == want[1]
    spec.spec_cache_release(t1.t, r1.t, i64(pos), ps, accepted_len=i32([0] * B2), window=6, sinks=2)
    c = {n: Guarded((m,), torch.int32, 99) for n, m in dict(src=P // 2, dst=P // 2, map=P, counts=2).items()}
    spec.spec_cache_compact(t1.t, r1.t, c["src"].t, c["dst"].t, c["map"].t, c["counts"].t)
    t2, r2 = ref.release(want[0], want[1], [p + 1 for p in pos], ps, 6, 2)
    assert t1.t.tolist() == ref.compact(t2, r2)[0]
    kv = Guarded((2, P, ps, 1, 8), torch.float32, 0)
    spec.spec_cache_copy(kv.t[0], kv.t[1], c["src"].t, c["dst"].t, c["counts"].t)
    assert_intact(table=t1, refs=r1, ws=ws, kv=kv, **o, **{"c" + n: x for n, x in c.items()})
