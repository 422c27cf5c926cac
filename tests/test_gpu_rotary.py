"""spec_rotary and spec_rotary_append against turns in 64 bits, and against
spec_cache_append for what they leave alone."""
import pytest
import torch

import paged_ref
import paper_2607_25852_gb300 as spec
import rows_ref as ref
from paper_2607_25852_gb300.paged import PagedCache

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def check(got, want, err, dtype):
    got = got.cpu().double()
    tol = err + want.abs() * ref.half_step(dtype) * 1.01 + 1e-38
    bad = (got - want).abs() > tol
    assert not bad.any(), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,rot,inter,heads", [
    (128, 128, False, 5), (128, 128, True, 3), (64, 32, False, 9), (64, 16, True, 1), (96, 24, False, 2),
    (80, 50, False, 7), (80, 50, True, 7), (256, 256, False, 1), (8, 2, False, 3), (128, 38, False, 40),
    (256, 12, True, 66)])
def test_rows(D, rot, inter, heads, dtype):
    depth, K = [2, 0, 3, 1], 3
    pos = [0, 131071, 1 << 30, 7]
    rows = paged_ref.Rows(depth, K)
    g = torch.Generator().manual_seed(D + rot)
    x = torch.randn((rows.R + 2, heads, D), generator=g).to(dtype)
    freq = ref.frequencies(rot, 10000.0, "linear", 2.0)
    f = spec.spec_rotary_frequencies(rot, 10000.0, "linear", 2.0)
    assert f.tolist() == pytest.approx(freq, rel=1e-14)
    out = torch.full(x.shape, 7.0, dtype=dtype, device=DEV)
    status = i32([0])
    xd = x.to(DEV)
    spec.spec_rotary(xd, f, torch.tensor(pos, device=DEV), 4, K, out, interleaved=inter, amplitude=1.25,
                     row_offsets=i32(rows.offsets), depth=i32(depth), status=status)
    same = xd.clone()
    spec.spec_rotary(same, f, torch.tensor(pos, device=DEV), 4, K, same, interleaved=inter, amplitude=1.25,
                     row_offsets=i32(rows.offsets), depth=i32(depth), status=status)
    assert int(status) == 0
    assert torch.equal(same[:rows.R], out[:rows.R]) and torch.equal(same[rows.R:], xd[rows.R:])
    assert bool((out[rows.R:] == 7).all())
    for i in range(4):
        for j in range(depth[i] + 1):
            r = rows.offsets[i] + j
            # the frequencies that the kernel got, to the last bit
            want, err = ref.rotate(x[r], pos[i] + j, f.tolist(), inter, 1.25)
            check(out[r], want, err, dtype)
            assert torch.equal(out[r, :, rot:].cpu(), x[r, :, rot:])


def test_turned_back():
    x = torch.randn((6, 4, 64), device=DEV)
    f = spec.spec_rotary_frequencies(64)
    pos = torch.tensor([12345, 99], device=DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    spec.spec_rotary(x, f, pos, 2, 2, y)
    spec.spec_rotary(y, -f, pos, 2, 2, z)
    # each way is off by at most 2^-20 of a pair's elements
    assert float((x - z).abs().max()) < 4 * float(x.abs().max()) * 2.0 ** -20


def test_skipped_rows_and_views():
    """Rows before position 0 and rows of no request are left alone; x and out may be views of wider rows."""
    wide, out = torch.randn((9, 6, 32), device=DEV), torch.full((9, 3, 32), 5.0, device=DEV)
    f = spec.spec_rotary_frequencies(32)
    status = i32([0])
    spec.spec_rotary(wide[:, 1:4], f, torch.tensor([-2, 4, -3], device=DEV), 3, 2, out, status=status)
    assert int(status) == 0
    assert bool((out[[0, 1, 6, 7, 8]] == 5).all())
    for r, p in [(2, 0), (3, 4), (4, 5), (5, 6)]:
        want, err = ref.rotate(wide[r, 1:4].cpu(), p, f.tolist(), False, 1.0)
        check(out[r], want, err, F32)


def test_bad_data():
    x, out = torch.randn((6, 1, 32), device=DEV), torch.full((6, 1, 32), 5.0, device=DEV)
    f, status, pos = spec.spec_rotary_frequencies(32), i32([0]), torch.tensor([1, 1], device=DEV)
    spec.spec_rotary(x, f, pos, 2, 2, out, row_offsets=i32([0, 3, 5]), depth=i32([2, 2]), status=status)
    assert int(status) == spec.ERR_BAD_INPUT and bool((out[3:] == 5).all())
    status.zero_()
    f[3] = float("nan")
    spec.spec_rotary(x, f, pos, 2, 2, out, status=status)
    assert int(status) == spec.ERR_BAD_INPUT
    assert torch.equal(out[:, :, [3, 19]], x[:, :, [3, 19]]) and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype,D,rot,inter,ps,fused", [
    (BF16, 128, 128, False, 16, True), (F32, 64, 32, True, 10, False), (BF16, 80, 24, False, 7, True),
    (BF16, 256, 256, True, 64, False)])
def test_append(dtype, D, rot, inter, ps, fused):
    """q, K and V of a round: the same as spec_rotary and spec_cache_append one after the other, and right."""
    Hq, Hkv, K = 6, 2, 5
    depth, pos = [5, 0, 3, 2], [0, 37, ps - 1, 1000]
    rows = paged_ref.Rows(depth, K)
    g = torch.Generator().manual_seed(D)
    need = [(p + n) // ps + 1 for p, n in zip(pos, depth)]
    pages = sum(need) + 2
    table = paged_ref.random_table(4, need, pages, max(need), g).to(DEV)
    if fused:
        r = torch.randn((rows.R, Hq + 2 * Hkv, D), generator=g).to(dtype).to(DEV)
        q, k, v = r[:, :Hq], r[:, Hq:Hq + Hkv], r[:, Hq + Hkv:]
    else:
        q, k, v = (torch.randn((rows.R, h, D), generator=g).to(dtype).to(DEV) for h in (Hq, Hkv, Hkv))
    caches = [torch.full((2, pages, ps, Hkv, D), 3.0, dtype=dtype, device=DEV) for _ in range(4)]
    f = spec.spec_rotary_frequencies(rot, 500000.0)
    at = dict(row_offsets=i32(rows.offsets), depth=i32(depth), status=i32([0]))
    where = torch.tensor(pos, device=DEV)
    out = torch.zeros((rows.R, Hq, D), dtype=dtype, device=DEV)
    spec.spec_rotary_append(q, k, v, caches[0], caches[1], table, where, 4, K, f, out, interleaved=inter, layer=1, **at)
    q2, k2 = torch.empty_like(out), torch.empty((rows.R, Hkv, D), dtype=dtype, device=DEV)
    spec.spec_rotary(q, f, where, 4, K, q2, interleaved=inter, **at)
    spec.spec_rotary(k, f, where, 4, K, k2, interleaved=inter, **at)
    spec.spec_cache_append(k2, v, caches[2], caches[3], table, where, 4, K, layer=1, **at)
    assert int(at["status"]) == 0
    assert torch.equal(out, q2) and torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
    spec.spec_rotary_append(None, k, v, caches[0].fill_(3.0), caches[1], table, where, 4, K, f, None, interleaved=inter,
                            layer=1, **at)
    assert torch.equal(caches[0], caches[2])
    for i in range(4):
        for j in range(depth[i] + 1):
            r, p = rows.offsets[i] + j, pos[i] + j
            check(out[r], *ref.rotate(q[r].cpu(), p, f.tolist(), inter, 1.0), dtype)
            page = int(table[i, p // ps])
            check(caches[0][1, page, p % ps], *ref.rotate(k[r].cpu(), p, f.tolist(), inter, 1.0), dtype)


def test_rows_without_a_page():
    """Their queries are turned, their keys and values go nowhere; the other requests are served."""
    table = i32([[0, -1], [1, 9], [2, 3]])
    kc, vc = torch.full((4, 2, 1, 32), 3.0, device=DEV), torch.full((4, 2, 1, 32), 3.0, device=DEV)
    q, k, v = (torch.randn((6, 1, 32), device=DEV) for _ in range(3))
    out, status, f = torch.zeros_like(q), i32([0]), spec.spec_rotary_frequencies(32)
    pos = torch.tensor([2, 2, 3], device=DEV)  # a hole; a page out of range; past the table
    spec.spec_rotary_append(q, k, v, kc, vc, table, pos, 3, 1, f, out, status=status)
    assert int(status) == spec.ERR_BAD_INPUT
    for r, p in enumerate([2, 3, 2, 3, 3, 4]):
        check(out[r], *ref.rotate(q[r].cpu(), p, f.tolist(), False, 1.0), F32)
    assert bool((kc[:3] == 3).all()) and bool((kc[3, 0] == 3).all())
    assert torch.equal(vc[3, 1], v[4]) and bool((vc[:3] == 3).all())


def test_paged_cache_captured():
    """PagedCache.append_rotary in a graph, replayed as the positions move."""
    B, K, Hq, Hkv, D = 3, 1, 4, 2, 64
    c = PagedCache(1, 16, 4, Hq, Hkv, D, B, 32, K, F32)
    f = spec.spec_rotary_frequencies(D)
    pos = torch.tensor([0, -2, 5], device=DEV)
    q, k, v = (torch.randn((B * 2, h, D), device=DEV) for h in (Hq, Hkv, Hkv))
    out = torch.zeros_like(q)

    def step():
        c.reserve(pos)
        c.append_rotary(0, q, k, v, pos, f, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
        for i, p in enumerate(pos.tolist()):
            for j in range(2):
                if p + j >= 0:
                    page = int(c.page_table[i, (p + j) // 4])
                    check(c.k[0, page, (p + j) % 4], *ref.rotate(k[2 * i + j].cpu(), p + j, f.tolist(), False, 1.0), F32)
                    check(out[2 * i + j], *ref.rotate(q[2 * i + j].cpu(), p + j, f.tolist(), False, 1.0), F32)
        pos += 2
    assert int(c.status) == 0


@pytest.mark.parametrize("dtype,Hq,Hkv,D,rot,inter,out_of_place", [
    (BF16, 6, 2, 128, 128, False, True), (BF16, 3, 1, 80, 50, True, False), (F32, 5, 5, 64, 32, False, True),
    (BF16, 40, 8, 64, 64, True, False)])
def test_many_ragged_rows(dtype, Hq, Hkv, D, rot, inter, out_of_place):
    """Thousands of rows: several to a CTA, of different requests, bad and early rows and pages among them."""
    B, K, ps = 211, 40, 16
    g = torch.Generator().manual_seed(Hq)
    depth = torch.randint(0, K + 1, (B,), generator=g).tolist()
    pos = torch.randint(0, 400, (B,), generator=g).tolist()
    pos[3], pos[50], pos[77] = -5, -K - 1, (1 << 40) + 12345
    rows = paged_ref.Rows(depth, K)
    need = [max(0, p + n) // ps + 1 if p < 1 << 20 else 0 for p, n in zip(pos, depth)]
    pages = sum(need) + 3
    table = paged_ref.random_table(B, need, pages, 32, g)
    table[8, pos[8] // ps] = pages  # out of range
    given = list(depth)
    given[120] = depth[120] + 1     # does not fit its rows
    q, k, v = (torch.randn((rows.R, h, D), generator=g).to(dtype).to(DEV) for h in (Hq, Hkv, Hkv))
    caches = [torch.full((1, pages, ps, Hkv, D), 3.0, dtype=dtype, device=DEV) for _ in range(2)]
    f = spec.spec_rotary_frequencies(rot, 10000.0)
    at = dict(row_offsets=i32(rows.offsets), depth=i32(given), status=i32([0]))
    out = torch.full(q.shape, 7.0, dtype=dtype, device=DEV) if out_of_place else q.clone()
    blank = out.clone()
    where, td = torch.tensor(pos, device=DEV), table.to(DEV)
    spec.spec_rotary_append(q if out_of_place else out, k, v, caches[0], caches[1], td, where, B, K, f, out,
                            interleaved=inter, **at)
    assert int(at["status"]) == spec.ERR_BAD_INPUT
    want = blank.cpu().double()
    err = torch.zeros_like(want)
    kept = [torch.full((pages, ps, Hkv, D), 3.0, dtype=torch.float64) for _ in range(2)]
    kept_err = torch.zeros_like(kept[0])
    qc, kc, vc = q.cpu(), k.cpu(), v.cpu()
    for i in range(B):
        if i == 120:
            continue
        for j in range(depth[i] + 1):
            r, p = rows.offsets[i] + j, pos[i] + j
            if not 0 <= p < 1 << 32:
                continue
            want[r], err[r] = ref.rotate(qc[r], p, f.tolist(), inter, 1.0)
            page = int(table[i, p // ps]) if p // ps < table.shape[1] else -1
            if 0 <= page < pages:
                kept[0][page, p % ps], kept_err[page, p % ps] = ref.rotate(kc[r], p, f.tolist(), inter, 1.0)
                kept[1][page, p % ps] = vc[r].double()
    check(out, want, err, dtype)
    check(caches[0][0], kept[0], kept_err, dtype)
    assert torch.equal(caches[1][0].cpu().double(), kept[1])


def test_many_rows_captured_on_a_stream():
    """Positions and depths that change between replays; what lies behind the last row stays."""
    B, K, H, D = 130, 31, 2, 64
    x = torch.randn((B * (K + 1) + 4, H, D), device=DEV)
    out = torch.full(x.shape, 5.0, device=DEV)
    f = spec.spec_rotary_frequencies(D)
    pos, depth, offsets = torch.zeros(B, dtype=torch.int64, device=DEV), i32([0] * B), i32([0] * (B + 1))
    status, side, graph = i32([0]), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        spec.spec_rotary(x, f, pos, B, K, out, row_offsets=offsets, depth=depth, status=status)
    for step in range(3):
        n = [(5 * i + 11 * step) % (K + 1) for i in range(B)]
        rows = paged_ref.Rows(n, K)
        where = [(1 << 20) * step + 7 * i for i in range(B)]
        pos.copy_(torch.tensor(where))
        depth.copy_(i32(n))
        offsets.copy_(i32(rows.offsets))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0 and bool((out[rows.R:] == 5).all())
        xc = x.cpu()
        want, err = xc.double(), torch.zeros(x.shape, dtype=torch.float64)
        for i in range(B):
            for j in range(n[i] + 1):
                r = rows.offsets[i] + j
                want[r], err[r] = ref.rotate(xc[r], where[i] + j, f.tolist(), False, 1.0)
        check(out[:rows.R], want[:rows.R], err[:rows.R], F32)
