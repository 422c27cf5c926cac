"""spec_attend against attention in 64 bits, at the sizes and masks where it can
go wrong.  Tolerances are the kernel's own error bounds (paged_ref.bounds)."""
import math

import pytest
import torch

import paged_ref as ref
import paper_2607_25852_gb300 as spec

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda")
BF16, F32 = torch.bfloat16, torch.float32


def make_cache(layout, pages, ps, Hkv, D, dtype, gen):
    """K and V as [pages, ps, Hkv, D] views of several memory orders, and their backing."""
    if layout == "token":
        k, v = (torch.randn((pages, ps, Hkv, D), generator=gen).to(dtype).to(DEV) for _ in range(2))
    elif layout == "head":
        k, v = (torch.randn((pages, Hkv, ps, D), generator=gen).to(dtype).to(DEV).transpose(1, 2) for _ in range(2))
    else:  # one buffer, keys and values of a token side by side
        both = torch.randn((pages, ps, 2, Hkv, D), generator=gen).to(dtype).to(DEV)
        k, v = both[:, :, 0], both[:, :, 1]
    return k, v


class Case:
    def __init__(self, pos, depth, K, Hq, Hkv, D, ps, dtype=BF16, window=0, sinks=0, layout="token", packed=True,
                 seed=1, q_scale=1.0, hole=None, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.rows = ref.Rows(depth, K, packed)
        self.B, self.K, self.Hq, self.Hkv, self.D, self.ps, self.dtype = len(pos), K, Hq, Hkv, D, ps, dtype
        self.window, self.sinks, self.pos = window, sinks, pos
        need = [max(0, (p + n) // ps + 1) for p, n in zip(pos, depth)]
        self.max_pages = max(1, max(need))
        pages = sum(need) + spare
        self.table = ref.random_table(self.B, need, pages, self.max_pages, g, hole or (lambda i, t: False))
        self.k, self.v = make_cache(layout, pages, ps, Hkv, D, dtype, g)
        self.q = (torch.randn((self.rows.R, Hq, D), generator=g) * q_scale).to(dtype).to(DEV)
        self.ws = spec.attend_workspace(self.B, K, Hq, Hkv, D, dtype, DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def call(self, q=None, ws=None, out=None, lse=None, **kw):
        q = self.q if q is None else q
        out = torch.full(q.shape, 7.0, dtype=self.dtype, device=DEV) if out is None else out
        lse = torch.full(q.shape[:2], 7.0, dtype=F32, device=DEV) if lse is None else lse
        r = self.rows
        spec.spec_attend(q, self.k, self.v, self.table.to(DEV), torch.tensor(self.pos, device=DEV), self.B, self.K,
                         out, self.ws if ws is None else ws,
                         row_offsets=torch.tensor(r.offsets, dtype=torch.int32, device=DEV) if r.packed else None,
                         depth=torch.tensor(r.depth, dtype=torch.int32, device=DEV), window=self.window,
                         sinks=self.sinks, lse_out=lse, status=self.status, **kw)
        return out, lse

    def check(self, out, lse, scale=None):
        scale = ref.sqrt_scale(self.D) if scale is None else scale
        want, want_lse, mass, big = ref.attend(self.q, self.k, self.v, self.table, self.pos, self.rows, scale,
                                               self.window, self.sinks)
        terms = max(1, max(p + n + 1 for p, n in zip(self.pos, self.rows.depth)))
        tol, tol_lse = ref.bounds(want, mass, big, terms, self.D, self.dtype == BF16)
        got, got_lse = out.cpu().double(), lse.cpu().double()
        mine = ~want_lse.isnan()
        assert mine.any()
        none = mine & (want_lse == -math.inf)
        assert (got[none] == 0).all() and (got_lse[none] == -math.inf).all()
        some = mine & ~none
        err = (got - want).abs()[some]
        assert not got[some].isnan().any()
        assert (err <= tol[some]).all(), (err / tol[some]).max()
        err = (got_lse - want_lse).abs()[some]
        assert (err <= tol_lse[some]).all(), (err / tol_lse[some]).max()
        assert (got[~mine] == 7.0).all()             # rows of no request are not written
        assert int(self.status.item()) == 0
        assert int(self.ws.view(torch.uint8)[:768].sum()) == 0  # the arrival counters are back at zero


SHAPES = [  # Hq, Hkv, D, page size
    (8, 2, 128, 16), (4, 4, 64, 16), (16, 1, 128, 64), (6, 2, 64, 32), (8, 1, 64, 128), (5, 5, 128, 8),
    (4, 2, 128, 48), (4, 2, 96, 16), (3, 1, 80, 10), (8, 2, 256, 16), (2, 1, 8, 1), (4, 1, 128, 24), (64, 1, 64, 256),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hq,Hkv,D,ps", SHAPES)
def test_ragged_rows_against_64_bits(Hq, Hkv, D, ps, dtype):
    pos = [0, 1, 127, 128, 300, 65, -1]
    depth = [0, 4, 0, 3, 4, 2, 0]
    c = Case(pos, depth, 4, Hq, Hkv, D, ps, dtype, seed=Hq + D + ps)
    c.check(*c.call())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["token", "head", "interleaved"])
def test_memory_orders(layout, dtype):
    c = Case([200, 17, 63], [2, 0, 2], 2, 8, 4, 64, 16, dtype, layout=layout, packed=False, seed=4)
    c.check(*c.call())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,Hq,Hkv", [(0, 1, 1), (0, 64, 1), (1, 24, 8), (7, 8, 1), (16, 16, 2), (16, 64, 4), (31, 4, 4),
                                      (255, 2, 1)])
def test_row_and_head_counts(K, Hq, Hkv, dtype):
    c = Case([140, 0, 700], [K, K // 2, K], K, Hq, Hkv, 64 if Hq > 16 else 128, 16, dtype, seed=K + Hq)
    c.check(*c.call())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (100, 0), (128, 128), (129, 130), (300, 64),
                                          (5000, 4), (37, 1000)])
def test_window_and_sinks(window, sinks, dtype):
    pos = [0, 5, 130, 511, 900, 1300]
    depth = [3, 0, 3, 1, 3, 2]
    c = Case(pos, depth, 3, 4, 2, 64, 16, dtype, window=window, sinks=sinks, seed=window + sinks)
    c.check(*c.call())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,ps", [(64, 16), (128, 32), (128, 128), (96, 10)])
def test_pages_between_sinks_and_window_may_be_gone(D, ps, dtype):
    window, sinks = 200, 5
    pos, depth = [1000, 40, 777], [2, 2, 0]

    def hole(i, t):
        return (t + 1) * ps <= pos[i] - window + 1 and t * ps >= sinks
    c = Case(pos, depth, 2, 8, 2, D, ps, dtype, window=window, sinks=sinks, hole=hole, seed=9)
    assert (c.table[0, 1:4] == -1).any()
    c.check(*c.call())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D,ps", [(64, 16), (128, 64), (128, 10)])
def test_what_masked_places_hold_does_not_matter(D, ps, bad, dtype):
    """Everything that no row sees is `bad`: the rest of the last page, free
    pages, and the positions between sinks and window."""
    for window, sinks in ((0, 0), (90, 3)):
        c = Case([333, 0, 95], [3, 0, 1], 3, 8, 2, D, ps, dtype, window=window, sinks=sinks, seed=11)
        seen = torch.zeros(c.k.shape[:2], dtype=torch.bool)
        for i, p in enumerate(c.pos):
            for j in range(c.rows.depth[i] + 1):
                for t in ref.visible(p + j, window, sinks):
                    seen[c.table[i, t // ps], t % ps] = True
        for x in (c.k, c.v):
            x[~seen.to(DEV)] = bad
        c.check(*c.call())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (128, 40), (96, 40)])
def test_a_later_draft_does_not_reach_an_earlier_row(D, window, bad, dtype):
    """Row j must not see the non-finite key and value of row j + 1, although
    both are done together; rows that see a value so get a result that is not
    finite either.  With a window, the same at its lower edge."""
    K, n = 3, 3
    for p in (60, 127, 300):
        c = Case([p], [n], K, 4, 2, D, 16, dtype, window=window, seed=p)
        want, want_lse, mass, big = ref.attend(c.q, c.k, c.v, c.table, c.pos, c.rows, ref.sqrt_scale(D), window)
        t = p + 2  # visible to rows 2 and 3 alone
        c.v[c.table[0, t // 16].long(), t % 16, 1, 5] = bad
        u = p - window + 2  # with a window: visible to rows 0..1 alone
        if window:
            c.v[c.table[0, u // 16].long(), u % 16, 0, 3] = bad
        out, lse = c.call()
        tol, tol_lse = ref.bounds(want, mass, big, p + 4, D, dtype == BF16)
        hit = torch.zeros(want.shape, dtype=torch.bool)
        hit[2:, 2:, 5] = True          # query heads 2, 3 share key-value head 1
        if window:
            hit[:2, :2, 3] = True
            hit[1, :2, 3] = True
        got = out.cpu().double()
        assert (~got[hit].isfinite()).all()
        assert ((got - want).abs() <= tol)[~hit].all()
        assert ((lse.cpu().double() - want_lse).abs() <= tol_lse).all()
        # a key that is not finite spoils the rows that see it, and no other
        c.k[c.table[0, t // 16].long(), t % 16, 1] = float("nan")
        out, lse = c.call()
        assert not lse[:2].isnan().any() and lse[2:, 2:].isnan().all() and not lse[2:, :2].isnan().any()
        got = out.cpu().double()
        assert ((got - want).abs() <= tol)[:2][~hit[:2]].all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_every_size(dtype):
    """Large scores (one weight close to 1), growing along the cache so that the
    running maximum keeps moving, and equal ones."""
    for ramp in (0.0, 0.02, -0.02):
        c = Case([1500], [1], 1, 4, 2, 64, 16, dtype, seed=5, q_scale=4.0)
        if ramp:
            t = torch.arange(1502)
            add = (ramp * t).to(dtype).to(DEV)
            c.k[c.table[0, t // 16].long().to(DEV), (t % 16).to(DEV)] += add[:, None, None]
            c.q[:] = c.q.abs()
        else:
            c.q.zero_()
        c.check(*c.call())


@pytest.mark.parametrize("dtype,D,B,p", [(BF16, 128, 1, 20000), (BF16, 64, 3, 7001), (F32, 128, 1, 9001),
                                         (BF16, 96, 2, 5000)])
def test_long_contexts_are_split_and_joined(dtype, D, B, p):
    for K in (0, 5):
        c = Case([p + 17 * i for i in range(B)], [K] * B, K, 8, 2, D, 64 if D == 128 else 16, dtype, seed=p)
        first = c.call()
        c.check(*first)
        again = c.call()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_many_requests_of_one_token():
    B = 700
    c = Case([(7 * i) % 90 - 1 for i in range(B)], [0] * B, 0, 2, 1, 64, 16, BF16, seed=3)
    c.check(*c.call())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scale_and_layer_arguments(dtype):
    c = Case([77], [2], 2, 4, 2, 128, 16, dtype, seed=8)
    out, lse = c.call(scale=0.3)
    c.check(out, lse, scale=0.3)
    k5 = torch.stack([torch.zeros_like(c.k), c.k])
    v5 = torch.stack([torch.zeros_like(c.v), c.v])
    k4, v4 = c.k, c.v
    c.k, c.v = k5, v5
    out5, lse5 = c.call(scale=0.3, layer=1)
    assert torch.equal(out, out5) and torch.equal(lse, lse5)
    c.k, c.v = k4, v4
    out2 = torch.empty_like(out)
    spec.spec_attend(c.q, c.k, c.v, c.table.to(DEV), torch.tensor(c.pos, device=DEV), 1, 2, out2, c.ws, scale=0.3)
    assert torch.equal(out, out2)


def test_queries_as_views_of_a_fused_projection():
    c = Case([90, 20], [3, 3], 3, 4, 2, 64, 16, BF16, packed=False, seed=12)
    fused = torch.randn((8, 4 * 64 + 2 * 2 * 64), device=DEV).to(BF16)
    fused[:, :256] = c.q.view(8, 256)
    q = fused[:, :256].view(8, 4, 64)
    assert not q.is_contiguous()
    c.check(*c.call(q=q))


@pytest.mark.parametrize("D", [64, 128, 96])
def test_offsets_past_32_bits(D):
    """Pages more than 2^32 elements from the cache's start."""
    ps, Hkv = 64, 2
    page = ps * Hkv * D
    pages = (1 << 32) // page + 40
    k = torch.empty((pages, ps, Hkv, D), dtype=BF16, device=DEV)
    v = torch.empty((pages, ps, Hkv, D), dtype=BF16, device=DEV)
    c = Case([150, 10], [1, 1], 1, 4, Hkv, D, ps, BF16, seed=2)
    used = c.table[c.table >= 0].long()
    to = torch.arange(pages - len(used), pages)
    k[to.to(DEV)] = c.k[used.to(DEV)]
    v[to.to(DEV)] = c.v[used.to(DEV)]
    out, lse = c.call()
    big = c.table.clone()
    big[c.table >= 0] = to.to(torch.int32)
    c.table, c.k, c.v = big, k, v
    out2, lse2 = c.call()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_on_a_side_stream_and_in_a_graph():
    c = Case([600, 31], [2, 1], 2, 8, 2, 128, 16, BF16, seed=6)
    want = c.call()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        side = c.call()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(want[0], side[0]) and torch.equal(want[1], side[1])
    table, pos = c.table.to(DEV), torch.tensor(c.pos, device=DEV)
    offsets = torch.tensor(c.rows.offsets, dtype=torch.int32, device=DEV)
    depth = torch.tensor(c.rows.depth, dtype=torch.int32, device=DEV)
    out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        spec.spec_attend(c.q, c.k, c.v, table, pos, c.B, c.K, out, c.ws, row_offsets=offsets, depth=depth,
                         lse_out=lse, status=c.status)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    pos -= 30  # a replay reads the lengths of its own time
    g.replay()
    c.pos = [p - 30 for p in c.pos]
    c.check(out, lse)


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 64), (BF16, 96)])
def test_bad_data_is_reported_and_contained(dtype, D):
    base = Case([100, 50, 70], [2, 2, 2], 2, 4, 2, D, 16, dtype, seed=21)
    want, _ = base.call()
    # a visible slot without a page: its keys are left out
    for entry in (-1, 10 ** 6, -7):
        c = Case([100, 50, 70], [2, 2, 2], 2, 4, 2, D, 16, dtype, seed=21)
        c.table[1, 1] = entry
        out, _ = c.call()
        assert int(c.status.item()) == spec.ERR_BAD_INPUT
        assert torch.equal(out[:3], want[:3]) and torch.equal(out[6:], want[6:])
        assert out[3:6].float().isfinite().all() and not torch.equal(out[3:6], want[3:6])
    # a position past the table: the request's rows see nothing
    c = Case([100, 50, 70], [2, 2, 2], 2, 4, 2, D, 16, dtype, seed=21)
    for p in (c.max_pages * 16 - 2, 1 << 40, (1 << 63) - 1):
        c.pos, c.status = [100, p, 70], torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = c.call()
        assert int(c.status.item()) == spec.ERR_BAD_INPUT
        assert (out[3:6] == 0).all() and (lse[3:6] == -math.inf).all()
        assert torch.equal(out[:3], want[:3]) and torch.equal(out[6:], want[6:])
    # depths that do not fit the offsets: nothing of the request is written
    for n in (-1, 3, 1, 1 << 30):
        c = Case([100, 50, 70], [2, 2, 2], 2, 4, 2, D, 16, dtype, seed=21)
        c.rows.depth[1] = n
        out, _ = c.call()
        assert int(c.status.item()) == spec.ERR_BAD_INPUT
        assert (out[3:6] == 7.0).all()
        assert torch.equal(out[:3], want[:3]) and torch.equal(out[6:], want[6:])


@pytest.mark.parametrize("dtype,D,ps", [(BF16, 128, 16), (BF16, 64, 64), (F32, 64, 16), (BF16, 80, 10)])
def test_writes_stay_inside(dtype, D, ps):
    from test_gpu_canaries import Guarded, assert_intact, guarded_workspace
    c = Case([3000, 0, 129, 64], [4, 0, 4, 2], 4, 8, 2, D, ps, dtype, seed=31)
    want = c.call()
    n = spec.spec_attend_workspace(c.B, c.K, c.Hq, c.Hkv, D, dtype)
    ws = guarded_workspace(n)
    out, lse = Guarded(c.q.shape, dtype, 7.0), Guarded(c.q.shape[:2], F32, 7.0)
    c.call(ws=ws.t, out=out.t, lse=lse.t)
    assert_intact(ws=ws, out=out, lse=lse)
    assert torch.equal(out.t, want[0]) and torch.equal(lse.t, want[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K,G", [(0, 8), (3, 8), (5, 8), (7, 8), (10, 8), (11, 8), (15, 8), (16, 8), (31, 4)])
def test_long_runs_of_every_width(D, K, G):
    """Many tiles per CTA at every number of columns: a pipeline that mixes up
    two uses of a buffer shows in runs longer than the buffers are deep.  Equal
    requests must get equal results, whatever share of the work they fall into."""
    B, p, Hkv = 40, 2900, 4
    g = torch.Generator().manual_seed(K)
    slots = (p + K) // 64 + 1
    k = torch.randn((slots, 64, Hkv, D), generator=g).to(BF16).to(DEV)
    v = torch.randn((slots, 64, Hkv, D), generator=g).to(BF16).to(DEV)
    q1 = torch.randn((K + 1, Hkv * G, D), generator=g).to(BF16)
    table = torch.arange(slots, dtype=torch.int32, device=DEV).repeat(B, 1)
    q = q1.repeat(B, 1, 1).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    ws = spec.attend_workspace(B, K, Hkv * G, Hkv, D, BF16, DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    pos = torch.full((B,), p, dtype=torch.int64, device=DEV)
    want, want_lse, mass, big = ref.attend(q1, k, v, table, [p], ref.Rows([K], K), ref.sqrt_scale(D))
    tol, tol_lse = ref.bounds(want, mass, big, p + K + 1, D, True)
    for _ in range(10):
        out.fill_(7.0)
        spec.spec_attend(q, k, v, table, pos, B, K, out, ws, lse_out=lse, status=st)
        assert int(st.item()) == 0
        got = out.view(B, K + 1, -1, D).cpu().double()
        assert ((got - want).abs() <= tol).all()
        assert ((lse.view(B, K + 1, -1).cpu().double() - want_lse).abs() <= tol_lse).all()
