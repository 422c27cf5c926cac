"""spec_linear_attend and spec_linear_commit against the recurrence in 64 bits."""
import math

import pytest
import torch

import paper_2607_25852_gb300 as spec
import rows_ref as ref
from paper_2607_25852_gb300.states import LinearStates

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Case:
    """Requests of `depth` + 1 rows; request i starts from slot start[i] of the pool (-1: zeros)."""

    def __init__(self, depth, K, Hq, H, Dk, Dv, dtype=BF16, gate="row", start=None, seed=1, strong=2.0, fused=False):
        g = torch.Generator().manual_seed(seed)
        self.depth, self.K, self.B, self.dtype = depth, K, len(depth), dtype
        self.Hq, self.H, self.Dk, self.Dv = Hq, H, Dk, Dv
        self.offsets = [0]
        for n in depth:
            self.offsets.append(self.offsets[-1] + n + 1)
        R = self.R = self.offsets[-1]
        if fused:
            w = Hq * Dk + H * Dk + H * Dv
            rows = torch.randn((R + 1, w + 8), generator=g).to(dtype).to(DEV)
            self.q = rows[:, :Hq * Dk].unflatten(1, (Hq, Dk))
            self.k = rows[:, Hq * Dk:(Hq + H) * Dk].unflatten(1, (H, Dk))
            self.v = rows[:, (Hq + H) * Dk:w].unflatten(1, (H, Dv))
        else:
            self.q, self.k, self.v = (torch.randn((R + 1, h, d), generator=g).to(dtype).to(DEV)
                                      for h, d in ((Hq, Dk), (H, Dk), (H, Dv)))
        if gate == "row":
            self.decay = -torch.exp(torch.empty((R + 1, H)).uniform_(math.log(1e-3), math.log(strong), generator=g))
        elif gate == "head":
            self.decay = -torch.exp2(-1.0 - torch.arange(H) * 7.0 / H)
        else:
            self.decay = gate
        self.slots = 2 * self.B + 1
        self.states = torch.randn((2, self.slots, H, Dk, Dv), generator=g).to(DEV)
        order = torch.randperm(self.slots, generator=g).tolist()
        self.start = order[:self.B] if start is None else start
        self.to = order[self.B:2 * self.B]
        self.status = i32([0])
        self.ws = spec.linear_workspace(self.B, K, Hq, H, Dk, Dv, dtype, DEV)
        self.scale = Dk ** -0.5
        self.pos = None

    def at(self):
        return dict(row_offsets=i32(self.offsets), depth=i32(self.depth), layer=1, status=self.status,
                    pos_base=None if self.pos is None else torch.tensor(self.pos, device=DEV))

    def attend(self, to="to", **kw):
        out = torch.full((self.R + 1, self.Hq, self.Dv), 7.0, dtype=self.dtype, device=DEV)
        slots_out = None if to is None else i32(self.to if to == "to" else to)
        spec.spec_linear_attend(self.q, self.k, self.v, self.decay.to(DEV), self.states, i32(self.start), slots_out, self.B,
                                self.K, out, self.ws, **{**self.at(), **kw})
        return out

    def commit(self, accepted, **kw):
        spec.spec_linear_commit(self.k, self.v, self.decay.to(DEV), self.states, i32(self.start), i32(self.to),
                                None if accepted is None else i32(accepted), self.B, self.K, self.ws,
                                **{**self.at(), **kw})

    def want(self, i, before, take=None):
        rows = slice(self.offsets[i], self.offsets[i + 1])
        g = self.decay if self.decay.dim() == 2 else self.decay.expand(self.R + 1, self.H)
        first = before[1, self.start[i]] if self.start[i] >= 0 else torch.zeros_like(before[1, 0])
        n = self.depth[i] + 1
        skip = 0 if self.pos is None else min(n, max(0, -self.pos[i]))
        out, state, o_size, s_size = ref.linear(
            self.q[rows][skip:].cpu(), self.k[rows][skip:].cpu(), self.v[rows][skip:].cpu(), g[rows][skip:],
            first.cpu(), self.scale, None if take is None else max(0, take - skip))
        o_tol, s_tol = ref.linear_bounds(out, o_size, state, s_size, n, self.Dk, self.dtype)
        pad = torch.zeros((skip,) + out.shape[1:], dtype=torch.float64)
        return torch.cat([pad, out]), torch.cat([pad, o_tol]), state, s_tol

    def check(self, out, before, accepted=None, states=True):
        for i in range(self.B):
            o, o_tol, s, s_tol = self.want(i, before, None if accepted is None else accepted[i] + 1)
            if out is not None:
                got = out[self.offsets[i]:self.offsets[i + 1]].cpu().double()
                assert bool(((got - o).abs() <= o_tol).all()), (i, float(((got - o).abs() / o_tol).max()))
            if states:
                got = self.states[1, self.to[i]].cpu().double()
                assert bool(((got - s).abs() <= s_tol).all()), (i, float(((got - s).abs() / s_tol).max()))
        if out is not None:
            assert bool((out[self.R] == 7).all())
        touched = {(1, t) for t in self.to} if states else set()
        for l in range(2):
            for t in range(self.slots):
                if (l, t) not in touched:
                    assert torch.equal(self.states[l, t], before[l, t]), (l, t)


SHAPES = [(4, 4, 128, 128), (4, 2, 64, 64), (8, 1, 64, 128), (2, 2, 128, 64)]
ODD = [(3, 3, 72, 96), (2, 1, 8, 8), (4, 4, 32, 160), (1, 1, 256, 256), (6, 2, 200, 40)]


@pytest.mark.parametrize("depth,K", [([0], 0), ([0] * 5, 0), ([7, 0, 3], 7), ([16, 8, 9], 16), ([40, 31, 0, 63], 63),
                                     ([64, 130, 127], 200), ([300, 5], 300)])
@pytest.mark.parametrize("shape", SHAPES + ODD)
def test_rows(shape, depth, K):
    c = Case(depth, K, *shape, start=None if len(depth) < 3 else [2, -1, 0, 3, 3][:len(depth)])
    c.to = [s for s in range(c.slots) if s not in c.start][:c.B]
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == 0
    c.check(out, before)


@pytest.mark.parametrize("gate", ["head", "row"])
@pytest.mark.parametrize("depth,K", [([0, 0], 0), ([11, 4], 16), ([100, 70], 150)])
@pytest.mark.parametrize("shape", [(2, 2, 128, 128), (4, 2, 64, 64), (3, 1, 36, 100)])
def test_fp32(shape, depth, K, gate):
    c = Case(depth, K, *shape, dtype=F32, gate=gate)
    before = c.states.clone()
    c.check(c.attend(), before)
    assert int(c.status) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,depth,accepted", [(7, [7, 0, 4], [3, 0, 4]), (70, [70, 64, 0], [64, 0, 0])])
def test_round(K, depth, accepted, dtype):
    """A verification leaves the states; the commit takes the accepted rows, whatever the rejected ones hold."""
    c = Case(depth, K, 4, 2, 128, 128, dtype=dtype, gate="head", fused=True)
    before = c.states.clone()
    out = c.attend(to=None)
    c.check(out, before, states=False)
    for i, a in enumerate(accepted):
        c.k[c.offsets[i] + a + 1:c.offsets[i + 1]] = math.nan
        c.v[c.offsets[i] + a + 1:c.offsets[i + 1]] = math.inf
    c.commit(accepted)
    assert int(c.status) == 0
    for i, a in enumerate(accepted):
        rows = slice(c.offsets[i] + a + 1, c.offsets[i + 1])
        c.k[rows], c.v[rows] = 0.0, 0.0
    c.check(None, before, accepted)


@pytest.mark.parametrize("K", [3, 130])
def test_in_place_and_shared_start(K):
    """New states in the old ones' slots; two requests from one slot, into slots of their own."""
    c = Case([K, K - 1, K], K, 2, 2, 64, 64)
    c.to = list(c.start)
    before = c.states.clone()
    out = c.attend()
    c.check(out, before)
    c = Case([K, K - 1, K], K, 2, 2, 64, 64)
    c.start[1] = c.start[0]
    before = c.states.clone()
    c.check(c.attend(), before)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [6, 150])
def test_strong_decays(K, dtype):
    """Decays of nothing, of everything, and far below fp32's range, next to slow ones; sums of many strong ones."""
    n = K + 1
    g = torch.full((2 * n + 1, 3), -0.01)
    g[:, 1] = -60.0
    g[n // 2, 0] = -math.inf
    g[n // 2 + 1, 2] = -1e30
    g[3:5, 2] = 0.0
    g[n:, 0] = -300.0
    c = Case([K, K], K, 3, 3, 128, 128, dtype=dtype, gate=g)
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == 0
    c.check(out, before)
    assert bool(torch.isfinite(out).all())


def test_growth_is_refused():
    g = torch.full((5, 2), -0.1)
    g[1, 0], g[2, 1] = 0.5, math.nan
    c = Case([3], 3, 2, 2, 64, 64, gate=g)
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == spec.ERR_BAD_INPUT
    c.decay[1, 0], c.decay[2, 1] = 0.0, 0.0
    c.check(out, before)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,at", [(5, 3), (140, 70), (140, 130), (200, 64)])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_not_finite(K, at, what, value, dtype):
    """Rows before it are as if it were not there, rows from it on and the state are not finite where it enters."""
    c = Case([K, K], K, 2, 2, 64, 64, dtype=dtype)
    before = c.states.clone()
    (c.k if what == "k" else c.v)[at, 1, 5] = value
    out = c.attend()
    c.k[at, 1], c.v[at, 1] = 0.0, 0.0
    o, o_tol, s, s_tol = c.want(0, before)
    got = out[:K + 1].cpu().double()
    fine = torch.ones_like(o, dtype=torch.bool)
    hit = slice(None) if what == "k" else 5
    fine[at:, 1, hit] = False
    if what == "v":  # the other elements of the row's product are what they were with the row
        fine[at:, 1] = False
    assert bool(((got - o).abs() <= o_tol)[fine].all())
    assert not bool(torch.isfinite(got[at:, 1, hit]).any())
    if what == "v":
        assert bool(torch.isfinite(got[at:, 1, 6:]).all()) and bool(torch.isfinite(got[at:, 1, :5]).all())
    state = c.states[1, c.to[0]].cpu()
    assert bool(torch.isfinite(state[0]).all())
    assert not bool(torch.isfinite(state[1][5] if what == "k" else state[1][:, 5]).any())
    o, o_tol, s, s_tol = c.want(1, before)
    assert bool(((out[K + 1:-1].cpu().double() - o).abs() <= o_tol).all())


@pytest.mark.parametrize("K", [4, 100])
def test_idle_and_early_rows(K):
    """Rows before position 0 give 0 and change nothing; an idle request's state moves as it is."""
    c = Case([K, K, K, K], K, 4, 2, 64, 128, start=[0, 1, -1, 2])
    c.to = [4, 5, 6, 7]
    c.pos = [-(K + 1), 3, -(K + 1), -2]
    for i in (0, 2):
        c.k[c.offsets[i]:c.offsets[i + 1]] = math.nan
        c.q[c.offsets[i]:c.offsets[i + 1]] = math.nan
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == 0
    assert torch.equal(c.states[1, 4], before[1, 0]) and not bool(c.states[1, 6].any())
    for i in (0, 2):
        assert not bool(out[c.offsets[i]:c.offsets[i + 1]].any())
        c.k[c.offsets[i]:c.offsets[i + 1]] = 0
        c.q[c.offsets[i]:c.offsets[i + 1]] = 0
    c.check(out, before)


@pytest.mark.parametrize("K", [2, 90])
def test_bad_requests(K):
    """Slots out of range, depths that do not fit: nothing of these requests is written, the others are served."""
    c = Case([K] * 5, K, 2, 2, 64, 64)
    before = c.states.clone()
    good_start, good_to = list(c.start), list(c.to)
    c.start[1], c.to[2] = c.slots, -2
    bad_depth = [K, K, K, K - 1, K]
    out = c.attend(depth=i32(bad_depth))
    assert int(c.status) == spec.ERR_BAD_INPUT
    for i in (1, 2, 3):
        assert bool((out[c.offsets[i]:c.offsets[i + 1]] == 7).all())
        assert torch.equal(c.states[1, good_to[i]], before[1, good_to[i]])
    c.start, c.to = good_start, good_to
    for i in (0, 4):
        o, o_tol, s, s_tol = c.want(i, before)
        assert bool(((out[c.offsets[i]:c.offsets[i + 1]].cpu().double() - o).abs() <= o_tol).all())
        assert bool(((c.states[1, c.to[i]].cpu().double() - s).abs() <= s_tol).all())
    c.status.zero_()
    kept = c.states.clone()
    c.commit([0, K + 1, -1, 0, 0])
    assert int(c.status) == spec.ERR_BAD_INPUT
    for i in (1, 2):
        assert torch.equal(c.states[1, c.to[i]], kept[1, c.to[i]])


@pytest.mark.parametrize("depth,K,B", [([2000], 2000, 1), ([1500, 3, 900], 1999, 3)])
def test_long(depth, K, B):
    """Prompts long enough to be divided; the result does not depend on the run."""
    c = Case(depth, K, 2, 1, 128, 128, strong=0.3)
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == 0
    c.check(out, before)
    again, states = c.attend(), c.states.clone()
    assert torch.equal(out, again)
    c.states.copy_(before)
    c.commit(None)
    for i in range(B):
        _, _, s, s_tol = c.want(i, before)
        assert bool(((c.states[1, c.to[i]].cpu().double() - s).abs() <= s_tol).all())
    del states


@pytest.mark.parametrize("Dk,Dv", [(128, 64), (64, 64), (64, 128), (128, 128)])
def test_every_run_is_the_same(Dk, Dv):
    """Warps that take part in a chunk and warps that do not (Dv = 64) keep step, call after call."""
    c = Case([2500, 2000, 1111], 2500, 16, 16, Dk, Dv, start=[-1, 1, 2])
    c.to = [4, 5, 6]
    out, first = c.attend(), c.states.clone()
    for _ in range(40):
        again = c.attend()
        c.commit(None)
        assert int(c.status) == 0
        assert torch.equal(out[:-1], again[:-1])
        # both calls' states: the same sums in the same order
        assert torch.equal(first, c.states)


@pytest.mark.parametrize("shape", [(64, 32, 64, 64), (48, 48, 128, 128)])
def test_many_heads(shape):
    """More requests' heads than the device has SMs: each works on several in turn, of all lengths."""
    c = Case([200, 64, 0, 130, 63, 191], 200, *shape)
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == 0
    c.check(out, before)


def test_prompt_in_parts_is_the_prompt():
    """One call, calls of 256 rows, and single tokens carry the same state."""
    n, H, D = 600, 2, 64
    c = Case([n - 1], n - 1, H, H, D, D, dtype=F32, start=[-1])
    before = c.states.clone()
    whole = c.attend()
    st = LinearStates(1, H, H, D, D, 1, 256, F32)
    out = torch.empty_like(whole[:n])
    at = 0
    for size in (256, 256, 60, 1, 1, 26):
        rows = slice(at, at + size)
        o = torch.empty((size, H, D), device=DEV)
        st.attend(0, c.q[rows], c.k[rows], c.v[rows], c.decay[rows].to(DEV), o, update=True, K=size - 1)
        out[rows] = o
        at += size
    assert at == n and int(st.status) == 0
    o, o_tol, s, s_tol = c.want(0, before)
    assert bool(((out.cpu().double() - o).abs() <= o_tol).all())
    assert bool(((st.states[0, int(st.slots[0])].cpu().double() - s).abs() <= s_tol).all())


def test_states_fork_in_a_graph():
    """Parallel samples: a fork copies states, in a captured graph at every replay."""
    H, D, B = 2, 64, 4
    st = LinearStates(2, H, H, D, D, B, 3, BF16)
    q, k, v = (torch.randn((B, H, D), device=DEV).to(BF16) for _ in range(3))
    decay, out = torch.full((H,), -0.1, device=DEV), torch.empty((B, H, D), dtype=BF16, device=DEV)
    parent = i32([0, 0, 2, -1])

    def step():
        for layer in range(2):
            st.attend(layer, q, k, v, decay, out, update=True, K=0)
        st.fork(parent)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    model = torch.zeros((B, H, D, D), dtype=torch.float64)
    kv = torch.einsum("bhd,bhe->bhde", k.cpu().double(), v.cpu().double())
    for n in range(3):
        graph.replay()
        torch.cuda.synchronize()
        model = math.exp(-float(torch.tensor(0.1))) * model + kv
        model = torch.stack([model[0], model[0], model[2], torch.zeros_like(model[0])])
        for layer in range(2):
            got = st.states[layer, st.slots.long()].cpu().double()
            # three rows' products, each rounded and rescaled a few times
            assert float((got - model).abs().max()) <= 16 * 2.0 ** -23 * float(model.abs().max())
    assert int(st.status) == 0 and sorted(st.slots.tolist() + st._spare.tolist()) == list(range(2 * B))


def test_another_stream():
    c = Case([5, 90], 90, 2, 2, 64, 64)
    before = c.states.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = c.attend()
    side.synchronize()
    c.check(out, before)


# Many requests of a few rows: from two heads' states per SM on, CTAs that stay and bring states by bulk copies.
FEW = [(8, 8, 128, 128), (16, 8, 64, 64), (32, 8, 64, 128), (8, 8, 128, 64)]


def few(shape, K, dtype=BF16, B=40, seed=2, **kw):
    g = torch.Generator().manual_seed(seed)
    return Case(torch.randint(0, K + 1, (B,), generator=g).tolist(), K, *shape, dtype=dtype, seed=seed, **kw)


@pytest.mark.parametrize("dtype,K", [(BF16, 0), (BF16, 2), (BF16, 7), (BF16, 10), (F32, 0), (F32, 1), (F32, 7)])
@pytest.mark.parametrize("shape", FEW)
def test_many_requests(shape, K, dtype):
    """Starts that are shared, fresh or in place, all in one call; then the same round by a commit."""
    c = few(shape, K, dtype)
    c.start[3] = c.start[5] = c.start[8]
    c.start[4] = -1
    c.to[6], c.to[20] = c.start[6], c.start[20]
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == 0
    c.check(out, before)
    c.states.copy_(before)
    assert torch.equal(c.attend(to=None), out)
    assert torch.equal(c.states, before)
    accepted = [(7 * i) % (n + 1) for i, n in enumerate(c.depth)]
    for i, a in enumerate(accepted):
        c.k[c.offsets[i] + a + 1:c.offsets[i + 1]] = math.nan
        c.v[c.offsets[i] + a + 1:c.offsets[i + 1]] = -math.inf
        c.decay[c.offsets[i] + a + 1:c.offsets[i + 1]] = math.nan  # a rejected row's decay is not looked at
    c.commit(accepted)
    assert int(c.status) == 0
    for i, a in enumerate(accepted):
        for x in (c.k, c.v, c.decay):
            x[c.offsets[i] + a + 1:c.offsets[i + 1]] = 0
    c.check(None, before, accepted)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", FEW)
def test_many_requests_early_and_idle(shape, dtype):
    c = few(shape, 3, dtype)
    c.pos = [(-4, -1, 5, -2, 0)[i % 5] for i in range(c.B)]
    for i in range(0, c.B, 5):  # idle, whatever their rows hold
        c.k[c.offsets[i]:c.offsets[i + 1]] = math.nan
        c.q[c.offsets[i]:c.offsets[i + 1]] = math.inf
    c.start[0] = -1
    before = c.states.clone()
    out = c.attend()
    assert int(c.status) == 0
    assert not bool(c.states[1, c.to[0]].any()) and torch.equal(c.states[1, c.to[5]], before[1, c.start[5]])
    for i in range(0, c.B, 5):
        assert not bool(out[c.offsets[i]:c.offsets[i + 1]].any())
        c.k[c.offsets[i]:c.offsets[i + 1]] = 0
        c.q[c.offsets[i]:c.offsets[i + 1]] = 0
    c.check(out, before)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_requests_bad_ones(dtype):
    """Bad slots, depths and accepted lengths among good requests, which are served (one's state, to slot -1, goes
    nowhere); growth and NaN stay where they are."""
    c = few(FEW[0], 3, dtype)
    before, start, to = c.states.clone(), list(c.start), list(c.to)
    bad = {1: "start", 2: "to", 7: "depth", 39: "start"}
    depth = list(c.depth)
    for i, what in bad.items():
        if what == "start":
            c.start[i] = (c.slots, -7)[i == 39]
        elif what == "to":
            c.to[i] = -1
        else:
            depth[i] = depth[i] + 1
    c.decay[c.offsets[9], 4] = 0.25
    c.v[c.offsets[11], 2, 3] = math.nan
    out = c.attend(depth=i32(depth))
    assert int(c.status) == spec.ERR_BAD_INPUT
    c.decay[c.offsets[9], 4] = 0
    c.start, c.to = start, to
    for i in range(c.B):
        rows = slice(c.offsets[i], c.offsets[i + 1])
        got, state = out[rows].cpu().double(), c.states[1, to[i]].cpu().double()
        if i in bad:
            assert torch.equal(c.states[1, to[i]], before[1, to[i]])
        if i in bad and i != 2:
            assert bool((got == 7).all())
            continue
        heads = [h for h in range(c.H) if (i, h) != (11, 2)]
        o, o_tol, s, s_tol = c.want(i, before)
        assert bool(((got - o).abs() <= o_tol)[:, heads].all())
        assert i == 2 or bool(((state - s).abs() <= s_tol)[heads].all())
    s = c.states[1, to[11], 2]
    assert bool(s[:, 3].isnan().all()) and bool(torch.isfinite(s[:, :3]).all()) and bool(torch.isfinite(s[:, 4:]).all())
    c.v[c.offsets[11], 2, 3] = 0
    c.status.zero_()
    c.states.copy_(before)
    c.commit([n + (i == 1) - (i == 2) * (n + 1) for i, n in enumerate(c.depth)])
    assert int(c.status) == spec.ERR_BAD_INPUT
    for i in range(c.B):
        state = c.states[1, to[i]].cpu().double()
        if i in (1, 2):
            assert torch.equal(c.states[1, to[i]], before[1, to[i]])
        else:
            _, _, s, s_tol = c.want(i, before)
            assert bool(((state - s).abs() <= s_tol).all())


@pytest.mark.parametrize("K", [3, 40])
def test_captured_round(K):
    """A verification and its commit in a graph on a stream of its own, replayed as rows, accepted lengths and slots
    change; another graph shares the workspace."""
    c = few((8, 8, 64, 64), K, B=48)
    accepted, start, to = i32([0] * c.B), i32(c.start), i32(c.to)
    out = torch.zeros((c.R + 1, c.Hq, c.Dv), dtype=c.dtype, device=DEV)
    decay, at = c.decay.to(DEV), c.at()

    def verify():
        spec.spec_linear_attend(c.q, c.k, c.v, decay, c.states, start, None, c.B, K, out, c.ws, **at)

    def commit():
        spec.spec_linear_commit(c.k, c.v, decay, c.states, start, to, accepted, c.B, K, c.ws, **at)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph, call in zip(graphs, (verify, commit)):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            call()
    for step in range(3):
        before = c.states.clone()
        kept = [(step + 3 * i) % (n + 1) for i, n in enumerate(c.depth)]
        accepted.copy_(i32(kept))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert int(c.status) == 0
        for i in range(c.B):
            o, o_tol, s, s_tol = c.want(i, before, kept[i] + 1)
            got = out[c.offsets[i]:c.offsets[i + 1]].cpu().double()
            assert bool(((got - o).abs() <= o_tol).all())
            assert bool(((c.states[1, c.to[i]].cpu().double() - s).abs() <= s_tol).all())
        c.q.copy_(torch.randn(c.q.shape, device=DEV))
        c.start, c.to = c.to, c.start  # the next round starts from this one's states
        start.copy_(i32(c.start))
        to.copy_(i32(c.to))


@pytest.mark.parametrize("dtype,shape", [(F32, (2, 2, 64, 64)), (F32, (6, 2, 128, 128)), (BF16, (3, 1, 72, 96)), (BF16, (4, 2, 256, 40))])
@pytest.mark.parametrize("K", [47, 200])
def test_parts_of_long_calls(K, shape, dtype):
    """Odd sizes and fp32 divided along the rows: in place, from a shared slot, from zeros, some rows before position 0,
    an idle request, one too long for its rows; then the same rows by a commit of some of them."""
    c = Case([K, K - 20, K, 15, K, K, 2], K, *shape, dtype=dtype)
    c.start[5] = c.start[1]
    c.start[2] = -1
    c.to[0] = c.start[0]
    c.pos = [0, 1000, -30, 7, -(K + 1), 0, -1]
    bad, bad_depth = 5, list(c.depth)
    bad_depth[bad] -= 1
    c.q[c.offsets[4]:c.offsets[5]] = math.nan
    before = c.states.clone()
    out = c.attend(depth=i32(bad_depth))
    assert int(c.status) == spec.ERR_BAD_INPUT
    assert bool((out[c.offsets[bad]:c.offsets[bad + 1]] == 7).all())
    assert torch.equal(c.states[1, c.to[bad]], before[1, c.to[bad]])
    c.q[c.offsets[4]:c.offsets[5]] = 0
    c.status.zero_()
    c.states.copy_(before)
    again = c.attend()
    assert int(c.status) == 0
    c.check(again, before)
    served = [i for i in range(c.B) if i != bad]
    for i in served:
        assert torch.equal(out[c.offsets[i]:c.offsets[i + 1]], again[c.offsets[i]:c.offsets[i + 1]])
    accepted = [n // (i + 1) for i, n in enumerate(c.depth)]
    c.states.copy_(before)
    for i, a in enumerate(accepted):
        c.k[c.offsets[i] + a + 1:c.offsets[i + 1]] = math.nan
    c.commit(accepted)
    assert int(c.status) == 0
    for i, a in enumerate(accepted):
        c.k[c.offsets[i] + a + 1:c.offsets[i + 1]] = 0
    c.check(None, before, accepted)


@pytest.mark.parametrize("K", [11, 12, 13, 14])
@pytest.mark.parametrize("B", [2, 40])
def test_between_the_forms(B, K):
    """Lengths around those at which another kernel takes over: single chunks, a verification and its commit."""
    c = Case([K - i % 3 for i in range(B)], K, 8, 8, 128, 128)
    before = c.states.clone()
    out = c.attend(to=None)
    c.check(out, before, states=False)
    accepted = [i % (n + 1) for i, n in enumerate(c.depth)]
    c.commit(accepted)
    assert int(c.status) == 0
    c.check(None, before, accepted)


@pytest.mark.parametrize("dtype,Hq,H,D", [(F32, 32, 32, 64), (BF16, 8, 2, 128), (F32, 3, 1, 96), (BF16, 4, 4, 64)])
def test_shorter_calls_in_the_same_workspace(dtype, Hq, H, D):
    """Calls of fewer rows than the workspace was made for, whose own best division would want a larger one."""
    rows = 700
    st = LinearStates(1, Hq, H, D, D, 1, rows, dtype)
    g = torch.Generator().manual_seed(4)
    for n in (1, 9, 17, 63, 64, 65, 127, 200, 255, 256, 300, 384, 449, 511, 512, 640, 700):
        q, k, v = (torch.randn((n, h, D), generator=g).to(dtype) for h in (Hq, H, H))
        decay = -torch.rand((n, H), generator=g)
        st.states.zero_()
        out = torch.empty((n, Hq, D), dtype=dtype, device=DEV)
        st.attend(0, q.to(DEV), k.to(DEV), v.to(DEV), decay.to(DEV), out, update=True, K=n - 1)
        o, state, o_size, s_size = ref.linear(q, k, v, decay, torch.zeros((H, D, D)), D ** -0.5)
        o_tol, s_tol = ref.linear_bounds(o, o_size, state, s_size, n, D, dtype)
        assert int(st.status) == 0
        assert bool(((out.cpu().double() - o).abs() <= o_tol).all())
        assert bool(((st.states[0, int(st.slots[0])].cpu().double() - state).abs() <= s_tol).all())


def test_fork_from_no_request():
    """A parent that is no request's is reported; the others' states move, and the next calls go on."""
    st = LinearStates(2, 1, 1, 64, 64, 4, 1, F32)
    st.states.copy_(torch.arange(2 * 8, device=DEV).view(2, 8, 1, 1, 1).expand_as(st.states))
    st.fork(i32([3, 4, -2, -1]))
    assert int(st.status) == spec.ERR_BAD_INPUT
    assert sorted(st.slots.tolist() + st._spare.tolist()) == list(range(8))
    for layer in range(2):
        assert bool((st.states[layer, st.slots[0]] == 8 * layer + 3).all()) and not bool(st.states[layer, st.slots[3]].any())
    with pytest.raises(ValueError):
        st.fork(i32([0, 1]))
    st.status.zero_()
    st.fork(i32([0, 0, 0, 0]))
    assert int(st.status) == 0
    assert bool((st.states[1, st.slots.long()] == 11).all())


@pytest.mark.parametrize("K", [11, 63])
def test_many_idle_requests_before_live_ones(K):
    """Chunks without rows, many more than are listed ahead, one after another, with a few requests behind them and some
    between: outputs and states by one call, states by a commit, on the tensor cores."""
    B, H, D = 120, 32, 64
    c = Case([K] * B, K, H, H, D, D)
    live = {0, 61, 62, 114, 116, 117, 118, 119}
    c.pos = [5 if i in live else -(K + 1) for i in range(B)]
    for i in range(B):
        if i not in live:
            c.k[c.offsets[i]:c.offsets[i + 1]] = math.nan
    before = c.states.clone()
    for call in (c.attend, lambda: c.commit(None)):
        c.states.copy_(before)
        c.states[1, c.to] = 9.0
        out = call()
        assert int(c.status) == 0
        for i in range(B):
            if i not in live:
                assert torch.equal(c.states[1, c.to[i]], before[1, c.start[i]])
                assert out is None or not bool(out[c.offsets[i]:c.offsets[i + 1]].any())
                continue
            o, o_tol, s, s_tol = c.want(i, before)
            assert bool(((c.states[1, c.to[i]].cpu().double() - s).abs() <= s_tol).all())
            assert out is None or bool(((out[c.offsets[i]:c.offsets[i + 1]].cpu().double() - o).abs() <= o_tol).all())


@pytest.mark.parametrize("depth,K,shape,dtype", [
    ([2500, 2000, 1111], 2500, (16, 16, 128, 128), BF16),  # the tensor cores, in segments
    ([100] * 20, 100, (16, 16, 64, 128), BF16),            # and whole, more heads than SMs
    ([2000], 2000, (2, 1, 128, 128), BF16),                # query heads in groups
    ([7, 3] * 20, 7, (8, 8, 128, 128), BF16),              # few rows of many heads
    ([150, 60, 201], 201, (4, 2, 72, 96), F32),            # the CUDA cores, in segments
    ([5, 1], 5, (2, 2, 256, 256), BF16)])                  # and whole
def test_every_run_leaves_the_same_states(depth, K, shape, dtype):
    """A call writes all of its outputs and states, the same at every run; a commit of all rows the same states."""
    c = Case(depth, K, *shape, dtype=dtype)
    before = c.states.clone()
    at = torch.tensor(c.to, device=DEV)
    first = None
    for run in range(12):
        c.states[1, at] = float(run)
        out = c.attend()
        attended = c.states.clone()
        c.states[1, at] = -float(run)
        c.commit(None)
        assert int(c.status) == 0
        if first is None:
            first = out, attended, c.states.clone()
            c.check(out, before)
        assert torch.equal(out, first[0])
        assert torch.equal(attended, first[1])
        assert torch.equal(c.states, first[2])


@pytest.mark.parametrize("K,B", [(16, 24), (80, 24), (300, 5)])
@pytest.mark.parametrize("shape", [(16, 4, 128, 128), (8, 2, 64, 64), (6, 2, 128, 64)])
def test_groups_in_place(shape, K, B):
    """Query heads in groups, many requests, new states in the old ones' slots, on the tensor cores: a head's outputs
    are those of the old state whichever of its group is done first.  Some start from zeros, some from a shared slot."""
    c = Case([(7 * i + 5) % K + 1 for i in range(B)], K, *shape)
    c.to = list(c.start)
    c.start[3] = -1
    spare = next(s for s in range(c.slots) if s not in c.start + c.to)
    c.start[1] = c.start[2] = spare
    before = c.states.clone()
    for _ in range(3):
        c.states.copy_(before)
        out = c.attend()
        assert int(c.status) == 0
        c.check(out, before)
