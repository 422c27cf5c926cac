"""Host-side checks of spec_rotary*, spec_linear_* and spec_logprobs: bad arguments
are refused before any launch, by the C ABI and by the Python binding."""
import ctypes
import math

import pytest
import torch

import rows_ref as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2607_25852_gb300 import build
    build.build()
    from paper_2607_25852_gb300 import _native
    return _native.load()


DUMMY = ctypes.c_void_p(4096)  # never dereferenced: every call fails a check
ODD = ctypes.c_void_p(4104)
STREAM = ctypes.c_void_p(0)
INF, NAN = float("inf"), float("nan")


def cache(**kw):
    from paper_2607_25852_gb300 import _native
    f = dict(k=4096, v=8192, dtype=0, layers=2, pages=10, page_size=16, kv_heads=2, head_dim=64, layer_stride=20480,
             page_stride=2048, token_stride=128, head_stride=64)
    f.update(kw)
    return ctypes.byref(_native.Cache(**f))


def states(**kw):
    from paper_2607_25852_gb300 import _native
    f = dict(state=4096, layers=2, slots=10, kv_heads=2, key_dim=64, value_dim=64, layer_stride=81920, slot_stride=8192)
    f.update(kw)
    return ctypes.byref(_native.States(**f))


BAD_STATES = [dict(state=0), dict(state=4104), dict(layers=0), dict(slots=0), dict(kv_heads=0), dict(key_dim=0),
              dict(key_dim=264), dict(value_dim=0), dict(value_dim=264), dict(slot_stride=8188), dict(slot_stride=8194),
              dict(slot_stride=-8192), dict(layer_stride=100), dict(layer_stride=1 << 62)]


@pytest.mark.parametrize("scaling,factor,original,low,high", [
    ("plain", 1.0, 0, 1.0, 32.0), ("linear", 4.0, 0, 1.0, 32.0), ("base", 8.0, 0, 1.0, 32.0),
    ("ramp", 32.0, 4096, 1.0, 32.0), ("ramp", 1.0, 1, 0.5, 0.6)])
@pytest.mark.parametrize("rot", [4, 50, 128, 256])
def test_frequencies(lib, rot, scaling, factor, original, low, high):
    import paper_2607_25852_gb300 as spec
    got = spec.spec_rotary_frequencies(rot, 10000.0, scaling, factor, original, low, high, device="cpu")
    assert got.dtype == torch.float64
    # pow and the divisions of both sides, a few roundings of 2^-53 each
    assert got.tolist() == pytest.approx(ref.frequencies(rot, 10000.0, scaling, factor, original, low, high), rel=2e-14)


def test_frequencies_refuse(lib):
    import paper_2607_25852_gb300 as spec
    out = (ctypes.c_double * 128)()

    def f(rot=8, base=1e4, s=0, factor=2.0, n=4096, low=1.0, high=32.0, to=out):
        return lib.spec_rotary_frequencies(rot, base, s, factor, n, low, high, to)
    assert f() == 0 and f(factor=0.0) == 0 and f(s=1, n=0, low=0.0) == 0 and f(s=3) == 0
    for kw in [dict(rot=0), dict(rot=7), dict(rot=258), dict(rot=-2), dict(base=1.0), dict(base=INF), dict(base=NAN),
               dict(s=4), dict(s=-1), dict(s=1, factor=0.5), dict(s=1, factor=NAN), dict(s=1, factor=INF),
               dict(s=2, rot=2), dict(s=3, n=0), dict(s=3, low=0.0), dict(s=3, low=2.0, high=2.0), dict(s=3, high=INF),
               dict(to=None)]:
        assert f(**kw) == 1, kw
    with pytest.raises(ValueError):
        spec.spec_rotary_frequencies(8, scaling="quadratic", device="cpu")
    with pytest.raises(spec.SpecError):
        spec.spec_rotary_frequencies(9, device="cpu")


def test_rotary_refuses(lib):
    def r(x=DUMMY, row=256, heads=4, D=64, t=0, f=DUMMY, rot=64, amp=1.0, pos=DUMMY, B=3, K=2, out=DUMMY, out_row=256):
        return lib.spec_rotary(x, row, heads, D, t, f, rot, 0, amp, None, None, pos, B, K, out, out_row, None, STREAM)

    def a(c=None, layer=0, q=DUMMY, row=256, heads=4, k=DUMMY, kr=128, v=DUMMY, vr=128, f=DUMMY, rot=64, amp=1.0,
          pos=DUMMY, table=DUMMY, M=4, B=3, K=2, out=DUMMY, out_row=256):
        return lib.spec_rotary_append(cache() if c is None else c, layer, q, row, heads, k, kr, v, vr, f, rot, 0, amp, None,
                                      None, pos, table, M, B, K, out, out_row, None, STREAM)
    both = [dict(f=None), dict(rot=0), dict(rot=63), dict(rot=66), dict(rot=-2), dict(amp=INF), dict(amp=NAN),
            dict(pos=None), dict(B=0), dict(K=-1), dict(K=256), dict(out=None), dict(out=ODD), dict(out_row=252),
            dict(out_row=260), dict(row=248), dict(row=260)]
    for kw in both + [dict(x=None), dict(x=ODD), dict(heads=0), dict(D=0), dict(D=60), dict(D=264), dict(t=2),
                      dict(row=264)]:  # in place, with another stride
        assert r(**kw) == 1, kw
    for kw in both + [dict(c=cache(head_dim=60)), dict(c=cache(k=0)), dict(layer=2), dict(layer=-1), dict(q=None),
                      dict(q=ODD), dict(heads=0), dict(heads=-1), dict(k=None), dict(k=ODD), dict(kr=120), dict(kr=132),
                      dict(v=None), dict(vr=64), dict(table=None), dict(M=0), dict(M=(1 << 26) + 1)]:
        assert a(**kw) == 1, kw


def test_linear_refuses(lib):
    import paper_2607_25852_gb300 as spec

    def n(*x):
        return lib.spec_linear_workspace(*x)
    assert n(1, 0, 2, 2, 64, 64, 0) >= 256 and n(64, 255, 32, 32, 128, 128, 0) % 256 == 0
    for bad in [(0, 0, 2, 2, 64, 64, 0), (1, -1, 2, 2, 64, 64, 0), (1, 1 << 20, 2, 2, 64, 64, 0),
                (1 << 20, 1023, 2, 2, 64, 64, 0), (1, 0, 3, 2, 64, 64, 0), (1, 0, 130, 2, 64, 64, 0),
                (1, 0, 2, 0, 64, 64, 0), (1, 0, 2, 2, 0, 64, 0), (1, 0, 2, 2, 60, 64, 0), (1, 0, 2, 2, 64, 264, 0),
                (1, 0, 2, 2, 64, 64, 2)]:
        assert n(*bad) == 0, bad

    def at(q=DUMMY, row=256, heads=4, k=DUMMY, kr=128, v=DUMMY, vr=128, t=0, g=DUMMY, gr=2, s=None, layer=0, i=DUMMY, B=3,
           K=2, scale=1.0, out=DUMMY, ws=DUMMY, nb=1 << 30):
        return lib.spec_linear_attend(q, row, heads, k, kr, v, vr, t, g, gr, states() if s is None else s, layer, i, DUMMY,
                                      None, None, None, B, K, scale, out, None, ws, nb, STREAM)

    def co(k=DUMMY, kr=128, v=DUMMY, vr=128, t=0, g=DUMMY, gr=2, s=None, layer=0, i=DUMMY, o=DUMMY, B=3, K=2, ws=DUMMY,
           nb=1 << 30):
        return lib.spec_linear_commit(k, kr, v, vr, t, g, gr, states() if s is None else s, layer, i, o, None, None, None,
                                      None, B, K, None, ws, nb, STREAM)
    both = [dict(s=states(**kw)) for kw in BAD_STATES] + [
        dict(s=ctypes.c_void_p(0)), dict(k=None), dict(k=ODD), dict(kr=120), dict(kr=132), dict(v=None), dict(v=ODD),
        dict(vr=64), dict(vr=-128), dict(t=2), dict(g=None), dict(g=ctypes.c_void_p(4098)), dict(gr=1), dict(gr=-2),
        dict(layer=2), dict(layer=-1), dict(i=None), dict(B=0), dict(K=-1), dict(K=1 << 20)]
    for kw in both + [dict(q=None), dict(q=ODD), dict(row=248), dict(row=260), dict(heads=3), dict(heads=0),
                      dict(heads=256, row=1 << 14), dict(scale=INF), dict(scale=NAN), dict(out=None), dict(out=ODD)]:
        assert at(**kw) == 1, kw
    for kw in both + [dict(o=None)]:
        assert co(**kw) == 1, kw
    for f in (at, co):
        assert f(ws=None) == 2 and f(ws=ctypes.c_void_p(4100)) == 2 and f(nb=100) == 2
    with pytest.raises(spec.SpecError):
        spec.linear_workspace(1, 0, 3, 2, 64, 64, device="cpu")


def test_logprobs_refuses(lib):
    import paper_2607_25852_gb300 as spec

    def n(*x):
        return lib.spec_logprobs_workspace(*x)
    assert n(1, 0, 1, 0) >= 256 and n(64, 16, 201088, 32) < 64 << 20
    for bad in [(0, 0, 10, 1), (1, -1, 10, 1), (1, 256, 10, 1), (1, 0, 0, 1), (1, 0, 1 << 30, 1), (1, 0, 10, 33),
                (1, 0, 10, -1)]:
        assert n(*bad) == 0, bad

    def f(x=DUMMY, t=0, tok=DUMMY, B=3, K=2, V=100, temp=1.0, top=4, lp=DUMMY, a=DUMMY, b=DUMMY, ws=DUMMY, nb=1 << 30):
        return lib.spec_logprobs(x, t, None, None, tok, None, B, K, V, temp, top, lp, None, None, a, b, None, ws, nb, STREAM)
    for kw in [dict(x=None), dict(x=ctypes.c_void_p(4097)), dict(x=ctypes.c_void_p(4098), t=1), dict(t=2), dict(tok=None),
               dict(B=0), dict(K=-1), dict(K=256), dict(V=0), dict(V=1 << 30), dict(temp=-1.0), dict(temp=INF),
               dict(temp=NAN), dict(top=-1), dict(top=33), dict(lp=None), dict(a=None, b=None)]:
        assert f(**kw) == 1, kw
    assert f(ws=None) == 2 and f(ws=ctypes.c_void_p(4100)) == 2 and f(nb=100) == 2
    with pytest.raises(spec.SpecError):
        spec.logprobs_workspace(1, 0, 10, 99, device="cpu")


def test_python_refuses():
    import paper_2607_25852_gb300 as spec
    f32, i32 = torch.float32, torch.int32
    pos, freq = torch.zeros(2, dtype=torch.int64), torch.ones(4, dtype=torch.float64)
    x = torch.zeros((4, 2, 8))

    def raises(call, *a, match=None, **kw):
        with pytest.raises((ValueError, TypeError), match=match):
            call(*a, **kw)
    r = spec.spec_rotary
    raises(r, x, freq, pos, 2, 1, torch.zeros((4, 2, 16)), match="same shape")
    raises(r, x, freq, pos, 2, 1, x.half(), match="dtype")
    raises(r, x.half(), freq, pos, 2, 1, x.half(), match="element type")
    raises(r, x, freq.float(), pos, 2, 1, x, match="frequencies")
    raises(r, x, freq, pos.int(), 2, 1, x, match="pos_base")
    raises(r, x, freq, pos, 2, 2, x, match="rows for every request")
    raises(r, x.transpose(0, 1), freq, pos, 1, 1, x.transpose(0, 1), match="contiguous")
    raises(r, x, freq, pos, 2, 1, x, match="CUDA device")  # tensors that no kernel could read
    k = torch.zeros((3, 4, 2, 8))
    table = torch.zeros((2, 2), dtype=i32)
    ap = spec.spec_rotary_append
    raises(ap, x, x, x, k, k, table, pos, 2, 1, freq, None, match="both or neither")
    raises(ap, x, x, x[:, :1], k, k, table, pos, 2, 1, freq, x, match="v_new")
    raises(ap, x, x, x, k, k, table.long(), pos, 2, 1, freq, x, match="page_table")
    raises(ap, x, x, x, k, k, table, pos, 2, 2, freq, x, match="rows for every request")
    raises(ap, None, x, x, k, k, table, pos, 2, 1, freq, None, match="CUDA device")
    la, lc = spec.spec_linear_attend, spec.spec_linear_commit
    st, g, slots, ws = torch.zeros((3, 2, 8, 8)), torch.zeros(2), torch.zeros(2, dtype=i32), torch.zeros(256)
    out = torch.zeros((4, 2, 8))
    raises(la, x, x, x, g, st.double(), slots, None, 2, 1, out, ws, match="states")
    raises(la, x, x, x, g, st.transpose(2, 3), slots, None, 2, 1, out, ws, match="states")
    raises(la, x, x, x, g[:1], st, slots, None, 2, 1, out, ws, match="log_decay")
    raises(la, x, x, x, g.double(), st, slots, None, 2, 1, out, ws, match="log_decay")
    raises(la, x, x, x, g.expand(3, 2), st, slots, None, 2, 1, out, ws, match="log_decay")
    raises(la, x, x, x, g, st, slots[:1], None, 2, 1, out, ws, match="slots_in")
    raises(la, x, x, x, g, st, slots, slots.long(), 2, 1, out, ws, match="slots_out")
    raises(la, x, x, x, g, st, slots, None, 2, 1, out.bfloat16(), ws, match="out")
    raises(la, x, x, x, g, st, slots, None, 2, 2, out, ws, match="rows for every request")
    raises(la, x, x[:, :1], x, g, st, slots, None, 2, 1, out, ws, match="k")
    raises(la, x, x, x, g, st, slots, None, 2, 1, out, ws, match="CUDA device")
    raises(lc, x, x, g, st, slots, slots, slots[:1], 2, 1, ws, match="accepted_len")
    raises(lc, x, x, g, st, slots, slots, None, 2, 1, ws, match="CUDA device")
    lp = spec.spec_logprobs
    z, tok, o = torch.zeros((4, 9)), torch.zeros((2, 2), dtype=i32), torch.zeros((2, 2))
    raises(lp, z, tok, 2, 1, 10, o, ws, match="logits")
    raises(lp, z[:3], tok, 2, 1, 9, o, ws, match="rows for every request")
    raises(lp, z, tok.long(), 2, 1, 9, o, ws, match="tokens")
    raises(lp, z, tok, 2, 1, 9, o.double(), ws, match="logprob_out")
    raises(lp, z, tok, 2, 1, 9, o, ws, top_tokens_out=torch.zeros((2, 2, 3), dtype=i32),
           top_logprobs_out=torch.zeros((2, 2, 4)), match="same n")
    raises(lp, z, tok, 2, 1, 9, o, ws, rank_out=tok[:1], match="rank_out")
    raises(lp, z, tok, 2, 1, 9, o, ws, match="CUDA device")
    from paper_2607_25852_gb300.states import LinearStates
    with pytest.raises(ValueError):
        LinearStates(1, 2, 2, 64, 64, 1, 0, device="cpu")


def test_reference_recurrence():
    """The plain forms of the tests against sums written out."""
    g = torch.Generator().manual_seed(1)
    n, Dk, Dv = 5, 3, 2
    q, k, v = (torch.randn((n, 1, d), generator=g) for d in (Dk, Dk, Dv))
    d = -torch.rand((n, 1), generator=g)
    s0 = torch.randn((1, Dk, Dv), generator=g)
    out, state, _, _ = ref.linear(q, k, v, d, s0, 0.5)
    for i in range(n):
        o = torch.zeros(Dv, dtype=torch.float64)
        f = math.exp(float(d[:i + 1].double().sum()))
        o += f * (q[i, 0].double() @ s0[0].double())
        for j in range(i + 1):
            f = math.exp(float(d[j + 1:i + 1].double().sum()))
            o += f * float(q[i, 0].double() @ k[j, 0].double()) * v[j, 0].double()
        assert torch.allclose(out[i, 0], 0.5 * o, rtol=1e-12)


def test_logprobs_refuses_denormal_temperatures(lib):
    """Their reciprocal is not finite."""
    for t, code in ((1e-39, 1), (2.0 ** -149, 1)):
        assert lib.spec_logprobs(DUMMY, 0, None, None, DUMMY, None, 1, 0, 100, t, 0, DUMMY, None, None, None, None, None,
                                 DUMMY, 1 << 20, STREAM) == code


def test_fork_refuses_another_shape():
    from paper_2607_25852_gb300.states import LinearStates
    st = LinearStates(1, 1, 1, 64, 64, 3, 1, device="cpu")
    with pytest.raises(ValueError, match="parent"):
        st.fork(torch.zeros(2, dtype=torch.int32))
