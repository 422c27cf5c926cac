"""Host-side checks of spec_attend and spec_cache_*: bad arguments are refused
before any launch, by the C ABI and by the Python binding.  No GPU needed."""
import ctypes

import pytest
import torch

import paged_ref as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2607_25852_gb300 import build
    build.build()
    from paper_2607_25852_gb300 import _native
    return _native.load()


DUMMY = ctypes.c_void_p(4096)  # never dereferenced: every call fails a check
STREAM = ctypes.c_void_p(0)


def cache(**kw):
    from paper_2607_25852_gb300 import _native
    f = dict(k=4096, v=8192, dtype=0, layers=2, pages=10, page_size=16, kv_heads=2, head_dim=64, layer_stride=20480,
             page_stride=2048, token_stride=128, head_stride=64)
    f.update(kw)
    return ctypes.byref(_native.Cache(**f))


BAD_CACHES = [dict(k=0), dict(v=0), dict(k=4104), dict(dtype=2), dict(layers=0), dict(pages=0), dict(page_size=0),
              dict(kv_heads=0), dict(head_dim=0), dict(head_dim=257), dict(head_dim=60), dict(head_stride=60),
              dict(head_stride=68), dict(token_stride=-128), dict(page_stride=2052), dict(layer_stride=0),
              dict(page_stride=1 << 62)]


def test_workspaces(lib):
    import paper_2607_25852_gb300 as spec
    ws = lib.spec_attend_workspace
    for bad in [(0, 4, 8, 2, 64, 0), (4, 256, 8, 2, 64, 0), (4, -1, 8, 2, 64, 0), (4, 4, 7, 2, 64, 0),
                (4, 4, 2, 4, 64, 0), (4, 4, 130, 2, 64, 0), (4, 4, 8, 0, 64, 0), (4, 4, 8, 2, 0, 0),
                (4, 4, 8, 2, 264, 0), (4, 4, 8, 2, 60, 0), (4, 4, 8, 2, 64, 7)]:
        assert ws(*bad) == 0, bad
    n = ws(1, 0, 64, 8, 128, 0)
    assert n > 0 and n % 256 == 0 and n < 64 << 20
    assert ws(64, 16, 64, 8, 128, 0) < 256 << 20
    assert lib.spec_cache_workspace(0, 4, 16) == 0 and lib.spec_cache_workspace(4, 256, 16) == 0
    assert lib.spec_cache_workspace(4, 4, 0) == 0 and lib.spec_cache_workspace(64, 255, 1) >= 64 * 257 * 4
    with pytest.raises(spec.SpecError):
        spec.attend_workspace(0, 4, 8, 2, 64, device="cpu")
    with pytest.raises(spec.SpecError):
        spec.cache_workspace(1, -1, 16, device="cpu")
    assert "free pages" in spec.spec_error_string(spec.ERR_CACHE_FULL)


def test_attend_refuses(lib):
    def d(q=DUMMY, row=512, Hq=8, c=None, layer=0, pos=DUMMY, table=DUMMY, M=4, B=3, K=2, scale=1.0, W=0, S=0,
          out=DUMMY, ws=DUMMY, ws_bytes=1 << 30):
        return lib.spec_attend(q, row, Hq, cache() if c is None else c, layer, None, None, pos, table, M, B, K, scale, W,
                               S, out, None, None, ws, ws_bytes, STREAM)
    for kw in BAD_CACHES:
        assert d(c=cache(**kw)) == 1, kw
    assert d(c=ctypes.c_void_p(0)) == 1
    for kw in [dict(q=None), dict(q=ctypes.c_void_p(4104)), dict(row=504), dict(row=516), dict(Hq=7), dict(Hq=0),
               dict(Hq=256, row=1 << 15), dict(layer=2), dict(layer=-1), dict(pos=None), dict(table=None), dict(M=0),
               dict(M=(1 << 26) + 1), dict(B=0), dict(K=-1), dict(K=256), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("inf")), dict(scale=float("nan")), dict(W=-1), dict(S=-1), dict(out=None),
               dict(out=ctypes.c_void_p(4104))]:
        assert d(**kw) == 1, kw
    assert d(ws=None) == 2 and d(ws=ctypes.c_void_p(4100)) == 2 and d(ws_bytes=1000) == 2


def test_append_and_copy_refuse(lib):
    def a(c=None, layer=0, k=DUMMY, kr=128, v=DUMMY, vr=128, pos=DUMMY, table=DUMMY, M=4, B=3, K=2):
        return lib.spec_cache_append(cache() if c is None else c, layer, k, kr, v, vr, None, None, pos, table, M, B, K,
                                     None, STREAM)

    def cp(c=None, src=DUMMY, dst=DUMMY, n=DUMMY, most=4):
        return lib.spec_cache_copy(cache() if c is None else c, src, dst, n, most, None, STREAM)
    for kw in BAD_CACHES:
        assert a(c=cache(**kw)) == 1 and cp(c=cache(**kw)) == 1, kw
    for kw in [dict(layer=2), dict(k=None), dict(v=None), dict(k=ctypes.c_void_p(4104)), dict(kr=120), dict(vr=132),
               dict(pos=None), dict(table=None), dict(M=0), dict(B=0), dict(K=256), dict(B=1 << 27, K=15)]:
        assert a(**kw) == 1, kw
    for kw in [dict(src=None), dict(dst=None), dict(n=None), dict(most=-1)]:
        assert cp(**kw) == 1, kw
    assert cp(most=0) == 0  # nothing to copy: no launch


def test_page_operators_refuse(lib):
    far = ctypes.c_void_p(1 << 20)

    def f(t=DUMMY, r=DUMMY, p=DUMMY, Bi=2, B=3, M=4, P=9, to=far, ro=DUMMY):
        return lib.spec_cache_fork(t, r, p, Bi, B, M, P, to, ro, None, STREAM)
    for kw in [dict(t=None), dict(r=None), dict(p=None), dict(to=None), dict(ro=None), dict(Bi=0), dict(B=0), dict(M=0),
               dict(P=0), dict(to=DUMMY), dict(to=ctypes.c_void_p(4096 + 28))]:
        assert f(**kw) == 1, kw

    def rs(t=DUMMY, r=DUMMY, pos=DUMMY, B=3, K=2, M=4, P=9, ps=16, s=DUMMY, d=DUMMY, n=DUMMY, g=DUMMY, ws=DUMMY, b=4096):
        return lib.spec_cache_reserve(t, r, None, None, pos, B, K, M, P, ps, s, d, n, g, None, ws, b, STREAM)
    for kw in [dict(t=None), dict(r=None), dict(pos=None), dict(s=None), dict(d=None), dict(n=None), dict(g=None),
               dict(B=0), dict(K=256), dict(M=0), dict(P=0), dict(ps=0), dict(M=1 << 20, ps=1 << 11)]:
        assert rs(**kw) == 1, kw
    assert rs(ws=None) == 2 and rs(b=4) == 2 and rs(ws=ctypes.c_void_p(4100)) == 2

    def rl(t=DUMMY, r=DUMMY, pos=DUMMY, B=3, M=4, P=9, ps=16, W=0, S=0):
        return lib.spec_cache_release(t, r, pos, None, B, M, P, ps, W, S, None, STREAM)
    for kw in [dict(t=None), dict(r=None), dict(pos=None), dict(B=0), dict(M=0), dict(P=0), dict(ps=0), dict(W=-1),
               dict(S=-1)]:
        assert rl(**kw) == 1, kw

    def co(t=DUMMY, r=DUMMY, B=3, M=4, P=9, s=DUMMY, d=DUMMY, m=DUMMY, n=DUMMY):
        return lib.spec_cache_compact(t, r, B, M, P, s, d, m, n, None, STREAM)
    for kw in [dict(t=None), dict(r=None), dict(B=0), dict(M=0), dict(P=0), dict(s=None), dict(d=None), dict(m=None),
               dict(n=None)]:
        assert co(**kw) == 1, kw


def test_python_binding_refuses_mismatched_tensors(lib):
    import paper_2607_25852_gb300 as spec
    bf, i32, i64 = torch.bfloat16, torch.int32, torch.int64
    k = torch.zeros((4, 8, 2, 64), dtype=bf)
    q = torch.zeros((3, 4, 64), dtype=bf)
    table, pos, ws = torch.zeros((1, 2), dtype=i32), torch.zeros(1, dtype=i64), torch.zeros(256, dtype=torch.uint8)

    def attend(q=q, k=k, v=None, table=table, pos=pos, out=None, **kw):
        spec.spec_attend(q, k, torch.zeros_like(k) if v is None else v, table, pos, 1, 2,
                         torch.zeros_like(q) if out is None else out, ws, **kw)
    for kw in [dict(v=k.float()), dict(v=k[:3]), dict(k=k[0], v=k[0]), dict(k=k.transpose(2, 3), v=k.transpose(2, 3)),
               dict(q=q[:2]), dict(q=q[..., :32]), dict(out=q.float()), dict(out=q[:2]), dict(table=table.long()),
               dict(table=table[0]), dict(pos=pos.int()), dict(pos=pos[:0]), dict(depth=torch.zeros(0, dtype=i32)),
               dict(row_offsets=torch.zeros(1, dtype=i32)), dict(lse_out=torch.zeros(3)),
               dict(lse_out=torch.zeros((3, 4), dtype=bf))]:
        with pytest.raises(ValueError):
            attend(**kw)
    with pytest.raises(TypeError):
        attend(q=q.float())
    with pytest.raises(TypeError):
        attend(k=k.half(), v=k.half(), q=q.half())
    with pytest.raises(ValueError):
        spec.spec_cache_append(q[:, :2], q[:2, :2], k, k.clone(), table, pos, 1, 2)
    with pytest.raises(ValueError):
        spec.spec_cache_fork(table, torch.zeros(4, dtype=i32), pos.int(), torch.zeros((2, 2), dtype=i32),
                             torch.zeros(4, dtype=i32))   # a parent per request
    with pytest.raises(ValueError):
        spec.spec_cache_compact(table, torch.zeros(9, dtype=i32), torch.zeros(3, dtype=i32),
                                torch.zeros(4, dtype=i32), torch.zeros(9, dtype=i32), torch.zeros(2, dtype=i32))


# ---------------------------------------------------------------------------
# The tests' own plain implementations, on cases worked out by hand
# ---------------------------------------------------------------------------
def test_plain_attention_by_hand():
    k = torch.tensor([[[[1.0]], [[2.0]]], [[[3.0]], [[0.0]]]])      # pages of two positions, one head, one d
    v = torch.tensor([[[[10.0]], [[20.0]]], [[[40.0]], [[0.0]]]])
    q = torch.tensor([[[0.0]], [[1.0]]])
    rows = ref.Rows([1], 1)
    table = torch.tensor([[0, 1]])
    out, lse, mass, big = ref.attend(q, k, v, table, [1], rows, 1.0)
    assert out[0, 0, 0] == 15.0                                      # positions 0 and 1, equal weights
    e = torch.exp(torch.tensor([1.0, 2.0, 3.0], dtype=torch.float64))
    assert torch.isclose(out[1, 0, 0], (e * torch.tensor([10.0, 20.0, 40.0])).sum() / e.sum())
    assert torch.isclose(lse[1, 0], torch.log(e.sum())) and big[1, 0] == 3.0
    out, lse, _, _ = ref.attend(q, k, v, table, [-1], rows, 1.0)
    assert out[0, 0, 0] == 0 and lse[0, 0] == float("-inf") and out[1, 0, 0] == 10.0
    assert ref.visible(9, 3, 2) == [0, 1, 7, 8, 9] and ref.visible(3, 3, 2) == [0, 1, 2, 3]
    assert ref.visible(2, 3, 9) == [0, 1, 2] and ref.visible(5, 1, 0) == [5]


def test_plain_pages_by_hand():
    table, refs = [[0, 1, -1], [0, 2, -1]], [2, 1, 1, 0, 0, 0]
    assert ref.fork(table, refs, [1, 1, -1]) == ([[0, 2, -1], [0, 2, -1], [-1] * 3], [2, 0, 2, 0, 0, 0])
    t, r, src, dst, used, granted, full = ref.reserve([[0, 2, -1], [0, 2, -1]], [2, 0, 2, 0, 0, 0], [7, 4], [1, 0], 4)
    assert t == [[0, 1, 3], [0, 4, -1]] and r == [2, 1, 0, 1, 1, 0]
    assert (src, dst, used, granted, full) == ([2, 2], [1, 4], 3, [1, 1], False)
    assert ref.release(table, refs, [4, 0], 4) == ([[0, -1, -1], [-1, -1, -1]], [1, 0, 0, 0, 0, 0])
    assert ref.release([[5, 6, 7]], [0] * 5 + [1] * 3, [12], 4, 5, 1)[0] == [[5, -1, 7]]
    assert ref.compact([[4, -1, 1]], [0, 2, 0, 0, 1]) == ([[0, -1, 1]], [1, 2, 0, 0, 0], [4], [0],
                                                          [-1, 1, -1, -1, 0], 2)
