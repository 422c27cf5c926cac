"""How spec_attend divides its work: the CTAs' segments cover every tile of every
item once, the parts of an item know one another, and the arrival counters are
back at zero after a call, also where CTAs leave their share unfinished (a
bounded wait that gave up).  The division's own functions run here in a small
kernel of their own, without the attention."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2607_25852_gb300 import build

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
DEV = "cuda"
FIELDS = ("request", "head", "col0", "cols", "tile0", "ntiles", "count", "slot", "first_cta", "step", "parts", "cta")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("shares") / "shares.so")
    subprocess.run([build.NVCC, *build.ARCH, *build.FLAGS, "-I", build.CSRC, "-shared", "-o", so,
                    os.path.join(HERE, "attend_shares.cu")], check=True, capture_output=True, timeout=300)
    return ctypes.CDLL(so)


def shares(lib, pos, depth, K, G, Hkv, tile, ct, ctas, lists, stop=None, window=0, sinks=0, page_size=128, max_pages=1 << 23,
           threads=256, part_cost=4, item_cost=4, part_tiles=6.0, arrived=None):
    """The listed segments, and the arrival counters after the call."""
    B, most = len(pos), 1 << 16
    off = [0]
    for n in depth:
        off.append(off[-1] + n + 1)
    i32 = dict(dtype=torch.int32, device=DEV)
    arrived = torch.zeros(ctas, **i32) if arrived is None else arrived
    t = dict(off=torch.tensor(off, **i32), depth=torch.tensor(depth, **i32), pos=torch.tensor(pos, device=DEV),
             stop=torch.tensor([1 << 30] * ctas if stop is None else stop, **i32),
             out=torch.zeros((most, len(FIELDS)), **i32), total=torch.zeros(1, **i32), status=torch.zeros(1, **i32))
    p = {n: ctypes.c_void_p(x.data_ptr()) for n, x in t.items()}
    torch.cuda.synchronize()
    code = lib.attend_shares(tile, threads, G, Hkv, page_size, max_pages, B, K, window, sinks, min(tile, page_size), ct, ctas,
                             lists, part_cost, item_cost, ctypes.c_float(part_tiles), p["off"], p["depth"], p["pos"],
                             ctypes.c_void_p(arrived.data_ptr()), p["stop"], p["out"], most, p["total"], p["status"])
    torch.cuda.synchronize()
    n = int(t["total"])
    assert code == 0 and n <= most and int(t["status"]) == 0
    return [dict(zip(FIELDS, row)) for row in t["out"][:n].tolist()], arrived


def check(listed, pos, depth, G, Hkv, tile, ct, window=0):
    items = {}
    for s in listed:
        items.setdefault((s["request"], s["head"], s["col0"]), []).append(s)
    want = {(i, h, c) for i in range(len(pos)) for h in range(Hkv) for c in range(0, (depth[i] + 1) * G, ct)}
    assert set(items) == want
    slots = [s["slot"] for s in listed if s["slot"] >= 0]
    assert len(slots) == len(set(slots))
    for (i, h, c0), parts in items.items():
        cols = min((depth[i] + 1) * G, c0 + ct) - c0
        last = pos[i] + (c0 + cols - 1) // G
        parts.sort(key=lambda s: s["tile0"])
        at = 0
        for s in parts:
            assert s["tile0"] == at and s["ntiles"] > 0 and s["cols"] == cols
            at += s["ntiles"]
        assert all(s["count"] == at for s in parts)
        if window == 0:
            assert at == max(0, last) // tile + 1
        if len(parts) == 1:
            assert parts[0]["slot"] == -1
            continue
        for x, s in enumerate(parts):
            assert s["parts"] == len(parts) and s["first_cta"] == parts[0]["cta"]
            assert s["cta"] == s["first_cta"] + x * s["step"] and s["slot"] == 2 * s["cta"] + (1 if x == 0 else 0)


CASES = [  # pos, depth, G, Hkv, tile, columns per item, CTAs, lists
    ([20000], [0], 8, 1, 128, 16, 152, 1),
    ([20000, 300], [0, 0], 8, 8, 128, 16, 152, 8),
    ([20000, 300, -1, 5], [4, 16, 0, 3], 8, 2, 128, 144, 152, 2),
    ([1000 + 37 * i for i in range(64)], [(5 * i) % 17 for i in range(64)], 8, 8, 128, 144, 152, 8),
    ([4000] * 4, [255] * 4, 4, 8, 128, 256, 152, 8),
    ([900 * (i % 7) for i in range(700)], [i % 3 for i in range(700)], 3, 1, 64, 32, 304, 1),
    ([3000, 10, 90], [31, 0, 40], 64, 1, 64, 32, 152, 1),
    # 2^33 tiles of one head: as far as positions, rows and heads of a group go
    ([(1 << 30) - 256], [255], 64, 1, 64, 32, 152, 1),
    ([(1 << 30) - 300, 7], [255, 255], 64, 2, 64, 32, 304, 2),
    ([(1 << 30) - 256] * 3, [255] * 3, 64, 1, 128, 256, 152, 1),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("window", [0, 500])
def test_every_tile_is_done_once(lib, case, window):
    pos, depth, G, Hkv, tile, ct, ctas, lists = CASES[case]
    listed, arrived = shares(lib, pos, depth, max(depth), G, Hkv, tile, ct, ctas, lists, window=window)
    check(listed, pos, depth, G, Hkv, tile, ct, window)
    assert int(arrived.abs().sum()) == 0


@pytest.mark.parametrize("case", range(len(CASES)))
def test_counters_are_ready_after_an_aborted_call(lib, case):
    pos, depth, G, Hkv, tile, ct, ctas, lists = CASES[case]
    g = torch.Generator().manual_seed(case)
    arrived = None
    for _ in range(6):  # CTAs that give up at once, after a segment, or not at all
        stop = torch.tensor([0, 0, 1, 1 << 30])[torch.randint(0, 4, (ctas,), generator=g)].tolist()
        listed, arrived = shares(lib, pos, depth, max(depth), G, Hkv, tile, ct, ctas, lists, stop, arrived=arrived)
        check(listed, pos, depth, G, Hkv, tile, ct)
        assert int(arrived.abs().sum()) == 0
