"""The paged key-value cache operators: cases, inputs, plain forms and exact values.

Five operators serve the target forward of a speculative round over a paged
key-value cache:

  attend  attention of the packed verification rows (one per request when
          nothing is drafted) over the whole cached context
  window  the same with a sliding window and a few first tokens (sinks) that
          stay visible; pages between the two have been given back
  append  the new rows' keys and values written into their pages
  branch  requests forked (pages shared by reference count), the pages that
          the next round writes reserved, shared ones copied
  sweep   rejected and finished requests' pages released, the live pages
          compacted to the low end of the cache

``run`` computes them with elementary torch operations, or through the
package's entry points where ``own`` is set.
"""
import math
import random

import torch

own = False

GOLDEN = 0.6180339887498949
DEVICE = "cuda"


def listed():
    return [
        # one request, one new token, a chat-length context: the call's latency counts
        dict(name="attend_token_short", op="attend", B=1, K=0, ragged=False, lo=913, hi=913, Hq=32, Hkv=8, D=128,
             page=16, dtype="bf16"),
        # two requests deep in a long document: the cache's length has to be split to fill the GPU
        dict(name="attend_token_long", op="attend", B=2, K=0, ragged=False, lo=70001, hi=131071, Hq=64, Hkv=8, D=128,
             page=64, dtype="bf16"),
        # a batch of 64 verified at up to 17 rows each, budgets cut per request, contexts of every length
        dict(name="attend_verify_batch", op="attend", B=64, K=16, ragged=True, lo=512, hi=8192, Hq=64, Hkv=8, D=128,
             page=32, dtype="bf16"),
        # the fp32 form, as a numerics run of a small target uses it
        dict(name="attend_verify_fp32", op="attend", B=8, K=4, ragged=True, lo=333, hi=2100, Hq=16, Hkv=4, D=64,
             page=16, dtype="f32"),
        # single tokens of a large batch with a local window; the sinks are the first four tokens
        dict(name="window_token_batch", op="window", B=128, K=0, ragged=False, lo=100, hi=32768, Hq=64, Hkv=8, D=64,
             page=16, dtype="bf16", window=1024, sinks=4),
        # a prompt's chunk of 256 rows per request with a local window
        dict(name="window_chunk", op="window", B=4, K=255, ragged=False, lo=700, hi=9000, Hq=32, Hkv=8, D=128,
             page=64, dtype="bf16", window=2048, sinks=16),
        # a round's rows, keys and values as views of one fused projection output
        dict(name="append_round", op="append", B=64, K=16, ragged=True, lo=512, hi=8192, Hkv=8, D=128, page=16,
             dtype="bf16", fused=True),
        # prompt chunks, fp32, pages that are no power of two
        dict(name="append_chunk_fp32", op="append", B=6, K=255, ragged=False, lo=300, hi=5001, Hkv=12, D=96, page=24,
             dtype="f32", fused=False),
        # a handful of prompts, each sampled three times
        dict(name="branch_few", op="branch", B=4, fan=3, K=4, lo=100, hi=1500, slots=128, page=16, pages=1024,
             L=2, Hkv=2, D=64, dtype="bf16"),
        # a serving batch branched four ways, long tables
        dict(name="branch_batch", op="branch", B=64, fan=4, K=16, lo=500, hi=4096, slots=320, page=16, pages=32768,
             L=2, Hkv=2, D=64, dtype="bf16"),
        # a small batch after a verification: rejected drafts' pages go back
        dict(name="sweep_few", op="sweep", B=6, K=7, lo=50, hi=900, slots=64, page=16, pages=509, L=2, Hkv=2, D=64,
             dtype="bf16", retire=3, window=0, sinks=0),
        # a serving batch, every third request finished, windowed layers: many pages move
        dict(name="sweep_batch", op="sweep", B=96, K=16, lo=500, hi=6000, slots=384, page=16, pages=32768, L=2, Hkv=2,
             D=64, dtype="bf16", retire=3, window=2048, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges, no dearer than the largest listed one."""
    op = rng.choice(["attend", "attend", "window", "append", "branch", "sweep"])
    if op in ("attend", "window"):
        f32 = rng.random() < 0.2
        Hkv = rng.choice([1, 2, 4, 8])
        group = rng.choice([1, 3, 4, 8])
        D = rng.choice([64, 128])
        page = rng.choice([16, 32, 64, 128])
        if rng.random() < 0.15:  # the layouts of less common models
            D, page = rng.choice([80, 96, 256]), rng.choice([10, 24, 48])
        K = rng.choice([0, 0, 3, 7, 16, _log_int(rng, 17, 255)])
        case = dict(op=op, B=_log_int(rng, 1, 128), K=K, ragged=rng.random() < 0.5 and K > 0, Hq=Hkv * group, Hkv=Hkv,
                    D=D, page=page, dtype="f32" if f32 else "bf16")
        if op == "window":
            case.update(window=_log_int(rng, 16, 4096), sinks=rng.choice([0, 1, 4, 64]))
        hi = _log_int(rng, 1, 131072)
        case.update(lo=max(1, int(hi * rng.uniform(0.05, 1.0))), hi=hi)
        slow = 8.0 if f32 or D not in (64, 128) or page % 16 else 1.0
        largest = work(listed()[2])
        while True:
            w = work(case)
            if w["bytes"] * slow <= largest["bytes"] and w["flops"] * slow <= largest["flops"] and \
                    case["B"] * (case["hi"] + 256) * Hkv * D <= 1 << 31:
                return case
            if case["B"] > 1:
                case["B"] = (case["B"] + 1) // 2
            elif case["hi"] > 1:
                case["hi"] = (case["hi"] + 1) // 2
                case["lo"] = max(1, min(case["lo"], case["hi"]))
            else:
                case["K"] = case["K"] // 2
    if op == "append":
        K = rng.choice([0, 4, 16, _log_int(rng, 17, 255)])
        B = min(_log_int(rng, 1, 128), max(1, 1600 // (K + 1)))
        hi = _log_int(rng, 8, 8192)
        return dict(op=op, B=B, K=K, ragged=rng.random() < 0.5 and K > 0, lo=max(1, hi // rng.randint(1, 16)), hi=hi,
                    Hkv=rng.choice([1, 4, 8]), D=rng.choice([64, 96, 128]), page=rng.choice([10, 16, 32, 64, 128]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), fused=rng.random() < 0.5)
    if op == "branch":
        B, fan = _log_int(rng, 1, 64), rng.randint(1, 4)
        page = rng.choice([16, 24, 32, 64])
        hi = _log_int(rng, 20, 4096)
        K = rng.choice([0, 3, 16, 40])
        slots = (hi + K) // page + 2 + rng.randint(0, 64)
        need = B * slots + B * fan * (K // page + 2)
        return dict(op=op, B=B, fan=fan, K=K, lo=max(1, hi // rng.randint(1, 8)), hi=hi, slots=slots, page=page,
                    pages=min(32768, need + rng.randint(0, need)), L=rng.randint(1, 2), Hkv=rng.choice([1, 2]), D=64,
                    dtype=rng.choice(["bf16", "f32"]) if need < 8000 else "bf16")
    B = _log_int(rng, 1, 96)
    page = rng.choice([16, 24, 32, 64])
    hi = _log_int(rng, 20, 6000)
    K = rng.choice([0, 3, 16, 40])
    slots = (hi + K) // page + 2 + rng.randint(0, 32)
    need = B * slots
    return dict(op="sweep", B=B, K=K, lo=max(1, hi // rng.randint(1, 8)), hi=hi, slots=slots, page=page,
                pages=max(64, min(32768, need + rng.randint(0, need))), L=rng.randint(1, 2), Hkv=rng.choice([1, 2]), D=64,
                dtype=rng.choice(["bf16", "f32"]) if need < 8000 else "bf16", retire=rng.randint(2, 5),
                window=rng.choice([0, 0, _log_int(rng, 16, 4096)]), sinks=rng.choice([0, 4, 40]))


# ---------------------------------------------------------------------------
# Lengths and depths: functions of the case alone
# ---------------------------------------------------------------------------
def _contexts(case):
    """pos_base per request (tokens already cached), spread over [lo, hi] on a log scale."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    if B == 1:
        return [hi]
    if B == 2:
        return [lo, hi]
    out = []
    for i in range(B):
        f = ((i + 1) * GOLDEN) % 1.0
        out.append(int(round(math.exp(math.log(lo) + f * (math.log(hi) - math.log(lo))))))
    return out


def _depths(case):
    K = case["K"]
    if not case.get("ragged"):
        return [K] * case["B"]
    return [(5 * i + 3) % (K + 1) for i in range(case["B"])]


def _element(case):
    return 4 if case["dtype"] == "f32" else 2


def _page_bytes(case):
    return case["page"] * case["Hkv"] * case["D"] * _element(case)


def _visible(case, p):
    """Keys that a row at position p sees."""
    W = case.get("window", 0)
    if not W or p + 1 <= W:
        return p + 1
    return W + min(case["sinks"], p + 1 - W)


def _covered(case, p0, p1):
    """Distinct keys that rows at positions p0..p1 see."""
    W = case.get("window", 0)
    if not W:
        return p1 + 1
    first = max(0, p0 - W + 1)
    return p1 + 1 - first + min(case["sinks"], first)


def work(case):
    e = _element(case)
    if case["op"] in ("attend", "window"):
        keys = pairs = rows = entries = 0
        for p, n in zip(_contexts(case), _depths(case)):
            c = _covered(case, p, p + n)
            keys += c
            entries += (c + case["page"] - 1) // case["page"]
            rows += n + 1
            pairs += sum(_visible(case, p + j) for j in range(n + 1))
        return {"bytes": keys * 2 * case["Hkv"] * case["D"] * e + 2 * rows * case["Hq"] * case["D"] * e +
                4 * rows * case["Hq"] + 4 * entries + 8 * case["B"],
                "flops": 4 * pairs * case["Hq"] * case["D"]}
    if case["op"] == "append":
        rows = sum(n + 1 for n in _depths(case))
        return {"bytes": 4 * rows * case["Hkv"] * case["D"] * e + 4 * rows + 8 * case["B"], "flops": 0}
    if case["op"] == "branch":
        B, F = case["B"], case["fan"]
        copies = sum(F for p in _contexts(case) if p % case["page"]) if F > 1 else 0
        return {"bytes": 4 * case["slots"] * B * (1 + F) + 8 * case["pages"] +
                2 * copies * 2 * case["L"] * _page_bytes(case), "flops": 0}
    moves, _ = _expected_moves(case)
    return {"bytes": 8 * case["slots"] * case["B"] + 8 * case["pages"] + 4 * case["pages"] +
            2 * moves * 2 * case["L"] * _page_bytes(case), "flops": 0}


def _expected_moves(case):
    """Live pages after a sweep and how many of them lie past the live count on
    average when the cache's pages are in random order."""
    live = 0
    for i, keep in enumerate(_kept(case)):
        if keep == 0:
            continue
        n = (keep + case["page"] - 1) // case["page"]
        W = case.get("window", 0)
        if W:
            lo = (min(case["sinks"], keep) + case["page"] - 1) // case["page"]
            first = max(0, keep - W + 1) // case["page"]
            n -= max(0, first - lo)
        live += n
    live = min(live, case["pages"])
    return int(live * (1.0 - live / case["pages"])), live


def _kept(case):
    """Tokens that stay per request after the round of a sweep (0: the request is done)."""
    out = []
    for i, p in enumerate(_contexts(case)):
        out.append(0 if i % case["retire"] == 0 else p + 1 + (3 * i) % (case["K"] + 1))
    return out


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(shape, dtype, g):
    return torch.randn(shape, device=DEVICE, dtype=torch.float32, generator=g).to(dtype) \
        if math.prod(shape) < 1 << 26 else torch.randn(shape, device=DEVICE, dtype=dtype, generator=g)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _i64(x):
    return torch.tensor(x, dtype=torch.int64, device=DEVICE)


def _row_layout(case):
    """row_offsets and depth on the host; packed rows of request i at row_offsets[i]."""
    depth = _depths(case)
    offsets = [0]
    for n in depth:
        offsets.append(offsets[-1] + n + 1)
    return offsets, depth


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"case": case, "op": op}
    if own:
        import paper_2607_25852_gb300 as spec
        s["spec"] = spec
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    if op in ("attend", "window", "append"):
        _prepare_rows(case, g, s)
    else:
        _prepare_pages(case, g, s)
    return s


def _prepare_rows(case, g, s):
    B, K, ps, Hkv, D, dt = case["B"], case["K"], case["page"], case["Hkv"], case["D"], _dtype(case)
    offsets, depth = _row_layout(case)
    ctx = _contexts(case)
    R = offsets[-1]
    W, S = case.get("window", 0), case.get("sinks", 0)
    slots = max((p + n) // ps + 1 for p, n in zip(ctx, depth))
    holders = []                                         # (request, slot) that hold a page
    for i, (p, n) in enumerate(zip(ctx, depth)):
        first = max(0, p - W + 1) // ps if W else 0      # pages between sinks and window were given back
        keep = (S + ps - 1) // ps if W else 0
        holders += [(i, t) for t in range((p + n) // ps + 1) if t >= first or t < keep]
    pages = len(holders) + len(holders) // 8 + 1
    perm = torch.randperm(pages, device=DEVICE, generator=g)[:len(holders)].to(torch.int32)
    table = torch.full((B, slots), -1, dtype=torch.int32, device=DEVICE)
    hi = _i64(holders)
    table[hi[:, 0], hi[:, 1]] = perm
    s.update(offsets=offsets, depth_host=depth, ctx=ctx, R=R, table=table, pos_base=_i64(ctx),
             row_offsets=_i32(offsets), depth=_i32(depth))
    s["k"] = _randn((pages, ps, Hkv, D), dt, g)
    s["v"] = _randn((pages, ps, Hkv, D), dt, g)
    if case["op"] == "append":
        if case["fused"]:  # rows of [queries | keys | values], as one projection writes them
            rows = _randn((R, 3, Hkv, D), dt, g)
            s["k_new"], s["v_new"] = rows[:, 1], rows[:, 2]
        else:
            s["k_new"], s["v_new"] = _randn((R, Hkv, D), dt, g), _randn((R, Hkv, D), dt, g)
        return
    # what no request has written yet is uninitialised memory: here NaN past every end
    last = _i64([p + n for p, n in zip(ctx, depth)])
    page = table[torch.arange(B, device=DEVICE), last // ps].long()
    past = torch.arange(ps, device=DEVICE)[None] > (last % ps)[:, None]
    for c in (s["k"], s["v"]):
        c[page] = torch.where(past[:, :, None, None], torch.full((), float("nan"), dtype=dt, device=DEVICE), c[page])
    # the first token draws much of the attention in trained models
    first = table[:, 0].long()
    s["k"][first, 0] *= 1.5
    s["q"] = _randn((R, case["Hq"], D), dt, g) * 1.25
    s["longest"] = max(p + n + 1 - (max(0, p - W + 1) if W else 0) for p, n in zip(ctx, depth))
    if own:
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((R, case["Hq"]), dtype=torch.float32, device=DEVICE)
        s["ws"] = s["spec"].attend_workspace(B, K, case["Hq"], Hkv, D, dt, DEVICE)


def _prepare_pages(case, g, s):
    B, ps, P, M = case["B"], case["page"], case["pages"], case["slots"]
    ctx = _contexts(case)
    sweep = case["op"] == "sweep"
    # a branch starts from the committed tokens, a sweep follows a round that wrote K+1 rows more
    have = [(p + case["K"]) // ps + 1 if sweep else (p + ps - 1) // ps for p in ctx]
    order = torch.randperm(P, generator=g, device=DEVICE).tolist()
    table = [[-1] * M for _ in range(B)]
    refs = [0] * P
    common = min(have) // 2 if B > 1 else 0             # a prompt's prefix that neighbours share
    nxt = 0
    for i in range(B):
        for t in range(min(have[i], M)):
            if i % 2 == 1 and t < common:
                page = table[i - 1][t]
            elif nxt < P:
                page = order[nxt]
                nxt += 1
            else:
                page = -1
            table[i][t] = page
            if page >= 0:
                refs[page] += 1
    for k in range(nxt, min(P, nxt + P // 64)):          # pages that a prefix store holds
        refs[order[k]] = 1
    s.update(table=_i32(table), refs=_i32(refs), ctx=ctx, pos_base=_i64(ctx))
    shape = (case["L"], P, ps, case["Hkv"], case["D"])
    s["k"], s["v"] = _randn(shape, _dtype(case), g), _randn(shape, _dtype(case), g)
    if not sweep:
        B2 = B * case["fan"]
        parent = torch.randperm(B2, generator=g, device=DEVICE) // case["fan"]
        s["parent"] = parent.to(torch.int32)
        s["pos_new"] = s["pos_base"][parent]
        cap = B2 * (case["K"] // ps + 2)
        s["cap"] = cap
        if own:
            s["out"] = dict(table=torch.empty((B2, M), dtype=torch.int32, device=DEVICE),
                            refs=torch.empty(P, dtype=torch.int32, device=DEVICE),
                            src=torch.empty(cap, dtype=torch.int32, device=DEVICE),
                            dst=torch.empty(cap, dtype=torch.int32, device=DEVICE),
                            counts=torch.empty(2, dtype=torch.int32, device=DEVICE),
                            granted=torch.empty(B2, dtype=torch.int32, device=DEVICE))
            s["ws"] = s["spec"].cache_workspace(B2, case["K"], ps, DEVICE)
        return
    accepted = [k - p - 1 for k, p in zip(_kept(case), ctx)]
    # a finished request keeps nothing: position -1 and nothing accepted
    s["pos_now"] = _i64([p if a >= 0 else -1 for p, a in zip(ctx, accepted)])
    s["accepted"] = _i32([max(a, 0) for a in accepted])
    if own:
        cap = max(1, P // 2)
        s["out"] = dict(src=torch.empty(cap, dtype=torch.int32, device=DEVICE),
                        dst=torch.empty(cap, dtype=torch.int32, device=DEVICE),
                        map=torch.empty(P, dtype=torch.int32, device=DEVICE),
                        counts=torch.empty(2, dtype=torch.int32, device=DEVICE))


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    return {"attend": _attend, "window": _attend, "append": _append, "branch": _branch,
            "sweep": _sweep}[state["op"]](state)


def _attend(s):
    c = s["case"]
    W, S = c.get("window", 0), c.get("sinks", 0)
    if own:
        s["spec"].spec_attend(s["q"], s["k"], s["v"], s["table"], s["pos_base"], c["B"], c["K"], s["out"], s["ws"],
                              row_offsets=s["row_offsets"], depth=s["depth"], window=W, sinks=S, lse_out=s["lse"],
                              status=s["status"])
        return {"out": s["out"], "lse": s["lse"]}
    # the whole batch at once, padded to its longest request: keys and rows past a request's own are masked
    B, N, Hq, Hkv, D, ps = c["B"], c["K"] + 1, c["Hq"], c["Hkv"], c["D"], c["page"]
    G, p = Hq // Hkv, s["pos_base"][:, None]
    first = (p - W + 1).clamp(min=0) if W else torch.zeros_like(p)
    pos = first + torch.arange(s["longest"], device=DEVICE)                       # [B, T]
    real = pos <= p + s["depth"][:, None]
    if W and S:
        sink = torch.arange(S, device=DEVICE).expand(B, S)
        pos, real = torch.cat([sink, pos], 1), torch.cat([sink < first, real], 1)
    page = s["table"].long().gather(1, torch.where(real, pos // ps, 0))
    at = (page * ps + pos % ps).clamp(min=0)
    k = s["k"].view(-1, Hkv, D)[at].float().permute(0, 2, 3, 1)                   # [B, Hkv, D, T]
    v = torch.where(real[..., None, None], s["v"].view(-1, Hkv, D)[at].float(), 0.0).transpose(1, 2)
    j = torch.arange(N, device=DEVICE)
    has = j <= s["depth"][:, None]                                                # [B, N]
    row = torch.where(has, s["row_offsets"][:-1, None] + j, 0).long()
    q = s["q"].float()[row].view(B, N, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, N * G, D)
    x = torch.matmul(q, k).mul_(1.0 / math.sqrt(D)).view(B, Hkv, N, G, -1)
    seen = real[:, None] & (pos[:, None] <= (p + j)[..., None])
    if W:
        seen &= (pos[:, None] > (p + j - W)[..., None]) | (pos[:, None] < S)
    x.masked_fill_(~seen[:, None, :, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)  # the rows that pad a request may see nothing
    e = x.sub_(m).exp_()
    l = e.sum(-1, keepdim=True)
    o = torch.matmul(e.div_(l).view(B, Hkv, N * G, -1), v).view(B, Hkv, N, G, D)
    out = o.transpose(1, 2)[has].reshape(-1, Hq, D).to(s["q"].dtype)
    lse = (m + torch.log(l)).squeeze(-1).transpose(1, 2)[has].reshape(-1, Hq)
    return {"out": out, "lse": lse}


def _append(s):
    c = s["case"]
    if own:
        s["spec"].spec_cache_append(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["pos_base"], c["B"], c["K"],
                                    row_offsets=s["row_offsets"], depth=s["depth"], status=s["status"])
        return {"k": s["k"], "v": s["v"]}
    ps = c["page"]
    off = s["row_offsets"].long()
    r = torch.arange(s["R"], device=DEVICE)
    i = (r[:, None] >= off[None, 1:]).sum(1)
    pos = s["pos_base"][i] + r - off[i]
    page = s["table"][i, pos // ps].long()
    s["k"][page, pos % ps] = s["k_new"]
    s["v"][page, pos % ps] = s["v_new"]
    return {"k": s["k"], "v": s["v"]}


def _branch(s):
    c = s["case"]
    ps, P, M, K = c["page"], c["pages"], c["slots"], c["K"]
    B2 = c["B"] * c["fan"]
    if own:
        spec, o = s["spec"], s["out"]
        spec.spec_cache_fork(s["table"], s["refs"], s["parent"], o["table"], o["refs"], status=s["status"])
        spec.spec_cache_reserve(o["table"], o["refs"], s["pos_new"], B2, K, ps, o["src"], o["dst"], o["counts"],
                                o["granted"], s["ws"], status=s["status"])
        spec.spec_cache_copy(s["k"], s["v"], o["src"], o["dst"], o["counts"], status=s["status"])
        return dict(o, k=s["k"], v=s["v"])
    # fork: rows follow their parents, counts follow the rows
    table = s["table"][s["parent"].long()]
    refs = s["refs"] + _count(table, P) - _count(s["table"], P)
    # reserve: slots that positions pos..pos+K touch and that are empty or shared
    slot = torch.arange(M, device=DEVICE)[None]
    touched = (slot >= (s["pos_new"] // ps)[:, None]) & (slot <= ((s["pos_new"] + K) // ps)[:, None])
    empty = table < 0
    shared = ~empty & (refs[table.clamp(min=0).long()] > 1)
    need = touched & (empty | shared)
    per = need.sum(1)
    free = (refs == 0).sum()
    granted = (per == 0) | (per.cumsum(0) <= free)
    need &= granted[:, None]
    rank = need.flatten().cumsum(0) - 1
    free_first = torch.argsort((refs != 0).to(torch.uint8), stable=True)
    flat, want = table.flatten(), need.flatten()
    page = torch.where(want, free_first[rank.clamp(min=0).clamp(max=P - 1)].to(torch.int32), flat)
    moved = (need & shared).flatten()
    at = moved.cumsum(0) - 1
    at = torch.where(moved, at, s["cap"])
    src = torch.full((s["cap"] + 1,), -1, dtype=torch.int32, device=DEVICE).scatter_(0, at, flat)[:-1]
    dst = torch.full((s["cap"] + 1,), -1, dtype=torch.int32, device=DEVICE).scatter_(0, at, page)[:-1]
    refs = refs + _count(torch.where(want, page, -1), P) - _count(torch.where(moved, flat, -1), P)
    counts = torch.stack([moved.sum(), want.sum()]).to(torch.int32)
    _copy(s, src, dst)
    return {"table": page.view(B2, M), "refs": refs, "src": src, "dst": dst, "counts": counts,
            "granted": granted.to(torch.int32), "k": s["k"], "v": s["v"]}


def _sweep(s):
    c = s["case"]
    ps, P, M = c["page"], c["pages"], c["slots"]
    W, S = c["window"], c["sinks"]
    table, refs = s["table"].clone(), s["refs"].clone()
    if own:
        spec, o = s["spec"], s["out"]
        spec.spec_cache_release(table, refs, s["pos_now"], ps, accepted_len=s["accepted"], window=W, sinks=S,
                                status=s["status"])
        spec.spec_cache_compact(table, refs, o["src"], o["dst"], o["map"], o["counts"], status=s["status"])
        spec.spec_cache_copy(s["k"], s["v"], o["src"], o["dst"], o["counts"], status=s["status"])
        return dict(o, table=table, refs=refs, k=s["k"], v=s["v"])
    # release: pages past the kept tokens, and those that no later row sees
    keep = (s["pos_now"] + s["accepted"] + 1)[:, None]
    begin = torch.arange(M, device=DEVICE)[None] * ps
    drop = begin >= keep
    if W:
        drop |= (begin + ps <= keep - W + 1) & (begin >= S)
    drop &= table >= 0
    refs = refs - _count(torch.where(drop, table, -1), P)
    table = torch.where(drop, -1, table)
    # compact: the live pages past the live count take the free places below it, in order
    live = refs > 0
    n = live.sum()
    index = torch.arange(P, device=DEVICE)
    leave, hole = live & (index >= n), ~live & (index < n)
    cap = max(1, P // 2)
    src = _ranked(leave, index, cap)
    dst = _ranked(hole, index, cap)
    page_map = torch.where(live, index, -1).to(torch.int32)
    to = dst[(leave.cumsum(0) - 1).clamp(min=0)]
    page_map = torch.where(leave, to, page_map)
    table = torch.where(table >= 0, page_map[table.clamp(min=0).long()], table)
    packed = torch.zeros(P + 1, dtype=torch.int32, device=DEVICE)
    packed.scatter_(0, torch.where(live, page_map.long(), P), refs)
    counts = torch.stack([leave.sum(), n]).to(torch.int32)
    _copy(s, src, dst)
    return {"src": src, "dst": dst, "map": page_map, "counts": counts, "table": table, "refs": packed[:-1], "k": s["k"],
            "v": s["v"]}


def _count(pages, P):
    """How often each page occurs among the entries that are not -1."""
    flat = pages.flatten().long()
    n = torch.zeros(P + 1, dtype=torch.int32, device=DEVICE)
    n.index_add_(0, torch.where(flat >= 0, flat, P), torch.ones_like(flat, dtype=torch.int32))
    return n[:-1]


def _ranked(mask, index, cap):
    at = torch.where(mask, mask.cumsum(0) - 1, cap).clamp(max=cap)
    out = torch.full((cap + 1,), -1, dtype=torch.int32, device=DEVICE)
    return out.scatter_(0, at, index.to(torch.int32))[:-1]


def _copy(s, src, dst):
    src, dst = src[src >= 0].long(), dst[dst >= 0].long()
    s["k"][:, dst] = s["k"][:, src]
    s["v"][:, dst] = s["v"][:, src]


# ---------------------------------------------------------------------------
# Exact values
# ---------------------------------------------------------------------------
def exact(case, seed):
    """The attention's outputs in 64 bits, one key-value head and one row at a
    time in the definition's terms; the other operators move whole numbers and
    copies, which have no exact value beside themselves."""
    if case["op"] not in ("attend", "window"):
        return None
    s = prepare(case, seed)
    Hq, Hkv, D, ps = case["Hq"], case["Hkv"], case["D"], case["page"]
    G = Hq // Hkv
    W, S = case.get("window", 0), case.get("sinks", 0)
    out = torch.zeros((s["R"], Hq, D), dtype=torch.float64, device=DEVICE)
    lse = torch.full((s["R"], Hq), float("-inf"), dtype=torch.float64, device=DEVICE)
    for i, p in enumerate(s["ctx"]):
        n = s["offsets"][i + 1] - s["offsets"][i]
        lo = max(0, p - W + 1) if W else 0                    # the lowest key that the first row's window holds
        keys = list(range(min(S, lo))) + list(range(lo, p + n))
        where = torch.tensor(keys, dtype=torch.int64, device=DEVICE)
        rows = s["table"][i].long().index_select(0, where // ps) * ps + where % ps
        distance = (p + torch.arange(n, dtype=torch.int64, device=DEVICE)).unsqueeze(1) - where.unsqueeze(0)
        hidden = distance < 0
        if W:
            hidden = hidden | ((distance >= W) & (where >= S).unsqueeze(0))
        for h in range(Hkv):
            keys64 = s["k"][:, :, h].reshape(-1, D).index_select(0, rows).double()
            vals64 = s["v"][:, :, h].reshape(-1, D).index_select(0, rows).double()
            for a in range(G):
                at = slice(s["offsets"][i], s["offsets"][i + 1])
                logit = s["q"][at, h * G + a].double().mm(keys64.t()).div_(math.sqrt(D))
                logit[hidden] = float("-inf")
                total = torch.logsumexp(logit, 1)
                lse[at, h * G + a] = total
                out[at, h * G + a] = torch.exp(logit - total.unsqueeze(1)).mm(vals64)
    return {"out": out, "lse": lse}


if __name__ == "__main__":
    for listed_case in listed():
        print(listed_case["name"], work(listed_case))
    rng = random.Random(1)
    for _ in range(6):
        drawn = draw(rng)
        print(drawn, work(drawn))
