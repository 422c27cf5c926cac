"""Operators around the paged cache's round: cases, inputs, plain forms and exact values.

  rotary    queries and keys turned by their positions' angles, keys and values
            written to their pages on the way
  linear    linear attention with a decay per head: outputs of the packed rows and
            the requests' states carried on, or (a round that verifies drafts) left
            alone until the accepted rows are known and taken in by a second call
  logprobs  log probabilities of given tokens with their ranks, the entropy and the
            most likely alternatives

``run`` computes them with elementary torch operations, or through the package's
entry points where ``own`` is set.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
GOLDEN = 0.6180339887498949


def listed():
    return [
        # one new token of one request: the call's latency counts
        dict(name="rotary_token", op="rotary", B=1, K=0, ragged=False, lo=913, hi=913, Hq=32, Hkv=8, D=128, rot=128,
             inter=False, base=10000.0, factor=1.0, amp=1.0, page=16, dtype="bf16"),
        # a round of 64 requests at up to 17 rows each, deep in long documents, angles scaled for the length
        dict(name="rotary_round", op="rotary", B=64, K=16, ragged=True, lo=512, hi=131072, Hq=64, Hkv=8, D=128, rot=128,
             inter=False, base=500000.0, factor=8.0, amp=1.2, page=32, dtype="bf16"),
        # prompt chunks, neighbouring elements paired, half of each head turned
        dict(name="rotary_chunk", op="rotary", B=16, K=255, ragged=False, lo=1, hi=8192, Hq=32, Hkv=8, D=128, rot=64,
             inter=True, base=10000.0, factor=1.0, amp=1.0, page=64, dtype="bf16"),
        # a numerics run in fp32 with heads and pages that are no power of two
        dict(name="rotary_chunk_fp32", op="rotary", B=6, K=255, ragged=True, lo=300, hi=5001, Hq=12, Hkv=12, D=96,
             rot=40, inter=False, base=10000.0, factor=4.0, amp=1.0, page=24, dtype="f32"),
        # one new token of one request over its layer's states
        dict(name="linear_token", op="linear", mode="step", B=1, K=0, ragged=False, Hq=16, Hkv=16, Dk=128, Dv=128,
             gate="row", dtype="bf16"),
        # single tokens of a serving batch: the states' bytes count
        dict(name="linear_token_batch", op="linear", mode="step", B=128, K=0, ragged=False, Hq=32, Hkv=32, Dk=128,
             Dv=128, gate="row", dtype="bf16"),
        # a verification of up to 8 rows each, then the accepted rows taken into the states
        dict(name="linear_round", op="linear", mode="round", B=64, K=7, ragged=True, Hq=32, Hkv=32, Dk=128, Dv=128,
             gate="head", dtype="bf16"),
        # two long prompts at once
        dict(name="linear_prompt", op="linear", mode="step", B=2, K=16383, ragged=True, Hq=32, Hkv=32, Dk=128, Dv=128,
             gate="row", dtype="bf16"),
        # prompt chunks in fp32, queries in groups, odd head sizes
        dict(name="linear_chunk_fp32", op="linear", mode="step", B=3, K=200, ragged=True, Hq=12, Hkv=4, Dk=72, Dv=96,
             gate="row", dtype="f32"),
        # the answer's next token with five alternatives for one request
        dict(name="logprobs_token", op="logprobs", B=1, K=0, ragged=False, V=32003, top=5, t=1.0, dtype="bf16"),
        # the committed rows of a verification of 64 requests
        dict(name="logprobs_round", op="logprobs", B=64, K=16, ragged=True, V=201088, top=8, t=1.0, dtype="bf16"),
        # the scores of a prompt's tokens in fp32 at a lower temperature, many alternatives
        dict(name="logprobs_prompt_fp32", op="logprobs", B=4, K=255, ragged=False, V=50021, top=20, t=0.7,
             dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges, no dearer than the largest listed one."""
    op = rng.choice(["rotary", "linear", "linear", "logprobs"])
    if op == "rotary":
        D = rng.choice([64, 128, 128, 80, 96, 256])
        f32 = rng.random() < 0.25
        Hkv = rng.choice([1, 2, 4, 8, 12])
        K = rng.choice([0, 0, 4, 16, _log_int(rng, 17, 255)])
        hi = _log_int(rng, 8, 131072)
        B = min(_log_int(rng, 1, 128), max(1, 4096 // (K + 1)), max(1, (1 << 20) // (hi + 512)))
        case = dict(op=op, B=B, K=K, ragged=rng.random() < 0.5 and K > 0, lo=max(1, hi // rng.randint(1, 16)), hi=hi,
                    Hq=Hkv * rng.choice([1, 3, 4, 8]), Hkv=Hkv, D=D, rot=rng.choice([D, D, D // 2, 2 * (D // 5)]),
                    inter=rng.random() < 0.4, base=rng.choice([10000.0, 500000.0, 1000000.0]),
                    factor=rng.choice([1.0, 4.0, 32.0]), amp=rng.choice([1.0, 1.0, 1.35]),
                    page=rng.choice([10, 16, 32, 64, 128]), dtype="f32" if f32 else "bf16")
        while work(case)["bytes"] > work(listed()[2])["bytes"]:
            case["B"], case["K"] = (case["B"] + 1) // 2, case["K"] if case["B"] > 1 else case["K"] // 2
        return case
    if op == "linear":
        f32 = rng.random() < 0.2
        Dk, Dv = rng.choice([(64, 64), (128, 128), (128, 128), (64, 128), (128, 64), (72, 96), (256, 256), (32, 160)])
        Hkv = rng.choice([1, 2, 4, 8, 16, 32])
        Hq = Hkv * rng.choice([1, 1, 1, 2, 4])
        mode = rng.choice(["step", "step", "round"])
        K = rng.choice([0, 0, 7, 16, _log_int(rng, 17, 255), _log_int(rng, 256, 16383)])
        if mode == "round":
            K = rng.choice([1, 4, 7, 16, 63])
        case = dict(op=op, mode=mode, B=_log_int(rng, 1, 128), K=K, ragged=rng.random() < 0.5 and K > 0, Hq=Hq, Hkv=Hkv,
                    Dk=Dk, Dv=Dv, gate=rng.choice(["row", "row", "head"]), dtype="f32" if f32 else "bf16")
        slow = 16.0 if f32 or Dk not in (64, 128) or Dv not in (64, 128) else 1.0
        most = 32768 * 32 * 128 * 128                       # rows x heads x state of the largest listed case
        while True:
            rows = case["B"] * (case["K"] + 1)
            if rows * Hq * Dk * Dv * (slow if K > 32 else 1.0) <= most and case["B"] * Hkv * Dk * Dv <= 1 << 26:
                return case
            if case["B"] > 1:
                case["B"] = (case["B"] + 1) // 2
            else:
                case["K"] //= 2
    K = rng.choice([0, 0, 4, 16, _log_int(rng, 17, 255)])
    V = _log_int(rng, 1000, 201088)
    f32 = rng.random() < 0.4
    B = _log_int(rng, 1, 64)
    while B > 1 and B * (K + 1) * V * (2 if f32 else 1) > 64 * 17 * 201088:
        B = (B + 1) // 2
    while B * (K + 1) * V * (2 if f32 else 1) > 64 * 17 * 201088:
        V //= 2
    return dict(op=op, B=B, K=K, ragged=rng.random() < 0.5 and K > 0, V=V, top=rng.choice([0, 1, 5, 8, 20, 32]),
                t=rng.choice([1.0, 1.0, 0.7, 1.3]), dtype="f32" if f32 else "bf16")


# ---------------------------------------------------------------------------
# Sizes: functions of the case alone
# ---------------------------------------------------------------------------
def _depths(case):
    """Drafts (rows less one) of each request: spread over 0 .. K where the batch is ragged."""
    K = case["K"]
    if not case["ragged"]:
        return [K] * case["B"]
    if case["B"] <= 4:
        return [max(0, K - i * (K + 2) // 3) for i in range(case["B"])]
    return [(5 * i + 3) % (K + 1) for i in range(case["B"])]


def _accepted(case):
    """Accepted drafts of each request: any number of them up to all."""
    return [(3 * i + 1) % (n + 1) for i, n in enumerate(_depths(case))]


def _element(case):
    return 4 if case["dtype"] == "f32" else 2


def work(case):
    e, rows = _element(case), sum(n + 1 for n in _depths(case))
    if case["op"] == "rotary":
        # queries in and out, keys and values into their pages
        return {"bytes": 2 * rows * (case["Hq"] + 2 * case["Hkv"]) * case["D"] * e + 4 * rows + 8 * case["B"],
                "flops": 3 * rows * (case["Hq"] + case["Hkv"]) * case["rot"]}
    if case["op"] == "linear":
        Hq, H, Dk, Dv = case["Hq"], case["Hkv"], case["Dk"], case["Dv"]
        io = rows * (Hq * Dk + H * Dk + H * Dv + Hq * Dv) * e + (4 * rows * H if case["gate"] == "row" else 4 * H)
        return {"bytes": io + 2 * 4 * case["B"] * H * Dk * Dv, "flops": 2 * rows * (Hq + H) * Dk * Dv}
    asked = sum(a + 1 for a in _accepted(case)) if case["ragged"] else rows
    return {"bytes": asked * (case["V"] * e + 16 + 8 * case["top"]), "flops": 4 * asked * case["V"]}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _randn(shape, dtype, g):
    return torch.randn(shape, device=DEVICE, dtype=dtype if math.prod(shape) > 1 << 26 else torch.float32,
                       generator=g).to(dtype)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    B, dt = case["B"], _dtype(case)
    depth = _depths(case)
    offsets = [0]
    for n in depth:
        offsets.append(offsets[-1] + n + 1)
    R = offsets[-1]
    s = {"case": case, "R": R, "offsets": offsets, "depth_host": depth, "row_offsets": _i32(offsets),
         "depth": _i32(depth), "status": torch.zeros(1, dtype=torch.int32, device=DEVICE)}
    if own:
        import paper_2607_25852_gb300 as spec
        s["spec"] = spec
    if case["op"] == "rotary":
        Hq, Hkv, D, ps, rot = case["Hq"], case["Hkv"], case["D"], case["page"], case["rot"]
        lo, hi = case["lo"], case["hi"]
        ctx = [hi] if B == 1 else [int(round(lo * (hi / lo) ** (((i + 1) * GOLDEN) % 1.0))) for i in range(B)]
        # the rows' pages alone: what a request has cached before is of no account here
        slots = max(p + n for p, n in zip(ctx, depth)) // ps + 1
        holders = [(i, t) for i, (p, n) in enumerate(zip(ctx, depth)) for t in range(p // ps, (p + n) // ps + 1)]
        pages = len(holders) + len(holders) // 8 + 1
        table = torch.full((B, slots), -1, dtype=torch.int32, device=DEVICE)
        at = torch.tensor(holders, device=DEVICE)
        table[at[:, 0], at[:, 1]] = torch.randperm(pages, device=DEVICE, generator=g)[:len(holders)].to(torch.int32)
        s["table"], s["pos_base"] = table, torch.tensor(ctx, device=DEVICE)
        s["k"], s["v"] = _randn((pages, ps, Hkv, D), dt, g), _randn((pages, ps, Hkv, D), dt, g)
        rows = _randn((R, Hq + 2 * Hkv, D), dt, g)  # [queries | keys | values], as one projection writes them
        s["q"], s["k_new"], s["v_new"] = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
        s["out"] = torch.empty((R, Hq, D), dtype=dt, device=DEVICE)
        exponent = torch.arange(0, rot, 2, dtype=torch.float64) / rot
        s["freq"] = (case["base"] ** -exponent / case["factor"]).to(DEVICE)
        return s
    if case["op"] == "linear":
        Hq, H, Dk, Dv = case["Hq"], case["Hkv"], case["Dk"], case["Dv"]
        s["q"], s["k"], s["v"] = _randn((R, Hq, Dk), dt, g), _randn((R, H, Dk), dt, g), _randn((R, H, Dv), dt, g)
        if case["gate"] == "row":  # each row's own, from nearly nothing forgotten to nearly all
            s["decay"] = -torch.exp(torch.empty((R, H), device=DEVICE).uniform_(math.log(1e-3), math.log(2.0), generator=g))
        else:                      # a head's own half-life, from a few rows to thousands
            s["decay"] = -torch.exp2(-1.0 - 10.0 * torch.arange(H, device=DEVICE) / H)
        # the requests' states lie in slots of a pool, in no order; the new ones go to other slots
        s["states"] = _randn((2 * B + 1, H, Dk, Dv), torch.float32, g)
        order = torch.randperm(2 * B + 1, device=DEVICE, generator=g).to(torch.int32)
        s["slots_in"], s["slots_out"] = order[:B].contiguous(), order[B:2 * B].contiguous()
        s["slots_in"][B // 2:B // 2 + (B > 1)] = -1  # one request has just begun
        s["accepted"] = _i32(_accepted(case))
        s["out"] = torch.empty((R, Hq, Dv), dtype=dt, device=DEVICE)
        if own:
            s["ws"] = spec.linear_workspace(B, case["K"], Hq, H, Dk, Dv, dt, DEVICE)
        return s
    V, top, N = case["V"], case["top"], case["K"] + 1
    s["logits"] = (_randn((R, V), torch.float32, g) * 2.5).to(dt)
    s["tokens"] = torch.randint(0, V, (B, N), device=DEVICE, generator=g, dtype=torch.int32)
    # most given tokens are likely ones: the first of 64 random entries' largest
    some = torch.randint(0, V, (R, 64), device=DEVICE, generator=g)
    best = some.gather(1, s["logits"].gather(1, some).float().argmax(1, keepdim=True)).squeeze(1).to(torch.int32)
    i, j = _places(s)
    s["tokens"][i, j] = torch.where(torch.rand(R, device=DEVICE, generator=g) < 0.8, best, s["tokens"][i, j])
    s["accepted"] = _i32(_accepted(case) if case["ragged"] else depth)
    f32 = dict(dtype=torch.float32, device=DEVICE)
    s["logprob"], s["entropy"] = torch.empty((B, N), **f32), torch.empty((B, N), **f32)
    s["rank"] = torch.empty((B, N), dtype=torch.int32, device=DEVICE)
    s["top_tokens"] = torch.empty((B, N, top), dtype=torch.int32, device=DEVICE) if top else None
    s["top_logprobs"] = torch.empty((B, N, top), **f32) if top else None
    if own:
        s["ws"] = spec.logprobs_workspace(B, case["K"], V, top, DEVICE)
    return s


def _places(s):
    """Request and place within it of every packed row."""
    off = s["row_offsets"].long()
    r = torch.arange(s["R"], device=DEVICE)
    i = torch.searchsorted(off, r, right=True) - 1
    return i, r - off[i]


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    return {"rotary": _rotary, "linear": _linear, "logprobs": _logprobs}[state["case"]["op"]](state)


def _turn(x, cos, sin, rot, inter):
    """x [R, heads, D] in fp32 with its first `rot` elements turned by pairs."""
    head = x[..., :rot]
    if inter:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = head.chunk(2, -1)
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _rotary(s):
    c = s["case"]
    if own:
        s["spec"].spec_rotary_append(s["q"], s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["pos_base"], c["B"],
                                     c["K"], s["freq"], s["out"], interleaved=c["inter"], amplitude=c["amp"],
                                     row_offsets=s["row_offsets"], depth=s["depth"], status=s["status"])
        return {"q": s["out"], "k": s["k"], "v": s["v"]}
    ps, dt = c["page"], s["q"].dtype
    i, j = _places(s)
    pos = s["pos_base"][i] + j
    angle = (pos.double()[:, None] * s["freq"]).unsqueeze(1)
    cos, sin = (torch.cos(angle) * c["amp"]).float(), (torch.sin(angle) * c["amp"]).float()
    page = s["table"][i, pos // ps].long()
    s["k"][page, pos % ps] = _turn(s["k_new"].float(), cos, sin, c["rot"], c["inter"]).to(dt)
    s["v"][page, pos % ps] = s["v_new"]
    return {"q": _turn(s["q"].float(), cos, sin, c["rot"], c["inter"]).to(dt), "k": s["k"], "v": s["v"]}


def _linear(s):
    c = s["case"]
    later = c["mode"] == "round"
    if own:
        spec, rows = s["spec"], dict(row_offsets=s["row_offsets"], depth=s["depth"], status=s["status"])
        spec.spec_linear_attend(s["q"], s["k"], s["v"], s["decay"], s["states"], s["slots_in"],
                                None if later else s["slots_out"], c["B"], c["K"], s["out"], s["ws"], **rows)
        if later:
            spec.spec_linear_commit(s["k"], s["v"], s["decay"], s["states"], s["slots_in"], s["slots_out"],
                                    s["accepted"], c["B"], c["K"], s["ws"], **rows)
        return {"out": s["out"], "states": s["states"]}
    # chunks of 64 rows: products within a chunk, and the chunks' own sums carried from chunk to chunk at once
    B, H, Dk, Dv = c["B"], c["Hkv"], c["Dk"], c["Dv"]
    G, C = c["Hq"] // H, min(64, c["K"] + 1)
    n = (c["K"] + C) // C
    j = torch.arange(n * C, device=DEVICE)
    has = j <= s["depth"][:, None]                                                # [B, n C]
    row = torch.where(has, s["row_offsets"][:-1, None] + j, 0).long()

    def heads(x, h, d):                                                           # [B, h, n, C, d]
        return torch.where(has[..., None, None], x[row].float(), 0.0).view(B, n, C, h, d).permute(0, 3, 1, 2, 4)

    q, k, v = heads(s["q"], c["Hq"], Dk), heads(s["k"], H, Dk), heads(s["v"], H, Dv)
    decay = s["decay"].expand(s["R"], H)[row].double()
    decay = torch.where(has[..., None], decay, 0.0).view(B, n, C, H).permute(0, 3, 1, 2)
    first = torch.where(s["slots_in"][:, None, None, None] >= 0, s["states"][s["slots_in"].clamp(min=0).long()], 0.0)

    def carry(k, decay):
        """The states before each chunk and after the last."""
        g = decay.cumsum(-1)
        chunk = torch.matmul((k * torch.exp(g[..., -1:] - g).float()[..., None]).transpose(-1, -2), v)
        upto = torch.cat([torch.zeros_like(g[..., :1, -1]), g[..., -1].cumsum(-1)], -1)  # [B, H, n + 1]
        w = upto[..., :, None] - upto[..., None, 1:]
        ahead = torch.arange(n + 1, device=DEVICE)[:, None] > torch.arange(n, device=DEVICE)
        w = torch.where(ahead, torch.exp(w.masked_fill(~ahead, 0.0)), 0.0).float()
        own_sums = torch.matmul(w, chunk.view(B, H, n, Dk * Dv)).view(B, H, n + 1, Dk, Dv)
        return own_sums.add_(torch.exp(upto).float()[..., None, None] * first[:, :, None]), g

    before, g = carry(k, decay)
    after = before[:, :, n]
    if later:
        kept = (j <= s["accepted"][:, None]).view(B, 1, n, C)
        after = carry(torch.where(kept[..., None], k, 0.0), torch.where(kept, decay, 0.0))[0][:, :, n]
    seen = torch.arange(C, device=DEVICE)[:, None] >= torch.arange(C, device=DEVICE)
    w = torch.exp((g[..., :, None] - g[..., None, :]).masked_fill_(~seen, -math.inf)).float().unsqueeze(2)
    q = q.view(B, H, G, n, C, Dk)
    p = torch.matmul(q, k.unsqueeze(2).transpose(-1, -2)).mul_(w)
    o = torch.matmul(p, v.unsqueeze(2))
    o.add_(torch.matmul(q, before[:, :, None, :n]).mul_(torch.exp(g).float()[:, :, None, ..., None])).mul_(Dk ** -0.5)
    s["states"][s["slots_out"].long()] = after
    out = o.view(B, c["Hq"], n * C, Dv).transpose(1, 2)[has].to(s["q"].dtype)
    return {"out": out, "states": s["states"]}


def _logprobs(s):
    c = s["case"]
    names = ("logprob", "rank", "entropy", "top_tokens", "top_logprobs")
    if own:
        s["spec"].spec_logprobs(s["logits"], s["tokens"], c["B"], c["K"], c["V"], s["logprob"], s["ws"],
                                temperature=c["t"], row_offsets=s["row_offsets"], depth=s["depth"],
                                accepted_len=s["accepted"], rank_out=s["rank"], entropy_out=s["entropy"],
                                top_tokens_out=s["top_tokens"], top_logprobs_out=s["top_logprobs"], status=s["status"])
        return {n: s[n] for n in names if s[n] is not None}
    j = torch.arange(c["K"] + 1, device=DEVICE)
    asked = j <= s["accepted"][:, None]
    raw = s["logits"][(s["row_offsets"][:-1, None] + j)[asked].long()].float()
    token = s["tokens"][asked].long()[:, None]
    x = raw / c["t"]
    x = x - x.amax(1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    norm = torch.log(total)
    given, index = raw.gather(1, token), torch.arange(c["V"], device=DEVICE)
    found = {"logprob": (x.gather(1, token) - norm).squeeze(1),
             "rank": 1 + ((raw > given) | ((raw == given) & (index < token))).sum(1),
             "entropy": (norm - (e * x).sum(1, keepdim=True) / total).squeeze(1)}
    if c["top"]:
        # the logits' order as whole numbers, the lower index first among equals
        bits = raw.view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 32) + (c["V"] - 1 - index)
        best = c["V"] - 1 - (torch.topk(order, c["top"], 1)[0] & 0xFFFFFFFF)
        found["top_tokens"], found["top_logprobs"] = best, x.gather(1, best) - norm
    nothing = {"logprob": -math.inf, "rank": 0, "entropy": 0.0, "top_tokens": -1, "top_logprobs": -math.inf}
    for n, value in found.items():
        s[n].fill_(nothing[n])
        s[n][asked] = value.to(s[n].dtype)
    return {n: s[n] for n in names if s[n] is not None}


# ---------------------------------------------------------------------------
# Exact values
# ---------------------------------------------------------------------------
def exact(case, seed):
    """The definitions in 64 bits: turns as complex products, the recurrence row by
    row, softmax sums a row at a time."""
    s = prepare(case, seed)
    off, depth = s["offsets"], s["depth_host"]
    if case["op"] == "rotary":
        def turned(x, position):
            x = x.double()
            rot, half = case["rot"], case["rot"] // 2
            pairs = x[:, :rot].reshape(-1, half, 2) if case["inter"] else x[:, :rot].reshape(-1, 2, half).transpose(1, 2)
            z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(s["freq"], case["amp"]),
                                                                        position * s["freq"])
            pairs = torch.view_as_real(z)
            y = pairs.reshape(-1, rot) if case["inter"] else pairs.transpose(1, 2).reshape(-1, rot)
            return torch.cat([y, x[:, rot:]], 1)
        q, k = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE), s["k"].double()
        table, base = s["table"].tolist(), s["pos_base"].tolist()
        for i, n in enumerate(depth):
            for j in range(n + 1):
                p = base[i] + j
                q[off[i] + j] = turned(s["q"][off[i] + j], p)
                k[table[i][p // case["page"]], p % case["page"]] = turned(s["k_new"][off[i] + j], p)
        return {"q": q, "k": k, "v": None}
    if case["op"] == "linear":
        Hq, H, Dk, Dv = case["Hq"], case["Hkv"], case["Dk"], case["Dv"]
        if (max(depth) + 1) * case["B"] * Hq * Dk * Dv > 1 << 36:
            return None
        states = s["states"].double()
        group = torch.arange(Hq, device=DEVICE) // (Hq // H)
        out = torch.zeros((s["R"], Hq, Dv), dtype=torch.float64, device=DEVICE)
        start = s["slots_in"].tolist()
        now = torch.stack([states[x] if x >= 0 else torch.zeros_like(states[0]) for x in start])
        after = now.clone()
        factor = torch.exp(s["decay"].double()).expand(s["R"], H)
        keep = _accepted(case) if case["mode"] == "round" else depth
        base = s["row_offsets"][:-1].long()
        for j in range(max(depth) + 1):
            live = torch.tensor([i for i, n in enumerate(depth) if n >= j], device=DEVICE)
            r = base[live] + j
            if len(live) < case["B"]:
                new = now[live]
            else:
                new = now
            new = new * factor[r][:, :, None, None] + s["k"][r].double()[..., None] * s["v"][r].double()[:, :, None]
            out[r] = (s["q"][r].double()[..., None] * (new if Hq == H else new[:, group])).sum(2) / math.sqrt(Dk)
            if len(live) < case["B"]:
                now[live] = new
            else:
                now = new
            last = [x for x, i in enumerate(live.tolist()) if keep[i] == j] if j in keep else []
            if last:
                after[live[last]] = new[last]
        states[s["slots_out"].long()] = after
        return {"out": out, "states": states}
    B, N, top = case["B"], case["K"] + 1, case["top"]
    lowest = dict(fill_value=-math.inf, dtype=torch.float64, device=DEVICE)
    logprob, entropy = torch.full((B, N), **lowest), torch.zeros((B, N), dtype=torch.float64, device=DEVICE)
    best = torch.full((B, N, top), **lowest)
    tokens, accepted = s["tokens"].tolist(), s["accepted"].tolist()
    for i in range(B):
        for j in range(accepted[i] + 1):
            lp = torch.log_softmax(s["logits"][off[i] + j].double() / case["t"], 0)
            logprob[i, j] = lp[tokens[i][j]]
            entropy[i, j] = -(lp.exp() * lp).sum()
            best[i, j] = lp.topk(top)[0]
    out = {"logprob": logprob, "rank": None, "entropy": entropy}
    return dict(out, top_tokens=None, top_logprobs=best) if top else out


if __name__ == "__main__":
    for listed_case in listed():
        print(listed_case["name"], work(listed_case))
    rng = random.Random(1)
    for _ in range(12):
        drawn = draw(rng)
        print(drawn, work(drawn))
