"""The operators of a K|V cache held in 4 bits, and those that copy and compact cached sequences, as cases that can be
timed and compared with a plain form.

A case is a dict of plain values.  `kind` says which operator it is:

  attend   attention of one query token per sequence over the rows of a 4-bit cache, layer by layer: sinks, a list of
           positions per KV head and a recent window, or every cached row (budget -1)
  ingest   new K and V rows enter a 4-bit cache behind `len` cached tokens and are read back as the values that the cache holds
           (what attention among the new tokens has to use)
  project  the keys of [len, len + new) are projected from their 4-bit rows
  fork     a sequence is copied into `copies` other slots: K|V rows and projected keys of every layer
  verify   drafted tokens enter the caches behind `len` tokens and are projected, then the accepted ones are kept
  prune    a copy of a sequence keeps a part of its tokens

A 4-bit row: blocks of 16 channels share a scale.  With a the block's largest magnitude the scale is the 8-bit float (5 exponent, 3
mantissa bits: e = 0: m 2^-17, else (8 + m) 2^(e - 18)) nearest to a / 6, at least 2^-17, at most 10240, and an element is the nearest of 0, 0.5,
1, 1.5, 2, 3, 4, 6 times the scale, with its sign (a zero has none); ties go to the even code.  144 bytes: 64 of K codes (channel 2 i in the low
half of byte i), 8 K scales, 8 V scales, 64 of V codes.

Shapes are those of an 8B model (32 query heads, 8 KV heads, head dimension 128) unless a case says otherwise."""
import math
import random

import numpy as np
import torch

own = False

HEAD_DIM = 128
BLOCK = 16
ROW = 144
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)         # magnitudes of the 4-bit codes
TOP_SCALE = 226                                          # the code of 10240

_BASE = dict(q_heads=32, kv_heads=8, imp_dim=32)
_ATTEND = dict(_BASE, kind="attend", layers=8, batch=1, len_lo=32768, len_hi=32768, budget=-1, sinks=0, recent=0, outliers=4)
_INGEST = dict(_BASE, kind="ingest", layers=4, batch=1, len_lo=0, len_hi=0, new_lo=1, new_hi=1, outliers=4)
_PROJECT = dict(_BASE, kind="project", layers=4, batch=1, len_lo=0, len_hi=0, new_lo=1, new_hi=1, outliers=4)
_FORK = dict(_BASE, kind="fork", dtype="fp4", layers=8, len_lo=16384, len_hi=16384, copies=8, share=1.0)
_VERIFY = dict(_BASE, kind="verify", dtype="fp4", layers=16, batch=4, len_lo=5000, len_hi=9000, new_lo=61, new_hi=61, keep_share=0.15)
_PRUNE = dict(_BASE, kind="prune", dtype="bf16", layers=4, len_lo=32768, len_hi=32768, keep_share=0.5, prefix_share=0.05)


def listed():
    return [
        # the smallest call: a first reply token over a few prompt tokens, one layer -- latency
        dict(_ATTEND, name="attend_37", layers=1, q_heads=8, len_lo=37, len_hi=37, outliers=0),
        # a decode step of a 32K-token sequence at a 10 % budget, eight layers
        dict(_ATTEND, name="attend_32k", budget=3276),
        # batched serving: sixteen ragged sequences, sinks and a recent window
        dict(_ATTEND, name="attend_batch16", layers=4, batch=16, len_lo=8192, len_hi=16384, budget=1024, sinks=4, recent=64),
        # the first decode token behind long prompts: every cached row
        dict(_ATTEND, name="attend_dense_128k", layers=1, batch=2, len_lo=100001, len_hi=131072),
        # a decoded token of three chats enters the cache, every layer called by itself
        dict(_INGEST, name="ingest_1", layers=16, batch=3, len_lo=700, len_hi=3100),
        # a chunk of two prompts, to be attended among itself
        dict(_INGEST, name="ingest_chunks", batch=2, len_lo=0, len_hi=9000, new_lo=4001, new_hi=8192),
        # eager projection: the newest token of sixteen sequences
        dict(_PROJECT, name="project_1", batch=16, len_lo=2000, len_hi=8191),
        # a 32K prompt is projected at once
        dict(_PROJECT, name="project_32k", new_lo=32768, new_hi=32768),
        # three samples of one chat prompt
        dict(_FORK, name="fork_chat", dtype="bf16", layers=16, len_lo=2100, len_hi=2100, copies=3, imp_dim=16),
        # eight beams from a 16K prompt
        dict(_FORK, name="fork_beams"),
        # a draft of 61 tokens is verified for four sequences
        dict(_VERIFY, name="verify_61"),
        # a branch that keeps half of a 32K context
        dict(_PRUNE, name="prune_32k"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_any(rng):
    kind = rng.choice(["attend"] * 4 + ["ingest", "project", "fork", "verify", "prune"])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 8), (8, 8), (16, 8), (16, 4), (28, 4), (32, 4)])
    shape = dict(q_heads=q_heads, kv_heads=kv_heads, imp_dim=rng.choice([16, 32, 32]))
    layers, batch = rng.choice([1, 2, 4, 8, 16]), _log_int(rng, 1, 32)
    hi = _log_int(rng, 1, 131072)
    lo = max(1, int(hi * rng.uniform(0.3, 1.0)))
    if kind == "attend":
        more = dict(outliers=rng.choice([0, 4]), layers=layers, batch=batch, len_lo=lo, len_hi=hi)
        if rng.random() < 0.6:
            more.update(budget=max(1, int(hi * math.exp(rng.uniform(math.log(0.01), math.log(0.2))))), sinks=rng.choice([0, 4, 16, 128]),
                        recent=rng.choice([0, 1, 64, 256]))
        return dict(_ATTEND, **{**shape, **more})
    if kind in ("ingest", "project"):
        new = _log_int(rng, 1, 16384)
        more = dict(layers=layers, batch=batch, len_lo=0, len_hi=_log_int(rng, 1, 8192), new_lo=max(1, int(new * rng.uniform(0.3, 1.0))), new_hi=new)
        return dict(_INGEST if kind == "ingest" else _PROJECT, **{**shape, **more, "outliers": rng.choice([0, 4])})
    dtype = rng.choice(["fp4", "fp4", "bf16", "fp32"])
    if kind == "fork":
        return dict(_FORK, **{**shape, "dtype": dtype, "layers": layers, "len_lo": lo, "len_hi": hi, "copies": _log_int(rng, 1, 16),
                              "share": rng.choice([1.0, 1.0, 0.4])})
    if kind == "verify":
        new = _log_int(rng, 1, 256)
        base = _log_int(rng, 1, 32768)
        return dict(_VERIFY, **{**shape, "dtype": dtype, "layers": layers, "batch": min(batch, 16), "len_lo": max(1, base // 2), "len_hi": base,
                                "new_lo": max(1, int(new * rng.uniform(0.5, 1.0))), "new_hi": new, "keep_share": rng.choice([0.05, 0.1, 0.4, 1.0])})
    return dict(_PRUNE, **{**shape, "dtype": dtype, "layers": layers, "len_lo": lo, "len_hi": hi, "keep_share": rng.choice([0.1, 0.5, 0.9]),
                           "prefix_share": rng.choice([0.0, 0.05, 0.5])})


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = _draw_any(rng)
        rows = c["layers"] * c.get("batch", 1) * c["kv_heads"] * (c["len_hi"] + c.get("new_hi", 0))
        slots = 1 + (c.get("copies", 1) if c["kind"] in ("fork", "prune") else 0)
        if work(c)["bytes"] <= most and rows <= 5e6 and rows * slots * _row_bytes(c) <= 3e9:
            return c


def _row_bytes(c):
    return {"fp4": ROW, "bf16": 512, "fp32": 1024}[c.get("dtype", "fp4")]


def _values(c):
    """The type of whatever is not held in 4 bits."""
    return torch.float32 if c.get("dtype") == "fp32" else torch.bfloat16


def _sizes(c):
    """Cached and new tokens of each sequence, and how many of the new (verify) or cached (prune) ones are kept."""
    rng = random.Random("%s" % sorted((k, v) for k, v in c.items() if k != "name"))
    cached = [rng.randint(c["len_lo"], c["len_hi"]) for _ in range(c.get("batch", 1))]
    new = [rng.randint(c["new_lo"], c["new_hi"]) for _ in cached] if "new_lo" in c else [0] * len(cached)
    if c["kind"] == "verify":
        kept = [min(n, int(rng.uniform(0, 2) * c["keep_share"] * n) if c["keep_share"] < 1 else n) for n in new]
        kept[0] = max(1, kept[0])
    elif c["kind"] == "prune":
        kept = [max(1, int((L - _prefix(c, L)) * c["keep_share"])) for L in cached]
    else:
        kept = [0] * len(cached)
    return cached, new, kept


def _prefix(c, L):
    return int(L * c["prefix_share"])


def _attended(c, L):
    return L if c["budget"] < 0 else min(L, min(c["sinks"], L) + c["budget"] + c["recent"])


def work(case):
    c = case
    cached, new, kept = _sizes(c)
    heads, layers, row, D = c["kv_heads"], c["layers"], _row_bytes(c), HEAD_DIM
    es = 4 if c.get("dtype") == "fp32" else 2
    imp = c["imp_dim"] * es
    if c["kind"] == "attend":
        rows = sum(_attended(c, L) for L in cached) * layers
        lists = 0 if c["budget"] < 0 else 4 * c["budget"] * heads * c["batch"] * layers
        return {"bytes": rows * heads * ROW + lists + layers * c["batch"] * c["q_heads"] * D * 6, "flops": 4.0 * D * c["q_heads"] * rows}
    if c["kind"] == "ingest":
        return {"bytes": sum(new) * layers * heads * 2 * (ROW + 512), "flops": 0}
    if c["kind"] == "project":
        return {"bytes": layers * heads * (sum(new) * (ROW // 2 + imp) + D * imp), "flops": 2.0 * D * c["imp_dim"] * layers * heads * sum(new)}
    if c["kind"] == "fork":
        return {"bytes": (1 + c["copies"]) * layers * heads * max(1, int(cached[0] * c["share"])) * (row + imp), "flops": 0}
    if c["kind"] == "verify":
        rows = sum(new) * (2 * D * es + row + D * es + imp) + sum(kept) * 2 * (row + imp)
        return {"bytes": layers * heads * (rows + D * imp), "flops": 2.0 * D * c["imp_dim"] * layers * heads * sum(new)}
    return {"bytes": 2 * layers * heads * (cached[0] + kept[0]) * (row + imp), "flops": 0}


class State:
    """What a serving program keeps, and the inputs of its next call."""


def _keys_values(c, gen, tokens):
    """K and V rows [layers][tokens][kv heads][head dim]; a few key channels per head are large where the case asks."""
    k, v = (torch.randn(c["layers"], tokens, c["kv_heads"], HEAD_DIM, generator=gen, device="cuda", dtype=_values(c)) for _ in range(2))
    if c.get("outliers"):
        ch = torch.argsort(torch.rand(c["kv_heads"], HEAD_DIM, generator=gen, device="cuda"), dim=1)[:, :c["outliers"]]
        k.mul_(torch.ones(c["kv_heads"], HEAD_DIM, device="cuda").scatter_(1, ch, 8.0).to(k.dtype))
    return k, v


def _rising(gen, rows, n, size, device="cuda"):
    """`n` different positions below `size` for each row, ascending."""
    return torch.argsort(torch.rand(rows, size, generator=gen, device=device), dim=1)[:, :n].sort(dim=1).values.to(torch.int32)


def _inputs(c, seed):
    """Everything that the seed decides."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    i = State()
    i.cached, i.new, i.kept = _sizes(c)
    B, layers, heads = len(i.cached), c["layers"], c["kv_heads"]
    i.k, i.v = _keys_values(c, gen, sum(i.cached))                       # the cached tokens, sequence behind sequence
    i.k_new, i.v_new = _keys_values(c, gen, sum(i.new))
    i.W = (torch.randn(layers, heads, HEAD_DIM, c["imp_dim"], generator=gen, device="cuda") / math.sqrt(HEAD_DIM)).to(_values(c))
    if c["kind"] == "attend":
        i.q = torch.randn(layers, B, c["q_heads"], HEAD_DIM, generator=gen, device="cuda", dtype=torch.bfloat16)
        if c["budget"] >= 0:
            i.cap = -(-c["budget"] // 4) * 4
            i.idx = torch.zeros(layers, B, heads, i.cap, dtype=torch.int32, device="cuda")
            i.cnt = torch.zeros(layers, B, heads, dtype=torch.int32, device="cuda")
            for b, L in enumerate(i.cached):
                lo = min(c["sinks"], L)
                hi = max(lo, L - c["recent"])
                n = min(c["budget"], hi - lo)
                for l in range(layers if n else 0):
                    i.idx[l, b, :, :n] = lo + _rising(gen, heads, n, hi - lo)
                    i.cnt[l, b] = n
    if c["kind"] in ("verify", "prune"):
        span = i.new if c["kind"] == "verify" else [L - _prefix(c, L) for L in i.cached]
        i.begin = i.cached if c["kind"] == "verify" else [_prefix(c, L) for L in i.cached]
        i.keep = torch.zeros(B, max(1, max(i.kept)), dtype=torch.int32, device="cuda")
        for b, n in enumerate(i.kept):
            if n:
                i.keep[b, :n] = i.begin[b] + _rising(gen, 1, n, span[b])[0]
    return i


def prepare(case, seed):
    c = case
    i = s = _inputs(c, seed)
    s.c = c
    B, layers, heads, total = len(i.cached), c["layers"], c["kv_heads"], [a + b for a, b in zip(i.cached, i.new)]
    slots = B + (c["copies"] if c["kind"] == "fork" else 1 if c["kind"] == "prune" else 0)
    room = -(-max(total) // 64) * 64
    fp4 = c.get("dtype", "fp4") == "fp4"
    s.ends = [a + n for a, n in zip(i.cached, i.kept)] if c["kind"] == "verify" else total
    s.n_fork = max(1, int(i.cached[0] * c["share"])) if c["kind"] == "fork" else 0
    if own:
        from paper_2503_07518_b200 import binding as tb
        dtype = tb.TB_FP4 if fp4 else tb.TB_BF16 if c["dtype"] == "bf16" else tb.TB_F32
        s.ctx = tb.Context(layers, c["q_heads"], heads, HEAD_DIM, c["imp_dim"], dtype, slots, room, max(1, c.get("budget", 1)))
        for l in range(layers):
            s.ctx.set_projection(l, i.W[l])
        s.kv, s.kimp = s.ctx.kv, s.ctx.kimp
        if sum(i.cached):
            s.ctx.append_kv(0, layers, list(range(B)), i.cached, i.k, i.v)
            s.ctx.project_keys(0, layers, list(range(B)), [0] * B, i.cached)
        if c["kind"] == "project":
            s.ctx.append_kv(0, layers, None, i.new, i.k_new, i.v_new)
        if c["kind"] == "attend":
            s.params = tb.select_params(c["budget"], c["sinks"], c["recent"])
            s.results = {"out": torch.empty(layers, B, c["q_heads"], HEAD_DIM, device="cuda"), "lse": torch.empty(layers, B, c["q_heads"], device="cuda")}
            lists = zip(i.idx, i.cnt) if c["budget"] >= 0 else [(None, None)] * layers
            s.by_layer = [(*t, *u) for t, u in zip(zip(i.q, s.results["out"], s.results["lse"]), lists)]      # a layer's tensors are its own in a decode step
        s.seen = _seen(s)
    else:
        s.kv = torch.zeros(layers, slots, heads, room, ROW, dtype=torch.uint8, device="cuda") if fp4 else \
            torch.zeros(layers, slots, heads, room, 2, HEAD_DIM, dtype=_values(c), device="cuda")
        s.kimp = torch.zeros(layers, slots, heads, room, c["imp_dim"], dtype=_values(c), device="cuda")
        _store(s, [0] * B, i.cached, i.k, i.v)
        _project(s, [0] * B, i.cached)
        if c["kind"] == "project":
            _store(s, i.cached, i.new, i.k_new, i.v_new)
    s.at = _places(i.cached, i.new)
    if c["kind"] == "ingest":
        s.k_out, s.v_out = torch.empty_like(i.k_new), torch.empty_like(i.v_new)
    if c["kind"] == "attend":
        s.out = torch.empty(layers, B, c["q_heads"], HEAD_DIM, device="cuda")
        s.lse = torch.empty(layers, B, c["q_heads"], device="cuda")
        s.lengths = torch.tensor(i.cached, device="cuda")
    if c["kind"] != "verify":
        s.k_new = s.k_new if c["kind"] == "ingest" else None
        s.v_new = s.v_new if c["kind"] == "ingest" else None
    s.k = s.v = None
    return s


def run(state):
    s = state
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    c, kind, B = s.c, s.c["kind"], len(s.cached)
    if kind == "attend":
        for l, (q, out, lse, idx, cnt) in enumerate(s.by_layer):
            s.ctx.sparse_decode_attention(l, 1, None, B, q, s.params, out, idx=idx, cnt=cnt, lse=lse)
        return s.results
    if kind == "ingest":
        s.ctx.compact_sequences(None, s.cached)                          # rolls the rows of the last pass back
        s.ctx.append_kv(0, c["layers"], None, s.new, s.k_new, s.v_new)
        s.ctx.read_kv(0, c["layers"], None, s.cached, s.ends, s.k_out, s.v_out)
        return {"k": s.k_out, "v": s.v_out}
    if kind == "project":
        s.ctx.project_keys(0, c["layers"], None, s.cached, s.ends)
        return s.seen
    if kind == "fork":
        s.ctx.fork_sequence(0, list(range(1, 1 + c["copies"])), s.n_fork)
        return s.seen
    if kind == "verify":
        s.ctx.compact_sequences(None, s.cached)
        s.ctx.append_kv(0, c["layers"], None, s.new, s.k_new, s.v_new)
        s.ctx.project_keys(0, c["layers"], None, s.cached, [a + n for a, n in zip(s.cached, s.new)])
        s.ctx.compact_sequences(None, s.cached, s.kept, s.keep)
        return s.seen
    s.ctx.fork_sequence(0, [1])
    s.ctx.compact_sequences([1], s.begin, s.kept, s.keep)
    return s.seen


def _seen(s):
    """The parts of the context's caches that a call writes: a program looks at them where they are."""
    c = s.c
    if c["kind"] == "project":
        return [s.kimp[:, b, :, lo:hi] for b, (lo, hi) in enumerate(zip(s.cached, s.ends))]
    if c["kind"] == "fork":
        return {"kv": s.kv[:, 1:, :, :s.n_fork], "kimp": s.kimp[:, 1:, :, :s.n_fork]}
    if c["kind"] == "verify":
        return _kept_rows(s)
    if c["kind"] == "prune":
        return {"kv": s.kv[:, 1, :, :s.begin[0] + s.kept[0]], "kimp": s.kimp[:, 1, :, :s.begin[0] + s.kept[0]]}


def _kept_rows(s):
    return {"kv": [s.kv[:, b, :, lo:hi] for b, (lo, hi) in enumerate(zip(s.cached, s.ends))],
            "kimp": [s.kimp[:, b, :, lo:hi] for b, (lo, hi) in enumerate(zip(s.cached, s.ends))]}


# ---- the plain form ------------------------------------------------------------------------------------------------


def _places(first, count):
    """(sequence, position) of every token of a call."""
    b = np.repeat(np.arange(len(first)), count)
    t = np.concatenate([np.arange(f, f + n) for f, n in zip(first, count)]) if len(first) else np.zeros(0)
    return torch.from_numpy(b).cuda(), torch.from_numpy(t.astype(np.int64)).cuda()


def _scales(codes):
    """The scales that 8-bit codes stand for."""
    e, m = (codes >> 3).to(torch.int32), (codes & 7).to(torch.float32)
    s = torch.where(e == 0, torch.ldexp(m, torch.full_like(e, -17)), torch.ldexp(8 + m, e - 18))
    return torch.where(e == 31, torch.full_like(s, math.nan), s)


def _encode(x):
    """Rows [..][128] -> codes [..][64] and scales [..][8], both uint8."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    a = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    a = torch.where(fine, a, torch.zeros_like(a))
    table = _scales(torch.arange(TOP_SCALE + 1, device=x.device, dtype=torch.uint8))
    six = 6 * table                                                      # exact, as are the midpoints below
    up = torch.searchsorted(six, a.contiguous()).clamp_(max=TOP_SCALE)   # the first scale with 6 s >= a
    down = (up - 1).clamp_(min=0)
    middle = (six[up] + six[down]) / 2
    code = torch.where((a > middle) | ((a == middle) & (up % 2 == 0)), up, down).clamp_(min=1)
    s = table[code]
    grid = torch.tensor(GRID, device=x.device)
    edge = (grid[1:] + grid[:-1]) / 2
    # (a magnitude on an edge goes to the even code: the edges below an even code belong to it)
    edge[1::2] = torch.nextafter(edge[1::2], torch.zeros_like(edge[1::2]))
    n = torch.bucketize(torch.where(fine[..., None], x.abs(), torch.zeros_like(x)) / s[..., None], edge, out_int32=True).to(torch.uint8)
    n = torch.where((x < 0) & (n > 0), n + 8, n).flatten(-2)
    return n[..., 0::2] | (n[..., 1::2] << 4), torch.where(fine, code, torch.full_like(code, 255)).to(torch.uint8)


def _decode(codes, scales):
    """The values of rows: codes [..][64], scales [..][8] -> [..][128] in 32 bits."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return (grid[n.to(torch.int32)].unflatten(-1, (-1, BLOCK)) * _scales(scales)[..., None]).flatten(-2)


def _keys(rows):
    return _decode(rows[..., :64], rows[..., 64:72])


def _vals(rows):
    return _decode(rows[..., 80:], rows[..., 72:80])


def _store(s, first, count, k, v):
    """K and V rows [layers][tokens][heads][128] enter the cache."""
    b, t = _places(first, count)
    if s.kv.dtype == torch.uint8:
        (kc, ks), (vc, vs) = _encode(k), _encode(v)
        s.kv[:, b, :, t] = torch.cat((kc, ks, vs, vc), -1).transpose(0, 1)
    else:
        s.kv[:, b, :, t] = torch.stack((k, v), -2).transpose(0, 1)


def _project(s, first, count):
    b, t = _places(first, count)
    rows = s.kv[:, b, :, t]                                              # [tokens][layers][heads][..]
    keys = _keys(rows) if s.kv.dtype == torch.uint8 else rows[..., 0, :].float()
    s.kimp[:, b, :, t] = torch.einsum("tlhc,lhcj->tlhj", keys, s.W.float()).to(s.kimp.dtype)


def _run_plain(s):
    c, kind, B = s.c, s.c["kind"], len(s.cached)
    if kind == "attend":
        return _attend_plain(s)
    if kind == "ingest":
        _store(s, s.cached, s.new, s.k_new, s.v_new)
        rows = s.kv[:, s.at[0], :, s.at[1]].transpose(0, 1)
        return {"k": _keys(rows).to(torch.bfloat16), "v": _vals(rows).to(torch.bfloat16)}
    if kind == "project":
        _project(s, s.cached, s.new)
        return [s.kimp[:, b, :, lo:hi] for b, (lo, hi) in enumerate(zip(s.cached, s.ends))]
    if kind == "fork":
        n = s.n_fork
        s.kv[:, 1:, :, :n] = s.kv[:, :1, :, :n]
        s.kimp[:, 1:, :, :n] = s.kimp[:, :1, :, :n]
        return {"kv": s.kv[:, 1:, :, :n], "kimp": s.kimp[:, 1:, :, :n]}
    if kind == "verify":
        _store(s, s.cached, s.new, s.k_new, s.v_new)
        _project(s, s.cached, s.new)
        b, t = _places(s.cached, s.kept)
        src = torch.cat([s.keep[j, :n] for j, n in enumerate(s.kept)]).long()
        s.kv[:, b, :, t] = s.kv[:, b, :, src]
        s.kimp[:, b, :, t] = s.kimp[:, b, :, src]
        return _kept_rows(s)
    L, p, n = s.cached[0], s.begin[0], s.kept[0]
    s.kv[:, 1, :, :L] = s.kv[:, 0, :, :L]
    s.kimp[:, 1, :, :L] = s.kimp[:, 0, :, :L]
    s.kv[:, 1, :, p:p + n] = s.kv[:, 1, :, s.keep[0, :n].long()]
    s.kimp[:, 1, :, p:p + n] = s.kimp[:, 1, :, s.keep[0, :n].long()]
    return {"kv": s.kv[:, 1, :, :p + n], "kimp": s.kimp[:, 1, :, :p + n]}


def _attend_plain(s):
    c, B, heads, layers = s.c, len(s.cached), s.c["kv_heads"], s.c["layers"]
    L = s.lengths[None, :, None, None]
    if c["budget"] < 0:
        rows = s.kv[:, :B, :, :max(s.cached)]
        valid = torch.arange(max(s.cached), device="cuda") < L
    else:
        sinks = torch.arange(c["sinks"], device="cuda").expand(layers, B, heads, -1)
        n_sink = L.clamp(max=c["sinks"])
        window = torch.maximum(n_sink, L - c["recent"]) + torch.arange(c["recent"], device="cuda")
        window = window.expand(layers, B, heads, -1)
        at = torch.cat((sinks, s.idx.long(), window), -1)
        valid = torch.cat((sinks < L, torch.arange(s.cap, device="cuda") < s.cnt[..., None], window < L), -1)
        at = torch.where(valid, at, torch.zeros_like(at))
        rows = torch.gather(s.kv[:, :B], 3, at[..., None].expand(-1, -1, -1, -1, ROW))
    q = s.q.float().view(layers, B, heads, -1, HEAD_DIM)
    x = torch.matmul(q, _keys(rows).transpose(-1, -2)) / math.sqrt(HEAD_DIM)
    x = torch.where(valid[..., None, :], x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    values = torch.where(valid[..., None], _vals(rows), torch.zeros((), device="cuda"))
    out = torch.matmul(p, values) / total
    return {"out": out.view(layers, B, -1, HEAD_DIM), "lse": (top + torch.log(total)).view(layers, B, -1)}


# ---- the definition, in 64 bits ------------------------------------------------------------------------------------


def _held(x):
    """What a 4-bit cache holds of rows [..][128]: every block scaled and rounded as the module's text says."""
    x = x.double()
    y = x.reshape(*x.shape[:-1], 8, 16)
    ideal = y.abs().amax(-1) / 6
    # the scale's unit in the last place: 2^-17 up to 2^-13, then an eighth of the power of two below the ideal
    unit = torch.exp2(torch.floor(torch.log2(ideal.clamp(min=2.0 ** -14))) - 3)
    scale = (torch.round(ideal / unit) * unit).clamp(2.0 ** -17, 10240.0)
    z = y / scale[..., None]
    m = z.abs().clamp(max=6)
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
    return (torch.sign(z) * torch.round(m / step) * step * scale[..., None]).reshape(x.shape)


def exact(case, seed):
    c, kind = case, case["kind"]
    i = _inputs(c, seed)
    fp4 = c.get("dtype", "fp4") == "fp4"
    held = _held if fp4 else torch.Tensor.double
    first = np.concatenate(([0], np.cumsum(i.cached))).tolist()
    first_new = np.concatenate(([0], np.cumsum(i.new))).tolist()
    if kind == "attend":
        outs, lses = [], []
        for l in range(c["layers"]):
            for b, L in enumerate(i.cached):
                k = held(i.k[l, first[b]:first[b] + L]).transpose(0, 1)      # [heads][tokens][128]
                v = held(i.v[l, first[b]:first[b] + L]).transpose(0, 1)
                x = i.q[l, b].double().reshape(c["kv_heads"], -1, HEAD_DIM) @ k.transpose(1, 2) / math.sqrt(HEAD_DIM)
                if c["budget"] >= 0:
                    seen = torch.zeros(c["kv_heads"], L, dtype=torch.bool, device="cuda")
                    seen[:, :c["sinks"]] = True
                    seen[:, max(min(c["sinks"], L), L - c["recent"]):] = True
                    for h in range(c["kv_heads"]):
                        seen[h, i.idx[l, b, h, :i.cnt[l, b, h]].long()] = True
                    x = x.masked_fill(~seen[:, None], -math.inf)
                lses.append(torch.logsumexp(x, -1).reshape(-1))
                outs.append((torch.softmax(x, -1) @ v).reshape(-1, HEAD_DIM))
        B = len(i.cached)
        return {"out": torch.stack(outs).reshape(c["layers"], B, -1, HEAD_DIM), "lse": torch.stack(lses).reshape(c["layers"], B, -1)}
    if kind == "ingest":
        return {"k": held(i.k_new), "v": held(i.v_new)}
    project = lambda k: torch.einsum("lthc,lhcj->lhtj", held(k), i.W.double())  # noqa: E731
    if kind == "project":
        return [project(i.k_new[:, lo:hi]) for lo, hi in zip(first_new, first_new[1:])]
    rows = lambda k, v: None if fp4 else torch.stack((k, v), -2).double().transpose(1, 2)  # noqa: E731   (a copy of codes: whole numbers)
    if kind == "fork":
        n = max(1, int(i.cached[0] * c["share"]))
        kv, kimp = rows(i.k[:, :n], i.v[:, :n]), project(i.k[:, :n])
        copies = lambda t: None if t is None else t[:, None].expand(-1, c["copies"], *t.shape[1:])  # noqa: E731
        return {"kv": copies(kv), "kimp": copies(kimp)}
    if kind == "verify":
        pick = [first_new[b] + (i.keep[b, :n].long() - i.cached[b]) for b, n in enumerate(i.kept)]
        return {"kv": [rows(i.k_new[:, p], i.v_new[:, p]) for p in pick], "kimp": [project(i.k_new[:, p]) for p in pick]}
    pick = torch.cat((torch.arange(i.begin[0], device="cuda"), i.keep[0, :i.kept[0]].long()))
    return {"kv": rows(i.k[:, pick], i.v[:, pick]), "kimp": project(i.k[:, pick])}
