"""Copying sequences into other slots and dropping tokens in place, for every type of rows: bytes land where they belong, nothing
else changes, and what is decoded afterwards is what a sequence that was built that way decodes."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_fp4 import generator, held, reference, tb  # noqa: E402,F401

TYPES = ["fp4", "bf16", "fp32"]


def dtype_of(tb, name):
    return {"fp4": tb.TB_FP4, "bf16": tb.TB_BF16, "fp32": tb.TB_F32}[name]


def make(tb, name, layers=2, hq=4, hkv=2, batch=4, room=300, imp=32, budget=16, seed=1, **more):
    ctx = tb.Context(layers, hq, hkv, 128, imp, dtype_of(tb, name), batch, room, budget, 0, **more)
    g = generator(seed)
    dt = tb.torch_dtype(ctx.cfg.kv_dtype)
    for l in range(layers):
        ctx.set_projection(l, (torch.randn(hkv, 128, imp, generator=g, device="cuda") / 11).to(dt))
    ctx.kv.view(torch.uint8).fill_(0x33)
    ctx.kimp.view(torch.uint8).fill_(0x33)
    ctx.g, ctx.dt = g, dt
    return ctx


def grow(ctx, seq, n, project=True):
    layers, hkv = ctx.cfg.n_layers, ctx.cfg.n_kv_heads
    k, v = (torch.randn(layers, n, hkv, 128, generator=ctx.g, device="cuda").to(ctx.dt) for _ in range(2))
    ctx.append_kv(0, layers, [seq], [n], k, v)
    if project:
        ctx.project_keys(0, layers, [seq], None, None, n_seq=1)
    return k, v


def raw(t):
    """Bytes, on the host."""
    return t.contiguous().view(torch.uint8).cpu()


def lengths(ctx, seq):
    got = {ctx.get_length(l, seq) for l in range(ctx.cfg.n_layers)}
    assert len(got) == 1
    return got.pop()


# ---- fork ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("imp,scope", [(16, 0), (32, 1), (32, 2)])
@pytest.mark.parametrize("n,part", [(1, -1), (257, -1), (257, 100), (300, 300), (40, 0), (0, -1)])
def test_fork_copies_rows_and_keys(tb, name, imp, scope, n, part):
    ctx = make(tb, name, imp=imp, list_scope=scope, batch=5)
    if n:
        grow(ctx, 1, n)
    grow(ctx, 3, 20)                                                       # a copy replaces what a slot held
    kv, kimp = raw(ctx.kv).clone(), raw(ctx.kimp).clone()
    ctx.fork_sequence(1, [3, 0], part)
    m = n if part < 0 else part
    row = lambda t: t.shape[3]  # noqa: E731
    for got, was in ((raw(ctx.kv), kv), (raw(ctx.kimp), kimp)):
        want = was.clone()
        for d in (3, 0):
            want[:, d, :, :m] = was[:, 1, :, :m]
        assert torch.equal(got, want) and row(got) == 300
    assert lengths(ctx, 0) == lengths(ctx, 3) == (m, m) and lengths(ctx, 1) == (n, n) and lengths(ctx, 2) == (0, 0)
    assert ctx.get_status() == 0


@pytest.mark.parametrize("name", TYPES)
def test_fork_to_many_and_a_part_that_is_not_projected(tb, name):
    ctx = make(tb, name, layers=3, hkv=1, batch=65, room=70)
    grow(ctx, 64, 50)
    grow(ctx, 64, 17, project=False)
    ctx.fork_sequence(64, list(range(64)), 60)
    assert lengths(ctx, 64) == (67, 50)
    for b in (0, 31, 63):
        assert lengths(ctx, b) == (60, 50)
    kv, kimp = raw(ctx.kv), raw(ctx.kimp)
    assert all(torch.equal(kv[:, b, :, :60], kv[:, 64, :, :60]) and torch.equal(kimp[:, b, :, :50], kimp[:, 64, :, :50]) for b in range(64))
    assert all((kv[:, b, :, 60:] == 0x33).all() for b in range(64))
    with pytest.raises(tb.TBError) as e:
        ctx.project_keys(0, 3, [0], [51], [60])                            # would leave a hole at 50
    assert e.value.status == tb.TB_ERR_INVALID_ARG


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("copies", [None, "resident", "important", "both"])
@pytest.mark.parametrize("host", [False, True])
def test_samples_go_on_in_the_middle_of_an_interval(tb, name, copies, host):
    """A forked sequence attends with the lists of its source on reuse steps, and both give the same bits until their tokens differ."""
    ctx = make(tb, name, hq=8, batch=3, room=300, budget=24, kv_on_host=host)
    if copies in ("resident", "both"):
        ctx.bind_resident_rows(4, 16)
    if copies in ("important", "both"):
        ctx.bind_important_buffer()
    layers = 2
    grow(ctx, 2, 200)
    qi = torch.randn(layers, 1, 8, 32, generator=ctx.g, device="cuda")
    p = [tb.select_params(24, 4, 16, interval=8, step=t) for t in range(4)]
    ctx.select_topk(0, layers, [2], 1, qi, p[0])
    ctx.fork_sequence(2, [0])
    k, v = (torch.randn(layers, 1, 2, 128, generator=ctx.g, device="cuda").to(ctx.dt) for _ in range(2))
    q = torch.randn(layers, 1, 8, 128, generator=ctx.g, device="cuda").to(ctx.dt)
    outs = {}
    for b in (2, 0):
        ctx.append_kv(0, layers, [b], [1], k, v)
        ctx.select_topk(0, layers, [b], 1, None, p[1])
        outs[b] = torch.full((layers, 1, 8, 128), math.nan, device="cuda")
        ctx.sparse_decode_attention(0, layers, [b], 1, q, p[1], outs[b])
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[2])
    ctx.fork_sequence(2, [1], 201)                                         # the first tokens only: no selection to reuse
    with pytest.raises(tb.TBError) as e:
        ctx.select_topk(0, layers, [1], 1, None, p[2])
    assert e.value.status == tb.TB_ERR_STATE
    ctx.project_keys(0, layers, [1], None, None, n_seq=1)
    ctx.project_keys(0, layers, [2], None, None, n_seq=1)
    for b in (1, 2):
        ctx.select_topk(0, layers, [b], 1, qi, p[0])
        outs[b] = torch.full((layers, 1, 8, 128), math.nan, device="cuda")
        ctx.sparse_decode_attention(0, layers, [b], 1, q, p[0], outs[b])
    assert torch.isfinite(outs[1]).all() and torch.equal(outs[1], outs[2])
    assert ctx.get_status() == 0


@pytest.mark.parametrize("name", TYPES)
def test_a_captured_fork_follows_its_source(tb, name):
    """With device lengths: append and fork replayed, the copy is always the source as it then is."""
    ctx = make(tb, name, batch=3, room=300)
    grow(ctx, 0, 50)
    ctx.use_device_lengths(True, growth_reserve=8)
    k, v = (torch.randn(2, 7, 2, 128, generator=ctx.g, device="cuda").to(ctx.dt) for _ in range(2))

    def step():
        ctx.append_kv(0, 2, [0], [7], k, v)
        ctx.project_keys(0, 2, [0], None, None, n_seq=1)
        ctx.fork_sequence(0, [2, 1])

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(5):
        k.copy_(torch.randn(k.shape, generator=ctx.g, device="cuda"))
        graph.replay()
    ctx.sync_lengths()
    n = 50 + 7 * 6
    assert lengths(ctx, 0) == lengths(ctx, 1) == lengths(ctx, 2) == (n, n)
    for t in (raw(ctx.kv), raw(ctx.kimp)):
        for b in (1, 2):
            assert torch.equal(t[:, b, :, :n], t[:, 0, :, :n]) and (t[:, b, :, n:] == 0x33).all()
    assert ctx.get_status() == 0


def test_fork_refusals(tb):
    ctx = make(tb, "fp4", batch=3)
    grow(ctx, 0, 30)
    n0 = ctx.launch_count()
    for src, dst, n in ((0, [0], -1), (0, [1, 1], -1), (0, [3], -1), (3, [0], -1), (-1, [0], -1), (0, [], -1), (0, [1], 31), (1, [0], 1), (0, [-1], -1)):
        with pytest.raises(tb.TBError) as e:
            ctx.fork_sequence(src, dst, n)
        assert e.value.status == tb.TB_ERR_INVALID_ARG and ctx.launch_count() == n0
    assert lengths(ctx, 0) == (30, 30) and lengths(ctx, 1) == (0, 0)
    wide = tb.Context(1, 1, 1, 128, 16, tb.TB_FP4, 66, 8, 4)
    with pytest.raises(tb.TBError) as e:
        wide.fork_sequence(65, list(range(65)))
    assert e.value.status == tb.TB_ERR_UNSUPPORTED


# ---- compact ----------------------------------------------------------------------------------------------------------------

def keep_lists(tb, g, begins, totals, counts, stride):
    idx = torch.full((len(begins), stride), 2 ** 30, dtype=torch.int32, device="cuda")      # (what lies behind the counts is not read)
    for b, n in enumerate(counts):
        at = torch.argsort(torch.rand(totals[b] - begins[b], generator=g, device="cuda"))[:n].sort().values
        idx[b, :n] = begins[b] + at.to(torch.int32)
    return idx


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("imp,scope,hkv,layers", [(16, 0, 2, 2), (32, 1, 3, 1), (32, 2, 1, 5)])
@pytest.mark.parametrize("totals,begins,counts", [([300, 5, 128], [0, 5, 100], [150, 0, 1]), ([2500], [3], [2400]), ([2500], [0], [1]), ([700, 700], [699, 0], [1, 700]),
                                                  ([1], [0], [1]), ([64, 65], [60, 1], [2, 63])])
def test_compaction_moves_rows_and_keys(tb, name, imp, scope, hkv, layers, totals, begins, counts):
    ctx = make(tb, name, layers, 6 if hkv == 3 else 4, hkv, len(totals) + 1, max(totals) + 3, imp, list_scope=scope)
    seqs = list(range(len(totals)))[::-1]                                  # listed in another order than stored
    for i, s in enumerate(seqs):
        grow(ctx, s, totals[i])
    kv, kimp = raw(ctx.kv).clone(), raw(ctx.kimp).clone()
    idx = keep_lists(tb, ctx.g, begins, totals, counts, max(counts) + 2)
    ctx.compact_sequences(seqs, begins, counts, idx)
    for got, was in ((raw(ctx.kv), kv), (raw(ctx.kimp), kimp)):
        want = was.clone()
        for i, s in enumerate(seqs):
            want[:, s, :, begins[i]:begins[i] + counts[i]] = was[:, s][:, :, idx[i, :counts[i]].long().cpu()]
        assert torch.equal(got, want)
    for i, s in enumerate(seqs):
        assert lengths(ctx, s) == (begins[i] + counts[i],) * 2
    assert ctx.get_status() == 0


@pytest.mark.parametrize("name", TYPES)
def test_long_compactions_of_every_share(tb, name):
    """Rows that move by little and by much, over many tiles."""
    ctx = make(tb, name, 1, 8, 8, 1, 40000, 32)
    grow(ctx, 0, 40000)
    for share in (0.999, 0.6, 0.1):
        n = ctx.get_length(0, 0)[0]
        kv, kimp = ctx.kv.clone(), ctx.kimp.clone()
        idx = keep_lists(tb, ctx.g, [17], [n], [int((n - 17) * share)], int((n - 17) * share))
        ctx.compact_sequences(None, [17], [idx.shape[1]], idx)
        m = 17 + idx.shape[1]
        at = idx[0].long()
        kv[:, :, :, 17:m] = kv[:, :, :, at]
        kimp[:, :, :, 17:m] = kimp[:, :, :, at]
        assert torch.equal(ctx.kv, kv) and torch.equal(ctx.kimp, kimp) and lengths(ctx, 0) == (m, m)
    assert ctx.get_status() == 0


@pytest.mark.parametrize("name", TYPES)
def test_truncation(tb, name):
    ctx = make(tb, name)
    grow(ctx, 0, 100)
    grow(ctx, 2, 60)
    grow(ctx, 2, 20, project=False)
    kv, n0 = raw(ctx.kv).clone(), ctx.launch_count()
    ctx.compact_sequences([2, 0], [70, 0])
    assert ctx.launch_count() == n0 and torch.equal(raw(ctx.kv), kv)       # nothing but the lengths
    assert lengths(ctx, 2) == (70, 60) and lengths(ctx, 0) == (0, 0)
    ctx.compact_sequences([2], [59])
    assert lengths(ctx, 2) == (59, 59)
    grow(ctx, 2, 4)
    assert lengths(ctx, 2) == (63, 63)
    ctx.use_device_lengths(True, 4)
    ctx.compact_sequences([2], [61])
    ctx.sync_lengths()
    assert lengths(ctx, 2) == (61, 61) and ctx.get_status() == 0


@pytest.mark.parametrize("bad", ["falls", "repeats", "early", "late", "negative", "huge"])
def test_bad_positions_are_reported(tb, bad):
    """The entry's row keeps what it held, every other one is right, and nothing outside is touched."""
    for name in TYPES:
        ctx = make(tb, name)
        grow(ctx, 1, 200)
        kv = raw(ctx.kv).clone()
        idx = torch.tensor([[20, 30, 40, 50, 60]], dtype=torch.int32)
        idx[0, 2] = {"falls": 25, "repeats": 30, "early": 5, "late": 200, "negative": -1, "huge": 2 ** 31 - 1}[bad]
        ctx.compact_sequences([1], [10], [5], idx.cuda())
        assert ctx.get_status() == tb.TB_ERR_BAD_INDEX and ctx.get_status() == 0
        want = kv.clone()
        for j, t in enumerate((20, 30, None, 50, 60)):
            # (behind an entry that is too large the next one does not ascend either)
            if t is not None and not (j == 3 and bad in ("late", "huge")):
                want[:, 1, :, 10 + j] = kv[:, 1, :, t]
        assert torch.equal(raw(ctx.kv), want) and lengths(ctx, 1) == (15, 15)


def test_compaction_refusals(tb):
    ctx = make(tb, "fp4", batch=3)
    grow(ctx, 0, 30)
    grow(ctx, 1, 30)
    grow(ctx, 1, 5, project=False)
    idx = torch.zeros(2, 8, dtype=torch.int32, device="cuda")
    n0 = ctx.launch_count()
    for status, *a in ((tb.TB_ERR_INVALID_ARG, [0], [31]), (tb.TB_ERR_INVALID_ARG, [0], [-1]), (tb.TB_ERR_INVALID_ARG, [0, 0], [1, 1]), (tb.TB_ERR_INVALID_ARG, [3], [0]),
                       (tb.TB_ERR_INVALID_ARG, [0], [0], [9], idx), (tb.TB_ERR_INVALID_ARG, [0], [23], [8], idx), (tb.TB_ERR_INVALID_ARG, [0], [0], [-1], idx),
                       (tb.TB_ERR_INVALID_ARG, [0], [0], [1], None), (tb.TB_ERR_INVALID_ARG, [0], [0], None, idx), (tb.TB_ERR_INVALID_ARG, [2], [1]),
                       (tb.TB_ERR_UNPROJECTED, [0, 1], [0, 20], [1, 1], idx)):
        with pytest.raises(tb.TBError) as e:
            ctx.compact_sequences(*a)
        assert e.value.status == status and ctx.launch_count() == n0, a
    wide = torch.zeros(2, 16, dtype=torch.int32, device="cuda")
    for bad in (wide[:, ::2], wide.long(), wide.cpu(), wide.t()):
        with pytest.raises(ValueError):
            ctx.compact_sequences([0], [0], [1], bad)
    for a in (([0], [0, 0], [1, 1], idx), ([0, 1], [0, 0], [1], idx), ([0, 1, 2], [0, 0, 0], [1, 1, 0], idx)):
        with pytest.raises(ValueError):
            ctx.compact_sequences(*a)
    assert lengths(ctx, 0) == (30, 30) and lengths(ctx, 1) == (35, 30)


def test_stored_selections_and_compaction(tb):
    """A selection made before the drafts came stays; one that could name what moved, or that a window could reach again, is gone."""
    ctx = make(tb, "fp4", hq=8, budget=24)
    grow(ctx, 0, 200)
    qi, q = torch.randn(2, 1, 8, 32, generator=ctx.g, device="cuda"), torch.randn(2, 1, 8, 128, generator=ctx.g, device="cuda").bfloat16()
    p = [tb.select_params(24, 4, 16, interval=8, step=t) for t in range(2)]
    ctx.select_topk(0, 2, [0], 1, qi, p[0])
    grow(ctx, 0, 8)
    idx = torch.tensor([[201, 204]], dtype=torch.int32, device="cuda")
    ctx.compact_sequences([0], [200], [2], idx)
    ctx.select_topk(0, 2, [0], 1, None, p[1])
    out = torch.full((2, 1, 8, 128), math.nan, device="cuda")
    ctx.sparse_decode_attention(0, 2, [0], 1, q, p[1], out)
    assert torch.isfinite(out).all()
    ctx.compact_sequences([0], [199])
    for call in (lambda: ctx.select_topk(0, 2, [0], 1, None, p[1]), lambda: ctx.sparse_decode_attention(0, 2, [0], 1, q, p[1], out)):
        with pytest.raises(tb.TBError) as e:
            call()
        assert e.value.status == tb.TB_ERR_STATE


# ---- all of it ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("host,resident", [(False, False), (True, True)])
@pytest.mark.parametrize("devlen", [False, True])
def test_speculative_decoding_of_two_samples(tb, name, host, resident, devlen):
    """A prompt, two samples of it, three rounds of drafts of which some are kept, selections and attention: as a context in which only the
    kept tokens were ever appended, and as the definition in 64 bits."""
    layers, hq, hkv = 2, 8, 2
    ctx, plain = (make(tb, name, layers, hq, hkv, 3, 400, 32, 40, kv_on_host=host and i == 0) for i in range(2))
    if resident:
        ctx.bind_resident_rows(4, 16)
    g = generator(77)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    k, v = rand(layers, 150, hkv, 128).to(ctx.dt), rand(layers, 150, hkv, 128).to(ctx.dt)
    kept = {b: ([k], [v]) for b in (1, 2)}
    ctx.append_kv(0, layers, [0], [150], k, v)
    ctx.project_keys(0, layers, [0], [0], [150])
    if devlen:
        ctx.use_device_lengths(True, 0)
    ctx.fork_sequence(0, [2, 1])
    for b in (1, 2):
        plain.append_kv(0, layers, [b], [150], k, v)
    n = {1: 150, 2: 150}
    for round_ in range(3):
        drafts = [13, 5]
        k, v = rand(layers, 18, hkv, 128).to(ctx.dt), rand(layers, 18, hkv, 128).to(ctx.dt)
        ctx.append_kv(0, layers, [1, 2], drafts, k, v)
        ctx.project_keys(0, layers, [1, 2], None, None, n_seq=2)
        take = [[0, 3, 4, 12], [] if round_ == 1 else [2]]
        idx = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
        for i, b in enumerate((1, 2)):
            idx[i, :len(take[i])] = torch.tensor([n[b] + t for t in take[i]], dtype=torch.int32)
            if take[i]:
                at = torch.tensor([13 * i + t for t in take[i]], device="cuda")
                plain.append_kv(0, layers, [b], [len(take[i])], k[:, at].contiguous(), v[:, at].contiguous())
                kept[b][0].append(k[:, at]), kept[b][1].append(v[:, at])
        ctx.compact_sequences([1, 2], [n[1], n[2]], [len(t) for t in take], idx)
        n = {b: n[b] + len(take[i]) for i, b in enumerate((1, 2))}
        plain.project_keys(0, layers, [1, 2], None, None, n_seq=2)
        qi, q = rand(layers, 2, hq, 32), rand(layers, 2, hq, 128).to(ctx.dt)
        p = tb.select_params(40, 4, 16)
        outs = []
        for c in (ctx, plain):
            cap = c.index_capacity
            lists, counts = torch.zeros(layers, 2, hkv, cap, dtype=torch.int32, device="cuda"), torch.zeros(layers, 2, hkv, dtype=torch.int32, device="cuda")
            c.select_topk(0, layers, [1, 2], 2, qi, p, lists, counts)
            out = torch.full((layers, 2, hq, 128), math.nan, device="cuda")
            c.sparse_decode_attention(0, layers, [1, 2], 2, q, p, out, idx=lists, cnt=counts)
            stored = torch.full((layers, 2, hq, 128), math.nan, device="cuda")
            c.sparse_decode_attention(0, layers, [1, 2], 2, q, p, stored)
            assert torch.allclose(out, stored, rtol=0, atol=1e-3)
            outs.append((out, lists, counts, stored))
        assert all(torch.equal(a, b) for a, b in zip(outs[0][1:3], outs[1][1:3]))
        if not devlen:
            assert torch.equal(outs[0][3], outs[1][3])
        for b in (1, 2):
            assert ctx.get_length(1, b) == plain.get_length(1, b) == (n[b], n[b])
            assert torch.equal(raw(ctx.kv[:, b, :, :n[b]]), raw(plain.kv[:, b, :, :n[b]])) and torch.equal(raw(ctx.kimp[:, b, :, :n[b]]), raw(plain.kimp[:, b, :, :n[b]]))
    out, lists, counts, _ = outs[0]
    for i, b in enumerate((1, 2)):
        kk, vv = (torch.cat(t, 1) for t in kept[b])
        kk, vv = (held(t) if name == "fp4" else t.double() for t in (kk, vv))
        for l in range(layers):
            seen = torch.zeros(hkv, n[b], dtype=torch.bool, device="cuda")
            seen[:, :4], seen[:, n[b] - 16:] = True, True
            for h in range(hkv):
                seen[h, lists[l, i, h, :counts[l, i, h]].long()] = True
            o, _, bound, _ = reference(q[l, i].double(), kk[l].transpose(0, 1), vv[l].transpose(0, 1), seen, 128 ** -0.5)
            # (bf16 rows: the weights are split into two bf16 parts, 2^-16)
            assert ((out[l, i].double() - o).abs() <= bound + 2.0 ** -15 * vv[l].abs().max()).all()
    if devlen:
        ctx.sync_lengths()
        assert lengths(ctx, 1)[0] == n[1] and lengths(ctx, 2)[0] == n[2]
    assert ctx.get_status() == 0 and plain.get_status() == 0


@pytest.mark.parametrize("name", TYPES)
def test_drafts_verified_in_a_replayed_graph(tb, name):
    """Truncate, append, project, compact and attend captured once: every replay verifies the new drafts at the same place."""
    ctx = make(tb, name, hq=8, batch=2, room=300)
    grow(ctx, 0, 150)
    k, v = (torch.zeros(2, 9, 2, 128, dtype=ctx.dt, device="cuda") for _ in range(2))
    idx, q, out = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, 8, 128, dtype=ctx.dt, device="cuda"), torch.zeros(2, 1, 8, 128, device="cuda")

    def step():
        ctx.compact_sequences([0], [150])
        ctx.append_kv(0, 2, [0], [9], k, v)
        ctx.project_keys(0, 2, [0], [150], [159])
        ctx.compact_sequences([0], [150], [4], idx)
        ctx.sparse_decode_attention(0, 2, [0], 1, q, tb.select_params(-1), out)

    idx.copy_(torch.tensor([[150, 151, 152, 153]], dtype=torch.int32))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=ctx.g, device="cuda"))
        at = torch.tensor([0, 2 + seed, 6, 8 - (seed == 2)])
        idx.copy_((150 + at)[None].to(torch.int32))
        graph.replay()
        direct = make(tb, name, hq=8, batch=2, room=300)
        grow(direct, 0, 150)
        direct.append_kv(0, 2, [0], [4], k[:, at].contiguous(), v[:, at].contiguous())
        direct.project_keys(0, 2, [0], [150], [154])
        want = torch.zeros_like(out)
        direct.sparse_decode_attention(0, 2, [0], 1, q, tb.select_params(-1), want)
        assert torch.equal(ctx.kv[:, 0, :, :154], direct.kv[:, 0, :, :154]) and torch.equal(ctx.kimp[:, 0, :, :154], direct.kimp[:, 0, :, :154])
        assert torch.equal(out, want) and torch.isfinite(out).all()
    assert ctx.get_status() == 0 and lengths(ctx, 0) == (154, 154)


def test_on_another_stream(tb):
    """Everything is enqueued on the stream that is passed or current."""
    ctx = make(tb, "fp4", batch=3)
    side = torch.cuda.Stream()
    grow(ctx, 0, 100)
    torch.cuda.synchronize()
    ref = raw(ctx.kv[:, 0, :, :100])
    busy = torch.randn(4096, 4096, device="cuda")
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy
            busy = busy / busy.norm()
        ctx.fork_sequence(0, [1])
    idx = torch.arange(1, 100, 2, dtype=torch.int32, device="cuda")[None]
    side.wait_stream(torch.cuda.current_stream())
    ctx.compact_sequences([1], [0], [50], idx, stream=side)
    side.synchronize()
    assert torch.equal(raw(ctx.kv[:, 1, :, :50]), ref[:, :, 1::2])
