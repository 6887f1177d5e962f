"""A K|V cache held in 4 bits (TB_FP4) against its definition in 64 bits: rows in and out, key projection, attention, and the
options that read or copy the rows.  The reference works on the values that the cache is defined to hold; it shares no code
with the library."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROW = 144
GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


@pytest.fixture(scope="module")
def tb():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2503_07518_b200 import binding, build
    build.build()
    return binding


# ---- the format, in 64 bits ------------------------------------------------------------------------------------------

def scale_values():
    b = np.arange(256)
    e, m = b >> 3, b & 7
    s = np.where(e == 0, m * 2.0 ** -17, (8 + m) * 2.0 ** (e - 18.0))
    s[255] = np.nan
    return s


def encode(x):
    """Rows [.., 128] in float64 -> codes 0..15 [.., 128], scale bytes [.., 8]."""
    blocks = x.reshape(*x.shape[:-1], 8, 16)
    fine = np.isfinite(blocks).all(-1)
    a = np.where(fine, np.abs(np.where(np.isfinite(blocks), blocks, 0)).max(-1), 0)
    table = scale_values()[:227]
    # nearest scale to a / 6: compared as a against 6 s, which is exact
    hi = np.clip(np.searchsorted(6 * table, a), 0, 226)
    lo = np.maximum(hi - 1, 0)
    dh, dl = np.abs(6 * table[hi] - a), np.abs(a - 6 * table[lo])
    b = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    b = np.maximum(b, 1)
    s = table[b][..., None]
    m = np.minimum(np.where(np.isfinite(blocks), np.abs(blocks), 0), 6 * s)     # (distances from far above would all round to one number)
    dist = np.abs(m[..., None] - GRID * s[..., None])           # exact: few significant bits
    best = dist.min(-1, keepdims=True)
    n = np.where((dist == best) & (np.arange(8) % 2 == 0), 2, (dist == best).astype(int)).argmax(-1)     # of two, the even code
    n = n + 8 * ((blocks < 0) & (n > 0))
    n = np.where(fine[..., None], n, 0)
    return n.reshape(x.shape), np.where(fine, b, 255)


def values(n, b):
    v = np.where(n >= 8, -1.0, 1.0) * GRID[n & 7]
    return (v.reshape(*n.shape[:-1], 8, 16) * scale_values()[b][..., None]).reshape(n.shape)


def held(t):
    """The values that the cache holds of bf16 rows, as float64 on the device."""
    n, b = encode(t.double().cpu().numpy())
    return torch.from_numpy(values(n, b)).cuda()


def pack(k, v):
    """Row bytes [.., 144] of float64 rows."""
    (kn, kb), (vn, vb) = encode(k), encode(v)
    half = lambda n: (n[..., 0::2] | n[..., 1::2] << 4).astype(np.uint8)  # noqa: E731
    return np.concatenate((half(kn), kb.astype(np.uint8), vb.astype(np.uint8), half(vn)), -1)


def rows(gen, *shape, spread=0.0):
    x = torch.randn(*shape, 128, generator=gen, device="cuda")
    if spread:
        x = x * torch.exp(spread * torch.randn(*shape, 1, generator=gen, device="cuda"))
    return x.bfloat16()


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def context(tb, layers=1, hq=8, hkv=2, batch=1, room=512, imp=32, budget=64, radius=0, **more):
    ctx = tb.Context(layers, hq, hkv, 128, imp, tb.TB_FP4, batch, room, budget, radius, **more)
    g = generator(99)
    ctx.W = (torch.randn(layers, hkv, 128, imp, generator=g, device="cuda") / 11).bfloat16()
    for l in range(layers):
        ctx.set_projection(l, ctx.W[l])
    return ctx


# ---- rows in and out -----------------------------------------------------------------------------------------------

def through(tb, x):
    """x [tokens, 128] as K rows and its negative as V rows: bytes and values that come back."""
    n = x.shape[0]
    ctx = context(tb, hq=1, hkv=1, room=n, layers=1)
    k = x.bfloat16().cuda()[:, None].contiguous()
    v = (-k).contiguous()
    ctx.append_kv(0, 1, None, [n], k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    ctx.read_kv(0, 1, None, [0], [n], ko, vo)
    assert ctx.get_status() == 0
    return k, v, ctx.kv[0, 0, 0].cpu().numpy(), ko, vo


def check_through(tb, x):
    k, v, got, ko, vo = through(tb, x)
    kd, vd = k.double().cpu().numpy()[:, 0], v.double().cpu().numpy()[:, 0]
    assert np.array_equal(got, pack(kd, vd))
    for out, d in ((ko, kd), (vo, vd)):
        assert np.array_equal(out.double().cpu().numpy()[:, 0], values(*encode(d)), equal_nan=True)


@pytest.mark.parametrize("spread", [0.0, 2.0, 8.0])
def test_rows_are_rounded_as_defined(tb, spread):
    check_through(tb, rows(generator(1), 777, spread=spread))


def test_every_magnitude_as_the_largest_of_its_block(tb):
    """All positive bf16 values as a block's largest, beside elements on and next to the edges between codes."""
    a = torch.arange(0x7f80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
    edge = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -2.5, -5, 1, 0, 6])
    x = torch.cat((a[:, None], a[:, None] / 6 * edge), 1)                 # [32640, 16]; rounded to bf16 on the way
    x = torch.cat((x, torch.zeros(-len(x) % 8, 16)))
    check_through(tb, x.reshape(-1, 128).float().clamp(-3e38, 3e38))


def test_elements_on_the_edges_between_codes(tb):
    """For every scale: elements exactly on each edge, where bf16 holds it, and one bf16 step on either side."""
    s = torch.from_numpy(scale_values()[1:227])
    edge = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5]).double()
    at = (s[:, None] * edge).bfloat16()                                   # at most 7 significant bits: exact
    assert torch.equal(at.double(), s[:, None] * edge)
    step = lambda t, d: (t.view(torch.int16) + d).view(torch.bfloat16)  # noqa: E731
    top = (6 * s[:, None]).bfloat16()
    for sign in (1, -1):
        for d in (-1, 0, 1):
            block = torch.cat((top, sign * step(at, d), torch.zeros(len(s), 8).bfloat16()), 1)
            check_through(tb, torch.cat((block, torch.zeros(-len(block) % 8, 16).bfloat16())).reshape(-1, 128))


def test_blocks_that_are_not_finite_read_as_nan(tb):
    x = rows(generator(2), 9).float().cpu()
    x[1, 17], x[3, 127], x[5, 0], x[6, 64] = math.inf, -math.inf, math.nan, 3e38
    check_through(tb, x)


@pytest.mark.parametrize("hkv,layers,counts", [(1, 1, [1]), (3, 2, [5, 0, 77]), (8, 3, [1, 1, 1, 1]), (8, 1, [1000, 3])])
def test_ragged_appends_and_reads(tb, hkv, layers, counts):
    """Rows of several sequences land behind what is cached; reads of any range give them back; nothing else is written."""
    g = generator(3)
    ctx = context(tb, layers, hkv, hkv, len(counts), room=max(counts) + 40)
    ctx.kv.fill_(0x5a)
    first = [7 * (i + 1) for i in range(len(counts))]
    want = torch.full_like(ctx.kv, 0x5a).cpu().numpy()
    at = [0] * len(counts)
    for n_new in (first, counts):
        k, v = rows(g, layers, sum(n_new), hkv), rows(g, layers, sum(n_new), hkv, spread=1.0)
        ctx.append_kv(0, layers, None, n_new, k, v)
        off = 0
        for b, n in enumerate(n_new):
            p = pack(k[:, off:off + n].double().cpu().numpy(), v[:, off:off + n].double().cpu().numpy())
            want[:, b, :, at[b]:at[b] + n] = p.transpose(0, 2, 1, 3)
            at[b] += n
            off += n
    assert np.array_equal(ctx.kv.cpu().numpy(), want)
    lo, hi = [a // 3 for a in at], [a - (a > 9) for a in at]
    n = sum(h - l for l, h in zip(lo, hi))
    ko, vo = (torch.empty(layers, n, hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.read_kv(0, layers, None, lo, hi, ko, vo)
    half = lambda c: np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], 128)  # noqa: E731
    wk = values(half(want[..., :64]), want[..., 64:72].astype(int))
    wv = values(half(want[..., 80:]), want[..., 72:80].astype(int))
    off = 0
    for b in range(len(counts)):
        m = hi[b] - lo[b]
        for got, w in ((ko, wk), (vo, wv)):
            assert np.array_equal(got[:, off:off + m].double().cpu().numpy(), w[:, b, :, lo[b]:hi[b]].transpose(0, 2, 1, 3))
        off += m


def test_rows_that_start_on_16_bytes(tb):
    """Inputs and outputs aligned to 16 bytes but not to 32: the same rows."""
    g = generator(43)
    ctx = context(tb, 2, 8, 2, 2, room=200)
    room = torch.zeros(2, 2 * 90 * 2 * 128 + 8, dtype=torch.bfloat16, device="cuda")
    k, v = (room[i, 8:].view(2, 90, 2, 128) for i in range(2))
    room = torch.zeros(2, 2 * 90 * 2 * 128 + 8, dtype=torch.bfloat16, device="cuda")
    ko, vo = (room[i, 8:].view(2, 90, 2, 128) for i in range(2))
    assert k.data_ptr() % 32 == 16 and ko.data_ptr() % 32 == 16
    k.copy_(rows(g, 2, 90, 2)), v.copy_(rows(g, 2, 90, 2))
    ctx.append_kv(0, 2, None, [40, 50], k, v)
    ctx.read_kv(0, 2, None, [0, 0], [40, 50], ko, vo)
    assert torch.equal(ko.double(), held(k)) and torch.equal(vo.double(), held(v)) and (room[:, :8] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_reads_of_the_other_types_return_what_was_appended(tb, dtype):
    dt = tb.TB_BF16 if dtype == "bf16" else tb.TB_F32
    ctx = tb.Context(2, 6, 3, 128, 16, dt, 3, 100, 8)
    counts = [40, 1, 100]
    k, v = (torch.randn(2, sum(counts), 3, 128, device="cuda").to(tb.torch_dtype(dt)) for _ in range(2))
    ctx.append_kv(0, 2, None, counts, k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    ctx.read_kv(0, 2, None, [0, 0, 0], counts, ko, vo)
    assert torch.equal(ko, k) and torch.equal(vo, v)
    ko, vo = torch.empty_like(k[1:, :33]), torch.empty_like(k[1:, :33])
    ctx.read_kv(1, 1, [2, 0], [67, 40], [100, 40], ko, vo)                # one empty range
    assert torch.equal(ko, k[1:, 41 + 67:]) and torch.equal(vo, v[1:, 41 + 67:])


# ---- projection -----------------------------------------------------------------------------------------------------

def check_projected(ctx, keys, lo, hi, l, b):
    """bf16 projections of float64 keys [heads, tokens, 128]: one rounding (half a step, 2^-8 of the value) and the forward error of a
    sum of 128 (or heads x 128) products in fp32."""
    W = ctx.W[l].double()
    ref = torch.einsum("htc,hcj->htj", keys, W)
    size = torch.einsum("htc,hcj->htj", keys.abs(), W.abs())
    if ctx.n_key_heads == 1 and W.shape[0] > 1:
        ref, size = ref.sum(0, keepdim=True), size.sum(0, keepdim=True)
    got = ctx.kimp[l, b, :, lo:hi].double()
    bound = ref.abs() * 2.0 ** -8 + 2.0 ** -133 + 128 * W.shape[0] * 2.0 ** -23 * size
    assert ((got - ref[:, lo:hi]).abs() <= bound[:, lo:hi]).all()


@pytest.mark.parametrize("scope", ["kv", "layer"])
@pytest.mark.parametrize("imp", [16, 32])
@pytest.mark.parametrize("counts", [[1], [15, 16, 17], [64, 65, 0, 1], [1000, 63]])
def test_projection_of_held_keys(tb, scope, imp, counts):
    g = generator(4)
    ctx = context(tb, 2, 6, 3, len(counts), room=max(counts) + 8, imp=imp, list_scope=tb.TB_SCOPE_LAYER if scope == "layer" else tb.TB_SCOPE_KV_HEAD)
    ctx.kimp.fill_(7.0)
    k, v = rows(g, 2, sum(counts), 3, spread=1.0), rows(g, 2, sum(counts), 3)
    ctx.append_kv(0, 2, None, counts, k, v)
    half = [n // 2 for n in counts]
    ctx.project_keys(0, 2, None, [0] * len(counts), half)
    assert all((ctx.kimp[:, b, :, h:] == 7.0).all() for b, h in enumerate(half))          # nothing behind the range
    ctx.project_keys(0, 2, None, None, None, n_seq=len(counts))                           # the rest, as everything not yet projected
    keys, off = held(k), 0
    for b, n in enumerate(counts):
        for l in range(2):
            check_projected(ctx, keys[l, off:off + n].transpose(0, 1), 0, n, l, b)
        assert (ctx.kimp[:, b, :, n:] == 7.0).all()
        off += n


def test_a_row_projects_alike_in_every_call(tb):
    g = generator(5)
    ctx = context(tb, 1, 8, 8, 1, room=300)
    k, v = rows(g, 1, 300, 8), rows(g, 1, 300, 8)
    ctx.append_kv(0, 1, None, [300], k, v)
    ctx.project_keys(0, 1, None, [0], [300])
    whole = ctx.kimp.clone()
    for lo, hi in ((0, 1), (37, 41), (299, 300), (100, 229)):
        ctx.kimp[:, :, :, lo:hi] = 0
        ctx.project_keys(0, 1, None, [lo], [hi])
        assert torch.equal(ctx.kimp, whole)


@pytest.mark.parametrize("n", [60, 700])
@pytest.mark.parametrize("kind", ["wide", "tiny", "huge", "zero", "inf"])
def test_projection_matrices_of_every_range(tb, n, kind):
    """Elements 2^-40 below the largest (more than f16 spans), matrices of the smallest and largest magnitudes, of zeros, and with an infinity."""
    g = generator(40)
    ctx = context(tb, 1, 2, 2, 1, room=n)
    W = torch.randn(1, 2, 128, 32, generator=g, device="cuda")
    if kind == "wide":
        W *= torch.exp2(torch.randint(-40, 1, W.shape, generator=g, device="cuda").float())
    W = (W * {"tiny": 2.0 ** -110, "huge": 2.0 ** 90, "zero": 0.0}.get(kind, 1.0)).bfloat16()
    if kind == "inf":
        W[0, 1, 5, 7] = math.inf
    ctx.W = W
    ctx.set_projection(0, W[0])
    k, v = rows(g, 1, n, 2, spread=1.0), rows(g, 1, n, 2)
    k[:, :, :, ::3] = 0                                                    # (large elements of W against zeros: small ones count)
    ctx.append_kv(0, 1, None, [n], k, v)
    ctx.project_keys(0, 1, None, [0], [n])
    if kind == "inf":
        at = held(k)[0, :, 1, 5]
        assert torch.equal(torch.isinf(ctx.kimp[0, 0, 1, :, 7]), at != 0) and torch.isnan(ctx.kimp[0, 0, 1, :, 7][at == 0]).all()
        ctx.kimp[0, 0, 1, :, 7] = 0
        ctx.W = torch.where(torch.isinf(W), torch.zeros_like(W), W)
        ctx.W[0, 1, :, 7] = 0
    check_projected(ctx, held(k)[0].transpose(0, 1), 0, n, 0, 0)


def test_scores_and_selections_are_those_of_bf16(tb):
    """The same projected keys: the same scores and lists, bit for bit."""
    g = generator(41)
    got = []
    kimp = torch.randn(2, 3, 4, 900, 32, generator=g, device="cuda").bfloat16()
    qi = torch.randn(2, 3, 8, 32, generator=g, device="cuda")
    k = torch.zeros(2, 2700, 4, 128, dtype=torch.bfloat16, device="cuda")
    for dt in (tb.TB_FP4, tb.TB_BF16):
        ctx = tb.Context(2, 8, 4, 128, 32, dt, 3, 900, 100, 1)
        ctx.append_kv(0, 2, None, [900] * 3, k, k)
        ctx.project_keys(0, 2, None, [0] * 3, [900] * 3)
        ctx.kimp.copy_(kimp)
        idx = torch.zeros(2, 3, 4, ctx.index_capacity, dtype=torch.int32, device="cuda")
        cnt = torch.zeros(2, 3, 4, dtype=torch.int32, device="cuda")
        ctx.select_topk(0, 2, None, 3, qi, tb.select_params(100, 4, 16, 1), idx, cnt)
        scores = torch.zeros(3, 4, 900, device="cuda")
        ctx.score_tokens(1, None, 3, qi[1].contiguous(), scores)
        assert ctx.get_status() == 0
        got.append((idx, cnt, scores))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and (got[0][1] > 100).all()


# ---- attention ----------------------------------------------------------------------------------------------------------

def reference(q, k, v, seen, scale):
    """q [hq, 128], k and v [hkv, tokens, 128], seen [hl, tokens] bool (hl divides hq): output, log-sum-exp and a bound on what fp32
    may be off by, in 64 bits."""
    hq, hkv = q.shape[0], k.shape[0]
    kk, vv = (t.repeat_interleave(hq // hkv, 0) for t in (k, v))
    seen = seen.repeat_interleave(hq // seen.shape[0], 0)
    x = torch.einsum("hc,htc->ht", q, kk) * scale
    x = x.masked_fill(~seen, -math.inf)
    out = torch.einsum("ht,htc->hc", torch.softmax(x, -1), vv)
    # Scores: a sum of 128 fp32 products (128 x 2^-23 of the sum of their magnitudes: the tensor core may truncate) and three roundings of
    # the scaled score and of the exponent, so a weight is off by that relative to itself, twice (it and the sum of all); the
    # weights' split (2^-21) and the sum over the tokens (n 2^-23 of the sum of magnitudes).
    size = torch.einsum("hc,htc->ht", q.abs(), kk.abs()) * scale
    e = (128 * 2.0 ** -23 * size + 2.0 ** -21 * (1 + x.abs())).masked_fill(~seen, 0).amax(-1)
    n = seen.sum(-1)
    largest = torch.einsum("ht,htc->hc", torch.softmax(x, -1), vv.abs())
    bound = largest * (2 * e + 2.0 ** -20 + n * 2.0 ** -23)[:, None] + vv.abs().amax((1, 2), keepdim=False)[:, None] * n[:, None] * 2.0 ** -39
    return out, torch.logsumexp(x, -1), bound, e + n * 2.0 ** -23 + 2.0 ** -20 * (1 + torch.logsumexp(x, -1).abs())


def check_attention(tb, ctx, k, v, lengths, p, q, idx=None, cnt=None, scale=0.0, layers=1, status=0):
    """k, v: float64 values [layers, sum of lengths, hkv, 128]."""
    B, hq = len(lengths), q.shape[2]
    out, lse = torch.full((layers, B, hq, 128), math.nan, device="cuda"), torch.full((layers, B, hq), math.nan, device="cuda")
    ctx.sparse_decode_attention(0, layers, None, B, q, p, out, idx=idx, cnt=cnt, sm_scale=scale, lse=lse)
    assert ctx.get_status() == status
    first = np.concatenate(([0], np.cumsum(lengths)))
    hl = 1 if idx is None else idx.shape[2]
    for l in range(layers):
        for b, L in enumerate(lengths):
            seen = torch.ones(hl, L, dtype=torch.bool, device="cuda")
            if p.budget >= 0:
                s = min(p.sinks, L)
                seen[:, s:max(s, L - p.recent)] = False
                for h in range(hl):
                    at = idx[l, b, h, :cnt[l, b, h]].long()
                    seen[h, at[(at >= 0) & (at < L)]] = True
            rows_ = slice(first[b], first[b] + L)
            o, s, bo, bs = reference(q[l, b].double(), k[l, rows_].transpose(0, 1), v[l, rows_].transpose(0, 1), seen, scale or 128 ** -0.5)
            assert ((out[l, b].double() - o).abs() <= bo).all(), ((out[l, b].double() - o).abs() / bo).max()
            assert ((lse[l, b].double() - s).abs() <= bs).all()
    return out, lse


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (8, 4), (9, 3), (32, 8), (7, 1), (16, 2)])
@pytest.mark.parametrize("lengths", [[1], [2, 15, 16, 17], [31, 33, 400, 129]])
def test_dense_attention(tb, hq, hkv, lengths):
    g = generator(6)
    ctx = context(tb, 1, hq, hkv, len(lengths), room=max(lengths))
    k, v = rows(g, 1, sum(lengths), hkv, spread=0.5), rows(g, 1, sum(lengths), hkv, spread=0.5)
    ctx.append_kv(0, 1, None, lengths, k, v)
    check_attention(tb, ctx, held(k), held(v), lengths, tb.select_params(-1), rows(g, 1, len(lengths), hq))


@pytest.mark.parametrize("batch,length,hq,hkv", [(1, 40001, 32, 8), (1, 9000, 8, 1), (3, 3000, 28, 4), (20, 2100, 32, 8), (40, 300, 32, 8), (1, 3000, 4, 1),
                                                 (5, 16500, 8, 1), (2, 700, 32, 32)])
def test_dense_attention_in_every_split(tb, batch, length, hq, hkv):
    """Cluster merges of every kind, the global merge and single blocks (which size takes which is the launcher's)."""
    g = generator(7)
    lengths = [max(5, length - 13 * b) for b in range(batch)]
    ctx = context(tb, 1, hq, hkv, batch, room=length)
    k, v = rows(g, 1, sum(lengths), hkv), rows(g, 1, sum(lengths), hkv)
    ctx.append_kv(0, 1, None, lengths, k, v)
    check_attention(tb, ctx, held(k), held(v), lengths, tb.select_params(-1), rows(g, 1, batch, hq))


def make_lists(g, lengths, hl, budget, sinks, recent, layers=1):
    cap = -(-budget // 4) * 4
    idx = torch.zeros(layers, len(lengths), hl, cap, dtype=torch.int32, device="cuda")
    cnt = torch.zeros(layers, len(lengths), hl, dtype=torch.int32, device="cuda")
    for l in range(layers):
        for b, L in enumerate(lengths):
            lo = min(sinks, L)
            hi = max(lo, L - recent)
            for h in range(hl):
                n = min(budget, hi - lo) - (h % 3)
                if n > 0:
                    idx[l, b, h, :n] = lo + torch.argsort(torch.rand(hi - lo, generator=g, device="cuda"))[:n].sort().values
                    cnt[l, b, h] = n
    return idx, cnt


@pytest.mark.parametrize("scope", ["kv", "q", "layer"])
@pytest.mark.parametrize("sinks,recent,budget,lengths", [(4, 16, 50, [1000, 3, 21, 300]), (0, 1, 1, [1, 2, 50]), (128, 256, 200, [5000, 100, 385]),
                                                         (0, 7, 2000, [12000]), (3, 3, 33, [200] * 17)])
def test_sparse_attention(tb, scope, sinks, recent, budget, lengths):
    g = generator(8)
    sc = {"kv": tb.TB_SCOPE_KV_HEAD, "q": tb.TB_SCOPE_Q_HEAD, "layer": tb.TB_SCOPE_LAYER}[scope]
    ctx = context(tb, 2, 12, 4, len(lengths), room=max(lengths), budget=budget, list_scope=sc)
    k, v = rows(g, 2, sum(lengths), 4, spread=0.3), rows(g, 2, sum(lengths), 4, spread=0.3)
    ctx.append_kv(0, 2, None, lengths, k, v)
    idx, cnt = make_lists(g, lengths, ctx.n_lists, budget, sinks, recent, layers=2)
    check_attention(tb, ctx, held(k), held(v), lengths, tb.select_params(budget, sinks, recent), rows(g, 2, len(lengths), 12), idx, cnt, layers=2)


def test_large_and_small_queries_and_values(tb):
    """Queries of every size (a head of zeros, one of the smallest and one of very large ones), keys and values at the ends of
    what the format holds."""
    g = generator(9)
    ctx = context(tb, 1, 8, 1, 1, room=200)
    k, v = rows(g, 1, 200, 1), rows(g, 1, 200, 1)
    k[:, 50:60] *= 2.0 ** -12
    v[:, 100:120] *= 2.0 ** 13
    v[:, 130:140] *= 2.0 ** -20
    ctx.append_kv(0, 1, None, [200], k, v)
    q = rows(g, 1, 1, 8)
    for h, s in enumerate((0.0, 2.0 ** -120, 2.0 ** -30, 2.0 ** -10, 1.0, 4.0, 30.0, 1.0)):
        q[0, 0, h] *= s
    q[0, 0, 7, :64] *= 2.0 ** -20
    check_attention(tb, ctx, held(k), held(v), [200], tb.select_params(-1), q)
    check_attention(tb, ctx, held(k), held(v), [200], tb.select_params(-1), q, scale=0.7)


def test_masked_scores_of_a_query_of_zeros(tb):
    """Lists shorter than a tile, a query of zeros and scales down to nearly nothing: the rows that are there share the weight."""
    g = generator(42)
    ctx = context(tb, 1, 4, 1, 1, room=64, budget=8)
    k, v = rows(g, 1, 50, 1), rows(g, 1, 50, 1)
    ctx.append_kv(0, 1, None, [50], k, v)
    idx = torch.tensor([[[[7, 9, 30, 41, 0, 0, 0, 0]]]], dtype=torch.int32, device="cuda")
    cnt = torch.tensor([[[4]]], dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    for scale in (0.0, 1e-12, 1e-30):
        out, _ = check_attention(tb, ctx, held(k), held(v), [50], tb.select_params(8), q, idx, cnt, scale=scale)
        assert (out[0, 0].double() - held(v)[0, [7, 9, 30, 41], 0].mean(0)).abs().max() <= 1e-6


def test_many_small_weights_beside_one_large(tb):
    """One token takes most of the weight, 60000 others share the rest evenly: each far below the step of a 16-bit float near the
    largest, none of them lost."""
    L = 60001
    ctx = context(tb, 1, 4, 1, 1, room=L)
    k = torch.zeros(1, L, 1, 128, dtype=torch.bfloat16, device="cuda")
    v = rows(generator(10), 1, L, 1).abs()
    k[0, 777, 0, 0] = 6.0
    v[0, 777] = 0
    ctx.append_kv(0, 1, None, [L], k, v)
    q = torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    for h, x in enumerate((2.5, 2.6875, 2.75, 3.0)):                      # e^15 .. e^18: 2^-21.6 .. 2^-26 beside 1
        q[0, 0, h, 0] = x
    check_attention(tb, ctx, held(k), held(v), [L], tb.select_params(-1), q, scale=1.0)


def test_nan_rows_reach_only_those_who_attend_them(tb):
    g = generator(11)
    lengths = [300, 300]
    ctx = context(tb, 1, 8, 2, 2, room=320, budget=40)
    k, v = rows(g, 1, 600, 2), rows(g, 1, 600, 2)
    k[0, 100, 0, 3] = math.nan
    v[0, 300 + 200, 1, 5] = math.inf
    ctx.append_kv(0, 1, None, lengths, k, v)
    q = rows(g, 1, 2, 8)
    p = tb.select_params(40, 4, 16)
    idx, cnt = make_lists(g, lengths, 2, 40, 4, 16)
    idx[idx == 100], idx[idx == 200] = 101, 201                           # (twice the same row at worst: still a list)
    for h in range(2):
        for b in range(2):
            u = torch.unique(idx[0, b, h, :cnt[0, b, h]])
            idx[0, b, h, :len(u)], cnt[0, b, h] = u, len(u)
    kh, vh = torch.nan_to_num(held(k), nan=0.0), torch.nan_to_num(held(v), nan=0.0)
    check_attention(tb, ctx, kh, vh, lengths, p, q, idx, cnt)             # nobody attends them
    out = torch.empty(1, 2, 8, 128, device="cuda")
    ctx.sparse_decode_attention(0, 1, None, 2, q, tb.select_params(-1), out)
    assert torch.isnan(out[0, 0, :4]).all() and torch.isfinite(out[0, 0, 4:]).all()
    assert torch.isfinite(out[0, 1, :4]).all() and torch.isnan(out[0, 1, 4:, :16]).all() and torch.isfinite(out[0, 1, 4:, 16:]).all()


def test_a_bad_list_entry_is_skipped_and_reported(tb):
    g = generator(12)
    ctx = context(tb, 1, 8, 2, 1, room=320, budget=40)
    k, v = rows(g, 1, 300, 2), rows(g, 1, 300, 2)
    ctx.append_kv(0, 1, None, [300], k, v)
    idx, cnt = make_lists(g, [300], 2, 40, 4, 16)
    idx[0, 0, 0, 5], idx[0, 0, 1, 39 - 2] = 300, -7
    check_attention(tb, ctx, held(k), held(v), [300], tb.select_params(40, 4, 16), rows(g, 1, 1, 8), idx, cnt, status=tb.TB_ERR_BAD_INDEX)
    assert ctx.get_status() == 0


def test_nothing_to_attend_is_what_the_other_types_make_of_it(tb):
    """No sinks, no window, an empty list: no weight to divide by.  NaN and a log-sum-exp of minus infinity, as with bf16 rows; the
    other heads' results are their own."""
    g = generator(13)
    k, v, q = rows(g, 1, 50, 2), rows(g, 1, 50, 2), rows(g, 1, 1, 8)
    idx = torch.zeros(1, 1, 2, 8, dtype=torch.int32, device="cuda")
    idx[0, 0, 1, 0] = 20
    cnt = torch.tensor([[[0, 1]]], dtype=torch.int32, device="cuda")
    got = []
    for dt in (tb.TB_FP4, tb.TB_BF16):
        ctx = tb.Context(1, 8, 2, 128, 32, dt, 1, 64, 8)
        ctx.append_kv(0, 1, None, [50], k, v)
        out, lse = torch.zeros(1, 1, 8, 128, device="cuda"), torch.zeros(1, 1, 8, device="cuda")
        ctx.sparse_decode_attention(0, 1, None, 1, q, tb.select_params(8), out, idx=idx, cnt=cnt, lse=lse)
        got.append((out, lse))
    for out, lse in got:
        assert torch.isnan(out[0, 0, :4]).all() and (lse[0, 0, :4] == -math.inf).all()
        assert torch.isfinite(out[0, 0, 4:]).all() and torch.isfinite(lse[0, 0, 4:]).all()
    assert (got[0][0][0, 0, 4:].double() - held(v)[0, 20, 1]).abs().max() == 0                   # a single row: its values


def test_offsets_past_32_bits(tb):
    """The last slots of a cache of 5.1 GB."""
    g = generator(14)
    L, heads, batch = 131072, 8, 34
    ctx = context(tb, 1, 32, heads, batch, room=L, budget=64)
    assert ctx.kv.numel() > 2 ** 32
    k, v = rows(g, 1, 3000, heads), rows(g, 1, 3000, heads)
    for b in (0, batch - 1):
        ctx.append_kv(0, 1, [b], [3000], k, v)
        ctx.project_keys(0, 1, [b], [0], [3000])
    assert torch.equal(ctx.kv[:, 0, :, :3000], ctx.kv[:, -1, :, :3000]) and torch.equal(ctx.kimp[:, 0, :, :3000], ctx.kimp[:, -1, :, :3000])
    q = rows(g, 1, 2, 32)
    q[0, 1] = q[0, 0]
    out = torch.zeros(1, 2, 32, 128, device="cuda")
    ctx.sparse_decode_attention(0, 1, [0, batch - 1], 2, q, tb.select_params(-1), out)
    assert torch.equal(out[0, 0], out[0, 1]) and torch.isfinite(out).all()
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    ctx.read_kv(0, 1, [batch - 1], [0], [3000], ko, vo)
    assert torch.equal(ko.double(), held(k)) and torch.equal(vo.double(), held(v))
    ctx.fork_sequence(0, [batch - 2])
    assert torch.equal(ctx.kv[:, 0, :, :3000], ctx.kv[:, -2, :, :3000])


# ---- the options that read or copy rows ---------------------------------------------------------------------------------

def decode_run(tb, host=False, resident=False, important=False, graph=False, every_step=False, steps=5):
    """A prompt and a few steps with a prediction interval: append, project, select, attend."""
    g = generator(15)
    layers, B, hq, hkv = 2, 2, 8, 2
    lengths = [700, 330]
    ctx = context(tb, layers, hq, hkv, B, room=800, budget=48, radius=1, kv_on_host=host)
    if resident:
        ctx.bind_resident_rows(4, 32)
    if important:
        ctx.bind_important_buffer()
    ctx.append_kv(0, layers, None, lengths, rows(g, layers, sum(lengths), hkv), rows(g, layers, sum(lengths), hkv))
    ctx.project_keys(0, layers, None, [0, 0], lengths)
    if graph:
        ctx.use_device_lengths(True, growth_reserve=16)
    k, v, q = (torch.empty(layers, B, n, 128, dtype=torch.bfloat16, device="cuda") for n in (hkv, hkv, hq))
    qi = torch.empty(layers, B, hq, 32, device="cuda")
    out = torch.empty(layers, B, hq, 128, device="cuda")
    p = [tb.select_params(48, 4, 32, 1, tb.TB_NEIGHBOR_DILATE, 1 if graph or every_step else 2, t) for t in range(steps)]

    def step(t):
        ctx.append_kv(0, layers, None, [1] * B, k, v)
        ctx.project_keys(0, layers, None, None, None, n_seq=B)
        ctx.select_topk(0, layers, None, B, qi, p[t])
        for l in range(layers):
            ctx.sparse_decode_attention(l, 1, None, B, q[l], p[t], out[l])

    captured, outs = None, []
    for t in range(steps):
        for x in (k, v, q):
            x.copy_(rows(g, *x.shape[:-1]))
        qi.copy_(torch.randn(qi.shape, generator=g, device="cuda"))
        if graph and t == 1:
            torch.cuda.synchronize()
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                step(0)
        if captured:
            captured.replay()
        else:
            step(t)
        outs.append(out.clone())
    assert ctx.get_status() == 0
    if graph:
        ctx.sync_lengths()
        assert ctx.get_length(1, 0) == (700 + steps, 700 + steps)
    return torch.stack(outs), ctx.kv[:, 0, :, :700 + steps].clone(), ctx.kimp[:, 0, :, :700 + steps].clone()


def test_offloaded_rows_and_their_copies_give_the_same_bits(tb):
    base = decode_run(tb)
    assert torch.isfinite(base[0]).all()
    for more in (dict(resident=True), dict(important=True), dict(host=True), dict(host=True, resident=True, important=True)):
        got = decode_run(tb, **more)
        assert torch.equal(got[0], base[0]) and torch.equal(got[1].cpu(), base[1].cpu()) and torch.equal(got[2], base[2]), more


def test_replayed_graph_of_a_growing_sequence(tb):
    """Rows and projections are those of direct calls, bit for bit.  Launches are sized for the reserve, so attention may be split
    otherwise: both are within 5e-4 of the exact result (scores: 128 x 2^-23 of a sum of magnitudes of about 8, twice, on values of about 1),
    so within 1e-3 of each other."""
    got, want = decode_run(tb, graph=True), decode_run(tb, every_step=True)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    assert torch.isfinite(got[0]).all() and (got[0] - want[0]).abs().max() <= 1e-3


def test_the_allocation_free_entry_point(tb):
    g = generator(16)
    lengths, hq, hkv = [900, 77], 8, 2
    ctx = context(tb, 1, hq, hkv, 2, room=1000, budget=64)
    k, v, q = rows(g, 1, sum(lengths), hkv), rows(g, 1, sum(lengths), hkv), rows(g, 2, hq)
    ctx.append_kv(0, 1, None, lengths, k, v)
    idx, cnt = make_lists(g, lengths, hkv, 64, 4, 16)
    kh, vh = held(k), held(v)
    for lists in (True, False):
        out, lse = torch.full((2, hq, 128), math.nan, device="cuda"), torch.full((2, hq), math.nan, device="cuda")
        more = dict(idx=idx, cnt=cnt, idx_stride=idx.shape[-1], sinks=4, recent=16) if lists else {}
        assert tb.sparse_decode_attention_static(ctx.kv[0], tb.TB_FP4, hq, hkv, 128, 1000, None, lengths, q, out, lse=lse, **more) == tb.TB_OK
        assert tb.static_get_status() == 0
        for b, L in enumerate(lengths):
            seen = torch.ones(hkv, L, dtype=torch.bool, device="cuda")
            if lists:
                seen[:, 4:max(4, L - 16)] = False
                for h in range(hkv):
                    seen[h, idx[0, b, h, :cnt[0, b, h]].long()] = True
            at = slice(sum(lengths[:b]), sum(lengths[:b]) + L)
            o, s, bo, bs = reference(q[b].double(), kh[0, at].transpose(0, 1), vh[0, at].transpose(0, 1), seen, 128 ** -0.5)
            assert ((out[b].double() - o).abs() <= bo).all() and ((lse[b].double() - s).abs() <= bs).all()
    odd = torch.zeros(2 * hq * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, hq, 128)
    assert tb.sparse_decode_attention_static(ctx.kv[0], tb.TB_FP4, hq, hkv, 128, 1000, None, lengths, odd, out) == tb.TB_ERR_INVALID_ARG


# ---- refusals ----------------------------------------------------------------------------------------------------------

def test_refusals(tb):
    ctx = context(tb, 2, 8, 2, 3, room=64)
    k = torch.zeros(2, 30, 2, 128, dtype=torch.bfloat16, device="cuda")
    odd = torch.zeros(k.numel() + 4, dtype=torch.bfloat16, device="cuda")[4:].view(k.shape)     # 8 bytes off
    n0 = ctx.launch_count()

    def refused(status, call, *a, **more):
        with pytest.raises(tb.TBError) as e:
            call(*a, **more)
        assert e.value.status == status and ctx.launch_count() == n0

    refused(tb.TB_ERR_INVALID_ARG, ctx.append_kv, 0, 2, None, [10, 10, 10], odd, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.append_kv, 0, 2, None, [10, 10, 10], k, odd)
    refused(tb.TB_ERR_CAPACITY, ctx.append_kv, 0, 2, None, [65], k, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, None, [0], [1], k, k)                     # nothing cached yet
    ctx.append_kv(0, 2, None, [10, 10, 10], k, k)
    n0 = ctx.launch_count()
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, None, [0, 0, 0], [10, 11, 10], k, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, None, [5], [4], k, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, None, [-1], [4], k, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 1, 2, None, [0], [4], k, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, [3], [0], [4], k, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, [1, 1], [0, 0], [4, 4], k, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, None, [0], [4], odd, k)
    refused(tb.TB_ERR_INVALID_ARG, ctx.read_kv, 0, 2, None, [0], [4], k, None)
    q, out = torch.zeros(2, 3, 8, 128 + 0, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 3, 8, 128, device="cuda")
    off = torch.zeros(q.numel() + 4, dtype=torch.bfloat16, device="cuda")[4:].view(q.shape)
    refused(tb.TB_ERR_INVALID_ARG, ctx.sparse_decode_attention, 0, 2, None, 3, off, tb.select_params(-1), out)
    refused(tb.TB_ERR_STATE, ctx.sparse_decode_attention, 0, 2, None, 3, q, tb.select_params(8), out)
    for bad in ([0], [0, 0], [0, 0, 0, 0]):
        with pytest.raises(ValueError):
            ctx.read_kv(0, 2, None, bad, [4, 4, 4], k, k)
    for bad in (k.transpose(0, 1), k.cpu(), k[:, ::2]):
        with pytest.raises(ValueError):
            ctx.read_kv(0, 2, None, [0] * 3, [10] * 3, bad, k)
    assert ctx.get_status() == 0
