"""The steady state of the 4-bit kernels: launches whose warps take dozens of tiles each, so that rings of stages wrap, sums are moved out of the
accumulators and rescaled there, and blocks pass over their tokens more than once.  The values that the cache holds are read back
from it (test_gpu_fp4.py compares reads with the definition, byte by byte)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_fp4 import check_attention, check_projected, context, generator, rows, tb  # noqa: E402,F401


def fill(ctx, g, lengths, make_k, make_v):
    """Appends sequence by sequence and returns the held values as float64 [1, sum of lengths, heads, 128]."""
    heads = ctx.cfg.n_kv_heads
    ks, vs = [], []
    for b, L in enumerate(lengths):
        k, v = make_k(L).bfloat16(), make_v(L).bfloat16()
        ctx.append_kv(0, 1, [b], [L], k[None], v[None])
        ko, vo = torch.empty_like(k[None]), torch.empty_like(v[None])
        ctx.read_kv(0, 1, [b], [0], [L], ko, vo)
        ks.append(ko), vs.append(vo)
    return torch.cat(ks, 1).double(), torch.cat(vs, 1).double()


def rising(g, heads, period):
    """Keys whose scores (for queries that are large in the first 16 channels) climb by 2^30 over `period` tokens, again and again."""
    def make(L):
        k = torch.randn(L, heads, 128, generator=g, device="cuda")
        k[:, :, :16] *= 0.25
        k[:, :, :16] += 3.75 * ((torch.arange(L, device="cuda") % period) / period)[:, None, None]
        return k
    return make


def drifting(g, heads):
    """Values around one that differ from stretch to stretch: what is lost or counted twice shows."""
    return lambda L: torch.rand(L, heads, 128, generator=g, device="cuda") + 0.5 + (torch.arange(L, device="cuda") / L)[:, None, None]


def queries(g, batch, hq):
    q = torch.randn(1, batch, hq, 128, generator=g, device="cuda")
    q[..., :16] = 4.0
    return q.bfloat16()


# (problems per launch and their length; a warp's tiles on 148 SMs: 29, 57, 41, 40)
@pytest.mark.parametrize("batch,hkv,group,length,period", [(8, 2, 4, 131072, 1500), (4, 8, 8, 131072, 2100), (40, 8, 4, 9000, 1500), (37, 8, 7, 8900, 700), (8, 2, 1, 131072, 131072)])
def test_dense_attention_with_many_tiles_per_warp(tb, batch, hkv, group, length, period):
    g = generator(50)
    hq = hkv * group
    lengths = [length - 37 * b for b in range(batch)]
    ctx = context(tb, 1, hq, hkv, batch, room=length)
    k, v = fill(ctx, g, lengths, rising(g, hkv, period), drifting(g, hkv))
    check_attention(tb, ctx, k, v, lengths, tb.select_params(-1), queries(g, batch, hq))


@pytest.mark.parametrize("group", [4, 8])
def test_long_lists_with_many_tiles_per_warp(tb, group):
    """The same by lists, with entries that are skipped far behind the first tiles."""
    g = generator(51)
    batch, hkv, L, n = 40, 8, 12000, 9000
    ctx = context(tb, 1, hkv * group, hkv, batch, room=L, budget=n)
    lengths = [L - 11 * b for b in range(batch)]
    k, v = fill(ctx, g, lengths, rising(g, hkv, 2000), drifting(g, hkv))
    idx = torch.zeros(1, batch, hkv, n, dtype=torch.int32, device="cuda")
    for b, length in enumerate(lengths):
        idx[0, b] = 4 + torch.argsort(torch.rand(hkv, length - 20, generator=g, device="cuda"), dim=1)[:, :n].sort(dim=1).values
    idx[0, 1, 3, 7777], idx[0, 39, 7, 8998], idx[0, 20, 0, 600] = L, -1, 2 ** 31 - 1
    cnt = torch.full((1, batch, hkv), n, dtype=torch.int32, device="cuda")
    check_attention(tb, ctx, k, v, lengths, tb.select_params(n, 4, 16), queries(g, batch, hkv * group), idx, cnt, status=tb.TB_ERR_BAD_INDEX)


@pytest.mark.parametrize("imp", [16, 32])
@pytest.mark.parametrize("kind", ["even", "wide"])
def test_projection_with_many_tiles_per_warp(tb, imp, kind):
    """Ten tiles per warp through a ring of six stages, on f16 matrices and on ones whose elements f16 does not hold; ragged ends, and a
    second range that starts inside a tile."""
    g = generator(52)
    lengths = [32768 - 5, 32768 - 1000]
    ctx = context(tb, 1, 4, 4, 2, room=32768, imp=imp)
    if kind == "wide":
        ctx.W *= torch.exp2(torch.randint(-40, 1, ctx.W.shape, generator=g, device="cuda").float()).bfloat16()
        ctx.set_projection(0, ctx.W[0])
    k, _ = fill(ctx, g, lengths, lambda L: rows(g, L, 4, spread=1.0), lambda L: rows(g, L, 4))
    ctx.kimp.fill_(7.0)
    first = [77, 30001]
    ctx.project_keys(0, 1, None, [0, 0], first)
    assert all((ctx.kimp[:, b, :, n:] == 7.0).all() for b, n in enumerate(first))
    ctx.project_keys(0, 1, None, first, lengths)
    assert all((ctx.kimp[:, b, :, n:] == 7.0).all() for b, n in enumerate(lengths))
    for b, n in enumerate(lengths):
        at = sum(lengths[:b])
        check_projected(ctx, k[0, at:at + n].transpose(0, 1), 0, n, 0, b)
    whole = ctx.kimp.clone()
    ctx.kimp.fill_(7.0)
    ctx.project_keys(0, 1, [1], [0], [lengths[1]])                        # in a launch of its own: other warps, the same bits
    assert torch.equal(ctx.kimp[:, 1], whole[:, 1])


@pytest.mark.parametrize("imp", [16, 32])
def test_layer_projection_in_several_passes(tb, imp):
    """One key stream per layer: a block that goes on to further tokens begins again with the first head's matrix."""
    g = generator(53)
    lengths = [32768 - 3 * b for b in range(8)]                           # 8 units: 111 blocks of 128 tokens, three passes
    ctx = context(tb, 1, 6, 3, 8, room=32768, imp=imp, list_scope=tb.TB_SCOPE_LAYER)
    ctx.kimp.fill_(7.0)
    k, _ = fill(ctx, g, lengths, lambda L: rows(g, L, 3, spread=1.0), lambda L: rows(g, L, 3))
    ctx.project_keys(0, 1, None, [0] * 8, lengths)
    for b, n in enumerate(lengths):
        at = sum(lengths[:b])
        check_projected(ctx, k[0, at:at + n].transpose(0, 1), 0, n, 0, b)
        assert (ctx.kimp[:, b, :, n:] == 7.0).all()
