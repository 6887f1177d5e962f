"""Calls on whole sequences whose lengths, or whose lists, only the device knows: replayed appends and forks, and lists that keep nothing."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_fp4 import tb  # noqa: E402,F401
from test_gpu_sequences import TYPES, grow, lengths, make, raw  # noqa: E402


def captured(step):
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    return graph


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("imp,scope", [(32, 0), (16, 2)])
def test_compaction_does_not_take_replayed_tokens_for_projected_ones(tb, name, imp, scope):
    """The host believes every token projected, replays have appended some that are not.  Kept among them, the projected length could not say which
    of the kept tokens are: the sequence is left as it is and reported.  Without kept tokens, or with all of them behind the projected
    ones, there is nothing to tell apart."""
    ctx = make(tb, name, hq=8, imp=imp, list_scope=scope)
    for s in (0, 1, 2):
        grow(ctx, s, 100)
    ctx.use_device_lengths(True, growth_reserve=16)
    k, v = (torch.randn(2, 30, 2, 128, generator=ctx.g, device="cuda").to(ctx.dt) for _ in range(2))
    graph = captured(lambda: ctx.append_kv(0, 2, [0, 1, 2], [10] * 3, k, v))                # the host counts them, the device has not run it
    ctx.project_keys(0, 2, [0, 1, 2], None, None, n_seq=3)                # nothing to project yet
    graph.replay()
    torch.cuda.synchronize()
    assert lengths(ctx, 0) == lengths(ctx, 1) == lengths(ctx, 2) == (110, 110)
    kv, kimp = raw(ctx.kv).clone(), raw(ctx.kimp).clone()
    idx = torch.tensor([[105, 106, 107, 108, 109]] * 2, dtype=torch.int32, device="cuda")
    ctx.compact_sequences([0], [90], [5], idx[:1])
    assert ctx.get_status() == tb.TB_ERR_UNPROJECTED and ctx.get_status() == 0
    assert torch.equal(raw(ctx.kv), kv) and torch.equal(raw(ctx.kimp), kimp)
    ctx.compact_sequences([1, 2], [100, 104], [5, 0], idx)
    assert ctx.get_status() == 0
    ctx.sync_lengths()
    assert lengths(ctx, 0) == (110, 100) and lengths(ctx, 1) == (105, 100) and lengths(ctx, 2) == (104, 100)
    # what is projected now is what a sequence of those tokens projects to
    ctx.project_keys(0, 2, [0, 1, 2], None, None, n_seq=3)
    ctx.sync_lengths()
    for s, m in ((0, 110), (1, 105), (2, 104)):
        assert lengths(ctx, s) == (m, m)
        kimp = ctx.kimp[:, s, :, :m].clone()
        ctx.kimp[:, s] = 0
        ctx.project_keys(0, 2, [s], [0], [m])
        assert torch.equal(ctx.kimp[:, s, :, :m], kimp)
    assert ctx.get_status() == 0


@pytest.mark.parametrize("name", TYPES)
def test_lists_and_ranges_with_nothing_in_them(tb, name):
    """A round that keeps no draft, and a read of no tokens, as a program that sizes its tensors by their counts calls them."""
    ctx = make(tb, name, batch=3)
    grow(ctx, 0, 40)
    grow(ctx, 2, 30)
    kv, n0 = raw(ctx.kv).clone(), ctx.launch_count()
    none = torch.empty(2, 0, dtype=torch.int32, device="cuda")
    ctx.compact_sequences([2, 0], [25, 40], [0, 0], none)
    assert lengths(ctx, 2) == (25, 25) and lengths(ctx, 0) == (40, 40)
    out = torch.empty(2, 0, 2, 128, dtype=ctx.dt, device="cuda")
    ctx.read_kv(0, 2, [0, 2], [7, 25], [7, 25], out, out)
    assert ctx.launch_count() == n0 and torch.equal(raw(ctx.kv), kv) and ctx.get_status() == 0
    for call, a in ((ctx.compact_sequences, ([0], [10], [1], none)), (ctx.compact_sequences, ([2, 0], [0, 0], [0, 1], none)),
                    (ctx.read_kv, (0, 2, [0], [7], [8], out, out)), (ctx.read_kv, (0, 2, [0], [41], [41], out, out)), (ctx.read_kv, (0, 2, [0], [8], [7], out, out))):
        with pytest.raises(tb.TBError) as e:
            call(*a)
        assert e.value.status == tb.TB_ERR_INVALID_ARG and ctx.launch_count() == n0
    ctx.use_device_lengths(True, 0)
    ctx.compact_sequences([0], [33], [0], none[:1])
    ctx.sync_lengths()
    assert lengths(ctx, 0) == (33, 33) and ctx.get_status() == 0


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("devlen", [False, True])
def test_a_fork_captured_before_the_first_selection_brings_the_rows_of_later_ones(tb, name, devlen):
    """Beams: the copy is captured once, then source and copy are selected, and the copy replaced by the source's state.  With an Important
    buffer its rows are those of the lists that came with it."""
    ctx = make(tb, name, hq=8, batch=2, room=300, budget=24)
    ctx.bind_important_buffer()
    grow(ctx, 0, 200)
    grow(ctx, 1, 200)
    if devlen:
        ctx.use_device_lengths(True, growth_reserve=0)
    graph = captured(lambda: ctx.fork_sequence(0, [1]))
    qi = torch.randn(2, 2, 8, 32, generator=ctx.g, device="cuda")
    q = torch.randn(2, 1, 8, 128, generator=ctx.g, device="cuda").to(ctx.dt).expand(-1, 2, -1, -1).contiguous()
    p = tb.select_params(24, 4, 16)
    ctx.select_topk(0, 2, None, 2, qi, p)
    graph.replay()
    out = torch.full((2, 2, 8, 128), math.nan, device="cuda")
    ctx.sparse_decode_attention(0, 2, None, 2, q, p, out)
    assert torch.isfinite(out).all() and torch.equal(out[:, 0], out[:, 1])
    assert ctx.get_status() == 0


def test_positions_come_as_a_matrix(tb):
    """Two sequences' lists in any other shape: refused, not read from the wrong places."""
    ctx = make(tb, "fp4", batch=2)
    grow(ctx, 0, 40)
    grow(ctx, 1, 40)
    idx, n0 = torch.arange(32, dtype=torch.int32, device="cuda").view(2, 16), ctx.launch_count()
    for bad in (idx.view(2, 4, 4), idx.view(2, 16, 1), idx.view(1, 2, 16)):
        with pytest.raises(ValueError, match="keep_idx"):
            ctx.compact_sequences([0, 1], [0, 0], [3, 3], bad)
    with pytest.raises((ValueError, IndexError)):
        ctx.compact_sequences([0], [0], [3], idx.view(-1))
    assert ctx.launch_count() == n0 and lengths(ctx, 0) == lengths(ctx, 1) == (40, 40)
    ctx.compact_sequences([0, 1], [0, 0], [3, 3], idx)
    assert lengths(ctx, 1) == (3, 3) and ctx.get_status() == 0
