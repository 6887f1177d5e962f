"""tb_read_kv through the extension module: an output that is too short, or of another type than the rows', is refused before anything runs."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_fp4 import tb  # noqa: E402,F401
from test_gpu_sequences import TYPES, grow, make  # noqa: E402


@pytest.mark.parametrize("name", TYPES)
def test_outputs_without_room_or_of_another_type(tb, name):
    ctx = make(tb, name, layers=3, hq=4, hkv=2, batch=3)
    k, v = grow(ctx, 0, 40)
    grow(ctx, 2, 30)
    n0 = ctx.launch_count()
    spans = ([0, 2], [5, 0], [40, 30])                                    # 65 tokens of 2 heads and 3 layers
    full = torch.full((3, 65, 2, 128), 9.0, dtype=ctx.dt, device="cuda")
    for short in (full[:, :64].contiguous(), full[:2], full.view(-1)[:-1], full[:0]):
        for pair in ((short, full), (full, short)):
            with pytest.raises(tb.TBError) as e:
                ctx.read_kv(0, 3, *spans, *pair)
            assert e.value.status == tb.TB_ERR_INVALID_ARG
    for other in {torch.float32, torch.bfloat16, torch.float16, torch.uint8, torch.int32} - {ctx.dt}:
        wrong = torch.zeros(4 * full.numel(), dtype=other, device="cuda")  # (long enough for every type's bytes)
        for pair in ((wrong, full), (full, wrong)):
            with pytest.raises(ValueError, match="_out"):
                ctx.read_kv(0, 3, *spans, *pair)
    with pytest.raises(ValueError, match="keep_idx"):
        ctx.compact_sequences([0], [0], [1], torch.zeros(1, 4, device="cuda"))
    assert ctx.launch_count() == n0 and (full == 9.0).all()
    # exactly enough, and more than enough, are served; one layer needs a third
    more = torch.full((3 * 65 * 2 * 128 + 256,), 9.0, dtype=ctx.dt, device="cuda")
    ctx.read_kv(0, 3, *spans, full, more)
    assert (more[-256:] == 9.0).all() and (more[:-256] != 9.0).all()
    ko, vo = torch.empty(1, 40, 2, 128, dtype=ctx.dt, device="cuda"), torch.empty(1, 40, 2, 128, dtype=ctx.dt, device="cuda")
    ctx.read_kv(1, 1, [0], [0], [40], ko, vo)
    assert torch.equal(ko[0, 5:], full[1, :35]) and torch.equal(vo[0, 5:], more[:-256].view(3, 65, 2, 128)[1, :35])
    if name != "fp4":
        assert torch.equal(ko[0], k[1]) and torch.equal(vo[0], v[1])
    assert ctx.get_status() == 0
