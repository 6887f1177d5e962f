"""What the entry points of the 4-bit cache and of whole sequences answer without a GPU."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2503_07518_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def test_sizes_of_a_4_bit_cache(b):
    L, sizes = b.lib(), [ctypes.c_size_t() for _ in range(4)]
    ask = lambda kv_dtype: L.tb_query_sizes(ctypes.byref(b.tb_config(3, 8, 4, 128, 32, kv_dtype, 2, 1000, 64, 1, 0, 0)),  # noqa: E731
                                            *[ctypes.byref(s) for s in sizes])
    assert ask(b.TB_BF16) == b.TB_OK
    bf16 = [s.value for s in sizes]
    assert ask(b.TB_FP4) == b.TB_OK
    fp4 = [s.value for s in sizes]
    assert fp4[0] == 3 * 2 * 4 * 1000 * 144 and bf16[0] == 3 * 2 * 4 * 1000 * 512
    assert fp4[1:] == bf16[1:]                                            # projected keys, state and workspace are those of bf16
    assert ask(3) == b.TB_ERR_INVALID_ARG and ask(-1) == b.TB_ERR_INVALID_ARG
    cfg = b.tb_config(3, 8, 4, 128, 32, b.TB_FP4, 2, 1000, 64, 1, 0, 0)
    assert L.tb_resident_rows_bytes(ctypes.byref(cfg), 4, 12) == 3 * 2 * 4 * 16 * 144
    assert L.tb_important_buffer_bytes(ctypes.byref(cfg)) == 3 * 2 * 4 * 192 * 144


def test_null_arguments_are_refused_before_anything_else(b):
    L, one, ints = b.lib(), ctypes.c_void_p(16), (ctypes.c_int32 * 1)(0)
    assert L.tb_read_kv(None, 0, 1, None, ints, ints, 1, one, one, None) == b.TB_ERR_INVALID_ARG
    assert L.tb_fork_sequence(None, 0, ints, 1, -1, None) == b.TB_ERR_INVALID_ARG
    assert L.tb_compact_sequences(None, None, 1, ints, None, None, 0, None) == b.TB_ERR_INVALID_ARG


def test_the_predictor_has_no_4_bit_weights(b):
    p = b.tb_predictor(dtype=b.TB_FP4, model_dim=4096, hidden_dim=512, n_q_heads=32, n_slots=4, imp_dim=32, activation=b.TB_ACT_GELU,
                       ln_eps=1e-5, ln_weight=16, ln_bias=16, w1=16, w2=16)
    one = ctypes.c_void_p(16)
    assert b.lib().tb_predict_importance_queries(ctypes.byref(p), one, 1, one, one, None) == b.TB_ERR_INVALID_ARG


def test_the_extension_module_checks_the_lengths_of_its_lists(b):
    s = type("Stream", (), {"cuda_stream": 0})()
    assert b._calls.read_kv(None, 0, 1, None, [0], [1], None, None, s) == b.TB_ERR_INVALID_ARG
    assert b._calls.fork_sequence(None, 0, (1, 2), -1, s) == b.TB_ERR_INVALID_ARG
    assert b._calls.compact_sequences(None, [0], [0], None, None, s) == b.TB_ERR_INVALID_ARG
    for bad in (lambda: b._calls.read_kv(None, 0, 1, [0, 1], [0], [1], None, None, s), lambda: b._calls.read_kv(None, 0, 1, None, [0], [1, 2], None, None, s),
                lambda: b._calls.compact_sequences(None, [0, 1], [0], None, None, s), lambda: b._calls.compact_sequences(None, None, [0], [1, 1], None, s)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        b._calls.fork_sequence(None, 0, None)


def test_tensors_that_a_kernel_could_not_read_are_refused(b):
    """On the host, of another type, or not one run of bytes (the type and the strides are asked for on the device too)."""
    import torch
    s = type("Stream", (), {"cuda_stream": 0})()
    for idx in (torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int64)):
        with pytest.raises(ValueError, match="keep_idx"):
            b._calls.compact_sequences(None, None, [0], [1], idx, s)
    for k, v in ((torch.zeros(4), None), (None, torch.zeros(4))):
        with pytest.raises(ValueError, match="_out"):
            b._calls.read_kv(None, 0, 1, None, [0], [1], k, v, s)


def test_types_that_a_4_bit_context_takes(b):
    import torch
    assert b.torch_dtype(b.TB_FP4) == b.torch_dtype(b.TB_BF16) == torch.bfloat16 and b.torch_dtype(b.TB_F32) == torch.float32
