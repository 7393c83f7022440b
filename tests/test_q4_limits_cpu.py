"""The 4-bit cache's attention and the sampled fill at the borders of what they take, on the host: refusals before any HIP call."""
import pytest

from paper_2505_21467_amd import binding as fc
from tests.test_q4_cpu import FAKE, _cfg, _raises


def test_row_tiles_whose_threads_do_not_fit_a_grid():
    """2^23 workgroups of 512 threads are 2^32: one more than a grid holds, by one sequence and by many."""
    A = fc.fc_q4_attention
    for cfg, rows in ((_cfg(batch=1, n_q_heads=1, n_kv_heads=1), 1 << 24), (_cfg(batch=1, n_q_heads=8, n_kv_heads=1), 1 << 21),
                      (_cfg(batch=1, n_q_heads=9, n_kv_heads=9), 1 << 23)):
        h = fc.fc_q4_alloc(cfg, FAKE)
        _raises(fc.FC_ERR_UNSUPPORTED, A, h, 0, FAKE, rows, 100, None, None, FAKE, FAKE, 1 << 30, 0)
        fc.fc_q4_free(h)


def test_workspace_of_logits_beyond_what_a_call_takes():
    """0 wherever the call refuses the shape."""
    W = fc.fc_sample_workspace_bytes
    assert W("bf16", 65535, 1 << 21) == 0 and W("f32", 4097, 1 << 24) == 0
    assert W("bf16", 4096, 1 << 24) > 0 and W("f32", 32768, 1 << 21) > 0        # 2^36 itself


def test_softmax_scales_whose_inverse_no_float_holds():
    """The scores start from the value rows' powers over the scale: from 2^-100 to 2^100, and the default."""
    for scale in (1e-38, 1e-44, 2.0 ** -101, 2.0 ** 101, 3e38):
        _raises(fc.FC_ERR_UNSUPPORTED, fc.fc_q4_alloc, _cfg(softmax_scale=scale), FAKE)
        assert fc.fc_q4_storage_bytes(_cfg(softmax_scale=scale)) == 0 and fc.fc_q4_workspace_bytes(_cfg(softmax_scale=scale), 4) == 0
    for scale in (0.0, 2.0 ** -100, 2.0 ** 100, 0.125):
        fc.fc_q4_free(fc.fc_q4_alloc(_cfg(softmax_scale=scale), FAKE))
