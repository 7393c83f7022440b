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
