"""Attention over the 4-bit cache with finite scores of any size: beyond 2^24 a score's own rounding is larger than what weights differ by, so that one key, or
the keys that are the same, take everything."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import inputs
from tests import q4_reference as ref
from tests.test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("e", [16, 24, 26, 28, 30, 34, 60, 100])
@pytest.mark.parametrize("n", [3, 64, 130, 700])
def test_one_key_takes_everything(dtype, Dh, e, n):
    """Queries times 2^e.  Rows count where the best key stands apart by 2^-15 of its score (fp32 sums of 128 terms: 2^-16 at worst) and e^40 in weight; in the
    second kv head every key is there twice, with another value."""
    B, Hq, Hkv, A = 1, 4, 2, 9
    c = Cache(dtype, B, Hq, Hkv, Dh, n)
    k, v = c.rows(90, n)
    k = k.clone()
    if n > 3:
        k[:, 1, 1::2] = k[:, 1, 0:n - n % 2:2][:, :k[:, 1, 1::2].shape[1]]  # the second kv head: every key twice
    c.store(k, v)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    q = (inputs.normal(91, "q", (B, Hq, A, Dh), 1.0, dtype).float() * 2.0 ** e).to(inputs.TORCH_DTYPE[dtype])
    got = c.attend(q, n)
    assert np.isfinite(got).all(), "not finite"
    compared = 0
    for h in range(Hq):
        kk, vv = hk[0, h // 2], hv[0, h // 2]
        s = ref.f64(q)[0, h] @ kk.T
        for a in range(A):
            best = s[a] >= s[a].max() - 2.0 ** -40 * abs(s[a].max())
            gap = s[a].max() - (s[a][~best].max() if not best.all() else -np.inf)
            if gap < 2.0 ** -15 * abs(s[a].max()) or gap * Dh ** -0.5 < 40:
                continue
            # the value of the best key, or, of two that are the same, something between theirs; half a step of the output
            lo, hi = vv[best].min(0), vv[best].max(0)
            off = (2.0 ** -8 + 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * np.abs(vv[best]).max(0)
            compared += 1
            assert (got[0, a, h] >= lo - off).all() and (got[0, a, h] <= hi + off).all(), (h, a, got[0, a, h][:4], lo[:4], hi[:4])
    assert compared >= 20 or e < 24


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_numbers_change_no_others_bits(dtype, Dh, what):
    c = Cache(dtype, 1, 2, 1, Dh, 400)
    c.store(*c.rows(92, 400))
    q = inputs.normal(93, "q", (1, 2, 12, Dh), 1.5, dtype).clone()
    want = c.attend(q, 400)
    q[0, 1, 4, 9] = what
    got = c.attend(q, 400)
    other = np.ones((12, 2), bool)
    other[4, 1] = False
    assert np.array_equal(got[0][other], want[0][other]) and np.isnan(got[0, 4, 1]).all()
