"""Attention over the 4-bit cache at the ends of the softmax scales that it takes."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import inputs
from tests import q4_reference as ref
from tests.test_gpu_q4 import Cache
from tests.test_gpu_q4_outliers import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("e", [-100, -60, -20, 20, 60, 100])
def test_scales_that_rows_make_up_for(dtype, Dh, e):
    """A scale of 2^e with queries over it: the scores of any other scale; rows of values 2^40 apart and rows never stored among them."""
    n = 150
    c = Cache(dtype, 1, 2, 1, Dh, n, scale=2.0 ** e)
    k, v = c.rows(80, n - 9)
    size = torch.exp2(torch.randint(-20, 21, (n - 9,), generator=torch.Generator().manual_seed(4)).float())[None, None, :, None]
    v = (v.float() * size).to(v.dtype)
    c.store(k, v)
    hk, hv = np.zeros((1, 1, n, Dh)), np.zeros((1, 1, n, Dh))
    hk[:, :, :n - 9], hv[:, :, :n - 9] = ref.held_rows(ref.f64(k), ref.f64(v))
    q = inputs.normal(81, "q", (1, 2, 7, Dh), 0.2, dtype)
    check(c, (q.float() * 2.0 ** -e).to(q.dtype), hk, hv, n, "scale 2^%d" % e)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("e", [-100, -40])
def test_scales_that_make_all_keys_alike(dtype, e):
    """Ordinary queries at a scale next to nothing: the mean of the values."""
    n = 200
    c = Cache(dtype, 1, 2, 1, 64, n, scale=2.0 ** e)
    k, v = c.rows(82, n)
    c.store(k, v)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    check(c, inputs.normal(83, "q", (1, 2, 3, 64), 1.0, dtype), hk, hv, n, "scale 2^%d" % e)
