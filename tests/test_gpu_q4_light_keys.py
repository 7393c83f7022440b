"""Attention over the 4-bit cache where a few keys take almost all of the weight and thousands of light ones share the rest: what they bring must show
where the heavy keys' values have nothing."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import inputs
from tests import q4_reference as ref
from tests.test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("below", [10.0, 18.5, 20.5])
@pytest.mark.parametrize("at", [0, 37, 63])
def test_light_keys_count(dtype, Dh, below, at):
    """16000 keys, one in every 64 of them `below` (in units of the exponent) above the others."""
    n, A = 16000, 3
    c = Cache(dtype, 1, 2, 1, Dh, n, scale=1.0)
    k, v = torch.zeros((1, 1, n, Dh)), torch.zeros((1, 1, n, Dh))
    k[:, :, at::64, 0] = 2.0
    v[..., 0::2], v[:, :, at::64, 0::2], v[:, :, at::64, 1::2] = 1.0, 0.0, 1.0  # even elements: the light keys'; odd ones: the heavy ones'
    c.store(k.to(inputs.TORCH_DTYPE[dtype]), v.to(inputs.TORCH_DTYPE[dtype]))
    q = torch.zeros((1, 2, A, Dh))
    q[..., 0] = below / 2
    got = c.attend(q.to(inputs.TORCH_DTYPE[dtype]), n)
    light, heavy = np.exp(-below), n // 64
    want = np.where(np.arange(Dh) % 2 == 0, (n - heavy) * light, heavy) / (heavy + (n - heavy) * light)
    # scores: one product, the scale to base 2 (2^-23 of the score); exponentials 2^-22; sums: 16000 additions of equal numbers, none of them
    # off by more than 2^-24 of the sum, or of half of it where a lane has a thousand: 1024 of 2^-24.  Weights to fp16: 2^-11 of themselves, or, where they
    # are subnormal, half a step of 2^-24, in units of which the largest weight is 2^7 or more: 2^-32 against e^-18.5 = 2^-26.7, e^-20.5 = 2^-29.6.  The output: half a step.
    u = 2.0 ** -24
    rel = 2 * (2 * u * below + 4 * u) + 1024 * u
    least = 2.0 ** -44 if dtype == "f32" else 2.0 ** -32
    rel += (2.0 ** -21 if dtype == "f32" else 2.0 ** -11) + least / light
    most = (rel + (2.0 ** -24 if dtype == "f32" else 2.0 ** -8)) * want
    assert (np.abs(got - want) <= most).all(), "largest error %.3g of the result" % (np.abs(got - want) / want).max()
