"""The sampled fill of logits far from zero in units of the temperature: bins lie on an absolute grid, whose places are rounded."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import inputs
from tests.test_gpu_sample import _call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,step,temperature", [(1e3, 2.0 ** -14, 1e-3), (-1e5, 2.0 ** -7, 2e-3), (131072.0, 2.0 ** -6, 0.0011), (-3e6, 0.25, 0.01), (6e7, 4.0, 0.7),
                                                     (-2.0 ** 40, 2.0 ** 17, 2.0 ** 15 * 1.1), (1e30, 0.0, 1e-3)])
@pytest.mark.parametrize("f", [dict(), dict(top_k=30), dict(top_p=0.97), dict(min_p=0.003)])
def test_logits_far_from_zero(dtype, offset, step, temperature, f):
    M, V = 24, 400
    g = torch.Generator().manual_seed(int(abs(offset)) % 1000)
    z = (offset + step * torch.randint(0, 40, (M, V), generator=g).double()).float().to(inputs.TORCH_DTYPE[dtype]).float()
    u = torch.rand(M, generator=g)
    tok, conf = _call(z, dtype, u, temperature=temperature, **f)
    T, x = float(np.float32(temperature)), z.double().numpy()
    far = np.abs(x).max() / T
    # a weight: 2^-32 of itself and |z| / T 2^-53 for its place in the grid (beyond 2^30 only equal logits are within 32 temperatures of one another, and
    # they have one place); the confidence has it in numerator and sum, and is rounded once
    rel = 2 * (2.0 ** -32 + (far * 2.0 ** -53 if far < 2.0 ** 30 else 0)) + 2.0 ** -24
    for m in range(M):
        order = np.lexsort((np.arange(V), -x[m]))
        w = np.exp((x[m][order] - x[m].max()) / T)
        w[w < np.exp(-31.9)] = 0
        n = f.get("top_k", V)
        if "top_p" in f:
            n = 1 + int(np.searchsorted(np.cumsum(w), float(np.float32(f["top_p"])) * w.sum(), side="left"))
        if "min_p" in f:
            n = int((w >= float(np.float32(f["min_p"]))).sum())
        w = w[:n]
        run = np.cumsum(w) / w.sum()
        # (the token at u, or one whose border u meets within what sums of such weights are off by)
        lo, hi = (int(np.searchsorted(run, min(max(float(u[m]) + s * (2 * rel), 0.0), 1 - 1e-12), side="right")) for s in (-1, 1))
        at = [i for i in range(lo, min(hi, n - 1) + 1) if order[i] == tok[m]]
        assert at, (m, int(tok[m]), order[lo], order[min(hi, n - 1)])
        c = w[at[0]] / w.sum()
        assert abs(float(conf[m]) - c) <= rel * c + V * 2.0 ** -44, (m, float(conf[m]), c)
