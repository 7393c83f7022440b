"""The end of the order in a sampled fill: u of 1 and more, and what is not a number, take the last kept entry, whichever filter ends the order
or none; u just below 1 takes what the definition in 64 bits says."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import inputs
from tests.test_gpu_sample import _call, _logits

pytestmark = pytest.mark.gpu
BEYOND = [1.0, 2.0, float("inf"), float("nan")]


def kept(z, temperature, top_k, top_p, min_p):
    """(indices in order, weights) of the entries that the filters keep, of one row (float32 numpy, finite)."""
    z = np.asarray(z, np.float64)
    if temperature == 0:  # the arg-max among all, no filter
        temperature, top_k, top_p, min_p = 1.0, 0, 1.0, 0.0
    order = np.lexsort((np.arange(len(z)), -z))
    far = (z[order] - z[order[0]]) / float(np.float32(temperature))
    assert not ((far < -31.9) & (far > -32.1)).any(), "an entry at the end of what has a weight"
    order, w = order[far > -32], np.exp(far[far > -32])
    if top_k:
        order, w = order[:top_k], w[:top_k]
    n = len(w)
    if top_p < 1:
        n = 1 + int(np.searchsorted(np.cumsum(w), float(np.float32(top_p)) * w.sum(), side="left"))
    n = min(n, int((w >= float(np.float32(min_p))).sum()))
    return order[:n], w[:n]


def check(z, dtype, u, what, **f):
    f = {**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **f}
    z = z.to(inputs.TORCH_DTYPE[dtype]).float()
    tok, conf = _call(z, dtype, u, **f)
    wrong = []
    for m in range(len(z)):
        order, w = kept(z[m].numpy(), **f)
        x = float(u[m])
        at = int(np.searchsorted(np.cumsum(w), x * w.sum(), side="right")) if x < 1 else len(w) - 1
        # the confidence: one rounding to fp32; weights to 2^-32 of themselves, and of every entry less than 2^-44 lost
        if tok[m] != order[at] or not abs(float(conf[m]) - w[at] / w.sum()) <= 2.0 ** -24 * w[at] / w.sum() + len(z[m]) * 2.0 ** -44:
            wrong.append((m, x, int(tok[m]), float(conf[m]), int(order[at]), w[at] / w.sum()))
    assert not wrong, "%s: %d of %d rows, first (row, u, token, confidence, token, confidence by definition) %s" % (what, len(wrong), len(z), wrong[0])


FILTERS = [dict(), dict(temperature=0.7), dict(min_p=0.01), dict(min_p=0.3), dict(min_p=1.0), dict(top_p=0.9), dict(top_p=0.9999), dict(top_k=1), dict(top_k=40),
           dict(top_p=0.99, min_p=0.02), dict(top_k=100, top_p=0.95, temperature=0.7), dict(top_k=60, min_p=0.05), dict(temperature=0.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(4, 1), (8, 3), (120, 300), (60, 4097), (60, 32000), (16, 152064)])
def test_the_last_kept_entry(dtype, M, V):
    for i, f in enumerate(FILTERS):
        print("[case]", dtype, M, V, f, flush=True)
        z, u = _logits(4000 + 20 * V + i, M, V, 1.5, peaks=4.0)
        u[:] = torch.tensor(BEYOND)[torch.arange(M) % 4]
        check(z, dtype, u if f.get("temperature") != 0.0 else torch.zeros(M), str(f), **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(120, 300), (60, 32000)])
def test_just_below_one_and_a_share_of_all(dtype, M, V):
    """u the largest number below 1, top-p likewise: the last entries of the order whatever the sums over the bins round to."""
    below = float(np.nextafter(np.float32(1), np.float32(0)))
    for i, f in enumerate([dict(), dict(top_p=below), dict(top_p=below, min_p=0.001), dict(min_p=0.01), dict(top_k=V // 2, top_p=below)]):
        print("[case]", dtype, M, V, f, flush=True)
        z, u = _logits(5000 + 20 * V + i, M, V, 1.5, peaks=4.0)
        u[:] = below
        check(z, dtype, u, str(f), **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ends_among_few_far_entries(dtype):
    """Entries far apart, most bins empty: the filters' ends, and the last entry with a weight, are bins apart from one another."""
    g = torch.Generator().manual_seed(6)
    z = -28 * torch.rand((200, 9), generator=g)
    u = torch.tensor(BEYOND).repeat(50)
    for f in (dict(), dict(top_k=4), dict(min_p=1e-6), dict(min_p=0.05), dict(top_p=0.999), dict(top_k=7, min_p=1e-4), dict(top_p=0.99, min_p=1e-9)):
        check(z, dtype, u, str(f), **f)
    # a weight that no sum in 64 bits shows is kept all the same: twelve equal ones, and one 31 temperatures below
    z = torch.zeros((4, 13))
    z[:, 5] = -31.0
    tok, conf = _call(z, dtype, torch.tensor(BEYOND))
    assert tok.tolist() == [5] * 4 and (conf > 0).all() and np.allclose(conf, np.exp(-31.0) / 12, rtol=2.0 ** -23, atol=0)
