"""Attention over the 4-bit cache where a few query channels are far larger than the others, as biased projections make them: what the other channels
hold must not be lost.  Against 64 bits, and bit for bit where the large channels meet keys of zero."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import inputs
from tests import q4_reference as ref
from tests.test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu
CHANNELS = {128: (3, 40, 77, 120), 64: (3, 40)}  # one in every block of 32


def bound(q, k, v, n, scale, dtype):
    """(out, largest error) [A][Dh] of one head: q [A][Dh], k, v [n][Dh] as held, in 64 bits.

    A product of a query element (one or three numbers of 8 bits) and a key is exact.  Sums: every addition of fp32 loses 2^-23 of the sum of
    magnitudes at most, Dh times the numbers of an element, and the power of the value row (40 at most) goes in as well; the scale is
    rounded twice, the exponential is off by 2^-22, in numerator and in sum each.  Sums over the keys: n + 16 of 2^-23.  Weights: fp16, 2^-11
    of themselves (fp32: two numbers, 2^-21), and 2^-25 of the largest weight times power of a value row where they are subnormal
    (fp32: 2^-36), times codes of 6 at most.  The output: half a step of the type."""
    s = q @ k.T * scale
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    out, spread = p @ v, p @ np.abs(v)
    size = (np.abs(q) @ np.abs(k).T * scale).max(-1, keepdims=True)
    power = np.exp2(np.maximum(np.ceil(np.log2(np.maximum(np.abs(v).max(-1), 1e-30) / 6)), ref.V_LOWEST))
    u, parts = 2.0 ** -23, 3 if dtype == "f32" else 1
    rel = 2 * ((parts * q.shape[-1] + 6) * u * size + 44 * u + 2 * u) + (n + 16) * u
    least = n * 6 * (p * power).max(-1, keepdims=True)
    if dtype == "f32":
        return out, (rel + 2.0 ** -21) * spread + 2.0 ** -36 * least + 2.0 ** -24 * np.abs(out)
    return out, (rel + 2.0 ** -11) * spread + 2.0 ** -25 * least + 2.0 ** -8 * np.abs(out)


def check(c, q, hk, hv, n, what):
    B, Hq, Hkv, Dh, _ = c.shape
    got = c.attend(q, n)
    for b in range(B):
        for h in range(Hq):
            out, most = bound(ref.f64(q[b, h]), hk[b, h // (Hq // Hkv), :n], hv[b, h // (Hq // Hkv), :n], n, c.scale, c.dtype)
            over = np.abs(got[b, :, h] - out) / most
            assert (over <= 1).all(), "%s: %.2f times the bound" % (what, over.max())
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [128, 64])
@pytest.mark.parametrize("n", [5, 63, 64, 65, 200, 700])
@pytest.mark.parametrize("factor", [16.0, 256.0, 4096.0, 2.0 ** 20])
def test_large_channels_against_64_bits(dtype, Dh, n, factor):
    """Keys are smaller in those channels by the same factor, or the same in all of them (which moves all scores alike)."""
    B, Hq, Hkv, A = 2, 6, 2, 11
    for same in (False, True):
        if same and factor > 256:
            continue  # (scores whose size alone decides the bound)
        c = Cache(dtype, B, Hq, Hkv, Dh, n)
        k, v = c.rows(70, n)
        q = inputs.normal(71, "q", (B, Hq, A, Dh), 1.5, dtype).clone()
        k = k.clone()
        for ch in CHANNELS[Dh]:
            q[..., ch] = (q[..., ch].float() * factor).to(q.dtype)
            k[..., ch] = torch.full_like(k[..., ch], 0.5) if same else (k[..., ch].float() / factor).to(k.dtype)
        c.store(k, v)
        hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
        check(c, q, hk, hv, n, "%s Dh %d, %d keys, factor %g%s" % (dtype, Dh, n, factor, ", keys the same there" if same else ""))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [128, 64])
@pytest.mark.parametrize("A,n", [(1, 130), (37, 1100)])
def test_channels_that_meet_zeros_change_no_bit(dtype, Dh, A, n):
    c = Cache(dtype, 1, 4, 2, Dh, n)
    k, v = c.rows(72, n)
    k = k.clone()
    for ch in CHANNELS[Dh]:
        k[..., ch] = 0
    c.store(k, v)
    q = inputs.normal(73, "q", (1, 4, A, Dh), 1.5, dtype).clone()
    for ch in CHANNELS[Dh]:
        q[..., ch] = 0
    want = c.attend(q, n)
    for factor in (1.0, 64.0, -1024.0, 1e5, 1e30):
        for ch in CHANNELS[Dh]:
            q[..., ch] = factor
        assert np.array_equal(c.attend(q, n), want), "queries of %g against keys of zero" % factor


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_queries_keep_their_bits(dtype):
    """A row times a power of two against keys over that power: the same scores, the same bits."""
    Dh, n, A = 128, 200, 5
    q = inputs.normal(74, "q", (1, 2, A, Dh), 1.5, dtype)
    k, v = inputs.normal(75, "k", (1, 1, n, Dh), 1.0, dtype), inputs.normal(76, "v", (1, 1, n, Dh), 1.0, dtype)
    want = None
    for e in (0, 30, -30, 70, -70):
        c = Cache(dtype, 1, 2, 1, Dh, n)
        c.store((k.float() * 2.0 ** -e).to(k.dtype), v)
        got = c.attend((q.float() * 2.0 ** e).to(q.dtype), n)
        want = got if want is None else want
        assert np.array_equal(got, want), "queries times 2^%d" % e
