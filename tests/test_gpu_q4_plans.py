"""Attention over the 4-bit cache under every launch plan: row tiles and waves of a workgroup, ranges of the keys from one to more than a merge takes
at once, by the tuning knob; the same bound whatever the plan, against plain definitions in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import binding as fc
from paper_2505_21467_amd import inputs
from tests import q4_reference as ref
from tests.test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("tiles,waves", [(1, 1), (1, 2), (1, 4), (1, 8), (2, 4), (2, 8)])
def test_every_plan(knob, dtype, Dh, tiles, waves):
    """37 rows of a kv head (a last row tile that is not full), 20 tiles of keys of which the last is not full; lengths of which some leave
    ranges, or all but a wave, without keys; rows that are padding."""
    B, Hq, Hkv, A, n = 3, 2, 2, 37, 1250
    c = Cache(dtype, B, Hq, Hkv, Dh, n + 40)
    k, v = c.rows(30, n + 40)
    c.store(k, v)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    q = inputs.normal(31, "q", (B, Hq, A, Dh), 1.5, dtype)
    lens = torch.tensor([n, 65, 0], dtype=torch.int32)
    pos = torch.arange(A, dtype=torch.int32).repeat(B, 1)
    pos[0, 5], pos[1, 36] = -1, -1
    for splits in (1, 2, 3, 9, 20):
        print("[case]", dtype, Dh, tiles, waves, splits, flush=True)
        knob("FC_Q4_TILES", "%d,%d,%d" % (tiles, waves, splits))
        space = 64 << 20
        c.check(q, hk, hv, n, what="%d ranges" % splits, space=space)
        a = c.check(q, hk, hv, n, lens, pos, what="%d ranges, lengths" % splits, space=space)
        assert not a[2].any() and not a[0, 5].any() and not a[1, 36].any()
        c.check(q, hk, hv, n, lens, pos, what="%d ranges, room for fewer" % splits, space=8 * 37 * 2 * 3 * (Dh + 2) * 4 + 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_ranges_than_a_merge_takes_at_once(knob, dtype):
    """64 ranges, of a long sequence and of one that fills eleven of them."""
    c = Cache(dtype, 2, 4, 1, 128, 5000)
    k, v = c.rows(32, 5000)
    c.store(k, v)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    q = inputs.normal(33, "q", (2, 4, 3, 128), 1.5, dtype)
    lens = torch.tensor([5000, 1300], dtype=torch.int32)
    for plan in ("1,4,64", "1,8,40"):
        knob("FC_Q4_TILES", plan)
        c.check(q, hk, hv, 5000, lens, what=plan, space=64 << 20)


def test_a_plan_never_exceeds_the_workspace_it_says(knob):
    """Whatever the shape, a call brings no more than the query's bytes into play: the bytes behind them stay as they were."""
    for dtype, B, Hq, Hkv, Dh, A, n in [("bf16", 1, 28, 4, 128, 32, 4000), ("bf16", 8, 28, 4, 128, 1, 1500), ("f32", 1, 4, 1, 64, 9, 4100), ("bf16", 1, 1, 1, 64, 1, 9000)]:
        c = Cache(dtype, B, Hq, Hkv, Dh, n)
        k, v = c.rows(34, n)
        c.store(k, v)
        q = inputs.normal(35, "q", (B, Hq, A, Dh), 1.0, dtype).to("cuda:0")
        bytes_ = fc.fc_q4_workspace_bytes(c.cfg, A)
        ws = torch.full((bytes_ + 4096,), 171, dtype=torch.uint8, device="cuda:0")
        out = torch.empty((B, A, Hq * Dh), dtype=c.tdt, device="cuda:0")
        for room in (bytes_, bytes_ // 3):
            ws.fill_(171)
            fc.fc_q4_attention(c.handle, 0, q, A, n, None, None, out, ws, room)
            torch.cuda.synchronize()
            assert bool((ws[room:] == 171).all())
            assert np.isfinite(ref.f64(out)).all()


def test_keys_beyond_2_to_the_31_bytes():
    """2^24 rows of which the last hundred are stored: places of their tiles pass 31 bits.  The others are zeros: score 0, value 0."""
    S, Dh, A = 1 << 24, 128, 3
    c = Cache("bf16", 1, 2, 1, Dh, S)
    q = inputs.normal(40, "q", (1, 2, A, Dh), 1.0, "bf16")
    k, v = c.rows(41, 100)
    k = (0.1 * k.float() + 0.5 * q[0, 0, 0].float() + 0.5 * q[0, 1, 1].float()).to(k.dtype)
    c.store(k, v, start=S - 100)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    s = np.einsum("had,kd->hak", ref.f64(q)[0], hk[0, 0]) * Dh ** -0.5
    top = np.maximum(s.max(-1, keepdims=True), 0)
    w = np.exp(s - top)
    total = w.sum(-1, keepdims=True) + (S - 100) * np.exp(-top)
    want = (w / total @ hv[0, 0]).transpose(1, 0, 2)[None]
    got = c.attend(q, S)
    # bf16 out, 2^-8; weights 2^-11; scores of at most 50 in magnitude by 2 * 132 roundings of 2^-24; sums of 2^24 weights in fp32: four lanes by four
    # waves by 64 ranges have 2^14 each, a rounding of 2^-24 every one, and the merges
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 264 * 50 * 2.0 ** -24 + (2.0 ** 14 + 100) * 2.0 ** -24) * ((w / total) @ np.abs(hv[0, 0])).transpose(1, 0, 2)[None] + 1e-9
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) - bound).max())
    assert np.abs(want[0, 0, 0]).max() > 1e-7
