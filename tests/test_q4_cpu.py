"""The 4-bit cache and the sampled fill on the host: refusals before any HIP call, sizes, and the pins of the reference that the GPU tests use."""
import ctypes

import numpy as np
import pytest

from paper_2505_21467_amd import binding as fc
from tests import q4_reference as ref

FAKE = 0x10000  # 16-byte aligned non-NULL "device pointer"; never dereferenced on the host


def _cfg(**kw):
    base = dict(n_layers=2, batch=2, hidden=256, n_q_heads=8, n_kv_heads=2, head_dim=128, max_seq=300, dtype="bf16")
    base.update(kw)
    return fc.make_config(**base)


def _raises(status, fn, *a, **k):
    with pytest.raises(fc.FreeCacheError) as e:
        fn(*a, **k)
    assert e.value.status == status, (e.value.status, str(e.value))
    assert fc.fc_last_error() != ""


@pytest.fixture()
def q4():
    h = fc.fc_q4_alloc(_cfg(), FAKE)
    yield h
    fc.fc_q4_free(h)


def test_storage_is_133_bytes_a_row():
    assert fc.fc_q4_storage_bytes(_cfg()) == 2 * 2 * 2 * 320 * 133        # 300 rows in tiles of 64
    assert fc.fc_q4_storage_bytes(_cfg(head_dim=64, dtype="f32")) == 2 * 2 * 2 * 320 * 67
    assert fc.fc_q4_storage_bytes(_cfg(head_dim=96)) == 0
    assert fc.fc_q4_storage_bytes(_cfg(batch=40000, n_kv_heads=2)) == 0


def test_alloc_refusals():
    for bad, st in [(dict(head_dim=96), fc.FC_ERR_UNSUPPORTED), (dict(n_q_heads=7), fc.FC_ERR_UNSUPPORTED),
                    (dict(max_seq=0), fc.FC_ERR_INVALID_ARG), (dict(max_seq=(1 << 24) + 1), fc.FC_ERR_UNSUPPORTED),
                    (dict(batch=40000), fc.FC_ERR_UNSUPPORTED)]:
        _raises(st, fc.fc_q4_alloc, _cfg(**bad), FAKE)
    _raises(fc.FC_ERR_INVALID_ARG, fc.fc_q4_alloc, _cfg(), FAKE + 8)
    assert fc.lib().fc_q4_alloc(None, FAKE, ctypes.byref(ctypes.c_void_p())) == fc.FC_ERR_INVALID_ARG
    assert fc.lib().fc_q4_alloc(ctypes.byref(_cfg()), FAKE, None) == fc.FC_ERR_INVALID_ARG
    fc.fc_q4_free(None)


def test_store_and_read_refusals(q4):
    S = fc.fc_q4_store_rows
    _raises(fc.FC_ERR_INVALID_ARG, S, None, 0, FAKE, FAKE, None, 0, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, S, q4, 2, FAKE, FAKE, None, 0, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, S, q4, -1, FAKE, FAKE, None, 0, 4, 0)
    _raises(fc.FC_ERR_INVALID_ARG, S, q4, 0, None, FAKE, None, 0, 4, 0)
    _raises(fc.FC_ERR_INVALID_ARG, S, q4, 0, FAKE, None, None, 0, 4, 0)
    _raises(fc.FC_ERR_INVALID_ARG, S, q4, 0, FAKE, FAKE, None, 0, 0, 0)
    _raises(fc.FC_ERR_BOUNDS, S, q4, 0, FAKE, FAKE, None, -1, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, S, q4, 0, FAKE, FAKE, None, 297, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, S, q4, 0, FAKE, FAKE, None, 2 ** 31 - 1, 4, 0)
    _raises(fc.FC_ERR_UNSUPPORTED, S, q4, 0, FAKE, FAKE, FAKE, 0, (1 << 24) + 1, 0)
    R = fc.fc_q4_read_rows
    _raises(fc.FC_ERR_INVALID_ARG, R, None, 0, FAKE, FAKE, 0, 4, 0)
    _raises(fc.FC_ERR_INVALID_ARG, R, q4, 0, FAKE, None, 0, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, R, q4, 5, FAKE, FAKE, 0, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, R, q4, 0, FAKE, FAKE, 297, 4, 0)
    _raises(fc.FC_ERR_INVALID_ARG, R, q4, 0, FAKE, FAKE, 0, 0, 0)


def test_store_from_wants_a_cache_of_the_same_geometry(q4):
    F = fc.fc_q4_store_from
    _raises(fc.FC_ERR_INVALID_ARG, F, q4, 0, None, 0, None, 0, 4, 0)
    for other in (dict(batch=1), dict(n_kv_heads=4), dict(head_dim=64), dict(max_seq=301), dict(dtype="f32")):
        src = fc.fc_cache_alloc(_cfg(**other), FAKE, FAKE)
        _raises(fc.FC_ERR_INVALID_ARG, F, q4, 0, src, 0, None, 0, 4, 0)
        fc.fc_cache_free(src)
    src = fc.fc_cache_alloc(_cfg(n_layers=1), FAKE, FAKE)
    _raises(fc.FC_ERR_BOUNDS, F, q4, 0, src, 1, None, 0, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, F, q4, 2, src, 0, None, 0, 4, 0)
    _raises(fc.FC_ERR_BOUNDS, F, q4, 0, src, 0, None, 298, 4, 0)
    _raises(fc.FC_ERR_INVALID_ARG, F, None, 0, src, 0, None, 0, 4, 0)
    fc.fc_cache_free(src)


def test_attention_refusals(q4):
    A = fc.fc_q4_attention
    _raises(fc.FC_ERR_INVALID_ARG, A, None, 0, FAKE, 4, 100, None, None, FAKE, FAKE, 1 << 30, 0)
    _raises(fc.FC_ERR_BOUNDS, A, q4, 2, FAKE, 4, 100, None, None, FAKE, FAKE, 1 << 30, 0)
    _raises(fc.FC_ERR_INVALID_ARG, A, q4, 0, None, 4, 100, None, None, FAKE, FAKE, 1 << 30, 0)
    _raises(fc.FC_ERR_INVALID_ARG, A, q4, 0, FAKE, 4, 100, None, None, None, FAKE, 1 << 30, 0)
    _raises(fc.FC_ERR_INVALID_ARG, A, q4, 0, FAKE, 0, 100, None, None, FAKE, FAKE, 1 << 30, 0)
    _raises(fc.FC_ERR_BOUNDS, A, q4, 0, FAKE, 4, 0, None, None, FAKE, FAKE, 1 << 30, 0)
    _raises(fc.FC_ERR_BOUNDS, A, q4, 0, FAKE, 4, 301, None, None, FAKE, FAKE, 1 << 30, 0)
    _raises(fc.FC_ERR_INVALID_ARG, A, q4, 0, FAKE, 4, 100, None, None, FAKE, FAKE + 4, 1 << 30, 0)
    _raises(fc.FC_ERR_UNSUPPORTED, A, q4, 0, FAKE, 1 << 24, 100, None, None, FAKE, FAKE, 1 << 30, 0)
    many = fc.fc_q4_alloc(_cfg(batch=1, n_q_heads=64, n_kv_heads=1), FAKE)
    _raises(fc.FC_ERR_UNSUPPORTED, A, many, 0, FAKE, (1 << 18) + 1, 100, None, None, FAKE, FAKE, 1 << 30, 0)
    fc.fc_q4_free(many)
    assert fc.fc_q4_workspace_bytes(_cfg(), 0) == 0 and fc.fc_q4_workspace_bytes(_cfg(head_dim=96), 4) == 0


def test_sampling_refusals():
    good = dict(dtype="bf16", logits=FAKE, ld=1000, M=4, V=1000, temperature=0.8, top_k=5, top_p=0.9, min_p=0.1, u=FAKE, tok=FAKE,
                conf=FAKE, workspace=FAKE, workspace_bytes=1 << 40, stream=0)
    for bad in (dict(logits=None), dict(tok=None), dict(conf=None), dict(u=None), dict(M=0), dict(V=0), dict(ld=999), dict(temperature=-0.1),
                dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.5),
                dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.1), dict(min_p=float("nan")), dict(workspace=FAKE + 4)):
        _raises(fc.FC_ERR_INVALID_ARG, fc.fc_sample_tokens, **{**good, **bad})
    _raises(fc.FC_ERR_UNSUPPORTED, fc.fc_sample_tokens, **{**good, "V": (1 << 24) + 1, "ld": 1 << 25})
    _raises(fc.FC_ERR_UNSUPPORTED, fc.fc_sample_tokens, **{**good, "M": (1 << 24) + 1})
    assert fc.lib().fc_sample_tokens(7, FAKE, 8, 1, 8, 1.0, 0, 1.0, 0.0, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0) == fc.FC_ERR_INVALID_ARG
    _raises(fc.FC_ERR_UNSUPPORTED, fc.fc_sample_tokens, **{**good, "M": 65535, "V": 1 << 21, "ld": 1 << 21})
    assert fc.fc_sample_workspace_bytes("bf16", 0, 10) == 0 and fc.fc_sample_workspace_bytes("bf16", 4, 0) == 0
    need = fc.fc_sample_workspace_bytes("bf16", 4, 1000)
    if need:
        _raises(fc.FC_ERR_WORKSPACE, fc.fc_sample_tokens, **{**good, "workspace_bytes": need - 1})
        _raises(fc.FC_ERR_WORKSPACE, fc.fc_sample_tokens, **{**good, "workspace": None})


def test_the_format_of_the_reference():
    x = np.zeros((4, 32))
    x[0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]       # ties go to the even code
    x[1, :3] = [12.5, 12.0, -0.1]                                 # 12.5 > 6 * 2: the scale is 4
    x[2, :2] = [6 * 2.0 ** -101, 2.0 ** -102]                     # the least scale
    got = ref.held(x, 32, ref.K_LOWEST)
    assert got[0, :8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    assert got[1, :3].tolist() == [12.0, 12.0, 0.0]
    assert got[2, :2].tolist() == [3 * 2.0 ** -100, 0.0]
    assert not got[3].any()
    k, v = ref.held_rows(np.array([[np.inf] + [0.0] * 63, [1.0] * 64, [1.0] * 64]), np.array([[1.0] * 64, [7 * 2.0 ** 40] * 64, [6 * 2.0 ** 40] * 64]))
    assert np.isnan(k[:2]).all() and np.isnan(v[:2]).all() and (k[2] == 1).all() and (v[2] == 6 * 2.0 ** 40).all()
    # half a step of the grid: a quarter of the scale below 2, a fifth of the number (midway between 2 and 3, 4 and 6) above; the scale is less
    # than a third of the block's largest magnitude
    g = np.random.default_rng(0).standard_normal((512, 128))
    for block, lowest in ((32, ref.K_LOWEST), (128, ref.V_LOWEST)):
        err, top = np.abs(ref.held(g, block, lowest) - g), np.abs(g).reshape(512, -1, block).max(-1).repeat(block, -1)
        assert (err <= np.maximum(top / 12, np.abs(g) / 5) * (1 + 1e-12)).all()


def test_the_filters_of_the_reference():
    z = np.log(np.array([0.1, 0.4, 0.3, 0.2], np.float64)).astype(np.float32)
    first = lambda **k: [ref.sample(z, **{**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **k}, u=u)[0] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91)]
    assert first() == [1, 1, 2, 2, 3, 3, 0]
    assert first(top_k=2) == [1, 1, 1, 2, 2, 2, 2]
    assert first(top_p=0.6) == [1, 1, 1, 2, 2, 2, 2]
    assert first(top_p=0.39) == [1] * 7
    assert first(min_p=0.45) == first(top_k=3)
    assert ref.sample(z, 0.0, 1, 0.1, 0.9, 0.99) == (1, pytest.approx(0.4, rel=1e-6))
    assert ref.sample(np.array([2.0, 5.0, 5.0, 1.0]), 1.0, 1, 1.0, 0.0, 0.99)[0] == 1   # the smaller index among equals
    assert ref.sample(np.array([-np.inf, np.nan]), 1.0, 0, 1.0, 0.0, 0.5) == (-1, 0.0)
    assert ref.sample(np.array([1.0, np.inf, np.inf]), 1.0, 0, 1.0, 0.0, 0.7) == (2, 0.5)
