"""The 4-bit cache on the GPU against plain definitions in 64 bits: what is stored bit for bit, attention within a bound by arithmetic."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import binding as fc
from paper_2505_21467_amd import inputs
from tests import q4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Cache:
    def __init__(self, dtype, B, Hq, Hkv, Dh, max_seq, n_layers=1, scale=0.0, fill=None):
        self.cfg = fc.make_config(n_layers, B, 256, Hq, Hkv, Dh, max_seq, dtype, 10000.0, scale)
        self.dtype, self.tdt, self.shape = dtype, inputs.TORCH_DTYPE[dtype], (B, Hq, Hkv, Dh, max_seq)
        self.storage = torch.zeros(fc.fc_q4_storage_bytes(self.cfg), dtype=torch.uint8, device=DEV)
        if fill is not None:
            self.storage.fill_(fill)
        self.handle = fc.fc_q4_alloc(self.cfg, self.storage)
        self.scale = scale or Dh ** -0.5

    def __del__(self):
        torch.cuda.synchronize()
        fc.fc_q4_free(self.handle)

    def rows(self, seed, rows, std=1.0):
        B, _, Hkv, Dh, _ = self.shape
        return tuple(inputs.normal(seed, "q4." + t, (B, Hkv, rows, Dh), std, self.dtype) for t in "kv")

    def store(self, k, v, pos=None, start=0, layer=0):
        fc.fc_q4_store_rows(self.handle, layer, k.to(DEV), v.to(DEV), None if pos is None else pos.to(DEV), start, k.shape[2])

    def read(self, start=0, rows=None, layer=0):
        B, _, Hkv, Dh, S = self.shape
        rows = S - start if rows is None else rows
        k, v = (torch.full((B, Hkv, rows, Dh), 7.0, dtype=self.tdt, device=DEV) for _ in "kv")
        fc.fc_q4_read_rows(self.handle, layer, k, v, start, rows)
        torch.cuda.synchronize()
        return ref.f64(k), ref.f64(v)

    def attend(self, q, n, lens=None, pos=None, layer=0, space=None, stream=None):
        B, Hq, _, Dh, _ = self.shape
        A = q.shape[2]
        out = torch.full((B, A, Hq * Dh), 5.0, dtype=self.tdt, device=DEV)
        bytes_ = fc.fc_q4_workspace_bytes(self.cfg, A) if space is None else space
        ws = torch.full((max(bytes_, 16),), 255, dtype=torch.uint8, device=DEV) if bytes_ else None
        dev = lambda t: None if t is None else t.to(DEV)
        fc.fc_q4_attention(self.handle, layer, dev(q), A, n, dev(lens), dev(pos), out, ws, bytes_, stream)
        torch.cuda.synchronize()
        return ref.f64(out).reshape(B, A, Hq, Dh)

    def check(self, q, k, v, n, lens=None, pos=None, what="", **kw):
        """k, v: held values of all rows."""
        B, _, _, Dh, _ = self.shape
        got = self.attend(q, n, lens, pos, **kw)
        each = [n] * B if lens is None else [min(max(int(x), 0), n) for x in lens]
        want, spread, score, most = ref.attend(ref.f64(q), k, v, each, self.scale, None if pos is None else pos.numpy())
        bound = ref.attention_bound(want, spread, score, most, each, Dh, self.dtype)
        assert np.isfinite(got).all(), what + ": non-finite values"
        over = np.abs(got - want) - bound
        assert (over <= 0).all(), "%s: %.3e beyond the bound" % (what, over.max())
        # and the norm: a wrong weight of one key in many would hide in the largest errors allowed.  bfloat16 out: 2^-8 of every element at
        # most, weights 2^-11; fp32: harness bound of the full-precision path
        rel = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300)
        assert rel <= (1e-5 if self.dtype == "f32" else 2.0 ** -8 + 2.0 ** -10), "%s: relative error %.3e" % (what, rel)
        return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [128, 64])
@pytest.mark.parametrize("start,rows", [(0, 1), (0, 64), (5, 1), (63, 2), (17, 200), (0, 300), (290, 10), (64, 64)])
def test_stored_rows_read_back_as_the_format_holds_them(dtype, Dh, start, rows):
    c = Cache(dtype, 2, 4, 2, Dh, 300, n_layers=2)
    k0, v0 = c.rows(1, 300)
    c.store(k0, v0, layer=1)
    k, v = c.rows(2, rows, 3.7)
    c.store(k, v, start=start, layer=1)
    hk, hv = ref.held_rows(ref.f64(k0), ref.f64(v0))
    hk[:, :, start:start + rows], hv[:, :, start:start + rows] = ref.held_rows(ref.f64(k), ref.f64(v))
    gk, gv = c.read(layer=1)
    assert np.array_equal(gk, hk) and np.array_equal(gv, hv)
    part = c.read(start, rows, layer=1)
    assert np.array_equal(part[0], hk[:, :, start:start + rows]) and np.array_equal(part[1], hv[:, :, start:start + rows])
    assert not any(x.any() for x in c.read(layer=0))       # the other layer: zeros as allocated


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_listed_places_padding_and_duplicates(dtype, Dh):
    c = Cache(dtype, 3, 4, 2, Dh, 200)
    k0, v0 = c.rows(3, 200)
    c.store(k0, v0)
    rows = 37
    k, v = c.rows(4, rows, 2.0)
    pos = torch.stack([torch.randperm(200, generator=torch.Generator().manual_seed(b))[:rows] for b in range(3)]).to(torch.int32)
    pos[0, 3], pos[0, 4], pos[1, 0], pos[2, :] = -1, 200, -2 ** 31, -1
    pos[1, 30] = pos[1, 2]                                  # twice: the later row is stored
    pos[0, 36], pos[0, 35] = 2 ** 31 - 1, pos[0, 7]
    c.store(k, v, pos)
    hk, hv = ref.held_rows(ref.f64(k0), ref.f64(v0))
    nk, nv = ref.held_rows(ref.f64(k), ref.f64(v))
    for b in range(3):
        for r in range(rows):
            if 0 <= pos[b, r] < 200:
                hk[b, :, pos[b, r]], hv[b, :, pos[b, r]] = nk[b, :, r], nv[b, :, r]
    gk, gv = c.read()
    assert np.array_equal(gk, hk) and np.array_equal(gv, hv)


def test_a_list_longer_than_a_workgroup():
    c = Cache("bf16", 1, 1, 1, 128, 1500)
    pos = torch.randperm(1500, generator=torch.Generator().manual_seed(9))[:1100].to(torch.int32)[None]
    k, v = c.rows(5, 1100)
    c.store(k, v, pos)
    gk, gv = c.read()
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    assert np.array_equal(gk[:, :, pos[0]], hk) and np.array_equal(gv[:, :, pos[0]], hv)
    rest = np.setdiff1d(np.arange(1500), pos[0].numpy())
    assert not gk[:, :, rest].any() and not gv[:, :, rest].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_at_the_ends_of_the_format(dtype):
    """Ties, zeros, the least scales, the largest numbers; rows that cannot be held read as NaN, K and V, and no other row does."""
    c = Cache(dtype, 1, 1, 1, 64, 64)
    k, v = (torch.zeros((1, 1, 64, 64)) for _ in "kv")
    k[0, 0, 0, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    k[0, 0, 0, 32:36] = torch.tensor([-0.25, -0.75, 48.0, -20.0])
    v[0, 0, 0, :8] = torch.tensor([0.25, -0.75, 1.25, -1.75, 2.5, -3.5, 5.0, -6.0])
    k[0, 0, 1, 0], v[0, 0, 1, 0] = 3.3e38, 6 * 2.0 ** 40
    k[0, 0, 2, 0], v[0, 0, 2, 0] = 2.0 ** -126, 2.0 ** -126
    k[0, 0, 3, 0], v[0, 0, 3, 0] = 3 * 2.0 ** -101, 3 * 2.0 ** -41
    k[0, 0, 4, 0], v[0, 0, 4, 0] = 6.25, 12.25
    v[0, 0, 5, 9] = 6.5 * 2.0 ** 40
    k[0, 0, 6, 63] = float("nan")
    k[0, 0, 7, 1] = float("-inf")
    v[0, 0, 8, 33] = float("inf")
    v[0, 0, 9, 0] = float("nan")
    k[0, 0, 10, 40] = 6 * 2.0 ** 120
    k, v = (x.to(inputs.TORCH_DTYPE[dtype]) for x in (k, v))
    c.store(k, v)
    gk, gv = c.read()
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    assert np.array_equal(gk, hk, equal_nan=True) and np.array_equal(gv, hv, equal_nan=True)
    bad = [1, 5, 6, 7, 8, 9]                                # (3.3e38 would round to 2^128)
    assert np.isnan(gk[0, 0, bad]).all() and np.isfinite(np.delete(gk[0, 0], bad, 0)).all()


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_store_from_a_full_precision_cache(dtype, Dh):
    B, Hkv, S = 2, 2, 150
    c = Cache(dtype, B, 4, Hkv, Dh, S)
    full = fc.fc_cache_alloc(fc.make_config(1, B, 256, 4, Hkv, Dh, S, dtype))
    k, v = c.rows(6, S)
    fc.fc_cache_write_rows(full, 0, k.to(DEV), v.to(DEV), 0, S)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    fc.fc_q4_store_from(c.handle, 0, full, 0, None, 30, 77)
    gk, gv = c.read()
    assert np.array_equal(gk[:, :, 30:107], hk[:, :, 30:107]) and np.array_equal(gv[:, :, 30:107], hv[:, :, 30:107])
    assert not gk[:, :, :30].any() and not gv[:, :, 107:].any()
    pos = torch.tensor([[0, -1, 149, 5], [3, 3, 200, 64]], dtype=torch.int32, device=DEV)
    fc.fc_q4_store_from(c.handle, 0, full, 0, pos, 0, 4)
    gk, gv = c.read()
    for b, p in ((0, 0), (0, 149), (0, 5), (1, 3), (1, 64)):
        assert np.array_equal(gk[b, :, p], hk[b, :, p]) and np.array_equal(gv[b, :, p], hv[b, :, p])
    assert not gk[0, :, 1:5].any() and not gv[1, :, 4:30].any()
    torch.cuda.synchronize()
    fc.fc_cache_free(full)


ATTEND = [
    # dtype, B, Hq, Hkv, Dh, A, keys
    ("f32", 1, 4, 4, 64, 32, 288), ("f32", 2, 4, 2, 128, 5, 77), ("f32", 1, 2, 1, 128, 1, 1), ("f32", 1, 8, 1, 64, 33, 700), ("f32", 2, 7, 1, 64, 3, 2500),
    ("bf16", 1, 28, 4, 128, 32, 1056), ("bf16", 1, 1, 1, 128, 1, 1), ("bf16", 1, 4, 4, 64, 1, 63), ("bf16", 2, 4, 4, 64, 17, 64),
    ("bf16", 3, 28, 4, 128, 19, 65), ("bf16", 8, 28, 4, 128, 1, 511), ("bf16", 1, 8, 8, 128, 64, 130), ("bf16", 2, 8, 1, 64, 9, 1500),
    ("bf16", 1, 6, 2, 128, 100, 333), ("bf16", 1, 2, 2, 128, 16, 5000), ("bf16", 1, 7, 1, 128, 32, 9000), ("bf16", 1, 4, 1, 64, 256, 256),
    ("bf16", 5, 3, 1, 128, 2, 192), ("bf16", 1, 64, 64, 128, 1, 128),
]


@pytest.mark.parametrize("dtype,B,Hq,Hkv,Dh,A,n", ATTEND)
def test_attention(dtype, B, Hq, Hkv, Dh, A, n):
    """Lengths from one key to several ranges, at and beside the ends of tiles; the cache has rows behind the attended ones."""
    print("[case]", dtype, B, Hq, Hkv, Dh, A, n, flush=True)
    c = Cache(dtype, B, Hq, Hkv, Dh, n + 70)
    k, v = c.rows(10, n + 70)
    c.store(k, v)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    q = inputs.normal(11, "q", (B, Hq, A, Dh), 1.5, dtype)
    a = c.check(q, hk, hv, n, what="with workspace")
    c.check(q, hk, hv, n, what="without workspace", space=0)
    assert np.array_equal(a, c.attend(q, n)), "another result the second time"


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_lengths_per_sequence_and_padded_rows(dtype, Dh):
    """Lengths of zero, one, beside the ends of tiles, beyond kv_len; padded rows; what lies behind a length is NaN and does not matter."""
    lens = torch.tensor([0, 1, 63, 64, 65, 700, 2 ** 31 - 1, -5], dtype=torch.int32)
    B, A, n = len(lens), 6, 700
    c = Cache(dtype, B, 4, 2, Dh, 760, fill=255)            # scales of 255 everywhere: not a number
    k, v = c.rows(12, 700)
    k, v = k.clone(), v.clone()
    for b in range(B):
        k[b, :, min(max(int(lens[b]), 0), n):] = float("nan")
    c.store(k, v)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    pos = torch.arange(A, dtype=torch.int32).repeat(B, 1)
    pos[3, 2], pos[5, 0], pos[6, :] = -1, -7, -1
    q = inputs.normal(13, "q", (B, 4, A, Dh), 1.5, dtype)
    for space in (None, 0):
        got = c.check(q, hk, hv, n, lens, pos, what="ragged", space=space)
        assert not got[0].any() and not got[7].any() and not got[6].any() and not got[3, 2].any() and got[3, 1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_numbers_show_where_they_are_attended(dtype):
    c = Cache(dtype, 2, 4, 2, 128, 300)
    k, v = c.rows(14, 300)
    v = v.clone()
    v[1, 1, 200, 5] = float("inf")
    c.store(k, v)
    q = inputs.normal(15, "q", (2, 4, 3, 128), 1.0, dtype)
    out = c.attend(q, 300)
    assert np.isfinite(out[0]).all() and np.isfinite(out[1, :, :2]).all() and np.isnan(out[1, :, 2:]).all()
    assert np.isfinite(c.attend(q, 200)).all()
    q[0, 1, 2, 7] = float("nan")
    out = c.attend(q, 200)
    assert np.isnan(out[0, 2, 1]).all() and np.isfinite(np.delete(out[0], 1, 1)).all() and np.isfinite(out[0, :2]).all() and np.isfinite(out[1]).all()


@pytest.mark.parametrize("dtype,Dh,n", [("bf16", 128, 2100), ("bf16", 64, 500), ("f32", 64, 500)])
def test_scores_that_grow_and_values_of_many_sizes(dtype, Dh, n):
    """Scores that rise along the keys, so that the running maximum moves all the way; value rows 2^-20 to 2^20 apart; one key that takes it all;
    a softmax scale of the caller's."""
    c = Cache(dtype, 1, 2, 1, Dh, n, scale=0.25)
    k, v = c.rows(16, n)
    ramp = torch.linspace(0, 6, n)[None, None, :, None]
    q = inputs.normal(17, "q", (1, 2, 20, Dh), 1.0, dtype).abs()
    k = (k.float() * 0.3 + ramp).to(k.dtype)
    size = torch.exp2(torch.randint(-20, 21, (n,), generator=torch.Generator().manual_seed(3)).float())[None, None, :, None]
    v = (v.float() * size).to(v.dtype)
    c.store(k, v)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    c.check(q, hk, hv, n, what="rising")
    c.store(k.flip(2), v.flip(2))
    c.check(q, hk[:, :, ::-1], hv[:, :, ::-1], n, what="falling")


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_rows_never_stored_are_zeros_that_count(dtype, Dh):
    """Zeroed storage: a row that was never stored has score 0 and value 0, beside rows with large values too."""
    c = Cache(dtype, 1, 2, 1, Dh, 200)
    k, v = c.rows(22, 200)
    v = (v.float() * 2.0 ** 39).to(v.dtype)
    c.store(k[:, :, 50:120], v[:, :, 50:120], start=50)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    for x in (hk, hv):
        x[:, :, :50], x[:, :, 120:] = 0, 0
    q = inputs.normal(23, "q", (1, 2, 9, Dh), 1.0, dtype)
    c.check(q, hk, hv, 200, what="rows never stored")
    assert not Cache(dtype, 1, 2, 1, Dh, 200).attend(q, 200).any()


def test_places_that_pass_32_bits():
    """A cache of 2^24 rows: the tiles of the last kv head lie beyond 2^31 bytes, and of the last sequence beyond 2^32."""
    B, Hkv, Dh, S = 2, 2, 128, 1 << 24
    c = Cache("bf16", B, 2, Hkv, Dh, S)
    assert c.storage.numel() > 2 ** 32
    k, v = c.rows(18, 100)
    c.store(k, v, start=S - 100)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    gk, gv = c.read(S - 100, 100)
    assert np.array_equal(gk, hk) and np.array_equal(gv, hv)
    c.store(k, v, start=0)
    gk, gv = c.read(0, 100)
    assert np.array_equal(gk, hk) and np.array_equal(gv, hv)
    q = inputs.normal(19, "q", (B, 2, 1, Dh), 1.0, "bf16")
    c.check(q, hk, hv, 100, what="first rows of a long cache")


def test_tensors_at_any_element():
    """Rows, queries and outputs that begin at an odd element."""
    c = Cache("bf16", 1, 2, 1, 128, 100)
    k, v = c.rows(20, 90)
    at = lambda t: torch.cat([torch.zeros(1, dtype=t.dtype), t.flatten()]).to(DEV)[1:]
    kd, vd = at(k), at(v)
    fc.fc_q4_store_rows(c.handle, 0, kd, vd, None, 3, 90)
    hk, hv = ref.held_rows(ref.f64(k), ref.f64(v))
    out = torch.full((1 + 2 * 90 * 128,), 3.0, dtype=torch.bfloat16, device=DEV)
    half = 90 * 128
    fc.fc_q4_read_rows(c.handle, 0, out[1:1 + half], out[1 + half:], 3, 90)
    assert np.array_equal(ref.f64(out[1:1 + half]).reshape(hk.shape), hk) and np.array_equal(ref.f64(out[1 + half:]).reshape(hv.shape), hv)
    q = inputs.normal(21, "q", (1, 2, 5, 128), 1.0, "bf16")
    o = torch.full((1 + 5 * 256 + 1,), 3.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(max(16, fc.fc_q4_workspace_bytes(c.cfg, 5)), dtype=torch.uint8, device=DEV)
    fc.fc_q4_attention(c.handle, 0, at(q), 5, 93, None, None, o[1:], ws)
    plain = c.attend(q, 93)
    assert np.array_equal(ref.f64(o[1:-1]).reshape(plain.shape), plain) and o[0] == 3 and o[-1] == 3


@pytest.mark.parametrize("dtype,Dh,B,rows", [("bf16", 128, 4, 4200), ("f32", 64, 4, 4333)])
def test_rows_beyond_what_a_cache_holds(dtype, Dh, B, rows):
    """More than 256 MB of rows in one call, which take another kind of load."""
    Hkv = 32 if dtype == "bf16" else 34
    c = Cache(dtype, B, Hkv, Hkv, Dh, rows + 9)
    g = torch.Generator(DEV).manual_seed(24)
    k, v = (torch.randn((B, Hkv, rows, Dh), generator=g, device=DEV).to(c.tdt) for _ in "kv")
    c.store(k, v, start=5)
    gk, gv = (torch.empty((B, Hkv, rows + 9, Dh), dtype=c.tdt, device=DEV) for _ in "kv")
    fc.fc_q4_read_rows(c.handle, 0, gk, gv, 0, rows + 9)
    for b, h in ((0, 0), (1, Hkv // 2), (B - 1, Hkv - 1)):
        hk, hv = ref.held_rows(ref.f64(k[b, h]), ref.f64(v[b, h]))
        assert np.array_equal(ref.f64(gk[b, h, 5:5 + rows]), hk) and np.array_equal(ref.f64(gv[b, h, 5:5 + rows]), hv)
    small = Cache(dtype, B, Hkv, Hkv, Dh, rows + 9)           # the same rows in two calls: the other kind
    half = rows // 2
    for a, b in ((0, half), (half, rows)):
        small.store(k[:, :, a:b].contiguous(), v[:, :, a:b].contiguous(), start=5 + a)
    assert torch.equal(c.storage, small.storage)


@pytest.mark.parametrize("dtype,Dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("from_cache", [False, True])
def test_few_listed_places_of_a_long_cache(dtype, Dh, from_cache):
    """Fewer entries than tiles: entries of one tile, apart and next to one another, a place named three times, padding, the last place."""
    S, B, Hkv = 2000, 2, 3
    c = Cache(dtype, B, 3, Hkv, Dh, S)
    k0, v0 = c.rows(25, S)
    c.store(k0, v0)
    hk, hv = ref.held_rows(ref.f64(k0), ref.f64(v0))
    pos = torch.tensor([[70, -1, 1999, 64, 70, 127, 640, 2000, 70, 0, 128], [5, 5, -9, 1990, 4, 6, 2 ** 31 - 1, 1300, 1301, 1299, 5]], dtype=torch.int32)
    rows = pos.shape[1]
    if from_cache:
        full = fc.fc_cache_alloc(fc.make_config(1, B, 256, 3, Hkv, Dh, S, dtype))
        k, v = c.rows(26, S)
        fc.fc_cache_write_rows(full, 0, k.to(DEV), v.to(DEV), 0, S)
        fc.fc_q4_store_from(c.handle, 0, full, 0, pos.to(DEV), 0, rows)
    else:
        k, v = c.rows(26, rows, 2.0)
        c.store(k, v, pos)
    nk, nv = ref.held_rows(ref.f64(k), ref.f64(v))
    for b in range(B):
        for r, p in enumerate(pos[b].tolist()):
            if 0 <= p < S:
                hk[b, :, p], hv[b, :, p] = nk[b, :, p if from_cache else r], nv[b, :, p if from_cache else r]
    gk, gv = c.read()
    assert np.array_equal(gk, hk) and np.array_equal(gv, hv)
    if from_cache:
        torch.cuda.synchronize()
        fc.fc_cache_free(full)
