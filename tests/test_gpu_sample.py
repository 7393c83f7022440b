"""The sampled fill on the GPU: tokens equal to the definition's in 64 bits, confidences within rounding."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import binding as fc
from paper_2505_21467_amd import inputs
from tests import q4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _call(z, dtype, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, V=None, offset=0):
    """z: float32 [M][ld] that the type holds; offset: elements in front of the first row."""
    M, ld = z.shape
    V = ld if V is None else V
    flat = torch.cat([torch.zeros(offset), z.flatten()]).to(inputs.TORCH_DTYPE[dtype]).to(DEV)[offset:]
    tok = torch.full((M + 1,), -77, dtype=torch.int32, device=DEV)
    conf = torch.full((M + 1,), -7.0, dtype=torch.float32, device=DEV)
    ws = torch.full((max(16, fc.fc_sample_workspace_bytes(dtype, M, V)),), 255, dtype=torch.uint8, device=DEV)
    ud = None if u is None else torch.as_tensor(u, dtype=torch.float32).to(DEV)
    for _ in range(2):  # (the second time over what the first left in the workspace)
        fc.fc_sample_tokens(dtype, flat, ld, M, V, temperature, top_k, top_p, min_p, ud, tok, conf, ws)
        torch.cuda.synchronize()
    assert tok[M] == -77 and conf[M] == -7
    return tok[:M].cpu().numpy(), conf[:M].cpu().numpy()


def _check(z, dtype, u, V=None, offset=0, what="", **k):
    z = z.to(inputs.TORCH_DTYPE[dtype]).float()
    tok, conf = _call(z, dtype, u, V=V, offset=offset, **k)
    for m in range(len(z)):
        p = {**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **k}
        t, c = ref.sample(z[m, :V].numpy(), u=0.0 if u is None else float(u[m]), **p)
        assert tok[m] == t, "%s row %d: token %d, %d by definition" % (what, m, tok[m], t)
        # weights and sums to 2^-33 of themselves, less than 2^-44 of each entry lost; one rounding to fp32
        assert abs(float(conf[m]) - c) <= 2.0 ** -24 * c + z.shape[1] * 2.0 ** -44, "%s row %d: confidence %r, %r" % (what, m, conf[m], c)


def _logits(seed, M, V, spread, peaks=14.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((M, V), generator=g) * spread
    z.scatter_add_(1, torch.randint(0, V, (M, 8), generator=g), peaks * torch.rand((M, 1), generator=g) * torch.rand((M, 8), generator=g))
    return z, torch.rand(M, generator=g)


FILTERS = [dict(), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(top_p=0.3, temperature=0.7), dict(min_p=0.05), dict(temperature=0.2, top_p=0.95),
           dict(temperature=1.5, top_k=200, top_p=0.8, min_p=0.01), dict(temperature=0.01, top_k=7), dict(temperature=30.0), dict(temperature=0.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4097, 32000])
def test_every_filter_at_many_vocabularies(dtype, V):
    for i, f in enumerate(FILTERS):
        z, u = _logits(100 * V + i, 5, V, 2.0)
        _check(z, dtype, u, what=str(f), **{"top_k": 0, **f})


@pytest.mark.parametrize("dtype,M,V,spread,f", [
    ("bf16", 3, 152064, 2.0, dict(temperature=0.2, top_p=0.95)), ("f32", 2, 152064, 1.0, dict()), ("bf16", 2, 152064, 0.5, dict(top_p=0.99)),
    ("f32", 2, 151669, 2.5, dict(temperature=0.8, top_k=200, top_p=0.9, min_p=0.02)), ("bf16", 1, 152063, 3.0, dict(top_k=5000)),
    ("f32", 65, 5003, 2.0, dict(top_p=0.9)), ("bf16", 300, 2049, 2.0, dict(top_k=40)), ("f32", 1, 1 << 20, 2.0, dict(top_p=0.7, top_k=100000)),
    ("bf16", 2, 152064, 0.0, dict(top_p=0.5, top_k=1000)), ("f32", 600, 700, 1.0, dict(top_p=0.5)),
])
def test_sizes_of_use(dtype, M, V, spread, f):
    print("[case]", dtype, M, V, spread, f, flush=True)
    z, u = _logits(V + M, M, V, spread, 14.0 if spread else 0.0)
    _check(z, dtype, u, what=str(f), **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,ld,offset", [(1000, 1003, 0), (1001, 1001, 1), (999, 1024, 3), (7, 9, 5), (20001, 20032, 7)])
def test_rows_of_padded_vocabularies_at_any_element(dtype, V, ld, offset):
    z, u = _logits(ld, 4, ld, 2.0)
    z[:, V:] = 100.0                                         # behind the vocabulary: not looked at
    for f in FILTERS[:6]:
        _check(z, dtype, u, V=V, offset=offset, what=str(f), **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_logits(dtype):
    """Ties go by the index: all equal, two values, a plateau across a filter's border; u on the borders between tokens."""
    V = 3001
    z = torch.zeros((6, V))
    u = torch.tensor([0.0, 0.25, 0.5, 1 / 3, 0.999, 0.75])
    for f in (dict(), dict(top_k=100), dict(top_p=0.1), dict(top_k=1000, top_p=0.5), dict(min_p=1.0)):
        _check(z, dtype, u, what="all equal " + str(f), **f)
    z = torch.where(torch.arange(V)[None] % 7 == 3, 2.0, 1.0).repeat(6, 1)
    for f in (dict(), dict(top_k=500), dict(top_p=0.9), dict(min_p=0.5), dict(temperature=0.1, top_k=429)):
        _check(z, dtype, u, what="two values " + str(f), **f)
    z = torch.zeros((6, 4))                                  # borders hit exactly: the next token
    tok, conf = _call(z, dtype, torch.tensor([0.0, 0.25, 0.5, 0.75, 0.2499999, 0.7499999]))
    assert tok.tolist() == [0, 1, 2, 3, 0, 2] and (conf == 0.25).all()
    z = torch.where(torch.arange(V)[None] % 2 == 0, 0.0, -0.0).repeat(6, 1)  # 0 and -0 are equal
    _check(z, dtype, u, what="zeros of both signs", top_k=10)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_nan_and_lowest_values(dtype):
    low, inf, nan = torch.finfo(inputs.TORCH_DTYPE[dtype]).min, float("inf"), float("nan")
    V = 500
    z, _ = _logits(7, 11, V, 2.0)
    z[0, :] = -inf
    z[1, :] = nan
    z[2, 1:] = -inf
    z[3, ::2] = nan
    z[4, 10], z[4, 20] = inf, inf
    z[5, 5:] = low
    z[6, :] = low
    z[7, :250], z[7, 250:] = -inf, nan
    z[8, 3] = -low
    z[9, 1:] = nan
    z[10, :490] = -inf
    u = torch.tensor([0.5, 0.5, 0.999, 0.3, 0.6, 0.9, 0.4, 0.1, 0.7, 0.999, 0.99])
    for f in FILTERS:
        _check(z, dtype, u, what=str(f), **f)
    tok, conf = _call(z, dtype, u)
    assert tok[[0, 1, 7]].tolist() == [-1] * 3 and not conf[[0, 1, 7]].any() and tok[4] == 20 and conf[4] == 0.5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_numbers_outside_the_unit_interval(dtype):
    z, _ = _logits(8, 6, 300, 1.0)
    u = torch.tensor([-1.0, 1.0, 2.0, float("inf"), -float("inf"), 0.0])
    _check(z, dtype, u, top_k=9, what="u")
    tok, _ = _call(z, dtype, torch.full((6,), float("nan")), top_k=9)
    last, _ = _call(z, dtype, torch.full((6,), 1.0), top_k=9)
    assert np.array_equal(tok, last)


def test_a_row_gives_the_same_whatever_is_around_it():
    z, u = _logits(9, 70, 20011, 2.0)
    f = dict(temperature=0.9, top_k=300, top_p=0.95)
    many = _call(z, "f32", u, **f)
    for m in (0, 33, 69):
        one = _call(z[m:m + 1], "f32", u[m:m + 1], **f)
        assert one[0][0] == many[0][m] and one[1][0] == many[1][m]


def test_temperature_zero_takes_no_numbers():
    z, _ = _logits(10, 5, 4000, 2.0)
    _check(z, "f32", None, temperature=0.0, what="greedy")
