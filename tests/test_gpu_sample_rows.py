"""The sampled fill's ways through a call: long and short parts, rows fetched by several workgroups, bins with more entries than are listed, rows whose
largest entries lie in one part, calls of many rows and of very long ones; tokens equal to the definition's in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2505_21467_amd import binding as fc
from tests.test_gpu_sample import _call, _check, _logits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
WIDE = [dict(), dict(top_p=0.9), dict(top_k=1000, top_p=0.9, temperature=1.5), dict(min_p=0.2), dict(top_p=0.5, min_p=0.001, temperature=1.5), dict(top_k=3000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,spread", [(2, 152064, 2.0), (3, 152061, 0.5), (5, 100003, 0.02), (2, 60001, 3.0)])
def test_rows_without_a_few_that_stand_out(dtype, M, V, spread):
    """Hardly decided rows: the bins in question hold thousands of entries, and are not among those that the parts list."""
    for i, f in enumerate(WIDE):
        print("[case]", dtype, M, V, spread, f, flush=True)
        z, u = _logits(70 + i, M, V, spread, peaks=0.0)
        _check(z, dtype, u, what=str(f), **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_entries_in_order_of_their_index(dtype):
    V = 70001
    z = torch.zeros(4, V)
    z[1, ::3] = 1.0
    z[2, 5000:5100] = 2.0
    z[3, :] = -1.0
    u = torch.tensor([0.25, 0.5, 0.01, 0.999])
    for f in (dict(), dict(top_k=20000), dict(top_p=0.3), dict(top_k=1), dict(min_p=1.0)):
        print("[case]", dtype, f, flush=True)
        _check(z, dtype, u, what=str(f), **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [4096, 4097, 8191, 16384, 16385, 32001])
def test_the_ends_of_parts(dtype, V):
    """The largest entries at the first and last place of a part, or all in one."""
    z, u = _logits(80, 6, V, 1.0, peaks=0.0)
    for m, at in enumerate((0, V - 1, min(4095, V - 1), min(4096, V - 1), min(8192, V - 1))):
        z[m, at] = 12.0
    z[5, :200] += 9.0
    for f in (dict(), dict(top_k=5), dict(top_p=0.99, temperature=0.7), dict(temperature=0.0)):
        _check(z, dtype, u, what=str(f), **f)


@pytest.mark.parametrize("dtype,V,room,offset", [("bf16", 151, 157, 3), ("f32", 5, 6, 1), ("bf16", 4103, 4109, 5), ("f32", 20003, 20010, 2)])
def test_rows_apart_and_beginning_anywhere(dtype, V, room, offset):
    """Rows of odd sizes at odd distances; what lies between them is larger than any logit."""
    z, u = _logits(81, 9, room, 2.0)
    z[:, V:] = 1e4
    for f in (dict(), dict(top_k=7, top_p=0.8), dict(min_p=0.01)):
        _check(z, dtype, u, V=V, offset=offset, what=str(f), **f)


def test_many_rows_and_long_ones():
    z, u = _logits(82, 65535, 9, 2.0, peaks=0.0)
    few = slice(None, None, 997)
    tok, conf = _call(z, "f32", u, top_k=4, top_p=0.9)
    one = _call(z[few].contiguous(), "f32", u[few], top_k=4, top_p=0.9)
    assert np.array_equal(tok[few], one[0]) and np.array_equal(conf[few], one[1])
    _check(z[few].contiguous(), "f32", u[few], top_k=4, top_p=0.9, what="of many")
    z, u = _logits(83, 700, 9001, 1.0, peaks=3.0)
    tok, conf = _call(z, "bf16", u, top_p=0.9)
    few = slice(None, None, 99)
    one = _call(z[few].contiguous(), "bf16", u[few], top_p=0.9)
    assert np.array_equal(tok[few], one[0]) and np.array_equal(conf[few], one[1])
    _check(z[few].contiguous(), "bf16", u[few], top_p=0.9, what="of 700")
    z, u = _logits(84, 1, 1 << 24, 2.0)
    for f in (dict(top_k=50, top_p=0.95), dict(top_p=0.9)):
        _check(z, "bf16", u, what="2^24 entries", **f)


def test_nothing_behind_the_workspace_is_touched():
    for dtype, M, V in [("f32", 3, 152064), ("bf16", 40, 32000), ("bf16", 1, 7), ("f32", 300, 5001)]:
        z, u = _logits(85, M, V, 1.0, peaks=0.0)
        bytes_ = fc.fc_sample_workspace_bytes(dtype, M, V)
        ws = torch.full((bytes_ + 4096,), 171, dtype=torch.uint8, device=DEV)
        t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        tok, conf = torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(M, dtype=torch.float32, device=DEV)
        for f in ((0, 1.0), (50, 0.9), (0, 0.9)):
            fc.fc_sample_tokens(dtype, z.to(t).to(DEV), V, M, V, 1.0, f[0], f[1], 0.0, u.to(DEV), tok, conf, ws, bytes_)
            torch.cuda.synchronize()
            assert bool((ws[bytes_:] == 171).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_which_filter_ends_first(dtype):
    """Top-k, top-p and min-p ending far before and behind one another, in every order, and near one another; hardly decided rows and peaked ones."""
    for peaks in (0.0, 12.0):
        z, u = _logits(86, 5, 50001, 1.2, peaks=peaks)
        for k in (0, 3, 600, 20000):
            for top_p in (1.0, 0.02, 0.5, 0.98):
                for min_p in (0.0, 0.7, 0.05, 0.0005):
                    _check(z, dtype, u, what="%s %s %s %s" % (peaks, k, top_p, min_p), top_k=k, top_p=top_p, min_p=min_p, temperature=0.9)


@pytest.mark.parametrize("f", [(0, 0.9), (0, 1.0), (40, 0.9)])
def test_replays_of_a_call_whose_workgroups_wait_for_nobody(f):
    """Rows that several workgroups fetch, recorded into a graph: other numbers and logits with every replay, over a workspace that was overwritten."""
    M, V = 2, 152064
    z = torch.empty((M, V), device=DEV)
    u, tok, conf = torch.empty(M, device=DEV), torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(M, device=DEV)
    ws = torch.empty(fc.fc_sample_workspace_bytes("f32", M, V), dtype=torch.uint8, device=DEV)
    call = lambda: fc.fc_sample_tokens("f32", z, V, M, V, 1.0, f[0], f[1], 0.0, u, tok, conf, ws)

    def fill(seed):
        a, b = _logits(seed, M, V, 1.0, peaks=0.0)
        z.copy_(a)
        u.copy_(b)

    fill(90)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for replay in range(5):
        fill(91 + replay)
        ws.fill_(255 if replay % 2 else 1)
        call()
        torch.cuda.synchronize()
        want = tok.clone(), conf.clone()
        ws.fill_(170)
        tok.zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok, want[0]) and torch.equal(conf, want[1]), replay
        assert int(tok.min()) >= 0 and int(tok.max()) < V
