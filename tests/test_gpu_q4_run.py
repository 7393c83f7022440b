"""The 4-bit cache and the sampled fill as a decoder uses them: new rows projected into a one-layer full-precision cache and stored from there, attention,
the rest of the layer, logits, a sampled fill, the unmasking step; each call against its definition in 64 bits on what the call before gave.  The
same step recorded into a graph and replayed; calls on other streams, and two at once."""
import numpy as np
import pytest
import torch

from oracle import fc_oracle as orc
from paper_2505_21467_amd import binding as fc
from paper_2505_21467_amd import inputs
from tests import q4_reference as ref
from tests.test_gpu_q4 import Cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Model:
    """Two layers, a vocabulary of an odd size, prompt rows stored already."""

    def __init__(self, dt):
        self.dt, self.tdt = dt, inputs.TORCH_DTYPE[dt]
        self.B, self.d, self.Hq, self.Hkv, self.Dh, self.F, self.V, self.NL = 2, 256, 4, 2, 64, 512, 1003, 2
        self.P, self.A, self.S = 75, 16, 75 + 64
        n = lambda tag, shape, std: inputs.normal(51, tag, shape, std, dt).to(DEV)
        N = (self.Hq + 2 * self.Hkv) * self.Dh
        self.w = [dict(qkv=n("qkv%d" % l, (N, self.d), 0.06), out=n("out%d" % l, (self.d, self.Hq * self.Dh), 0.04),
                       gate=n("gate%d" % l, (self.F, self.d), 0.04), up=n("up%d" % l, (self.F, self.d), 0.04),
                       down=n("down%d" % l, (self.d, self.F), 0.04)) for l in range(self.NL)]
        self.norm, self.vocab, self.emb = n("norm", (self.d,), 1.0), n("vocab", (self.V, self.d), 0.1), n("emb", (self.V + 1, self.d), 1.0)
        self.q4 = Cache(dt, self.B, self.Hq, self.Hkv, self.Dh, self.S, n_layers=self.NL)
        self.one_cfg = fc.make_config(1, self.B, self.d, self.Hq, self.Hkv, self.Dh, self.S, dt)
        self.one = fc.fc_cache_alloc(self.one_cfg)
        for l in range(self.NL):
            k, v = self.q4.rows(52 + l, self.P)
            self.q4.store(k, v, layer=l)
        B, A, d = self.B, self.A, self.d
        e = lambda *shape, t=self.tdt: torch.empty(shape, dtype=t, device=DEV)
        self.x, self.h, self.y, self.q, self.o = e(B, A, d), e(B, A, d), e(B, A, d), e(B, self.Hq, A, self.Dh), e(B, A, self.Hq * self.Dh)
        self.f, self.logits = e(B, A, self.F), e(B * A, self.V)
        self.tok, self.conf, self.u = e(B * A, t=torch.int32), e(B * A, t=torch.float32), torch.rand(B * A, device=DEV, generator=torch.Generator(DEV).manual_seed(5))
        self.tokens, self.pos = torch.full((B, self.S), self.V, dtype=torch.int32, device=DEV), e(B, A, t=torch.int32)
        self.pos_next, self.count, self.idx = e(B, A, t=torch.int32), e(B, t=torch.int32), e(B, A, t=torch.int32)
        self.tokens[:, :self.P] = 7
        self.lens = torch.tensor([self.S, self.P + 20], dtype=torch.int32, device=DEV)
        self.q4_ws = e(max(16, fc.fc_q4_workspace_bytes(self.q4.cfg, A)), t=torch.uint8)
        self.ws = e(max([16] + [fc.fc_linear_workspace_bytes(dt, B * A, kk, nn) for kk, nn in
                                ((self.Hq * self.Dh, d), (d, 2 * self.F), (self.F, d), (d, self.V))]), t=torch.uint8)
        self.s_ws = e(fc.fc_sample_workspace_bytes(dt, B * A, self.V), t=torch.uint8)

    def close(self):
        torch.cuda.synchronize()
        fc.fc_cache_free(self.one)

    def step(self, stream, seen=lambda *a: None):
        B, A, d, M = self.B, self.A, self.d, self.B * self.A
        self.idx.copy_(torch.gather(self.tokens, 1, self.pos.clamp(min=0).long()))
        for b in range(B):
            fc.fc_gather_rows(self.dt, self.emb, self.V + 1, d, self.idx[b], A, self.x[b], stream)
        for l in range(self.NL):
            w = self.w[l]
            fc.fc_rmsnorm(self.dt, self.x, self.norm, 1e-6, M, d, self.h, stream)
            fc.fc_qkv_project_scatter(self.one, 0, self.h, w["qkv"], None, 0, A, self.pos, self.q, stream)
            fc.fc_q4_store_from(self.q4.handle, l, self.one, 0, self.pos, 0, A, stream)
            fc.fc_q4_attention(self.q4.handle, l, self.q, A, self.S, self.lens, self.pos, self.o, self.q4_ws, None, stream)
            seen("layer", l)
            fc.fc_linear_residual(self.dt, self.o, w["out"], self.x, M, self.Hq * self.Dh, d, self.y, self.ws, None, stream)
            fc.fc_rmsnorm(self.dt, self.y, self.norm, 1e-6, M, d, self.h, stream)
            fc.fc_ffn_gate_up(self.dt, self.h, w["gate"], w["up"], M, d, self.F, self.f, self.ws, None, stream)
            fc.fc_linear_residual(self.dt, self.f, w["down"], self.y, M, self.F, d, self.x, self.ws, None, stream)
        fc.fc_rmsnorm(self.dt, self.x, self.norm, 1e-6, M, d, self.h, stream)
        fc.fc_linear_residual(self.dt, self.h, self.vocab, None, M, d, self.V, self.logits, self.ws, None, stream)
        fc.fc_sample_tokens(self.dt, self.logits, self.V, M, self.V, 0.8, 50, 0.95, 0.01, self.u, self.tok, self.conf, self.s_ws, None, stream)
        seen("tokens", None)
        fc.fc_unmask_select(self.tok, self.conf, self.pos, 0, B, A, 3, self.V, self.tokens, self.S, self.pos_next, self.count, stream)

    def window(self, at):
        self.pos.copy_((at + torch.arange(self.A, dtype=torch.int32, device=DEV)).repeat(self.B, 1))
        self.pos[1, 3] = -1


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_steps_of_a_decoder(dt):
    m = Model(dt)
    try:
        held = [list(m.q4.read(layer=l)) for l in range(m.NL)]

        def seen(what, l):
            torch.cuda.synchronize()
            if what == "layer":
                k, v = (torch.empty((m.B, m.Hkv, m.S, m.Dh), dtype=m.tdt, device=DEV) for _ in "kv")
                fc.fc_cache_read_rows(m.one, 0, k, v, 0, m.S)
                nk, nv = ref.held_rows(ref.f64(k), ref.f64(v))
                for b in range(m.B):
                    for p in m.pos[b].tolist():
                        if p >= 0:
                            held[l][0][b, :, p], held[l][1][b, :, p] = nk[b, :, p], nv[b, :, p]
                got = m.q4.read(layer=l)
                assert np.array_equal(got[0], held[l][0]) and np.array_equal(got[1], held[l][1]), "rows held after the store"
                each = m.lens.tolist()
                want, spread, score, most = ref.attend(ref.f64(m.q), held[l][0], held[l][1], each, m.Dh ** -0.5, m.pos.cpu().numpy())
                bound = ref.attention_bound(want, spread, score, most, each, m.Dh, dt)
                assert (np.abs(ref.f64(m.o).reshape(want.shape) - want) <= bound).all(), "attention of layer %d" % l
            else:
                z = m.logits.float().cpu().numpy()
                for r in range(m.B * m.A):
                    t, c = ref.sample(z[r], 0.8, 50, 0.95, 0.01, float(m.u[r]))
                    assert int(m.tok[r]) == t and abs(float(m.conf[r]) - c) <= 2.0 ** -24 * c + m.V * 2.0 ** -44, "row %d" % r

        for step in range(5):
            m.window(m.P + 16 * (step // 2))
            tokens = m.tokens.cpu().numpy().copy()
            m.step(None, seen)
            torch.cuda.synchronize()
            pos_next, count = orc.unmask_select(m.tok.cpu().numpy(), m.conf.cpu().numpy(), m.pos.cpu().numpy(), 3, m.V, tokens)
            assert np.array_equal(tokens, m.tokens.cpu().numpy()) and np.array_equal(pos_next, m.pos_next.cpu().numpy())
            assert np.array_equal(count, m.count.cpu().numpy())
        assert int((m.tokens[:, m.P:] != m.V).sum()) == 2 * 3 * 5
    finally:
        m.close()


def test_the_step_replayed_from_a_graph():
    m = Model("bf16")
    try:
        storage, tokens = m.q4.storage.clone(), m.tokens.clone()

        def reset(replay):
            m.window(m.P + 16 * (replay // 2))
            m.q4.storage.copy_(storage)
            m.tokens.copy_(tokens)
            m.u.copy_(torch.rand(m.B * m.A, generator=torch.Generator().manual_seed(replay)))

        state = lambda: [t.clone() for t in (m.o, m.x, m.logits, m.tok, m.conf, m.tokens, m.pos_next, m.count, m.q4.storage)]
        reset(0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            m.step(side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.step(torch.cuda.current_stream().cuda_stream)
        for replay in range(5):
            reset(replay)
            m.step(torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            want = state()
            reset(replay)
            for t in (m.o, m.x, m.logits, m.tok, m.conf):
                t.zero_()
            m.q4_ws.fill_(255)
            m.s_ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(state(), want)):
                assert torch.equal(a, b), "replay %d: tensor %d differs from the eager step" % (replay, i)
    finally:
        m.close()


def test_calls_at_the_same_time_on_two_streams():
    """Two attentions over one cache and two sampled fills, each pair on streams of its own with workspaces of its own, many times over."""
    B, Hq, Hkv, Dh, A, n, V = 2, 8, 2, 128, 24, 3000, 40001
    c = Cache("bf16", B, Hq, Hkv, Dh, n)
    k, v = c.rows(60, n)
    c.store(k, v)
    q = [inputs.normal(61 + i, "q", (B, Hq, A, Dh), 1.5, "bf16").to(DEV) for i in range(2)]
    z = [inputs.normal(63 + i, "z", (9, V), 2.0, "f32").to(DEV) for i in range(2)]
    u = torch.rand(9, generator=torch.Generator().manual_seed(1)).to(DEV)
    space = [torch.empty(fc.fc_q4_workspace_bytes(c.cfg, A), dtype=torch.uint8, device=DEV) for _ in range(2)]
    s_space = [torch.empty(fc.fc_sample_workspace_bytes("f32", 9, V), dtype=torch.uint8, device=DEV) for _ in range(2)]
    out = [torch.empty((20, B, A, Hq * Dh), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    tok = [torch.empty((20, 9), dtype=torch.int32, device=DEV) for _ in range(2)]
    conf = [torch.empty((20, 9), dtype=torch.float32, device=DEV) for _ in range(2)]

    def call(i, r, stream):
        fc.fc_q4_attention(c.handle, 0, q[i], A, n, None, None, out[i][r], space[i], None, stream)
        fc.fc_sample_tokens("f32", z[i], V, 9, V, 1.0, 0, 0.9, 0.0, u, tok[i][r], conf[i][r], s_space[i], None, stream)

    for i in range(2):
        call(i, 0, None)
    torch.cuda.synchronize()
    want = [(out[i][0].clone(), tok[i][0].clone(), conf[i][0].clone()) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for r in range(20):
        for i in range(2):
            call(i, r, streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        for r in range(20):
            assert torch.equal(out[i][r], want[i][0]) and torch.equal(tok[i][r], want[i][1]) and torch.equal(conf[i][r], want[i][2]), (i, r)
