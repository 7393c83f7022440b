"""Measured work of the operators around a cache held in 4 bits and of the sampled fill.

A case is one pass of one of these:

  store   rows of keys and values into a cache held in 4 bits, and back as the values they stand for
          (fc_q4_store_rows, fc_q4_read_rows): what a block is put through when it is frozen
  attend  bidirectional attention of window queries over such a cache, a length per sequence
          (fc_q4_attention)
  sample  a token and its confidence for every masked position from given logits and given uniform
          numbers: temperature, top-k, top-p, min-p (fc_sample_tokens)

The 4-bit format.  A value is an E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times a
power of two: one per 32 elements of a key row, one per value row.  The power is the smallest one, 2^-100
(keys) or 2^-40 (values) at least, with which the block's largest magnitude is at most 6; values round to
the nearest number, ties to the even code.

Geometries are those of paper_2505_21467_amd.inputs and, for draws, any in between.
"""
import torch

own = False  # set by who measures: False the plain forms, True the framework's calls

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _store(dtype, batch, hkv, dh, rows, room, ragged=False):
    """rows: rows per sequence; room: rows that the cache has; ragged: a list of places, some of them padding."""
    return {"op": "store", "dtype": dtype, "batch": batch, "hkv": hkv, "dh": dh, "rows": rows, "room": room, "ragged": ragged}


def _attend(dtype, batch, hq, hkv, dh, rows, keys, ragged=False):
    """rows: query rows per sequence; ragged: every sequence has a length of its own, up to `keys`."""
    return {"op": "attend", "dtype": dtype, "batch": batch, "hq": hq, "hkv": hkv, "dh": dh, "rows": rows, "keys": keys, "ragged": ragged}


def _sample(dtype, rows, vocab, temperature, top_k, top_p, min_p, spread, room=0):
    """spread: standard deviation of the logits below their peaks; room: entries from row to row (0: vocab)."""
    return {"op": "sample", "dtype": dtype, "rows": rows, "vocab": vocab, "temperature": temperature, "top_k": top_k,
            "top_p": top_p, "min_p": min_p, "spread": spread, "room": room or vocab}


def listed():
    return [
        # the masked rows of three sequences' blocks, a list of places padded with -1
        dict(_store("bf16", 3, 4, 128, 19, 1581, True), name="store ragged block"),
        # a long document's rows of one layer, after its initial pass
        dict(_store("bf16", 1, 4, 128, 16384, 16800), name="store prompt 16384"),
        # the prompts of four sequences of the multi-head geometry
        dict(_store("bf16", 4, 32, 128, 4096, 4160), name="store multi-head B4 4096"),
        # the smallest call: the full-precision configuration
        dict(_attend("f32", 1, 4, 4, 64, 32, 288), name="attend tiny f32"),
        # one user, one block of 32 tokens behind a prompt of 1024
        dict(_attend("bf16", 1, 28, 4, 128, 32, 1056), name="attend L1024"),
        # the same behind a long document
        dict(_attend("bf16", 1, 28, 4, 128, 32, 16800), name="attend L16384"),
        # four users of the multi-head geometry, blocks of 64
        dict(_attend("bf16", 4, 32, 32, 128, 64, 4160), name="attend multi-head B4 L4096"),
        # eight users, single tokens, every one at a length of its own
        dict(_attend("bf16", 8, 28, 4, 128, 1, 8192, True), name="attend single tokens B8"),
        # one row of a guide's logits
        dict(_sample("f32", 1, 32000, 0.7, 50, 1.0, 0.0, 2.0), name="sample one row"),
        # a block of 32 masked positions
        dict(_sample("bf16", 32, 152064, 0.2, 0, 0.95, 0.0, 2.0), name="sample block"),
        # nothing but the temperature, an odd vocabulary in rows of a padded one
        dict(_sample("f32", 57, 50001, 1.0, 0, 1.0, 0.0, 1.0, 50048), name="sample unfiltered odd"),
        # the blocks of eight users, every filter on
        dict(_sample("bf16", 256, 152064, 0.8, 200, 0.9, 0.02, 2.5), name="sample B8 all filters"),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choices(("store", "attend", "sample"), (1, 3, 2))[0]
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if op == "sample":
        vocab = rng.choice((152064, 32000, _log(rng, 300, 152064) | 1))
        rows = _log(rng, 1, max(1, min(512, 32 * 152064 * (1 if dtype == "f32" else 8) // vocab)))
        return _sample(dtype, rows, vocab, rng.choice((0.2, 0.5, 0.8, 1.0, round(rng.uniform(0.1, 1.5), 3))),
                       rng.choice((0, 0, 1, _log(rng, 2, 1000))), rng.choice((1.0, 0.95, round(rng.uniform(0.3, 0.99), 3))),
                       rng.choice((0.0, 0.0, round(rng.uniform(0.005, 0.2), 4))), round(rng.uniform(0.5, 3.0), 2),
                       vocab + rng.choice((0, 0, rng.randint(1, 63))))
    dh = rng.choice((128, 128, 64))
    batch = _log(rng, 1, 8)
    hkv = rng.choice((1, 2, 4, 4, 8, 32))
    wide = 2 if dtype == "f32" else 1
    most = 4 * 32 * 4160 * 128 // (batch * hkv * dh * wide)  # the values of the largest listed cache
    if op == "store":
        rows = _log(rng, 1, min(16384, most))
        ragged = rows <= 512 and rng.random() < 0.5
        return _store(dtype, batch, hkv, dh, rows, rows + rng.randint(0, 512) + (rows if ragged else 0), ragged)
    keys = _log(rng, 1, min(16800, most))
    hq = hkv * (1 if hkv == 32 else rng.choice((1, 2, 4, 7, 8)))
    flops = 4 * 32 * 64 * 4160 * 128 // (8 if dtype == "f32" else 1)
    rows = _log(rng, 1, max(1, min(256, flops // (batch * hq * keys * dh))))
    return _attend(dtype, batch, hq, hkv, dh, rows, keys, rng.random() < 0.4)


def _generator(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + what)
    return g


def _rows(case, seed, n):
    """Keys and values [batch][hkv][n][dh]: some channels of the keys are larger than others, in every head its own."""
    g = _generator(seed, 1)
    shape = (case["batch"], case["hkv"], n, case["dh"])
    channels = torch.exp(0.5 * torch.randn((1, case["hkv"], 1, case["dh"]), generator=g, device=DEV))
    k = torch.randn(shape, generator=g, device=DEV).mul_(channels).to(TYPES[case["dtype"]])
    v = torch.randn(shape, generator=g, device=DEV).to(TYPES[case["dtype"]])
    return k, v


def _places(case, seed):
    """A block's places behind a prompt, in order, one in five of them padding; None where rows are stored in one piece."""
    if not case["ragged"]:
        return None
    g = _generator(seed, 2)
    n, room = case["rows"], case["room"]
    place = torch.stack([torch.randperm(room, generator=g, device=DEV)[:n].sort().values for _ in range(case["batch"])])
    return torch.where(torch.rand(place.shape, generator=g, device=DEV) < 0.2, -1, place).to(torch.int32)


def _queries(case, seed):
    q = torch.randn((case["batch"], case["hq"], case["rows"], case["dh"]), generator=_generator(seed, 3), device=DEV)
    return q.to(TYPES[case["dtype"]])


def _lengths(case, seed):
    """A length per sequence; None where all have the same."""
    if not case["ragged"]:
        return None
    part = torch.rand(case["batch"], generator=_generator(seed, 4), device=DEV)
    return (1 + part * case["keys"]).long().clamp(max=case["keys"]).to(torch.int32)


def _logits(case, seed):
    """Rows from nearly decided to undecided: a few entries stand out, by an amount of the row's own."""
    g = _generator(seed, 5)
    m, v = case["rows"], case["vocab"]
    z = torch.randn((m, case["room"]), generator=g, device=DEV).mul_(case["spread"])
    peaks = torch.randint(0, v, (m, 8), generator=g, device=DEV)
    z.scatter_add_(1, peaks, 14 * torch.rand((m, 1), generator=g, device=DEV) * torch.rand((m, 8), generator=g, device=DEV))
    return z.to(TYPES[case["dtype"]]), torch.rand(m, generator=g, device=DEV)


class _Cache:
    """The framework's cache in 4 bits and the storage that it borrows."""

    def __init__(self, case, room):
        from paper_2505_21467_amd import binding as fc
        self.fc = fc
        heads = case.get("hq", case["hkv"])
        self.cfg = fc.make_config(1, case["batch"], heads * case["dh"], heads, case["hkv"], case["dh"], room, case["dtype"])
        self.storage = torch.zeros(fc.fc_q4_storage_bytes(self.cfg), dtype=torch.uint8, device=DEV)
        self.handle = fc.fc_q4_alloc(self.cfg, self.storage)

    def __del__(self):
        torch.cuda.synchronize()
        self.fc.fc_q4_free(self.handle)


def _pack(x, block, lowest):
    """Rows [..., dh] to (two codes a byte, the lower four bits first; exponents, one per `block` elements)."""
    y = x.float().unflatten(-1, (-1, block))
    top = y.abs().amax(-1, keepdim=True)
    part, e = torch.frexp(top)  # top = part 2^e, part from a half to one; 6 = 0.75 2^3
    e = torch.where(part <= 0.75, e - 3, e - 2)
    e = torch.where(top > 0, e, lowest).clamp(min=lowest)
    y = torch.ldexp(y, -e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step  # (to even)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, 2 + a, 4 + a / 2)).to(torch.uint8)
    code = (code + 8 * (y < 0).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], e.squeeze(-1).to(torch.int8)


def _unpack(codes, e, block):
    """The values that codes and exponents stand for, in 32 bits."""
    grid = torch.tensor(GRID + tuple(-x for x in GRID), device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return torch.ldexp(grid[code.int()].unflatten(-1, (-1, block)), e.int().unsqueeze(-1)).flatten(-2)


def prepare(case, seed):
    state = dict(case)
    if case["op"] == "store":
        state["k"], state["v"] = _rows(case, seed, case["rows"])
        state["pos"] = _places(case, seed)
        if own:
            state["cache"] = _Cache(case, case["room"])
        return state
    if case["op"] == "attend":
        k, v = _rows(case, seed, case["keys"])
        if own:
            cache = state["cache"] = _Cache(case, case["keys"])
            cache.fc.fc_q4_store_rows(cache.handle, 0, k, v, None, 0, case["keys"])
            state["workspace"] = torch.empty(cache.fc.fc_q4_workspace_bytes(cache.cfg, case["rows"]), dtype=torch.uint8, device=DEV)
        else:
            state["k"], state["v"] = _pack(k, 32, -100), _pack(v, case["dh"], -40)
        state["q"], state["lens"] = _queries(case, seed), _lengths(case, seed)
        return state
    state["logits"], state["u"] = _logits(case, seed)
    if own:
        from paper_2505_21467_amd import binding as fc
        state["fc"] = fc
        state["workspace"] = torch.empty(fc.fc_sample_workspace_bytes(case["dtype"], case["rows"], case["vocab"]), dtype=torch.uint8, device=DEV)
    return state


def _run_store(s):
    room, rows, pos = s["room"], s["rows"], s["pos"]
    if own:
        fc, cache = s["cache"].fc, s["cache"].handle
        fc.fc_q4_store_rows(cache, 0, s["k"], s["v"], pos, 0, rows)
        n = room if s["ragged"] else rows
        k = torch.empty((s["batch"], s["hkv"], n, s["dh"]), dtype=TYPES[s["dtype"]], device=DEV)
        v = torch.empty_like(k)
        fc.fc_q4_read_rows(cache, 0, k, v, 0, n)
        return k, v
    t = TYPES[s["dtype"]]
    k, v = _unpack(*_pack(s["k"], 32, -100), 32).to(t), _unpack(*_pack(s["v"], s["dh"], -40), s["dh"]).to(t)
    if pos is None:
        return k, v
    shape = (s["batch"], s["hkv"], room + 1, s["dh"])  # (padding goes to a row of its own)
    at = torch.where(pos < 0, room, pos).long()[:, None, :, None].expand(k.shape)
    return tuple(torch.zeros(shape, dtype=t, device=DEV).scatter_(2, at, x)[:, :, :room].contiguous() for x in (k, v))


def _run_attend(s):
    b, hq, hkv, a, dh, n = s["batch"], s["hq"], s["hkv"], s["rows"], s["dh"], s["keys"]
    if own:
        fc = s["cache"].fc
        out = torch.empty((b, a, hq * dh), dtype=TYPES[s["dtype"]], device=DEV)
        fc.fc_q4_attention(s["cache"].handle, 0, s["q"], a, n, s["lens"], None, out, s["workspace"])
        return out
    k, v = _unpack(*s["k"], 32), _unpack(*s["v"], dh)
    score = torch.matmul(s["q"].float().view(b, hkv, -1, dh), k.transpose(2, 3).contiguous()) * dh ** -0.5
    if s["lens"] is not None:
        beyond = torch.arange(n, device=DEV)[None] >= s["lens"][:, None]
        score = score.masked_fill(beyond[:, None, None], float("-inf"))
    weight = torch.exp(score - score.amax(-1, keepdim=True))
    out = torch.matmul(weight, v) / weight.sum(-1, keepdim=True)
    return out.view(b, hq, a, dh).transpose(1, 2).reshape(b, a, hq * dh).to(TYPES[s["dtype"]])


def _run_sample(s):
    m, v = s["rows"], s["vocab"]
    if own:
        tok = torch.empty(m, dtype=torch.int32, device=DEV)
        conf = torch.empty(m, dtype=torch.float32, device=DEV)
        s["fc"].fc_sample_tokens(s["dtype"], s["logits"], s["room"], m, v, s["temperature"], s["top_k"], s["top_p"], s["min_p"],
                                 s["u"], tok, conf, s["workspace"])
        return tok, conf
    # in 64 bits: borders between tokens decide whole numbers
    z, order = torch.sort(s["logits"][:, :v].double(), dim=1, descending=True, stable=True)
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))  # (the call takes its parameters in 32 bits)
    w = torch.exp((z - z[:, :1]) / f32(s["temperature"]))
    kept = torch.ones_like(w, dtype=torch.bool)
    if s["top_k"]:
        kept[:, s["top_k"]:] = False
    if s["top_p"] < 1:
        of = w * kept
        before = torch.cumsum(of, 1) - of
        kept &= before < f32(s["top_p"]) * of.sum(1, keepdim=True)
    kept &= w >= f32(s["min_p"])
    w = w * kept
    upto = torch.cumsum(w, 1)
    at = (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1, keepdim=True)
    at = torch.minimum(at, kept.sum(1, keepdim=True) - 1)
    return order.gather(1, at)[:, 0].to(torch.int32), (w.gather(1, at) / upto[:, -1:])[:, 0].float()


def run(state):
    return {"store": _run_store, "attend": _run_attend, "sample": _run_sample}[state["op"]](state)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * 12, "flops": 4 * n}
    dh = case["dh"]
    held = dh + dh // 32 + 1  # bytes of a row's codes and exponents, keys and values
    if case["op"] == "store":
        rows = case["batch"] * case["hkv"] * case["rows"]
        back = case["batch"] * case["hkv"] * (case["room"] if case["ragged"] else case["rows"])
        return {"bytes": rows * (2 * dh * size + held) + back * (2 * dh * size + held), "flops": 4 * dh * rows}
    keys = case["batch"] * (case["keys"] + 1) // 2 if case["ragged"] else case["batch"] * case["keys"]
    ends = 2 * case["batch"] * case["hq"] * case["rows"] * dh * size
    return {"bytes": case["hkv"] * keys * held + ends, "flops": 4 * case["hq"] * case["rows"] * keys * dh}


def _held(x, block, lowest):
    """What the format makes of rows, by the definition: the least power of two, the nearest number, the even code of two."""
    y = x.double().unflatten(-1, (-1, block))
    top = y.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -130)
    s = torch.exp2(torch.ceil(torch.log2(top / 6)))
    s = torch.where(top > 6 * s, 2 * s, torch.where(top <= 3 * s, s / 2, s)).clamp(min=2.0 ** lowest)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    y = y / s
    a = y.abs()
    low = (torch.bucketize(a, grid, right=True) - 1).clamp(max=6)
    off = (a - grid[low]) - (grid[low + 1] - a)
    code = low + ((off > 0) | ((off == 0) & (low % 2 == 1))).long()
    return (grid[code] * y.sign() * s).flatten(-2)


def exact(case, seed):
    if case["op"] == "store":
        k, v = _rows(case, seed, case["rows"])
        k, v = _held(k, 32, -100), _held(v, case["dh"], -40)
        pos = _places(case, seed)
        if pos is None:
            return k, v
        out = tuple(torch.zeros((case["batch"], case["hkv"], case["room"], case["dh"]), dtype=torch.float64, device=DEV) for _ in "kv")
        for b, places in enumerate(pos.tolist()):
            for r, p in enumerate(places):
                if p >= 0:
                    out[0][b, :, p], out[1][b, :, p] = k[b, :, r], v[b, :, r]
        return out
    if case["op"] == "attend":
        k, v = _rows(case, seed, case["keys"])
        q, lens = _queries(case, seed).double(), _lengths(case, seed)
        n = [case["keys"]] * case["batch"] if lens is None else lens.tolist()
        group = case["hq"] // case["hkv"]
        out = torch.empty((case["batch"], case["rows"], case["hq"], case["dh"]), dtype=torch.float64, device=DEV)
        for b in range(case["batch"]):
            for j in range(case["hkv"]):
                kk, vv = _held(k[b, j, :n[b]], 32, -100), _held(v[b, j, :n[b]], case["dh"], -40)
                for h in range(j * group, (j + 1) * group):
                    p = torch.softmax(q[b, h] @ kk.T / case["dh"] ** 0.5, -1)
                    out[b, :, h] = p @ vv
        return out.flatten(2)
    import numpy as np
    z, u = _logits(case, seed)
    z, u = z[:, :case["vocab"]].float().cpu().numpy(), u.cpu().numpy()
    tok, conf = [], []
    for row, x in zip(z, u):
        order = np.argsort(-row, kind="stable")
        w = np.exp((row[order].astype(np.float64) - float(row.max())) / float(np.float32(case["temperature"])))
        if case["top_k"]:
            w = w[:case["top_k"]]
        if case["top_p"] < 1:
            w = w[:1 + int(np.searchsorted(np.cumsum(w), float(np.float32(case["top_p"])) * w.sum(), side="left"))]
        w = w[w >= float(np.float32(case["min_p"]))]
        at = min(int(np.searchsorted(np.cumsum(w), float(x) * w.sum(), side="right")), len(w) - 1)
        tok.append(int(order[at]))
        conf.append(w[at] / w.sum())
    return torch.tensor(tok, dtype=torch.int32), torch.tensor(conf, dtype=torch.float64)
