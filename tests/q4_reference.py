"""Plain definitions in 64 bits for the tests of the 4-bit cache and of the sampled fill, written from the format's and the filters'
definitions (numpy; no code shared with the library or with perf/)."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
K_LOWEST, V_LOWEST, K_MOST, V_MOST = -100, -40, 6.0 * 2.0 ** 120, 6.0 * 2.0 ** 40


def held(x, block, lowest):
    """The values that the format holds for rows x [..., dh] (finite float64)."""
    x = np.asarray(x, np.float64)
    y = x.reshape(x.shape[:-1] + (-1, block))
    top = np.abs(y).max(-1, keepdims=True)
    e = np.full(top.shape, lowest, np.int64)
    while True:  # the least exponent that is enough
        short = top > 6.0 * np.exp2(e.astype(np.float64))
        if not short.any():
            break
        e = np.where(short, np.maximum(e + 1, np.frexp(np.maximum(top, 1e-300))[1] - 4), e)
    y = y / np.exp2(e.astype(np.float64))
    near = np.abs(np.abs(y)[..., None] - GRID)
    best = near.min(-1, keepdims=True)
    # of two as near the even code: prefer it by looking at the even codes first
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.argmax((near == best)[..., order], -1)]
    return (np.sign(y) * GRID[code] * np.exp2(e.astype(np.float64))).reshape(x.shape)


def held_rows(k, v):
    """K and V rows [..., dh] as they read back: NaN in both where either cannot be held."""
    k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
    bad = ~(np.abs(k) <= K_MOST).all(-1) | ~(np.abs(v) <= V_MOST).all(-1)
    hk = held(np.where(bad[..., None], 0, k), 32, K_LOWEST)
    hv = held(np.where(bad[..., None], 0, v), v.shape[-1], V_LOWEST)
    hk[bad], hv[bad] = np.nan, np.nan
    return hk, hv


def attend(q, k, v, n, scale, pos=None):
    """out [B][A][Hq][Dh] and what bounds its error: (sum of |p v|, largest sum of |q k| scale, largest |v|) per output row.
    k, v: held values [B][Hkv][S][Dh]; n: length per sequence."""
    B, Hq, A, Dh = q.shape
    g = Hq // k.shape[1]
    out = np.zeros((B, A, Hq, Dh))
    spread, score, most = np.zeros_like(out), np.zeros((B, A, Hq, 1)), np.zeros((B, A, Hq, 1))
    for b in range(B):
        if n[b] < 1:
            continue
        for h in range(Hq):
            kk, vv = k[b, h // g, :n[b]], v[b, h // g, :n[b]]
            s = q[b, h] @ kk.T * scale
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, :, h] = p @ vv
            spread[b, :, h] = p @ np.abs(vv)
            score[b, :, h, 0] = (np.abs(q[b, h]) @ np.abs(kk).T * scale).max(-1)
            most[b, :, h, 0] = np.abs(vv).max()
        if pos is not None:
            out[b][pos[b] < 0] = 0
            spread[b][pos[b] < 0] = 0
            most[b][pos[b] < 0] = 0
    return out, spread, score, most


def attention_bound(ref, spread, score, most, n, dh, dtype):
    """Largest error per element.  Scores: products of dh terms summed in fp32, dh + 4 roundings of 2^-24 of the sum of magnitudes (fp32 queries are held to
    2^-29 of the largest of 32 elements: within the same); the error of a score is the relative error of its weight, in numerator and in
    sum.  Sums over n keys in fp32: n + 8 roundings; an fp32 weight is two fp16 numbers, 2^-23 of itself: within the same.  bf16: weights
    rounded to fp16 (2^-11, or half a subnormal step, 2^-25 of at most the largest), queries in three 6-bit parts, which lack up to 2^-14 of the largest
    of 32 elements, terms of either sign: 2^-11 of the largest |v| where keys of several tiles differ by it; the output to bfloat16
    (2^-8)."""
    n = np.asarray(n).reshape(-1, 1, 1, 1)
    u = 2.0 ** -24
    err = (2 * (dh + 4) * u * score + (n + 8) * u) * spread
    if dtype == "f32":
        return err + u * np.abs(ref)
    return err + 2.0 ** -11 * spread + n * 2.0 ** -25 * most + 2.0 ** -11 * most * (n > 64) + 2.0 ** -8 * np.abs(ref)


def sample(z, temperature, top_k, top_p, min_p, u):
    """(token, confidence) of one row of logits (float32 numpy)."""
    z = np.asarray(z, np.float64)
    index = np.flatnonzero(~np.isnan(z) & (z > -np.inf))
    if not len(index):
        return -1, 0.0
    order = index[np.lexsort((index, -z[index]))]
    z = z[order]
    greedy = temperature == 0
    with np.errstate(invalid="ignore"):
        w = np.where(z == z[0], 1.0, np.exp((z - z[0]) / (1.0 if greedy else float(np.float32(temperature)))))
    if greedy:
        return int(order[0]), 1.0 / w.sum()
    keep = len(w)
    if top_k:
        w = w[:top_k]
    if top_p < 1:
        keep = 1 + int(np.searchsorted(np.cumsum(w), float(np.float32(top_p)) * w.sum(), side="left"))
    w = w[:keep]
    w = w[w >= float(np.float32(min_p))]
    run = np.cumsum(w)
    at = np.flatnonzero(run > min(max(float(u), 0.0), 1.0) * run[-1]) if u == u else ()
    at = at[0] if len(at) else np.flatnonzero(w > 2.0 ** -44)[-1]
    return int(order[at]), float(w[at] / run[-1])


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().double().numpy()
