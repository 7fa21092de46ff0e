"""FP8 with fine-grained scales, scored routing and the layer of the two (float64 numpy).

The paper's FP8 rollout (Sec. 2.2 "FP8" paragraph) uses E4M3 codes with
fine-grained scales; the block shapes and the router are readings:

  S1  a block of 128 elements of an activation row, or of 128 x 128 of a weight
      matrix (the last one may be short), with m = max |x|: enc = fl(448 / m),
      dec = fl(1 / enc) for m >= 2^-100, else enc = dec = 1.
  S2  code = E4M3_RNE(min(|fl(x * enc)|, 448)) with the sign in bit 7.
  S3  out[r, n] = sum over the blocks b of K of
      dec_a[b, r] * dec_w[e, n / 128, b] * sum_{k in b} a_k w_k.
  S4  scored routing: see `route`.
  S5  layer: S4, S3 with SwiGLU, S1-S2 on that float32 value, S3, z held as
      bf16, y = bf16_RNE(sum_s w[t, s] z[row(t, s)]).
"""

import numpy as np

from .formats import e4m3_decode, e4m3_encode_pos, bf16_round_f64

BLOCK = 128


def _scale(m):
    m = np.asarray(m, np.float32)
    some = m >= np.float32(2.0 ** -100)
    enc = np.where(some, np.float32(448.0) / np.where(some, m, np.float32(1.0)),
                   np.float32(1.0)).astype(np.float32)
    return enc, (np.float32(1.0) / enc).astype(np.float32)


def _codes(x, enc):
    v = np.minimum(np.abs(x * enc).astype(np.float32), np.float32(448.0))
    return (e4m3_encode_pos(v) | (np.signbit(x).astype(np.uint8) << 7)).astype(np.uint8)


def values(codes):
    """The signed E4M3 values of codes (float64)."""
    v = np.asarray(e4m3_decode(codes & 0x7F), np.float64)
    return np.where(codes & 0x80, -v, v)


def quantize_act(x):
    """S1-S2 per 1 x 128.  x float32 [rows][K] -> (codes u8, dec f32 [blocks][rows])."""
    x = np.asarray(x, np.float32)
    rows, K = x.shape
    codes = np.empty((rows, K), np.uint8)
    dec = np.empty((-(-K // BLOCK), rows), np.float32)
    for b in range(dec.shape[0]):
        s = slice(BLOCK * b, BLOCK * (b + 1))
        enc, dec[b] = _scale(np.abs(x[:, s]).max(1))
        codes[:, s] = _codes(x[:, s], enc[:, None])
    return codes, dec


def quantize_weight(w):
    """S1-S2 per 128 x 128.  w float32 [E][N][K] -> (codes u8, dec f32 [E][..][..])."""
    w = np.asarray(w, np.float32)
    E, N, K = w.shape
    codes = np.empty((E, N, K), np.uint8)
    dec = np.empty((E, -(-N // BLOCK), -(-K // BLOCK)), np.float32)
    for i in range(dec.shape[1]):
        for j in range(dec.shape[2]):
            a, s = slice(BLOCK * i, BLOCK * (i + 1)), slice(BLOCK * j, BLOCK * (j + 1))
            enc, dec[:, i, j] = _scale(np.abs(w[:, a, s]).max((1, 2)))
            codes[:, a, s] = _codes(w[:, a, s], enc[:, None, None])
    return codes, dec


def act_values(codes, dec):
    K = codes.shape[1]
    return values(codes) * np.repeat(dec.astype(np.float64), BLOCK, 0)[:K].T


def weight_values(codes, dec):
    N, K = codes.shape[-2:]
    s = np.repeat(np.repeat(dec.astype(np.float64), BLOCK, -2), BLOCK, -1)
    return values(codes) * s[..., :N, :K]


def grouped_gemm(a, dec_a, row_token, offsets, w, dec_w):
    """S3.  Returns (out, the sum of |products| behind each element), float64."""
    av = act_values(a, dec_a)
    if row_token is not None:
        av = av[np.maximum(row_token, 0)]
    rows, N = int(offsets[-1]), w.shape[1]
    out, mag = np.zeros((rows, N)), np.zeros((rows, N))
    for e in range(len(offsets) - 1):
        r = slice(int(offsets[e]), int(offsets[e + 1]))
        if r.stop > r.start:
            wv = weight_values(w[e], dec_w[e])
            out[r] = av[r] @ wv.T
            mag[r] = np.abs(av[r]) @ np.abs(wv).T
    return out, mag


def silu(g):
    return g / (1.0 + np.exp(-g))


def scores(logits, scoring):
    x = np.asarray(logits, np.float64)
    if scoring == "sigmoid":
        return 1.0 / (1.0 + np.exp(-x))
    m = x.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):          # a NaN or +inf: the whole row is NaN
        p = np.where(np.isneginf(m), 0.0, np.exp(x - np.where(np.isneginf(m), 0.0, m)))
    z = p.sum(1, keepdims=True)
    return p / np.where(z == 0, 1.0, z)


def choice_scores(logits, scoring):
    """The scores that choose: those of `scores`, where it leaves numbers.  Of a softmax row
    with a NaN or +inf, the softmax of its numbers, of which +inf ones share alike; a NaN
    stays NaN."""
    s = scores(logits, scoring)
    x = np.asarray(logits, np.float64)
    for t in range(x.shape[0]) if scoring == "softmax" else ():
        num = ~np.isnan(x[t])
        if num.all() and not np.isposinf(x[t]).any():
            continue
        s[t] = np.nan
        if np.isposinf(x[t]).any():
            top = np.isposinf(x[t])
            s[t, num] = top[num] / top.sum()
        elif num.any():
            s[t, num] = scores(x[t:t + 1, num], scoring)[0]
    return s


def route(logits, k, scoring="softmax", bias=None, groups=1, top_groups=1, group_sum=1,
          renorm=True, scale=1.0, live=None):
    """S4, token by token: c = s + bias chooses (without bias and groups the logits do),
    the top_groups groups by the sum of their group_sum largest c, then the k largest c
    of theirs; ties to the lower index, a NaN after every number (`choice_scores`); weight
    scale * s / sum(s chosen) or scale * s.
    Returns dict(ids, w, offsets, row_token, inv_row); w float64."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    s = scores(x, scoring)
    chooses = choice_scores(x, scoring)
    ids = np.full((T, k), -1, np.int64)
    w = np.zeros((T, k))
    n = E // groups
    for t in range(T):
        if live is not None and not live[t]:
            continue
        c = list(x[t] if bias is None and groups == 1 else chooses[t] + (
            0.0 if bias is None else np.asarray(bias, np.float64)))
        first = lambda v: (np.isnan(v), 0.0 if np.isnan(v) else -v)
        best = [sum(sorted(c[g * n:(g + 1) * n], key=first)[:group_sum]) for g in range(groups)]
        part = sorted(range(groups), key=lambda g: (first(best[g]), g))
        pool = [e for g in part[:top_groups] for e in range(g * n, (g + 1) * n)]
        ids[t] = sorted(pool, key=lambda e: (first(c[e]), e))[:k]
        w[t] = s[t][ids[t]]
        if renorm:
            tot = w[t].sum()
            w[t] = w[t] / tot if tot else 0.0
    w *= float(np.float32(scale))
    flat = [(int(ids[t, j]), t, j) for t in range(T) for j in range(k) if ids[t, j] >= 0]
    flat.sort()
    row_token = np.full(T * k, -1, np.int64)
    inv = np.full((T, k), -1, np.int64)
    count = np.zeros(E + 1, np.int64)
    for r, (e, t, j) in enumerate(flat):
        row_token[r], inv[t, j] = t, r
        count[e + 1] += 1
    return dict(ids=ids, w=w, offsets=np.cumsum(count), row_token=row_token, inv_row=inv)


def chosen_weights(logits, ids, scoring, renorm, scale):
    """The weights as a function of the logits, the choice fixed (for differences)."""
    s = np.take_along_axis(scores(logits, scoring), ids, 1)
    if renorm:
        s = s / s.sum(1, keepdims=True)
    return float(np.float32(scale)) * s


def route_backward(logits, ids, grad_w, scoring="softmax", renorm=True, scale=1.0):
    """The gradient of the logits, row by row through the Jacobian of the weights
    (float64); rows of ids that are -1 have none.  Where the weights depend on the chosen
    logits alone, the other experts' gradients are 0, beside NaN ones too."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    out = np.zeros((T, E))
    for t in range(T):
        if ids[t, 0] < 0:
            continue
        s = scores(x[t:t + 1], scoring)[0]
        ds = np.diag(s * (1.0 - s)) if scoring == "sigmoid" else np.diag(s) - np.outer(s, s)
        v, J = s[ids[t]], ds[ids[t]]             # chosen scores, their Jacobian
        if renorm:
            n = v.sum()
            J = (np.eye(len(v)) / n - np.outer(v, np.ones(len(v))) / n ** 2) @ J if n else 0 * J
        out[t] = float(np.float32(scale)) * np.asarray(grad_w[t], np.float64) @ J
        if renorm or scoring == "sigmoid":
            out[t, np.setdiff1d(np.arange(E), ids[t])] = 0.0
    return out


def moe_layer(x, logits, w13, w2, k, **router):
    """S5.  w13, w2: (codes, dec).  Returns dict(y, h, z, r)."""
    r = route(logits, k, **router)
    T, I = x.shape[0], w13[0].shape[1] // 2
    gu, _ = grouped_gemm(*quantize_act(x), r["row_token"], r["offsets"], *w13)
    h = silu(gu[:, :I]) * gu[:, I:]
    z, _ = grouped_gemm(*quantize_act(h.astype(np.float32)), None, r["offsets"], *w2)
    z = bf16_round_f64(z)
    y = np.zeros((T, w2[0].shape[1]))
    for t in range(T):
        for j in range(k):
            if r["inv_row"][t, j] >= 0:
                y[t] += r["w"][t, j] * z[r["inv_row"][t, j]]
    return dict(y=y, h=h, z=z, r=r)
