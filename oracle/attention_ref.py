"""fp64 oracle of the attention block: rotary positions, attention with its
gradients, the clip of query and key weights.  Test infrastructure only.

Each result comes with an elementwise bound on the rounding error of an
implementation that holds products and sums in binary32 and rounds
probabilities, their gradients and results to the storage type:

  u    half a step of the storage type (2^-8 bf16, 2^-24 fp32)
  e    what binary32 may do to a probability, relatively: the exponent is a sum
       of D products of size up to S = max sum_d |q_d k_d| scale and carries the
       log-sum-exp L, each within (D + 8) 2^-24 of its size, doubled for the
       exponent's own rounding, plus 2^-22 for the exponential and n 2^-24 for
       a sum over n of them.
"""
from __future__ import annotations

import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
E32 = 2.0 ** -24


def visible(nq, nk, causal=False, window=0):
    gap = np.arange(nq)[:, None] + (nk - nq) - np.arange(nk)[None, :]
    see = np.ones((nq, nk), dtype=bool)
    if causal:
        see &= gap >= 0
        if window:
            see &= gap < window
    return see


def attention_head(q, k, v, scale, see, dtype, dout=None):
    """One head of one sequence: dict name -> (value, bound) of out, lse, top
    and, with dout, dq, dk, dv."""
    u = HALF_STEP[dtype]
    nq, nk, d = len(q), len(k), q.shape[1]
    s = np.where(see, scale * (q @ k.T), -np.inf)
    size = scale * (np.abs(q) @ np.abs(k).T)
    big = float(np.where(see, size, 0.0).max(initial=0.0))
    top = s.max(axis=1, initial=-np.inf)
    base = np.where(np.isfinite(top), top, 0.0)
    p = np.exp(s - base[:, None])
    total = p.sum(axis=1)
    some = total > 0
    p = p / np.where(some, total, 1.0)[:, None]
    lse = np.where(some, base + np.log(np.where(some, total, 1.0)), -np.inf)
    reach = float(np.abs(lse[some]).max(initial=0.0))
    e = E32 * (2 * (d + 8) * (big + reach + 1) + nk) + 2.0 ** -22
    out = p @ v
    weight = p @ np.abs(v)
    got = {"out": (out, (u + e) * weight + u * (np.abs(out) + u * weight)),
           "lse": (lse, np.full(nq, 2 * e + 4 * E32 * (reach + 1))),
           "top": (float(top.max(initial=-np.inf)), E32 * (d + 8) * (big + 1))}
    if dout is None:
        return got
    r = u if dtype == "bf16" else 0.0       # rounding of p and ds before the products
    ea = E32 * (max(nq, nk, d) + 8)         # any binary32 sum, relative to its terms' sizes
    dp = dout @ v.T
    dp_err = ea * (np.abs(dout) @ np.abs(v).T)
    delta = (dout * out).sum(axis=1)
    # out is given to the backward pass as two bfloat16 (2^-16), or one binary32
    delta_err = ((2.0 ** -16 if dtype == "bf16" else E32) + ea) * (np.abs(dout) * np.abs(out)).sum(axis=1)
    ds = p * (dp - delta[:, None])
    ds_err = (r + 2 * e + 4 * E32) * np.abs(ds) + p * (dp_err + delta_err[:, None]) * (1 + r + e)
    dq, dk, dv = scale * ds @ k, scale * ds.T @ q, p.T @ dout
    sized = np.abs(ds) + ds_err
    for name, val, err in (
            ("dq", dq, scale * (ds_err @ np.abs(k) + ea * sized @ np.abs(k))),
            ("dk", dk, scale * (ds_err.T @ np.abs(q) + ea * sized.T @ np.abs(q))),
            ("dv", dv, (r + 2 * e + ea) * (p.T @ np.abs(dout)))):
        got[name] = (val, err)              # before the result's own rounding (heads are summed first)
    return got


def attention(q, k, v, dtype, scale=None, causal=False, window=0, seqs=None, dout=None):
    """q [B, Sq, Hq, D], k and v [B, Sk, Hkv, D].  seqs: (batch, q start, q
    length, k start, k length) of each sequence; default whole batches.  Rows
    of no sequence: zeros, lse -inf."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    B, sq, hq, d = q.shape
    sk, hkv = k.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    u = HALF_STEP[dtype]
    if seqs is None:
        seqs = [(b, 0, sq, 0, sk) for b in range(B)]
    got = {n: [np.zeros(s), np.zeros(s)] for n, s in (("out", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}
    got["lse"] = [np.full((B, hq, sq), -np.inf), np.zeros((B, hq, sq))]
    got["top"] = [np.full(hq, -np.inf), np.zeros(hq)]
    for b, i, nq, j, nk in seqs:
        see = visible(nq, nk, causal, window)
        for h in range(hq):
            g = h // (hq // hkv)
            do = None if dout is None else np.asarray(dout, dtype=np.float64)[b, i:i + nq, h]
            one = attention_head(q[b, i:i + nq, h], k[b, j:j + nk, g], v[b, j:j + nk, g], scale, see, dtype, do)
            for x in (0, 1):
                got["out"][x][b, i:i + nq, h] = one["out"][x]
                got["lse"][x][b, h, i:i + nq] = one["lse"][x]
                if do is not None:
                    got["dq"][x][b, i:i + nq, h] = one["dq"][x]
                    got["dk"][x][b, j:j + nk, g] += one["dk"][x]
                    got["dv"][x][b, j:j + nk, g] += one["dv"][x]
            got["top"][1][h] = max(got["top"][1][h], one["top"][1])
            got["top"][0][h] = max(got["top"][0][h], one["top"][0])
    for n in ("dq", "dk", "dv"):
        got[n][1] += u * (np.abs(got[n][0]) + got[n][1]) + (hq // hkv) * E32 * np.abs(got[n][0])
    return {n: tuple(x) for n, x in got.items()}


def rotary(x, positions, freqs, dtype, layout="half", scale=1.0, inverse=False):
    """x [B, S, H, D], positions [B, S]: (value, bound)."""
    x = np.asarray(x, dtype=np.float64)
    n = len(freqs)
    angle = np.asarray(positions, dtype=np.float64)[..., None, None] * np.asarray(freqs, dtype=np.float64)
    c, s = scale * np.cos(angle), scale * np.sin(angle) * (-1.0 if inverse else 1.0)
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    # the angle as a fraction of a turn in binary32 (2^-24 of up to pi), its
    # sine and cosine, their scaling, two products and a sum: 12 half steps of
    # the largest possible result; 64-bit reduction adds 2^-52 of the angle
    size = np.zeros_like(x)
    size[..., a] = size[..., b] = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    far = 2.0 ** -50 * (np.abs(angle).max(initial=0.0) + 1)
    bound = (12 * E32 + far) * size
    u = HALF_STEP[dtype]
    turned = np.zeros(x.shape[-1], dtype=bool)
    turned[: 2 * n] = True
    return y, np.where(turned, bound + u * (np.abs(y) + bound), 0.0)


def qk_clip(wq, wk, logits, threshold, dtype):
    """((wq', bound), (wk', bound))."""
    logits = np.asarray(logits, dtype=np.float64)
    hq = len(logits)
    hd = wq.shape[0] // hq
    hkv = wk.shape[0] // hd
    with np.errstate(invalid="ignore", divide="ignore"):
        gamma = np.where(np.isfinite(logits) & (logits > threshold), threshold / logits, 1.0)
    least = gamma.reshape(hkv, -1).min(axis=1)
    fq = np.repeat(gamma / np.repeat(np.sqrt(least), hq // hkv), hd)[:, None]
    fk = np.repeat(np.sqrt(least), hd)[:, None]
    u = HALF_STEP[dtype]
    res = []
    for w, f in ((wq, fq), (wk, fk)):
        y = np.asarray(w, dtype=np.float64) * f
        # factor: a quotient, a square root and a quotient in binary32, then
        # the product; rows with factor 1 keep their bits
        res.append((y, np.where(f == 1.0, 0.0, (u + 6 * E32) * np.abs(y) * (1 + u))))
    return res
