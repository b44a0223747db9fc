"""fp64 oracle of 8-bit integer products and of the way from logits to probabilities
(test infrastructure only; shares no code with the kernels)."""
from __future__ import annotations

import numpy as np

import oracle

LEAST = 127.0 * 2.0 ** -126
MOST_COUNT = 32767


# ------------------------------------------------------- 8-bit products

def quantize(x):
    """Codes and scales of rows: 127 x / a to the nearest integer, ties to even.  127 x is
    exact in fp64 for x of 24 bits; the quotient of such numbers is a middle of two integers
    exactly or is farther from one than fp64 rounds."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x).all(axis=1)
    a = np.maximum(np.abs(np.where(fine[:, None], x, 0.0)).max(axis=1), LEAST)
    codes = np.rint(127.0 * np.where(fine[:, None], x, 0.0) / a[:, None]).astype(np.int64)
    return codes, np.where(fine, a / 127.0, np.nan)


def matmul_i8(a, a_scale, w, w_scale, bias=None):
    """(result, magnitude of the scaled sum) of the product, in 64 bits; sums in integers."""
    acc = np.asarray(a, np.int64) @ np.asarray(w, np.int64).T
    y = acc * (np.asarray(a_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64))
    return (y if bias is None else y + np.asarray(bias, np.float64)), np.abs(y)


def project_i8(H, wf, wf_scale, wkv, wkv_scale, f_e, carried, pos, L, Hkv, hd, theta, z_norm=None,
               k_norm=None, doubt=2.0 ** -11):
    """K and V rows [M][L][Hkv][hd] of the projection with 8-bit weights, and how far each may be
    off because z lies within ``doubt`` of the middle of two codes (fp32 sums decide there)."""
    q, s = quantize(H)
    z, _ = matmul_i8(q, s, wf, wf_scale)
    if f_e is not None:
        z = z + np.asarray(carried)[:, None] * np.asarray(f_e, np.float64)
    if z_norm is not None:
        z = oracle.rms_norm(z, np.asarray(z_norm, np.float64))
    q, s = quantize(z)
    unit = 127.0 * z / np.maximum(np.abs(z).max(axis=1, keepdims=True), LEAST)
    open_ = np.abs(np.abs(unit - np.floor(unit)) - 0.5) < doubt
    y, _ = matmul_i8(q, s, wkv, wkv_scale)
    off = (open_ * s[:, None]) @ np.abs(np.asarray(wkv, np.float64) * np.asarray(wkv_scale)[:, None]).T
    M = len(y)
    y, off = y.reshape(M, L, 2, Hkv, hd), off.reshape(M, L, 2, Hkv, hd)
    k, v = y[:, :, 0], y[:, :, 1]
    k_off, v_off = off[:, :, 0], off[:, :, 1]
    if k_norm is not None:
        g = np.asarray(k_norm, np.float64)[None, :, None]
        r = 1.0 / np.sqrt((k ** 2).mean(axis=-1, keepdims=True) + 1e-6)
        # (a key moves by its own change and by that of its head's root mean square)
        k_off = (k_off + np.abs(k) * np.sqrt((k_off ** 2).mean(-1, keepdims=True)) * r) * r * np.abs(g)
        k = k * r * g
    half = hd // 2
    k = oracle.rope(k, np.asarray(pos)[:, None, None], theta)
    pair = k_off[..., :half] + k_off[..., half:]
    size = np.abs(k[..., :half]) + np.abs(k[..., half:])
    return k, v, np.concatenate([pair, pair], -1), v_off, np.concatenate([size, size], -1)


# ------------------------------------------------------------- history

def count_tokens(seen, tokens, lens, prompt, fresh):
    """History words after one call; (words, status)."""
    seen = np.array(seen, dtype=np.uint16)
    S, V = seen.shape
    status = oracle.OK
    for s in range(S):
        n = tokens.shape[1] if lens is None else int(lens[s])
        if not 0 <= n <= tokens.shape[1]:
            status = oracle.ERR_LENGTH
            continue
        if fresh and n > 0:
            seen[s] = 0
        for t in tokens[s][:n]:
            if t < 0:
                continue
            if t >= V:
                status = oracle.ERR_TOKEN
                continue
            w = int(seen[s, t])
            seen[s, t] = w | 0x8000 if prompt else (w & 0x8000) | min((w & 0x7FFF) + 1, MOST_COUNT)
    return seen, status


# --------------------------------------------------------- logits' rules

def rules_row(x, word=None, window=(), repetition=1.0, presence=0.0, frequency=0.0, biases=(),
              allowed=None):
    """One row of logits after the rules, in 64 bits, and how far the same in fp32 may be off
    (half a step, 2^-24 of the value, at every operation).  word: the sequence's history words;
    window: proposals before the row; biases: (token, value) in their order; allowed: bools."""
    x = np.array(x, dtype=np.float64)
    err = np.zeros_like(x)
    V, half = len(x), 2.0 ** -24

    def put(at, y, e):
        with np.errstate(invalid="ignore"):
            err[at] = e + half * np.abs(y)
        x[at] = y

    with np.errstate(invalid="ignore", divide="ignore"):
        if word is not None:
            word = np.asarray(word).astype(np.int64) & 0xFFFF
            c = (word & 0x7FFF).astype(np.float64)
            for t in window:
                if 0 <= t < V:
                    c[t] = min(c[t] + 1, MOST_COUNT)
            known = np.flatnonzero(((word & 0x8000) != 0) | (c > 0))
            r = float(repetition)
            put(known, np.where(x[known] > 0, x[known] / r, x[known] * r), 0.0)
            made = np.flatnonzero(c > 0)
            fc = float(frequency) * c[made]
            put(made, x[made] - fc, err[made] + half * np.abs(fc))
            put(made, x[made] - float(presence), err[made])
        last = {int(t): float(b) for t, b in biases if 0 <= t < V}
        if last:
            at = np.array(list(last))
            put(at, x[at] + np.array(list(last.values())), err[at])
    if allowed is not None:
        allowed = np.asarray(allowed, dtype=bool)
        x[~allowed] = -np.inf
        err[~allowed] = 0.0
    return x, err


def probabilities_row(x, err, temperature=1.0):
    """(probabilities, tolerance, lowest token of the largest logit or -1) of one row after the
    rules.  Tolerance: a weight's exponent t = (x - max) / T, held in fp32 through the
    difference, the slope 1 / T in two operations and the product, moves by 2^-24 of itself at
    each, and with the logits' own error over T; the exponential is good to 2^-22; sums of up
    to 256 terms behind each other add 2^-24 each."""
    x = np.where(np.isnan(x), -np.inf, x)
    V = len(x)
    top = x.max()
    if top == -np.inf:
        return np.zeros(V), np.zeros(V), -1
    first = int(np.flatnonzero(x == top)[0])
    if not temperature > 0:
        p = np.zeros(V)
        p[first] = 1.0
        return p, np.zeros(V), first
    with np.errstate(invalid="ignore", over="ignore"):
        t = np.where(x == top, 0.0, (x - top) / temperature)
    w = np.exp(t)
    p = w / w.sum()
    ok = np.isfinite(t)
    t0 = np.where(ok, np.abs(t), 0.0)
    d = np.where(ok & np.isfinite(err), err, 0.0)
    rel = t0 * 8 * 2.0 ** -24 + 2 * (d + d[first]) / temperature
    # the sum moves as its terms do, weighted
    rel = rel + (rel * p).sum() + 2.0 ** -21 + 256 * 2.0 ** -24
    return p, p * np.expm1(rel) + 2.0 ** -126, first
