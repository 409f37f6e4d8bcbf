"""The operators over label logits from their definitions, in 64 bits on the CPU (NumPy)."""
from __future__ import annotations

import numpy as np
import torch

EMPTY = 2 ** 31 - 1
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(t, dtype):
    """Half a step of a 16- or 32-bit type at the values t (its smallest step near zero)."""
    fi = torch.finfo(DTYPES[dtype])
    return np.maximum(np.abs(t) * fi.eps / 2, fi.smallest_normal * fi.eps / 2)


# ---------------------------------------------------------------- MXFP4
def quantize(x):
    """(values, codes [rows, cols], scale bytes) of MXFP4 for float64 x."""
    rows, cols = x.shape
    b = x.reshape(rows, cols // 32, 32)
    big = np.abs(b).max(-1)
    bad = ~np.isfinite(big)
    with np.errstate(all="ignore"):
        e = np.floor(np.log2(np.where(bad | (big == 0), 1.0, big))).astype(int)
    # log2 may round up next to a power of two
    e = np.where(np.ldexp(1.0, e) > np.where(bad | (big == 0), 1.0, big), e - 1, e)
    e = np.clip(np.where(big == 0, -127, e - 2), -127, 127)
    y = np.where(bad[..., None], 0.0, b) * np.ldexp(1.0, -e)[..., None]
    a = np.abs(y)
    code = np.zeros(a.shape, int)
    for c in range(7):
        mid = (GRID[c] + GRID[c + 1]) / 2
        code += (a > mid) | ((a == mid) & (c % 2 == 1))  # ties to the even code
    sign = (y < 0).astype(int)
    values = np.where(bad[..., None], np.nan, np.where(sign == 1, -1.0, 1.0) * GRID[code] * np.ldexp(1.0, e)[..., None])
    return (values.reshape(rows, cols), (code + 8 * sign).reshape(rows, cols), np.where(bad, 255, e + 127))


def unpack(codes):
    """[rows, cols / 2] bytes as [rows, cols] codes."""
    out = np.empty((codes.shape[0], codes.shape[1] * 2), int)
    out[:, 0::2], out[:, 1::2] = codes & 15, codes >> 4
    return out


def values_of(codes, scales):
    c = unpack(codes)
    v = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return v * np.repeat(s, 32, 1)


# ---------------------------------------------------------------- ranking
def scores(z, bias=None, seen=None, row_bias=None, repetition=1.0, frequency=0.0, presence=0.0):
    """float32 scores; seen: list of id lists, row_bias: list of (ids, values)."""
    B, L = z.shape
    x = z.astype(np.float64).copy()
    for r in range(B):
        if seen is not None:
            ids = np.asarray(seen[r], np.int64)
            ids, n = np.unique(ids[(ids >= 0) & (ids < L)], return_counts=True)
            with np.errstate(all="ignore"):
                t = np.where(x[r, ids] > 0, x[r, ids] / repetition, x[r, ids] * repetition)
                x[r, ids] = t - frequency * n - presence
        with np.errstate(all="ignore"):
            if bias is not None:
                x[r] += bias
            if row_bias is not None:
                last = {int(i): float(v) for i, v in zip(*row_bias[r]) if 0 <= i < L}
                for i, v in last.items():
                    x[r, i] += v
    with np.errstate(all="ignore"):
        return x.astype(np.float32)


def topk(s, k, allowed=None):
    """(ids, scores, lse) of float32 scores s."""
    B, L = s.shape
    ids = np.full((B, k), EMPTY, np.int64)
    top = np.full((B, k), -np.inf, np.float32)
    lse = np.full(B, -np.inf)
    for r in range(B):
        ok = ~np.isnan(s[r])
        if allowed is not None:
            ok &= allowed[r]
        j = np.nonzero(ok)[0]
        v = s[r, j]
        order = np.argsort(-v.astype(np.float64), kind="stable")[:k]
        ids[r, :len(order)], top[r, :len(order)] = j[order], v[order]
        if len(j):
            m = v.max().astype(np.float64)
            lse[r] = m if np.isinf(m) else m + np.log(np.exp(v.astype(np.float64) - m).sum())
    return ids, top, lse


def lse_bound(lse, columns):
    """How far a float32 log-sum-exp may be: its own rounding, one step of every exponential
    and its argument (at most 0.4 steps, x e^-x being at most 1 / e), and one rounding of the sum per
    addition, at most columns / 256 on a lane, 64 lanes and waves, and 20 pieces' merges."""
    return np.abs(np.where(np.isfinite(lse), lse, 0)) * 2.0 ** -23 + (columns / 256 + 32) * 2.0 ** -23


# ---------------------------------------------------------------- distillation
def distill(z, t_ids, t_logits, T, weights=None):
    """(loss rows, gradient, p, target distribution)."""
    B, L = z.shape
    z = z.astype(np.float64)
    loss, grad, p_all, q_all = np.zeros(B), np.zeros((B, L)), np.zeros((B, L)), np.zeros((B, L))
    w = np.full(B, 1.0 / B) if weights is None else np.asarray(weights, np.float64)
    for r in range(B):
        on = (t_ids[r] >= 0) & (t_ids[r] < L) & np.isfinite(t_logits[r])
        if not on.any():
            continue
        if np.isnan(z[r]).any() or np.isposinf(z[r]).any():
            loss[r], grad[r], p_all[r] = np.nan, np.nan, np.nan
            continue
        ids, t = t_ids[r][on].astype(np.int64), t_logits[r][on].astype(np.float64) / T
        q = np.exp(t - t.max())
        q /= q.sum()
        x = z[r] / T
        m = x.max()
        if np.isneginf(m):
            p, log_p = np.zeros(L), np.full(L, -np.inf)
        else:
            with np.errstate(all="ignore"):
                log_p = x - m - np.log(np.exp(x - m).sum())
            p = np.exp(log_p)
        with np.errstate(all="ignore"):
            loss[r] = T * T * np.where(q > 0, q * (np.log(np.where(q > 0, q, 1.0)) - log_p[ids]), 0.0).sum()
        np.add.at(q_all[r], ids, q)
        p_all[r] = p
        grad[r] = w[r] * T * (p - q_all[r])
    return loss, grad, p_all, q_all
