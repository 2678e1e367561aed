"""Plain CPU oracle for the model operators of a stage: query/key norm with rotary positions, the loss against a teacher's
top logits, 8-bit products.

TEST INFRASTRUCTURE.  Only the tests, the smoke check and the benchmark's CPU-baseline leg may import this file.  It shares no
code with the CUDA library and never calls it.  Everything is numpy in float64, written from the definitions.

Pins (tests/test_stage_oracle_pins.py): the rotation keeps the norm of every pair and composes (angle of a plus angle of b is
the angle of a + b); both gradients agree with central differences; the loss is 0 where student and teacher agree on the
whole vocabulary and never negative; the quantised rows are within half a step.
"""

from __future__ import annotations

import numpy as np


def rope_table(max_pos: int, rot_dim: int, theta: float) -> np.ndarray:
    freq = float(theta) ** (-np.arange(0, rot_dim, 2, dtype=np.float64) / rot_dim)
    angle = np.arange(max_pos, dtype=np.float64)[:, None] * freq
    return np.concatenate((np.cos(angle), np.sin(angle)), axis=1)


def pair_columns(rot_dim: int, pairing: str):
    """The two columns of every pair."""
    i = np.arange(rot_dim // 2)
    return (i, i + rot_dim // 2) if pairing == "halves" else (2 * i, 2 * i + 1)


def rotate(x: np.ndarray, rows: np.ndarray, pairing: str, sign: float = 1.0) -> np.ndarray:
    """x [n, heads, D] with its pairs turned by sign times the angles of rows [n, rot_dim] (cosines, then sines)."""
    half = rows.shape[1] // 2
    a, b = pair_columns(2 * half, pairing)
    c, s = rows[:, None, :half], sign * rows[:, None, half:]
    out = np.array(x, dtype=np.float64)
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    return out


def table_rows(table: np.ndarray, pos: np.ndarray):
    """The table row of every position (zeros where there is none), and whether any position was outside the table."""
    ok = (pos >= 0) & (pos < len(table))
    rows = np.where(ok[:, None], np.asarray(table, dtype=np.float64)[np.where(ok, pos, 0)], 0.0)
    return rows, bool((~ok).any())


def qk_norm(x: np.ndarray, w, eps: float):
    """(x / sqrt(mean x^2 + eps) * w, the reciprocal root per row)"""
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    n = x * r
    return (n if w is None else n * w), r


def qk_rope_forward(x, w, rows, pairing: str, eps: float) -> np.ndarray:
    return rotate(qk_norm(x, w, eps)[0], rows, pairing)


def qk_rope_backward(dy, x, w, rows, pairing: str, eps: float):
    """(dx, dw)"""
    r = qk_norm(x, None, eps)[1]
    u = x * r
    g = rotate(dy, rows, pairing, -1.0)
    h = g if w is None else g * w
    return r * (h - u * (h * u).mean(axis=-1, keepdims=True)), (g * u).sum(axis=(0, 1))


def distill_loss(logits, ids, top, weight, tau: float):
    """(loss [n], dlogits [n, vocab]) row by row; ids outside [0, vocab) are padding."""
    logits, top = np.asarray(logits, np.float64), np.asarray(top, np.float64)
    n, vocab = logits.shape
    loss, grad = np.zeros(n), np.zeros((n, vocab))
    for t in range(n):
        there = (ids[t] >= 0) & (ids[t] < vocab)
        w = 1.0 if weight is None else float(weight[t])
        if w == 0.0 or not (there & (top[t] != -np.inf)).any():
            continue
        a = top[t][there] / tau
        p = np.exp(a - a.max())
        p = p / p.sum()
        x = logits[t] / tau
        m = x.max()
        e = np.exp(x - m)
        logq = x - m - np.log(e.sum())
        for j, pj in zip(ids[t][there], p):
            if pj > 0:
                loss[t] += w * tau * tau * pj * (np.log(pj) - logq[j])
        grad[t] = w * tau * e / e.sum()
        np.subtract.at(grad[t], ids[t][there], w * tau * p)
    return loss, grad


def int8_quantize(x: np.ndarray):
    """(q [n, K], scale [n] as the fp32 number it is) of a float64 matrix that holds fp32 or bf16 values.  A row with a value
    that is not finite: q = 0, scale NaN."""
    x = np.asarray(x, dtype=np.float64)
    top = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(len(x))
    fine = np.isfinite(top)
    scale = (np.where(fine, top, 0.0).astype(np.float32) / np.float32(127)).astype(np.float32)
    q = np.zeros(x.shape)
    for t in range(len(x)):
        if fine[t] and scale[t] > 0:
            q[t] = np.clip(np.rint(x[t] / float(scale[t])), -127, 127)   # a quotient of an fp32 pair is exact enough in 64 bits
    return q, np.where(fine, scale, np.float32(np.nan))


def int8_matmul(xq, xs, wq, ws) -> np.ndarray:
    total = np.asarray(xq, np.int64) @ np.asarray(wq, np.int64).T
    return total.astype(np.float64) * np.asarray(xs, np.float64)[:, None] * np.asarray(ws, np.float64)
