"""The gated feed-forward block, 4-bit weights and gradient clipping (oracle; test infrastructure).

Section 2.2 of the zip2zip paper trains a transformer as hyper-encoder; the gated form of its feed-forward block is
    G = X W1[:f]^T,  U = X W1[f:]^T,  F = act(G) * U,  Y = F W2^T + residual,
act = SiLU or GELU (erf).  A 4-bit weight is scale[column // group, row] times one of
0, 1/2, 1, 3/2, 2, 3, 4, 6, with a sign.  Everything is float64; with each result comes an
elementwise bound on how far a computation may be off that rounds F (and, backward, dG and dU) to bf16 once
and forms its sums in float32.
"""
from __future__ import annotations

import math

import numpy as np

HALF_BF16 = 2.0 ** -8                    # half a step of bf16, relative to the value
HALF_F32 = 2.0 ** -24
KEPT = 2.0 ** -16                        # half a step of 15 bits of fraction: a number's upper 24 bits are its sign, 8 of exponent and these
ACT_ERROR = 1e-6                         # of the activations' and slopes' own arithmetic in float32 (their erf: 1.5e-7; exponentials, reciprocals: a few steps)

_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(x: np.ndarray, kind: str):
    """(value, slope) of the activation."""
    if kind == "silu":
        with np.errstate(over="ignore"):
            p = 1.0 / (1.0 + np.exp(-x))
        return x * p, p + x * p * (1.0 - p)
    p = 0.5 * (1.0 + _erf(x / math.sqrt(2.0)))
    return x * p, p + x * np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)


def _sum_bound(A: np.ndarray, B: np.ndarray) -> np.ndarray:
    """How far A @ B may be off in float32: every one of n additions rounds a partial sum of at most the terms' magnitudes."""
    return (A.shape[1] + 8) * HALF_F32 * (np.abs(A) @ np.abs(B))


def _sixteen_bits(x, err):
    """How far numbers that are `err` off x may be moved by 16 bits: half a step of 9 bits of fraction from 2^-16 to 2^16, of 6 elsewhere."""
    size = np.abs(x)
    near = (size - err >= 2.0 ** -16) & (size + err < 2.0 ** 16 * (1 - 2.0 ** -10))
    return np.where(near, 2.0 ** -10, 2.0 ** -7) * (size + err)


def gated_ffn(X, W1, W2, kind: str, residual=None, round_weights: bool = False, kept16: bool = False):
    """dict(Y, Y_bound, G, U, F and their bounds).  round_weights: the weights may each be rounded to bf16; kept16: G and U to 16 bits (as a gradient may have them)."""
    f = W2.shape[1]
    GU = X @ W1.T
    gu_err = _sum_bound(X, W1.T) + (HALF_BF16 * (np.abs(X) @ np.abs(W1).T) if round_weights else 0.0)
    if kept16:
        gu_err = gu_err + _sixteen_bits(GU, gu_err)
    G, U = GU[:, :f], GU[:, f:]
    g_err, u_err = gu_err[:, :f], gu_err[:, f:]
    a, _ = act(G, kind)
    F = a * U
    a_err = 1.13 * g_err + ACT_ERROR * (np.abs(G) + 1e-30)       # (neither activation is steeper than 1.13)
    F_err = (a_err * (np.abs(U) + u_err) + np.abs(a) * u_err) * 1.01 + HALF_BF16 * np.abs(F) * 1.01
    Y = F @ W2.T + (0.0 if residual is None else residual)
    w2 = np.abs(W2).T
    Y_err = F_err @ w2 + _sum_bound(F, W2.T) + (HALF_BF16 * (np.abs(F) @ w2) if round_weights else 0.0)
    Y_bound = (Y_err * 1.02 + HALF_BF16 * (np.abs(Y) + Y_err)) * 1.001 + 1e-30
    # what the gradient needs: act(G) and U act'(G), which may be stored with 15 bits of fraction
    slope = act(G, kind)[1]
    slope_err = 0.8 * g_err + 4 * ACT_ERROR                      # (neither slope changes faster than 0.8)
    a_bound = a_err + KEPT * (np.abs(a) + a_err) + 1e-30
    s_bound = (u_err * (np.abs(slope) + slope_err) + np.abs(U) * slope_err) * 1.01
    s_bound = s_bound + KEPT * (np.abs(U * slope) + s_bound) + 1e-30
    return dict(Y=Y, Y_bound=Y_bound, Y_err=Y_err, G=G, U=U, F=F, F_err=F_err, a=a, a_bound=a_bound, s=U * slope, s_bound=s_bound)


def gated_ffn_backward(X, W1, W2, kind: str, dY, kept16: bool = False):
    """dict of dX, dW1, dW2 and their bounds (name + "_bound").  kept16: from G and U in 16 bits."""
    f = W2.shape[1]
    forward = gated_ffn(X, W1, W2, kind, kept16=kept16)
    F, F_err, a, a_err, s, s_err = (forward[k] for k in ("F", "F_err", "a", "a_bound", "s", "s_bound"))
    dF = dY @ W2
    dF_err = _sum_bound(dY, W2)
    dG, dU = dF * s, dF * a
    big = np.abs(dF) + dF_err
    dG_err = (big * s_err + dF_err * np.abs(s)) * 1.01 + HALF_BF16 * np.abs(dG) * 1.01
    dU_err = (big * a_err + dF_err * np.abs(a)) * 1.01 + HALF_BF16 * np.abs(dU) * 1.01
    D, D_err = np.concatenate([dG, dU], axis=1), np.concatenate([dG_err, dU_err], axis=1)
    out = {}
    for name, A, A_err, B in (("dX", D, D_err, W1), ("dW1", D.T, D_err.T, X), ("dW2", dY.T, np.zeros_like(dY.T), F)):
        value = A @ B
        err = A_err @ np.abs(B) + _sum_bound(A, B)
        if name == "dW2":
            err = err + np.abs(A) @ F_err
        out[name] = value
        out[name + "_err"] = err
        out[name + "_bound"] = (err * 1.02 + HALF_BF16 * (np.abs(value) + err)) * 1.001 + 1e-30
    return out


Q4_VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def quantize_q4(W: np.ndarray, group: int, round_bf16):
    """W [rows, cols] float64 (bf16 values) -> codes [rows, cols] in 0..15 and scales [cols / group, rows] as float64.  round_bf16: float64 -> the nearest bf16
    value.  The quotient by 6 is rounded to float32 first, as the definition's arithmetic is."""
    rows, cols = W.shape
    w = W.reshape(rows, cols // group, group)
    most = np.max(np.abs(w), axis=2)
    finite = np.isfinite(w).all(axis=2)
    with np.errstate(invalid="ignore"):
        scale = round_bf16((most.astype(np.float32) / np.float32(6)).astype(np.float64))
    scale = np.where(finite, scale, np.nan)
    with np.errstate(invalid="ignore", divide="ignore"):
        x = np.abs(w / scale[:, :, None])
        off = np.abs(x[..., None] - Q4_VALUES[:8])
    off = np.where(np.isfinite(off), off, np.inf)
    even_first = [0, 2, 4, 6, 1, 3, 5, 7]                       # (the first of the nearest: of two as near, the even code)
    code = np.array(even_first)[np.argmin(off[..., even_first], axis=-1)]
    code = np.where(finite[:, :, None] & (scale[:, :, None] > 0), code, 0)
    code = np.where((code > 0) & (w < 0), code + 8, code)
    return code.astype(np.int64).reshape(rows, cols), scale.T


def q4_words(q: np.ndarray) -> np.ndarray:
    """codes [rows, cols] -> words uint32 [rows / 16, ceil(cols / 128), 64, 4], element by element."""
    rows, cols = q.shape
    out = np.zeros((rows // 16, (cols + 127) // 128, 64, 4), dtype=np.uint32)
    for row in range(rows):
        for col in range(cols):
            block, in_block = divmod(col, 128)
            m, rest = divmod(in_block, 32)
            j, c = divmod(rest, 8)
            out[row // 16, block, 16 * j + row % 16, m] |= np.uint32(q[row, col]) << np.uint32(4 * c)
    return out


def q4_weights(q: np.ndarray, scale: np.ndarray, group: int) -> np.ndarray:
    return Q4_VALUES[q] * scale.T.repeat(group, axis=1)


def clip(gradients, max_norm: float):
    """(norm, coefficient, clipped float64 tensors)."""
    total = 0.0
    for g in gradients:
        total += float(np.sum(np.square(g.astype(np.float64))))
    norm = math.sqrt(total) if total == total else math.nan
    c = max_norm / norm if math.isfinite(norm) and norm > max_norm else 1.0
    return norm, c, [g.astype(np.float64) * c for g in gradients]
