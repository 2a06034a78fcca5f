"""Negative log-likelihood of target codes under the joint softmax (oracle; test infrastructure).

Section 2.4 of the zip2zip paper trains with the usual next-token objective, taken over the compressed
sequence (its second displayed equation): every position contributes -log of the probability the joint
softmax over base tokens and hypertokens gives to the code that actually follows.  For hidden row r with
target code t (a base token, or V + e for entry e of the row's sequence):

    nll[r] = log-sum-exp_v(logits[r, v]) - logits[r, t]

over the V + C existing columns.  A negative target marks a position without a target (it contributes 0);
a target that names no existing column has probability zero (nll = +inf).
"""
from __future__ import annotations

import numpy as np

from .logits import extended_logits


def extended_nll(H: np.ndarray, W_base: np.ndarray, W_hyper: np.ndarray, C: int, dtype: str,
                 targets: np.ndarray) -> dict:
    """Rows of ONE sequence.  Returns dict(nll float64 [rows], lse float64 [rows])."""
    r = extended_logits(H, W_base, W_hyper, C, dtype, return_logits=True)
    lg, lse = r["logits"], r["lse"]
    n_cols = lg.shape[1]
    nll = np.zeros(lg.shape[0], dtype=np.float64)
    for i, t in enumerate(np.asarray(targets).tolist()):
        if t < 0:
            nll[i] = 0.0
        elif t >= n_cols:
            nll[i] = np.inf
        else:
            nll[i] = lse[i] - lg[i, t]
    return dict(nll=nll, lse=lse)


def extended_nll_backward(H: np.ndarray, W_base: np.ndarray, W_hyper: np.ndarray, C: int, dtype: str,
                          targets: np.ndarray, grad_nll: np.ndarray) -> dict:
    """Gradient of sum_r grad_nll[r] * nll[r] for the rows of ONE sequence (float64).

    With p = softmax(logits[r, :]) over the V + C existing columns and t the row's target,
    d nll[r] / d logits[r, v] = p[v] - [v == t].  Rows without a target (t < 0) and rows whose target names
    no existing column (nll = +inf: no finite gradient) contribute nothing.  From dZ = grad_nll[:, None] *
    (P - onehot):  dH = dZ W,  dW_base = dZ[:, :V]^T H,  dW_hyper[:C] = dZ[:, V:]^T H  (rows at and beyond C: 0).
    """
    from .numfmt import to_f64

    r = extended_logits(H, W_base, W_hyper, C, dtype, return_logits=True)
    lg, lse = r["logits"], r["lse"]
    V = W_base.shape[0]
    n_cols = lg.shape[1]
    H64, Wb, Wh = to_f64(H, dtype), to_f64(W_base, dtype), to_f64(W_hyper, dtype)
    dZ = np.exp(lg - lse[:, None])
    g = np.asarray(grad_nll, dtype=np.float64).copy()
    for i, t in enumerate(np.asarray(targets).tolist()):
        if 0 <= t < n_cols:
            dZ[i, t] -= 1.0
        else:
            g[i] = 0.0
    dZ *= g[:, None]
    W = np.concatenate([Wb, Wh[:C]])
    dWh = np.zeros_like(Wh)
    dWh[:C] = dZ[:, V:].T @ H64
    return dict(dH=dZ @ W, dW_base=dZ[:, :V].T @ H64, dW_hyper=dWh, dZ=dZ)


def hyper_embed_backward(dW_hyper: np.ndarray, entries, V: int, pool: str = "mean", w=()) -> np.ndarray:
    """Gradient through the pooling of ONE sequence's entries (float64): W_hyper[e] = sum_j a_j E[t_j], so
    dE[t_j] += a_j * dW_hyper[e] for every token of every entry (a token that occurs twice receives twice)."""
    from .embed import pool_coefficients

    dE = np.zeros((V, dW_hyper.shape[1]), dtype=np.float64)
    for e, toks in enumerate(entries):
        a = pool_coefficients(len(toks), pool, w)
        for j, t in enumerate(toks):
            dE[t] += a[j] * dW_hyper[e]
    return dE


def teacher_distribution(ids, teacher, T: float, n_cols: int):
    """One row's (columns, q, ln q) over what it lists, and whether some of it lies on a column that does not exist."""
    used = [(int(c), float(t)) for c, t in zip(ids, teacher) if c >= 0 and not float(t) == -np.inf]
    if not used:
        return np.zeros(0, dtype=np.int64), np.zeros(0), np.zeros(0), False
    cols = np.array([c for c, _ in used], dtype=np.int64)
    t = np.array([x for _, x in used], dtype=np.float64) / T
    keep = ~(t - t.max() < -87.0)                      # (what is e^-87 of the best listed column counts as nothing)
    cols, t = cols[keep], t[keep]
    ln_q = t - t.max()
    ln_q = ln_q - np.log(np.exp(ln_q).sum())
    return cols, np.exp(ln_q), ln_q, bool((cols >= n_cols).any())


def extended_distill(H: np.ndarray, W_base: np.ndarray, W_hyper: np.ndarray, C: int, dtype: str, ids: np.ndarray,
                     teacher: np.ndarray, T: float) -> dict:
    """Rows of ONE sequence against a teacher's listed logits: with q the softmax of the row's listed teacher logits / T
    and p the joint softmax at temperature T, kl[r] = sum_k q_k (ln q_k - ln p_{id_k}).  Negative ids, logits of -inf and
    those more than 87 T below the row's largest list nothing; a row that lists nothing has 0, one with mass on a column that does not exist +inf.
    Returns dict(kl, lse: ln sum exp(logit / T), student: the logits at ids, 0 where none is listed, logits), float64."""
    lg = extended_logits(H, W_base, W_hyper, C, dtype, return_logits=True)["logits"]
    n_cols = lg.shape[1]
    m = lg.max(axis=1, keepdims=True)
    lse = m[:, 0] / T + np.log(np.exp((lg - m) / T).sum(axis=1))
    kl = np.zeros(lg.shape[0])
    student = np.zeros(ids.shape)
    for r in range(lg.shape[0]):
        there = (ids[r] >= 0) & (ids[r] < n_cols)
        student[r, there] = lg[r, ids[r][there]]
        cols, q, ln_q, outside = teacher_distribution(ids[r], teacher[r], T, n_cols)
        if outside:
            kl[r] = np.inf
        elif len(cols):
            kl[r] = (q * (ln_q - (lg[r, cols] / T - lse[r]))).sum()
    return dict(kl=kl, lse=lse, student=student, logits=lg)


def extended_distill_backward(H: np.ndarray, W_base: np.ndarray, W_hyper: np.ndarray, C: int, dtype: str, ids: np.ndarray,
                              teacher: np.ndarray, T: float, grad_kl: np.ndarray) -> dict:
    """Gradient of sum_r grad_kl[r] * kl[r] for the rows of ONE sequence (float64): d kl / d logit_v = (p_v - sum of q on v) / T;
    rows that list nothing and rows with an infinite loss contribute nothing.  P: g p / T, for error bounds."""
    from .numfmt import to_f64

    f = extended_distill(H, W_base, W_hyper, C, dtype, ids, teacher, T)
    lg, lse = f["logits"], f["lse"]
    V, n_cols = W_base.shape[0], lg.shape[1]
    P = np.exp(lg / T - lse[:, None])
    dZ = P.copy()
    g = np.asarray(grad_kl, dtype=np.float64).copy() / T
    for r in range(lg.shape[0]):
        cols, q, _, outside = teacher_distribution(ids[r], teacher[r], T, n_cols)
        if outside or len(cols) == 0:
            g[r] = 0.0
            continue
        np.add.at(dZ[r], cols, -q)
    dZ *= g[:, None]
    P = P * np.abs(g)[:, None]
    H64, Wb, Wh = to_f64(H, dtype), to_f64(W_base, dtype), to_f64(W_hyper, dtype)
    W = np.concatenate([Wb, Wh[:C]])
    dWh = np.zeros_like(Wh)
    dWh[:C] = dZ[:, V:].T @ H64
    return dict(dH=dZ @ W, dW_base=dZ[:, :V].T @ H64, dW_hyper=dWh, dZ=dZ, P=P)
