"""Lookup of code streams in the joint embedding table (oracle; test infrastructure).

Section 2.2 of the zip2zip paper embeds a compressed sequence through the base embeddings and the hyper-embeddings of
its own codebook: position i of a sequence with code c has the row c of [E ; W_hyper[:C]], times a scale.  A code that names
no row gives zeros.  The gradient is the transpose: every row receives scale times the sum over its positions.
"""
from __future__ import annotations

import numpy as np

from .numfmt import to_f64


def embed_codes(codes, E: np.ndarray, W_hyper: np.ndarray, C: int, dtype: str, scale: float) -> dict:
    """Codes of ONE sequence.  Returns dict(X float64 [n, d], bad bool): scale * rows, not rounded."""
    V, d = E.shape
    X = np.zeros((len(codes), d), dtype=np.float64)
    bad = False
    for i, c in enumerate(int(c) for c in codes):
        if 0 <= c < V:
            X[i] = to_f64(E[c], dtype) * scale
        elif V <= c < V + C:
            X[i] = to_f64(W_hyper[c - V], dtype) * scale
        else:
            bad = True
    return dict(X=X, bad=bad)


def embed_codes_backward(codes, dX: np.ndarray, V: int, C: int, cap: int, dtype: str, scale: float) -> dict:
    """Gradient for the codes of ONE sequence: dict(dE [V, d], dW_hyper [cap, d], terms: per row of [dE ; dW_hyper] how many
    positions named it, mass: the sum of |scale * dX| over them), float64."""
    g = to_f64(dX, dtype) * scale
    both = np.zeros((V + cap, dX.shape[1]), dtype=np.float64)
    mass = np.zeros_like(both)
    terms = np.zeros(V + cap, dtype=np.int64)
    for i, c in enumerate(int(c) for c in codes):
        if 0 <= c < V + C:
            both[c] += g[i]
            mass[c] += np.abs(g[i])
            terms[c] += 1
    return dict(dE=both[:V], dW_hyper=both[V:], terms=terms, mass=mass)
