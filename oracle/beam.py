"""The pick of a beam search over the joint softmax, and the move of the beams' codebooks (oracle; test infrastructure).

Section 2.3 of the zip2zip paper, step 9, leaves open how the next token is picked from the joint distribution; here it
is the step of a beam search over a prompt's beams: every continuation (beam r, column v) is worth

    score[r] + logit[r, v] - lse[r]

and the n best are picked, largest first, equal ones by lower beam, then lower column.  Continuations that are not finite
are left out.
"""
from __future__ import annotations

import copy

import numpy as np


def continuations(logits, lse, score) -> list:
    """Per beam the float64 values of its columns.  logits: per beam an array over its own V + C columns."""
    return [score[r] + np.asarray(logits[r], dtype=np.float64) - lse[r] for r in range(len(logits))]


def beam_pick(values, n: int) -> list:
    """The n best (value, beam, column) of `continuations`, in order; fewer where there are fewer."""
    every = [(float(v), r, c) for r, row in enumerate(values) for c, v in enumerate(row) if np.isfinite(v)]
    every.sort(key=lambda x: (-x[0], x[1], x[2]))
    return every[:n]


def beam_reorder(states, source) -> list:
    """One prompt's beam states after the move: state k becomes a copy of state source[k] (no such beam: stays)."""
    n = len(states)
    return [copy.deepcopy(states[s if 0 <= s < n else k]) for k, s in enumerate(source)]
