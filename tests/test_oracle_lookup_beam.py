"""Pins of the oracle's code lookup, its gradient and the beam search's pick (CPU)."""
import itertools

import numpy as np
import pytest
import torch

import oracle


@pytest.mark.parametrize("scale", [1.0, 8.0, 0.3])
def test_lookup_is_the_librarys_embedding_of_the_joint_table_and_its_gradient(scale):
    rng = np.random.default_rng(3)
    V, cap, C, d, n = 20, 6, 4, 5, 40
    E, W = rng.normal(size=(V, d)).astype(np.float32), rng.normal(size=(cap, d)).astype(np.float32)
    codes = rng.integers(0, V + C, size=n)
    table = torch.tensor(np.concatenate([E, W]).astype(np.float64), requires_grad=True)
    X = torch.nn.functional.embedding(torch.tensor(codes), table) * scale
    r = oracle.embed_codes(codes, E, W, C, "f32", scale)
    assert not r["bad"] and np.allclose(r["X"], X.detach().numpy(), rtol=1e-15, atol=0)
    g = rng.normal(size=(n, d)).astype(np.float32)
    X.backward(torch.tensor(g.astype(np.float64)))
    b = oracle.embed_codes_backward(codes, g, V, C, cap, "f32", scale)
    assert np.allclose(np.concatenate([b["dE"], b["dW_hyper"]]), table.grad.numpy(), rtol=1e-13, atol=1e-15)
    assert b["terms"].sum() == n
    # central differences of the forward pass along a random direction
    D, eps = rng.normal(size=(V + cap, d)), 1e-4
    f = lambda t: (oracle.embed_codes(codes, t[:V].astype(np.float32), t[V:].astype(np.float32), C, "f32", scale)["X"] * g).sum()
    T = np.concatenate([E, W]).astype(np.float64)
    num = (f(T + eps * D) - f(T - eps * D)) / (2 * eps)
    assert abs(num - (np.concatenate([b["dE"], b["dW_hyper"]]) * D).sum()) < 2e-2 * max(1.0, abs(num))


@pytest.mark.parametrize("code", [-1, -2**31, 24, 26, 2**31 - 1])
def test_codes_that_name_nothing(code):
    E, W = np.ones((20, 3), dtype=np.float32), np.ones((6, 3), dtype=np.float32)
    r = oracle.embed_codes([1, code, 23], E, W, 4, "f32", 2.0)
    assert r["bad"] and (r["X"] == [[2.0] * 3, [0.0] * 3, [2.0] * 3]).all()
    b = oracle.embed_codes_backward([1, code, 23], np.ones((3, 3), dtype=np.float32), 20, 4, 6, "f32", 2.0)
    assert b["terms"].sum() == 2 and b["dE"].sum() + b["dW_hyper"].sum() == 12.0


def test_pick_is_the_best_of_all_sequences_of_one_step():
    rng = np.random.default_rng(5)
    logits = [rng.normal(size=9), rng.normal(size=7), rng.normal(size=8)]
    score = np.array([-0.5, -0.1, -2.0])
    lse = [np.log(np.exp(x).sum()) for x in logits]
    got = oracle.beam_pick(oracle.continuations(logits, lse, score), 5)
    every = sorted((score[r] + np.log(np.exp(logits[r][c]) / np.exp(logits[r]).sum()) for r in range(3) for c in range(len(logits[r]))), reverse=True)
    assert np.allclose([v for v, _, _ in got], every[:5], atol=1e-12)
    assert all(abs(score[r] + logits[r][c] - lse[r] - v) < 1e-12 for v, r, c in got)
    # equal values: lower beam, then lower column; dead beams and NaN are left out
    flat = oracle.continuations([np.zeros(3)] * 3, [0.0] * 3, [-1.0, -np.inf, -1.0])
    assert [(r, c) for _, r, c in oracle.beam_pick(flat, 10)] == [(0, 0), (0, 1), (0, 2), (2, 0), (2, 1), (2, 2)]
    flat[0][1] = np.nan
    assert [(r, c) for _, r, c in oracle.beam_pick(flat, 10)] == [(0, 0), (0, 2), (2, 0), (2, 1), (2, 2)]


def test_reordered_streams_go_on_as_if_they_had_read_the_sources_history():
    V, M, cap = 5, 3, 20
    hist = [[1, 2, 1, 2, 3], [4, 4, 4, 4], [0, 1, 0, 1, 0]]
    for source in itertools.product([-1, 0, 1, 2, 3], repeat=3):
        states = []
        for h in hist:
            s = oracle.LZWStream(V, M, cap)
            s.encode_chunk(h)
            states.append(s)
        moved = oracle.beam_reorder(states, source)
        for k, s in enumerate(source):
            fresh = oracle.LZWStream(V, M, cap)
            fresh.encode_chunk(hist[s if 0 <= s < 3 else k])
            assert moved[k].entries == fresh.entries
            assert moved[k].encode_chunk([1, 2, 1, 0]) == fresh.encode_chunk([1, 2, 1, 0])
