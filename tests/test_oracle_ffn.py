"""The oracle of the gated block, 4-bit weights and clipping: against finite differences, library routines and closed forms."""
import math

import numpy as np
import pytest
import torch

import oracle


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_block_and_gradient(kind):
    rng = np.random.default_rng(5)
    n, d, f = 5, 12, 7
    X, W1, W2, R, dY = (rng.normal(size=s) for s in ((n, d), (2 * f, d), (d, f), (n, d), (n, d)))
    t = [torch.tensor(x, dtype=torch.float64, requires_grad=True) for x in (X, W1, W2)]
    GU = t[0] @ t[1].T
    a = torch.nn.functional.silu(GU[:, :f]) if kind == "silu" else torch.nn.functional.gelu(GU[:, :f])
    Y = (a * GU[:, f:]) @ t[2].T + torch.tensor(R)
    Y.backward(torch.tensor(dY))
    ref = oracle.gated_ffn(X, W1, W2, kind, R)
    assert np.allclose(ref["Y"], Y.detach().numpy(), rtol=1e-12, atol=1e-12)
    back = oracle.gated_ffn_backward(X, W1, W2, kind, dY)
    for name, x in zip(("dX", "dW1", "dW2"), t):
        assert np.allclose(back[name], x.grad.numpy(), rtol=1e-10, atol=1e-12), name
    # differences
    eps = 1e-6
    for name, x, at in (("dX", X, (2, 3)), ("dW1", W1, (9, 4)), ("dW1", W1, (1, 4)), ("dW2", W2, (5, 6))):
        kept = x[at]
        x[at] = kept + eps
        up = np.sum(oracle.gated_ffn(X, W1, W2, kind, R)["Y"] * dY)
        x[at] = kept - eps
        down = np.sum(oracle.gated_ffn(X, W1, W2, kind, R)["Y"] * dY)
        x[at] = kept
        assert abs((up - down) / (2 * eps) - back[name][at]) < 1e-6 * max(1, abs(back[name][at]))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_steepness_that_the_bounds_assume(kind):
    x = np.linspace(-12, 12, 200001)
    value, slope = oracle.ffn.act(x, kind)
    assert np.max(np.abs(slope)) < 1.13
    assert np.max(np.abs(np.diff(slope) / np.diff(x))) < 0.8
    assert np.allclose(np.diff(value) / np.diff(x), (slope[1:] + slope[:-1]) / 2, atol=1e-6)


def _bf16(x):
    return oracle.bf16_bits_to_f64(oracle.f64_to_bf16_bits(np.nan_to_num(x, nan=0.0, posinf=0.0)))


def test_four_bits():
    rng = np.random.default_rng(6)
    W = oracle.bf16_bits_to_f64(oracle.f64_to_bf16_bits(rng.normal(size=(16, 192))))
    W[3, 64:128] = 0.0
    W[4, 5] = math.inf
    W[5, 70] = math.nan
    W[6, 128:136] = [6, 0.25, 0.75, 1.25, -1.75, 2.5, -3.5, 5]
    W[6, 136:192] = 0
    q, scale = oracle.quantize_q4(W, 64, _bf16)
    value = oracle.q4_weights(q, scale, 64)
    ok = np.isfinite(value)
    assert (~ok).sum() == 2 * 64 and np.isnan(scale[0, 4]) and np.isnan(scale[1, 5])
    # the widest gap is from 4 to 6; where the scale was rounded down, the largest by what that leaves of six steps
    assert np.all(np.abs(value - W)[ok] <= (scale.T.repeat(64, axis=1) * (1.0 + 6 * 2.0 ** -8))[ok])
    nearest = np.min(np.abs(W[0, :64, None] - scale[0, 0] * oracle.ffn.Q4_VALUES), axis=1)
    assert np.allclose(np.abs(value - W)[0, :64], nearest, atol=1e-15)
    assert np.all(q[3, 64:128] == 0) and scale[1, 3] == 0
    assert value[6, 128:136].tolist() == [6, 0, 1, 1, -2, 2, -4, 4] and scale[2, 6] == 1
    words = oracle.q4_words(q)
    assert words.shape == (1, 2, 64, 4)
    assert np.all(words[0, 1, :, 2:] == 0)                                             # columns 192 .. 255
    row, col = 7, 64 + 32 + 16 + 5                                                     # m = 3, j = 2, column 5 of eight
    assert (int(words[0, 0, 2 * 16 + row, 3]) >> 20) & 15 == q[row, col]


def test_clip():
    a, b = np.array([3.0, 0.0]), np.array([[4.0]])
    norm, c, out = oracle.clip([a, b], 1.0)
    assert norm == 5 and c == 0.2 and np.allclose(out[0], [0.6, 0]) and np.allclose(out[1], 0.8)
    assert oracle.clip([a, b], 6.0)[1] == 1.0 and oracle.clip([a * 0], 0.0)[:2] == (0.0, 1.0)
    assert oracle.clip([np.array([math.inf])], 1.0)[1] == 1.0 and math.isnan(oracle.clip([np.array([math.nan])], 1.0)[0])


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_encoder(kind):
    """A gated layer is the attention layer and the block behind it; its gradient, against differences."""
    from paper_2506_01084_amd import workloads as wl

    cfg = dict(d=16, M=3, dtype="f32", seed=4)
    enc = wl.make_encoder(cfg, n_layers=2, n_heads=2, d_ff=24, gated=kind)
    assert enc["layers"][0]["w_1"].shape == (48, 16) and "b_1" not in enc["layers"][0]
    E = wl.normal_matrix(8, 9, 16, 0.6, "f32")
    entries = [(0, 3), (4, 4, 1), (2, 8)]
    one = dict(enc, layers=enc["layers"][:1])
    attention = dict(one, gated=None, attention_only=True)
    lay = one["layers"][0]
    for e in entries:                                       # one slot at a time of a layer's output: the mean of one
        X = E[list(e)].astype(np.float64) + enc["pos"][:len(e)]
        A64, full = oracle.encoder.widen_encoder(attention, "f32"), oracle.encoder.widen_encoder(one, "f32")
        Y = X + oracle.encoder.attention(oracle.encoder.layer_norm(X, lay["ln1_g"], lay["ln1_b"]), lay["w_qkv"].astype(np.float64),
                                         lay["b_qkv"], lay["w_o"].astype(np.float64), lay["b_o"], 2)
        assert np.allclose(Y.mean(axis=0), oracle.encoder.encode_entry(X, A64))
        block = oracle.gated_ffn(oracle.encoder.layer_norm(Y, lay["ln2_g"], lay["ln2_b"]), lay["w_1"].astype(np.float64),
                                 lay["w_2"].astype(np.float64), kind, Y)["Y"]
        assert np.allclose(block.mean(axis=0), oracle.encoder.encode_entry(X, full), atol=1e-12)
    rng = np.random.default_rng(2)
    dW = rng.normal(size=(3, 16))
    grad = oracle.hyper_encode_backward(E, "f32", entries, enc, dW)

    def loss(enc64, table):
        total = 0.0
        for i, e in enumerate(entries):
            total += float(dW[i] @ oracle.encoder.encode_entry(table[list(e)] + enc64["pos"][:len(e)], enc64))
        return total

    e64, table, eps = oracle.encoder.widen_encoder(enc, "f32"), E.astype(np.float64), 1e-6
    for where, x, at, want in [(l, e64["layers"][l][k], at, grad["layers"][l][k][at]) for l in (0, 1)
                               for k, at in (("w_1", (30, 5)), ("w_1", (3, 7)), ("w_2", (9, 20)), ("ln2_g", (4,)), ("w_qkv", (40, 2)))] + [("E", table, (4, 6), grad["dE"][4, 6])]:
        was = x[at]
        x[at] = was + eps
        up = loss(e64, table)
        x[at] = was - eps
        down = loss(e64, table)
        x[at] = was
        assert abs((up - down) / (2 * eps) - want) < 1e-7 * max(1, abs(want)), where
