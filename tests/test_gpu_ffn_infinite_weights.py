"""Infinities and NaN among a gated block's bf16 weights: an output is what the sum over its own columns is, whichever kernel serves the rows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ffn import _context, _host, _tensors  # noqa: E402


# few rows in one launch (widths of whole units of 128 columns, and of half a one more), small tiles, weights that are streamed, the tile kernel
SHAPES = [(1, 64, 64), (3, 192, 64), (16, 128, 192), (16, 320, 448), (2, 256, 128), (33, 512, 320), (70, 192, 192), (300, 64, 64), (40, 8192, 5504), (1100, 3520, 1792)]


@pytest.mark.parametrize("rows,d,f", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_second_matrix(rows, d, f, act):
    from paper_2506_01084_amd import api

    X, W1, W2, R, _ = _tensors(rows, d, f, rows + f)
    ctx = _context(d)
    Y, Z = torch.empty_like(X), torch.empty_like(X)
    # every column of F is one, so that no product is a zero's
    W1[:f], W1[f:] = 0, 0
    X[:, 0] = 1
    W1[:f, 0], W1[f:, 0] = 4, 2
    ctx.gated_ffn(X, api.GatedFFN(W1, W2, act=act), Y, residual=R)
    at = {0: (f - 64, float("inf")), 1: (f - 1, float("-inf")), 2: (f - 40, float("nan")), 3: (0, float("inf")), 5: (f - 33, float("inf"))}
    for row, (column, value) in at.items():
        W2[row, column] = value
    W2[6, f - 64], W2[6, f - 63] = float("inf"), float("-inf")
    ctx.gated_ffn(X, api.GatedFFN(W1, W2, act=act), Z, residual=R)
    for row, (_, value) in at.items():
        got = Z[:, row].float()
        assert torch.isnan(got).all() if np.isnan(value) else (got == value).all(), (row, value, got[:4].tolist())
    assert torch.isnan(Z[:, 6].float()).all()
    assert torch.equal(Z[:, 7:], Y[:, 7:]) and torch.equal(Z[:, 4], Y[:, 4])


@pytest.mark.parametrize("rows,d,f", SHAPES)
def test_first_matrix(rows, d, f):
    from paper_2506_01084_amd import api

    X, W1, W2, R, dY = _tensors(rows, d, f, rows + d)
    ctx = _context(d)
    W1[5, d - 64], W1[6, d - 1], W1[f + 7, d - 50], W1[f + 8, 0] = float("inf"), float("-inf"), float("inf"), float("nan")
    X[:, d - 64], X[:, d - 1], X[:, d - 50] = 1, -0.5, -2
    kept = torch.empty((rows, 2 * f), dtype=torch.bfloat16, device="cuda")
    ctx.gated_ffn(X, api.GatedFFN(W1, W2), torch.empty_like(X), kept=kept)
    # (G and U in 16 bits: exponents of ones, and a fraction that a NaN has)
    words = kept.view(torch.int32).cpu().numpy().view(np.uint32).reshape(rows, f)
    G, U = words & 0xFFFF, words >> 16
    assert (G[:, 5] == 0x7FC0).all() and (G[:, 6] == 0x7FC0).all() and (U[:, 7] == 0xFFC0).all() and ((U[:, 8] & 0x7FE0) == 0x7FE0).all()
    others = np.delete(np.arange(f), [5, 6, 7, 8])
    for words in (G, U):
        assert ((words[:, others] & 0x7FC0) != 0x7FC0).all()
