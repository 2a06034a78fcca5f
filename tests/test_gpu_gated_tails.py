"""The activations of a gated block where they are small: F and what is kept, relative to the values themselves, against the error function's complement in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ffn import _context  # noqa: E402

KEPT = 2.0 ** -16                         # 15 bits of fraction, rounded


def _values(act, x):
    """Activation and slope in 64 bits, no difference of nearly equal numbers."""
    if act == "silu":
        p = np.exp(np.minimum(x, 0)) / (1 + np.exp(-np.abs(x)))
        q = np.exp(np.minimum(-x, 0)) / (1 + np.exp(-np.abs(x)))
        return x * p, p * (1 + x * q), p
    p = np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in x])
    return x * p, p + x * np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi), p


# (a kernel each: few rows in one launch, small tiles, the weight-streaming kernel's sum, the tile kernel)
@pytest.mark.parametrize("rows,d,f", [(2, 128, 1088), (200, 256, 1088), (40, 8192, 5504), (1031, 3520, 1792)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_small_values(rows, d, f, act):
    from paper_2506_01084_amd import api

    x = torch.linspace(-12, 6, f).bfloat16()
    x[:8] = torch.tensor([-4.5, -5.0, -5.5, -6.0, -0.0, 0.0, 1e-20, -1e-20])
    W1, X = torch.zeros((2 * f, d), dtype=torch.bfloat16), torch.zeros((rows, d), dtype=torch.bfloat16)
    W1[:f, 3], W1[f:, 3], X[:, 3] = x, 1, 1
    W2 = torch.zeros((d, f), dtype=torch.bfloat16)
    kept = torch.empty((rows, 2 * f), device="cuda")
    _context(d).gated_ffn(X.cuda(), api.GatedFFN(W1.cuda(), W2.cuda(), act=act), torch.empty((rows, d), dtype=torch.bfloat16, device="cuda"), kept=kept)
    n, raw = rows * f, kept.view(torch.uint8).flatten().cpu()
    F = raw[:2 * n].view(torch.bfloat16).reshape(rows, f).double().numpy()
    hi, lo = raw[2 * n:6 * n].reshape(n, 4).int(), raw[6 * n:].reshape(n, 2).int()
    a, s = ((lo[:, i] << 8 | hi[:, 2 * i] << 16 | hi[:, 2 * i + 1] << 24).view(torch.float32).reshape(rows, f).double().numpy() for i in range(2))
    x = x.double().numpy()
    value, slope, p = _values(act, x)
    # the fit, five roundings of the polynomial's larger terms, the exponential's and the reciprocal's last bits, their product and the exponent's rounding: 2^-24 each of
    # them, the last x^2 / 2 (SiLU: x) times; half a bit more of everything for products that round
    arithmetic = 6.7e-7 + (12 + 2 * (0.5 * x * x if act == "gelu" else np.abs(x))) * 2.0 ** -24
    # (a slope is the sum of two terms, with errors of their own)
    terms = p + np.abs(x) * (np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi) if act == "gelu" else p)
    least = 2.0 ** -120
    for row in (0, rows - 1):
        assert np.all(np.abs(a[row] - value) <= np.abs(value) * (KEPT + arithmetic) + least), (x[np.argmax(np.abs(a[row] - value) / (np.abs(value) + least))])
        assert np.all(np.abs(F[row] - value) <= np.abs(value) * (2.0 ** -8 + arithmetic) + least)
        assert np.all(np.abs(s[row] - slope) <= np.abs(slope) * KEPT + terms * 2 * arithmetic + least)
