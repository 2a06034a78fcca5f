"""The rounding of what a gated block keeps in 32 bits a pair: a number's upper 24 bits, the nearest."""
import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ffn import _context  # noqa: E402


def test_upper_24_bits():
    """SiLU's slope at zero is 1/2: U act'(G) is U / 2 there, any number that a sum of three bf16 is."""
    from paper_2506_01084_amd import api

    step = 2.0 ** -15
    want = {1.0: 1.0, 1 + step: 1 + step, 1 + step / 2: 1 + step, 1 + step / 4: 1.0, 1 + 3 * step / 4: 1 + step, 1 + step / 2 - 2.0 ** -22: 1.0, 1 + 3 * step / 2: 1 + 2 * step,
            2 - step / 2: 2.0, 2 - step: 2 - step, -1 - step / 2: -1 - step, -1 - step / 4: -1.0, 0.0: 0.0, 3e38: 3e38, 2.0 ** -60 * (1 + step / 2): 2.0 ** -60 * (1 + step)}
    d = f = 128
    x, y = torch.tensor(list(want), dtype=torch.float64), np.array(list(want.values()))
    W1, rest = torch.zeros((2 * f, d), dtype=torch.bfloat16), 2 * x
    rest[rest.abs() > 3.4e38] = 3e38
    for column in range(3):
        part = rest.bfloat16()
        W1[f:f + len(x), column] = part
        rest = rest - part.double()
    assert not rest[x.abs() < 1e38].any()
    for rows in (1, 70, 600):
        X = torch.zeros((rows, d), dtype=torch.bfloat16)
        X[:, :3] = 1
        kept = torch.empty((rows, 2 * f), device="cuda")
        _context(d).gated_ffn(X.cuda(), api.GatedFFN(W1.cuda(), torch.zeros((d, f), dtype=torch.bfloat16, device="cuda")), torch.empty_like(X.cuda()), kept=kept)
        n, raw = rows * f, kept.view(torch.uint8).flatten().cpu()
        hi, lo = raw[2 * n:6 * n].reshape(n, 4).int(), raw[6 * n:].reshape(n, 2).int()
        s = (lo[:, 1] << 8 | hi[:, 2] << 16 | hi[:, 3] << 24).view(torch.float32).reshape(rows, f).double().numpy()[:, :len(x)]
        inside = np.abs(y) < 1e38
        assert np.array_equal(s[0][inside], y[inside]) and np.array_equal(s[-1], s[0]), (s[0], y)
        off = np.abs(s[0] - x.numpy())[inside]
        assert np.all(off <= oracle.ffn.KEPT * np.abs(x.numpy())[inside]) and np.max(off / np.maximum(np.abs(x.numpy()[inside]), 1e-30)) > oracle.ffn.KEPT * (1 - 2.0 ** -14)
