"""The gated block and its gradient on the largest number of rows that a call takes: matrices of more than 2^32 elements."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ffn import _context  # noqa: E402


@pytest.mark.parametrize("form", [torch.bfloat16, torch.float32])
def test_most_rows(form):
    from paper_2506_01084_amd import api

    rows, d, f = 1 << 22, 64, 1088
    gen = torch.Generator(device="cuda").manual_seed(8)
    make = lambda shape, std: (torch.randn(shape, generator=gen, device="cuda") * std).bfloat16()
    X, dY, W1, W2 = make((rows, d), 1.0), make((rows, d), 1e-2), make((2 * f, d), d ** -0.5), make((d, f), f ** -0.5)
    ctx, block = _context(d), api.GatedFFN(W1, W2, act="silu")
    Y, dX = (torch.full_like(X, float("nan")) for _ in range(2))
    dW1, dW2 = torch.full_like(W1, float("nan")), torch.full_like(W2, float("nan"))
    kept = torch.empty((rows, 2 * f), dtype=form, device="cuda")
    ctx.gated_ffn(X, block, Y, kept=kept)
    ctx.gated_ffn_backward(X, block, kept, dY, dX, api.GatedFFN(dW1, dW2))
    del kept
    w1, w2 = W1.double(), W2.double()
    off, size = torch.zeros(2, device="cuda", dtype=torch.float64), torch.zeros(2, device="cuda", dtype=torch.float64)
    want1, want2 = torch.zeros_like(w1), torch.zeros_like(w2)
    step = 1 << 17
    for r in range(0, rows, step):
        x, dy = X[r:r + step].double(), dY[r:r + step].double()
        G, U = x @ w1[:f].T, x @ w1[f:].T
        p = torch.sigmoid(G)
        a = G * p
        dF = dy @ w2
        D = torch.cat([dF * U * (p + a * (1 - p)), dF * a], dim=1)
        want1 += D.T @ x
        want2 += dy.T @ (a * U)
        for i, (got, want) in enumerate(((Y, (a * U) @ w2.T), (dX, D @ w1))):
            e = (got[r:r + step].double() - want).norm()
            # two roundings to bf16, each 2^-8 sqrt(0.54 / 3) of the numbers' norm in the mean, and three of a quarter; no piece of the rows is further off than all of them
            assert float(e) <= 2.6e-3 * float(want.norm()), (r, i)
            off[i] += e * e
            size[i] += want.norm() ** 2
    assert torch.all(off.sqrt() <= 2.6e-3 * size.sqrt())
    for got, want in ((dW1, want1), (dW2, want2)):
        assert float((got.double() - want).norm()) <= 2.6e-3 * float(want.norm())
    ctx.close()
    torch.cuda.empty_cache()
