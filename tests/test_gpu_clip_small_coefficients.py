"""Gradients clipped to a norm that is smaller than theirs by more than floats span: each is its share of the norm all the same."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size,max_norm", [(1e30, 1e-12), (1e34, 1e-8), (3e37, 1e-5), (1e25, 1e-20), (1e20, 1e-10), (1e-3, 1e-33), (1e30, 0.0), (1e10, 1e-34), (1e30, 1e-3)])
@pytest.mark.parametrize("in_place", [True, False])
def test_small_coefficients(size, max_norm, in_place):
    from paper_2506_01084_amd import api

    gen = torch.Generator().manual_seed(3)
    ctx = api.Context(B=1, V=8, M=2, cap=0, d=64)
    # (starts between 16-byte boundaries, too)
    tensors = [(torch.randn(n, generator=gen, dtype=torch.float64) * size).to(t).cuda()[lead:] for n, t, lead in ((20000, torch.float32, 0), (20001, torch.bfloat16, 3), (37, torch.float32, 1))]
    host = [t.double() for t in tensors]
    out = tensors if in_place else [torch.full_like(t, 7.0) for t in tensors]
    norm = torch.empty(2, device="cuda")
    ctx.clip_gradients(api.Gradients(tensors, out), max_norm, norm)
    total = float(torch.sqrt(sum((h * h).sum() for h in host)))
    c = float(np.float32(max_norm)) / total
    assert abs(float(norm[1]) - c) <= c * 36 * 2.0 ** -24 + 2.0 ** -149
    for o, h in zip(out, host):
        step = 2.0 ** -8 if o.dtype == torch.bfloat16 else 2.0 ** -24
        least = 2.0 ** -133 if o.dtype == torch.bfloat16 else 2.0 ** -148        # (subnormal results: half a step, twice)
        # the coefficient: a sum of at most 64 squares in 32 bits, halved by the root, and one rounding; a product's two
        assert torch.all((o.double() - h * c).abs() <= (h * c).abs() * (step + 40 * 2.0 ** -24) + least)
    if max_norm > 1e-30:
        got = float(torch.sqrt(sum((o.double() * o.double()).sum() for o in out)))
        assert abs(got - max_norm) <= max_norm * 1e-3
