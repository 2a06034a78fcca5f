"""GPU: the lookup's gradient where rows that the sort's launches have not cleared are named very often (a padding or special token at the vocabulary's
end, a popular entry), beside rows that nobody names.  Whole numbers: every sum is exact."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,d,N", [(300_000, 128, 4096), (600_000, 128, 4097), (400_000, 256, 12_345)])
@pytest.mark.parametrize("popular", [(1,), (1, 2, 3), tuple(range(1, 40)), (16, 17, 33), "entry"])
def test_popular_rows_behind_the_cleared_ones(V, d, N, popular):
    import torch
    from paper_2506_01084_amd import api

    print(f"[case] lookup gradient, popular rows V={V} d={d} N={N} {popular}", flush=True)
    cap = 40
    ctx = api.Context(B=1, V=V, M=2, cap=cap, d=d, dtype="bf16")
    phrases = torch.tensor([[[0, e + 1] for e in range(cap)]], dtype=torch.int32, device="cuda")
    added, st = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    ctx.codebook_prefill(phrases, torch.full((1, cap), 2, dtype=torch.int32, device="cuda"), torch.tensor([cap], dtype=torch.int32, device="cuda"), added, st,
                         api.RESET)
    assert added.tolist() == [cap]
    rng = np.random.default_rng(V + N)
    often = [V + 7, V + 8] if popular == "entry" else [V - k for k in popular]
    codes = rng.choice(often, size=N)
    some = rng.random(N) < 0.02
    codes[some] = rng.integers(0, V + cap, size=int(some.sum()))
    dX = rng.integers(-1, 2, size=(N, d)).astype(np.float32)
    want = torch.zeros((V + cap, d), device="cuda")
    want.index_add_(0, torch.from_numpy(codes).cuda(), torch.from_numpy(dX).cuda())
    dE, dW = torch.ones((V, d), device="cuda"), torch.ones((1, cap, d), dtype=torch.bfloat16, device="cuda")
    ctx.embed_codes_backward(torch.from_numpy(codes[None].astype(np.int32)).cuda(), None, torch.from_numpy(dX[None]).cuda().bfloat16(), dE, dW)
    torch.cuda.synchronize()
    assert torch.equal(dE, want[:V]) and torch.equal(dW[0], want[V:].bfloat16())
    ctx.close()
