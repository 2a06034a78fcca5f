"""4-bit weights through the C ABI: how they are made, bit by bit, and the gated block over them, against the oracle."""
import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ffn import _context, _host, _tensors, _within  # noqa: E402


def _bf16(x):
    return oracle.bf16_bits_to_f64(oracle.f64_to_bf16_bits(np.nan_to_num(x, nan=0.0, posinf=0.0)))


def _quantized(ctx, W, group):
    from paper_2506_01084_amd import api

    words, scales = api.q4_shapes(W.shape[0], W.shape[1], group)
    q = torch.full(words, -1, dtype=torch.int32, device="cuda")
    s = torch.full(scales, 9.0, dtype=torch.bfloat16, device="cuda")
    ctx.quantize_q4(W, group, q, s)
    return q, s


@pytest.mark.parametrize("rows,cols,group", [(16, 64, 32), (16, 64, 64), (16, 128, 128), (48, 192, 64), (64, 448, 32), (80, 256, 128), (16, 1088, 64)])
def test_quantize(rows, cols, group):
    gen = torch.Generator().manual_seed(rows + cols)
    W = (torch.randn((rows, cols), generator=gen) * 0.02).bfloat16()
    # runs of zeros, of one value, of subnormal and of the largest numbers, at a tie of the quotient, with an infinity and a NaN
    W[0, :group] = 0
    W[1, :group] = -0.5
    W[2, :group] = 1e-39
    W[3, :group] = torch.linspace(-3.3e38, 3.3e38, group).bfloat16()
    W[4, :group] = (torch.arange(group) % 29 - 14).float() * 0.5 + 0.25
    W[4, 0] = 6.0
    W[4, :16] = torch.tensor([6, 0.25, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, 0.2490234375, 0.25195312, -0.7460938, 4.9687, -5.0313, 0.5])
    W[5, group - 1] = float("inf")
    W[6, 0] = float("nan")
    ctx = _context(64)
    q, s = _quantized(ctx, W.cuda(), group)
    want_q, want_s = oracle.quantize_q4(W.double().numpy(), group, _bf16)
    assert np.array_equal(s.double().cpu().numpy(), want_s, equal_nan=True)
    assert np.array_equal(q.cpu().numpy().view(np.uint32), oracle.q4_words(want_q))


# rows on both sides of the product's blocks of 16 and of the change to expanded weights; widths that no block of 128 columns divides
@pytest.mark.parametrize("rows", [1, 2, 8, 9, 15, 16, 17, 32, 33, 48, 49, 64, 65, 100, 192, 193, 320, 321, 400])
@pytest.mark.parametrize("d,f,group,act", [(64, 64, 32, "silu"), (192, 448, 64, "gelu"), (320, 64, 32, "gelu"), (512, 1152, 128, "silu"), (1088, 320, 64, "silu"),
                                           (2048, 192, 32, "silu")])
def test_forward(rows, d, f, group, act):
    from paper_2506_01084_amd import api

    X, W1, W2, R, _ = _tensors(rows, d, f, rows + d + f + group)
    ctx = _context(d)
    (q1, s1), (q2, s2) = _quantized(ctx, W1, group), _quantized(ctx, W2, group)
    host = []
    for W in (W1, W2):
        q, s = oracle.quantize_q4(_host(W), group, _bf16)
        host.append(oracle.q4_weights(q, s, group))
    block = api.GatedFFN(q1, q2, act=act, scale_1=s1, scale_2=s2)
    assert (block.desc.group, block.d, block.d_ff) == (group, d, f)
    Y = torch.full_like(X, float("nan"))
    ctx.gated_ffn(X, block, Y, residual=R)
    ref = oracle.gated_ffn(_host(X), *host, act, _host(R), round_weights=rows > 320)
    _within(Y, ref["Y"], ref["Y_bound"], "Y")
    Z = torch.full_like(X, float("nan"))
    ctx.gated_ffn(X, block, Z, residual=None)
    ref = oracle.gated_ffn(_host(X), *host, act, None, round_weights=rows > 320)
    _within(Z, ref["Y"], ref["Y_bound"], "Y without a residual")


def test_exact_sums():
    """Whole numbers: products of few rows are exact, whatever the group."""
    from paper_2506_01084_amd import api

    d, f = 192, 64
    gen = torch.Generator().manual_seed(3)
    for group in (32, 64):
        grid = torch.tensor(oracle.ffn.Q4_VALUES, dtype=torch.float32)
        W1 = torch.zeros((2 * f, d))
        W1[:f] = grid[torch.randint(0, 16, (f, d), generator=gen)]
        W1[:, ::group] = 6                                       # scale 1 in every run
        W1[f:] = 0
        W1[f:, 0] = 6
        W2 = torch.zeros((d, f))
        W2[torch.arange(d), torch.arange(d) % f] = 6
        X = torch.randint(-3, 4, (20, d), generator=gen).float()
        X[:, 0] = 1
        ctx = _context(d)
        X, W1, W2 = (t.bfloat16().cuda() for t in (X, W1, W2))
        (q1, s1), (q2, s2) = _quantized(ctx, W1, group), _quantized(ctx, W2, group)
        assert set(s1.float().cpu().unique().tolist()) <= {0.0, 1.0}
        Y = torch.empty_like(X)
        ctx.gated_ffn(X, api.GatedFFN(q1, q2, act="silu", scale_1=s1, scale_2=s2), Y)
        G = _host(X) @ _host(W1)[:f].T
        F = oracle.ffn.act(G, "silu")[0] * 6
        want = (F * 6)[:, np.arange(d) % f]
        # two roundings to bf16 and the activation's own error
        assert np.all(np.abs(_host(Y) - want) <= np.abs(want) * (2.02 * 2.0 ** -8) + 36 * 1e-6 * np.abs(G)[:, np.arange(d) % f] + 1e-30)


def test_rows_do_not_meet_and_graphs():
    from paper_2506_01084_amd import api

    d, f = 512, 320
    X, W1, W2, R, _ = _tensors(40, d, f, 8)
    ctx = _context(d)
    (q1, s1), (q2, s2) = _quantized(ctx, W1, 64), _quantized(ctx, W2, 64)
    block = api.GatedFFN(q1, q2, scale_1=s1, scale_2=s2)
    Y, Z = torch.full_like(X, 7.0), torch.empty_like(X)
    ctx.gated_ffn(X[:39], block, Y[:39], residual=R[:39])
    assert (Y[39] == 7).all()
    other = X.clone()
    other[5] = float("nan")
    ctx.gated_ffn(other[:39], block, Z[:39], residual=R[:39])
    same = [i for i in range(39) if i != 5]
    assert torch.equal(Y[same], Z[same]) and torch.isnan(Z[5]).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.gated_ffn(X[:39], block, Z[:39], residual=R[:39])
    for i in range(3):
        X.copy_(torch.randn((40, d), generator=torch.Generator().manual_seed(i)).bfloat16())
        graph.replay()
        ctx.gated_ffn(X[:39], block, Y[:39], residual=R[:39])
        torch.cuda.synchronize()
        assert torch.equal(Y[:39], Z[:39])
    # many rows: the weights are expanded; a group whose scale is NaN reaches every row
    s1[0, 0] = float("nan")
    ctx.gated_ffn(X, block, Y)
    assert torch.isnan(Y).all()


def test_kept_needs_bf16_weights():
    from paper_2506_01084_amd import api

    X, W1, W2, _, _ = _tensors(4, 64, 64, 8)
    ctx = _context(64)
    (q1, s1), (q2, s2) = _quantized(ctx, W1, 32), _quantized(ctx, W2, 32)
    block = api.GatedFFN(q1, q2, scale_1=s1, scale_2=s2)
    with pytest.raises(api.Z2ZError) as e:
        ctx.gated_ffn(X, block, torch.empty_like(X), kept=torch.empty((4, 128), device="cuda"))
    assert e.value.code == api.E_UNSUPPORTED
