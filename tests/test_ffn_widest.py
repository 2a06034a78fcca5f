"""The widest hidden layers of a gated block: what is refused, without a GPU (stub_hip.cpp), and rows that are as far apart as they may be."""
import numpy as np
import pytest

import oracle
from test_ffn_clip_refusals import BLOCK
from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


def test_refusals(without_a_device):
    """Offsets inside 256 rows of dG | dU, 4 d_ff bytes each, have 32 bits: a block that needs more is refused, whichever call it is."""
    without_a_device(BLOCK + """
K, D, G, Y = (P + (i << 44) for i in range(1, 5))         # (these tensors are large)
W1, W2, S1, S2, GW1, GW2 = (P + (i << 46) for i in range(3, 9))
narrow = {d: context(B=1, V=8, M=2, cap=0, d=d) for d in (64, 128, 192)}
for d, c in narrow.items():
    for d_ff in (1 << 22, (1 << 22) + 64, (1 << 23) + 64, 64 * ((1 << 30) // d // 64 - 2)):
        if d_ff < 1 << 22:
            continue
        for rows in (1, 16, 256, 4000):
            for f in (block(d_ff=d_ff), four(d_ff=d_ff)):
                assert fwd(c, f, rows=rows) == api.E_UNSUPPORTED, (d, d_ff, rows)
            assert bwd(c, block(d_ff=d_ff), rows=rows) == api.E_UNSUPPORTED, (d, d_ff, rows)
    assert launches() == []
    assert fwd(c, block(d_ff=(1 << 22) - 64), rows=256, kept=K) == 0 and bwd(c, block(d_ff=(1 << 22) - 64), rows=256) == 0
    assert fwd(c, four(d_ff=(1 << 22) - 64), rows=320) == 0
    launches()
g = api.GatedEncoderDesc()
g.encoder = encoder(64, 1)
g.encoder.attention_only = api.ENC_GATED
one = (api.FfnDesc * 1)(block(d_ff=1 << 22))
g.ffn = ctypes.cast(one, ctypes.POINTER(api.FfnDesc))
c = context(B=2, V=100, M=3, cap=50, d=64)
assert lib.z2z_hyper_encode(c, P, ctypes.byref(g.encoder), P, None, 1, None) == api.E_UNSUPPORTED
assert lib.z2z_hyper_encode_backward(c, P, ctypes.byref(g.encoder), P, ctypes.byref(g.encoder), P, 0, None) == api.E_UNSUPPORTED
assert launches() == []
""")


@pytest.mark.gpu
def test_rows_as_far_apart_as_they_may_be():
    """A hidden layer of 2^22 - 64 columns, all but 64 of which have weights of zero: what the products add up is what a block of those 64 gives."""
    torch = pytest.importorskip("torch")
    from paper_2506_01084_amd import api
    from test_gpu_gated_ffn import _context, _host, _tensors, _within

    rows, d, f = 256, 64, (1 << 22) - 64
    X, w1, w2, R, dY = _tensors(rows, d, 64, 5)
    at = torch.from_numpy(np.random.default_rng(6).choice(f, 64, replace=False)).cuda()
    at[:4] = torch.tensor([0, f - 1, f // 2, f - 64])
    assert len(set(at.tolist())) == 64
    W1, W2 = torch.zeros((2 * f, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((d, f), dtype=torch.bfloat16, device="cuda")
    W1[at], W1[at + f], W2[:, at] = w1[:64], w1[64:], w2
    ctx, block = _context(d), api.GatedFFN(W1, W2, act="silu")
    Y, dX = torch.full_like(X, float("nan")), torch.full_like(X, float("nan"))
    kept = torch.empty((rows, 2 * f), dtype=torch.bfloat16, device="cuda")
    dW1, dW2 = torch.full_like(W1, float("nan")), torch.full_like(W2, float("nan"))
    ctx.gated_ffn(X, block, Y, residual=R, kept=kept)
    ctx.gated_ffn_backward(X, block, kept, dY, dX, api.GatedFFN(dW1, dW2))
    x, a, b, dy = _host(X), _host(w1), _host(w2), _host(dY)
    ref = oracle.gated_ffn(x, a, b, "silu", _host(R))
    _within(Y, ref["Y"], ref["Y_bound"], "Y")
    want = oracle.gated_ffn_backward(x, a, b, "silu", dy, kept16=True)
    _within(dX, want["dX"], want["dX_bound"], "dX")
    _within(torch.cat([dW1[at], dW1[at + f]]), want["dW1"], want["dW1_bound"], "dW1")
    _within(dW2[:, at], want["dW2"], want["dW2_bound"], "dW2")
    # (columns without weights: act(0) = 0 and U = 0 leave no gradient)
    dW1[at] = 0
    dW1[at + f] = 0
    dW2[:, at] = 0
    assert not dW1.any() and not dW2.any()
