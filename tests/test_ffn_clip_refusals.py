"""What the gated block's, the 4-bit weights' and the clipping's entry points refuse, what they launch, and what their work buffers do: without a GPU, against a
HIP runtime that launches nothing (stub_hip.cpp)."""
from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)

BLOCK = """
def ffn(d_ff=256, act=0, group=0, w_1=P, w_2=P, scale_1=None, scale_2=None, reserved=0):
    f = api.FfnDesc()
    f.d_ff, f.act, f.group, f.reserved, f.w_1, f.w_2, f.scale_1, f.scale_2 = d_ff, act, group, reserved, w_1, w_2, scale_1, scale_2
    return f
X, R, Y, K, D, G = (P + (i << 32) for i in range(1, 7))   # (nothing near anything else)
W1, W2, S1, S2, GW1, GW2 = (P + (i << 34) for i in range(3, 9))
def block(**kw):
    return ffn(**{**dict(w_1=W1, w_2=W2), **kw})
def four(**kw):
    return ffn(**{**dict(w_1=W1, w_2=W2, scale_1=S1, scale_2=S2, group=64), **kw})
def fwd(c, f, X=X, rows=24, residual=R, Y=Y, kept=None):
    return lib.z2z_gated_ffn(c, X, rows, ctypes.byref(f) if f else None, residual, Y, kept, None)
def bwd(c, f, X=X, rows=24, kept=K, dY=D, dX=G, grad=None, flags=0):
    g = grad or ffn(w_1=GW1, w_2=GW2)
    return lib.z2z_gated_ffn_backward(c, X, rows, ctypes.byref(f) if f else None, kept, dY, dX, ctypes.byref(g), flags, None)
h = context(B=1, V=8, M=2, cap=0, d=512)
"""


def test_block_refusals(without_a_device):
    without_a_device(BLOCK + """
bad = [dict(f=None), dict(f=block(d_ff=0)), dict(f=block(d_ff=-64)), dict(f=block(act=2)), dict(f=block(act=-1)), dict(f=block(reserved=1)), dict(f=block(w_1=None)),
       dict(f=block(w_2=None)), dict(f=block(w_1=W1 + 8)), dict(f=block(w_2=W2 + 2)), dict(f=block(group=16)), dict(f=block(group=-32)), dict(f=four(scale_1=None)),
       dict(f=four(scale_2=None)), dict(f=four(scale_1=S1 + 2))]
for kw in bad:
    assert fwd(h, kw["f"]) == api.E_INVAL, kw
    if kw["f"] is None or not kw["f"].group:
        assert bwd(h, kw["f"]) == api.E_INVAL, kw
assert fwd(None, block()) == api.E_INVAL and bwd(None, block()) == api.E_INVAL
for kw in (dict(X=None), dict(Y=None), dict(rows=-1), dict(X=X + 2), dict(Y=Y + 8), dict(residual=R + 4), dict(kept=K + 8)):
    assert fwd(h, block(), **kw) == api.E_INVAL, kw
for kw in (dict(X=None), dict(kept=None), dict(dY=None), dict(dX=None), dict(rows=-1), dict(X=X + 2), dict(kept=K + 4), dict(dY=D + 8), dict(dX=G + 8), dict(flags=2), dict(flags=-1),
           dict(grad=ffn(w_1=None)), dict(grad=ffn(w_1=GW1, w_2=None)), dict(grad=ffn(w_1=GW1 + 8, w_2=GW2))):
    assert bwd(h, block(), **kw) == api.E_INVAL, kw
# shapes and types
for f in (block(d_ff=96), four(d_ff=320, group=128), block(d_ff=64 * 40000)):
    assert fwd(h, f) == api.E_UNSUPPORTED, f.d_ff
assert bwd(h, four()) == api.E_UNSUPPORTED and fwd(h, four(), kept=K) == api.E_UNSUPPORTED
assert fwd(h, block(), rows=(1 << 22) + 1) == api.E_UNSUPPORTED
assert fwd(context(B=1, V=8, M=2, cap=0, d=512, dtype=api.F32), block()) == api.E_UNSUPPORTED
assert fwd(context(B=1, V=8, M=2, cap=0, d=96), block()) == api.E_UNSUPPORTED
assert fwd(context(B=1, V=8, M=2, cap=0, d=192), four(group=128)) == api.E_UNSUPPORTED
assert launches() == []
# overlaps
rows, row, keep = 24, 24 * 512 * 2, 24 * 256 * 8
assert fwd(h, block(), Y=X) == api.E_INVAL and fwd(h, block(), Y=X + row - 16) == api.E_INVAL and fwd(h, block(), Y=R + 16) == api.E_INVAL
assert fwd(h, block(), Y=W2 + 2 * 512 * 256 - 16) == api.E_INVAL and fwd(h, four(), Y=S1) == api.E_INVAL and fwd(h, four(), Y=W1 + 512 * 512 // 2 - 16) == api.E_INVAL
assert fwd(h, block(), kept=Y) == api.E_INVAL and fwd(h, block(), kept=X - keep + 16) == api.E_INVAL and fwd(h, block(), kept=R) == api.E_INVAL
assert fwd(h, block(), kept=R, Y=R) == api.E_INVAL and fwd(h, block(), kept=W1 + 16) == api.E_INVAL
for kw in (dict(dX=X), dict(dX=D), dict(dX=K + keep - 16), dict(dX=W1), dict(grad=ffn(w_1=W1, w_2=GW2)), dict(grad=ffn(w_1=GW1, w_2=GW1 + 16)), dict(dX=GW2), dict(grad=ffn(w_1=GW1, w_2=K))):
    assert bwd(h, block(), **kw) == api.E_INVAL, kw
assert launches() == []
assert fwd(h, block(), Y=R) == 0 and fwd(h, block(), Y=X + row) == 0 and fwd(h, block(), kept=X - keep) == 0
launches()
# empty calls
assert fwd(h, block(), rows=0, X=None, Y=None, residual=None) == 0 and launches() == []
assert bwd(h, block(), rows=0, X=None, kept=None, dY=None, dX=None, flags=api.GRAD_ADD) == 0 and launches() == []
assert bwd(h, block(), rows=0, X=None, kept=None, dY=None, dX=None) == 0 and [n for n, _ in launches()] != []
clean()
""")


def test_block_launches_and_work_space(without_a_device):
    without_a_device(BLOCK + """
names = lambda: [next(k for k in ("few_rows_kernel", "q4_kernel", "few_sum_kernel", "q4_expand", "logits_mid_kernel", "logits_fast_kernel", "linear_sum_kernel", "tile_sum_kernel",
                                  "small_tile_kernel", "small_pair_kernel", "fill_zero") if k in n) for n, _ in launches()]
big = context(B=1, V=8, M=2, cap=0, d=2048)
wide = dict(d_ff=4096)
assert fwd(big, block(**wide), rows=16) == 0 and names() == ["few_rows_kernel"] * 2
assert fwd(big, block(**wide), rows=17) == 0 and names() == ["small_tile_kernel"] * 2 + ["few_sum_kernel"]
assert fwd(big, block(d_ff=22016), rows=17) == 0 and names() == ["logits_mid_kernel", "few_sum_kernel", "logits_mid_kernel", "linear_sum_kernel"]
assert fwd(big, block(**wide), rows=767) == 0 and names() == ["small_tile_kernel"] * 2
assert fwd(big, block(**wide), rows=768) == 0 and names() == ["small_tile_kernel"] * 2
assert fwd(big, block(**wide), rows=769) == 0 and names()[0] == "logits_fast_kernel"
assert fwd(big, block(**wide), rows=5000) == 0 and names()[0] == "logits_fast_kernel"
assert fwd(big, four(**wide), rows=8) == 0 and names() == ["few_rows_kernel"] * 2
for rows in (9, 320):
    assert fwd(big, four(**wide), rows=rows) == 0 and names() == ["q4_kernel", "few_sum_kernel"] * 2
assert fwd(big, four(**wide), rows=321) == 0 and names()[:4] == ["q4_expand", "q4_expand"] + ["small_tile_kernel"] * 2
assert fwd(big, four(**wide), rows=769) == 0 and names()[:3] == ["q4_expand", "q4_expand", "logits_fast_kernel"]
pairs = ["small_pair_kernel"] * 2                                                         # (dF with dW2, dX with dW1)
for rows in (1, 64, 639, 640):
    assert bwd(big, block(**wide), rows=rows) == 0
    assert [n for n in names() if n != "few_sum_kernel"] == pairs, rows
for rows, d_ff, small in ((641, 4096, 1), (1280, 4096, 1), (1281, 4096, 0), (16, 22016, None), (17, 22016, 2), (71, 22016, 2), (72, 22016, 1)):
    assert bwd(big, block(d_ff=d_ff), rows=rows) == 0
    now = names()
    assert [n for n in now if n != "few_sum_kernel"] == pairs if small is None else now.count("small_tile_kernel") == small, (rows, now)
assert bwd(big, block(d_ff=2048), rows=60) == 0 and names() == ["small_pair_kernel"] * 2 + ["few_sum_kernel"]
assert fwd(h, block(), rows=256) == 0 and names() == ["few_rows_kernel"] * 2             # (small weights)
# nothing grows under capture; what a graph names stays
fresh = context(B=1, V=8, M=2, cap=0, d=512)
stub.stub_capturing(1)
assert fwd(fresh, block(), rows=400) == api.E_CAPTURE and bwd(fresh, block(), rows=400) == api.E_CAPTURE and launches() == []
stub.stub_capturing(0)
assert bwd(fresh, block(), rows=400) == 0
launches()
stub.stub_capturing(1)
assert bwd(fresh, block(), rows=400) == 0
stub.stub_capturing(0)
used = stub.stub_used()
assert bwd(fresh, block(), rows=4000) == 0 and stub.stub_used() >= used + 4000 * 4 * 256
launches()
stub.stub_capacity(stub.stub_used())
assert bwd(fresh, block(), rows=1 << 20) == api.E_NOMEM and launches() == []
clean()
assert bwd(fresh, block(), rows=4000) == 0
stub.stub_capacity(1 << 50)
for c in (h, big, fresh):
    assert lib.z2z_destroy(c) == 0
assert stub.stub_used() == 0
""")


def test_four_bits_refusals(without_a_device):
    without_a_device(BLOCK + """
q4 = lambda c=h, W=X, rows=64, cols=256, group=64, q=Y, s=K: lib.z2z_quantize_q4(c, W, rows, cols, group, q, s, None)
for kw in (dict(c=None), dict(W=None), dict(q=None), dict(s=None), dict(rows=0), dict(cols=0), dict(rows=-16), dict(group=0), dict(group=48), dict(group=256), dict(W=X + 8),
           dict(q=Y + 4), dict(s=K + 2), dict(q=X), dict(s=X + 64 * 256 * 2 - 16), dict(s=Y + 64 * 2 * 64 - 16)):
    assert q4(**kw) == api.E_INVAL, kw
for kw in (dict(rows=24), dict(cols=96), dict(cols=192, group=128), dict(c=context(B=1, V=8, M=2, cap=0, d=512, dtype=api.F32))):
    assert q4(**kw) == api.E_UNSUPPORTED, kw
assert launches() == []
assert q4() == 0 and q4(s=Y + 64 * 2 * 64) == 0 and q4(cols=192) == 0 and q4(cols=128, group=128) == 0 and len(launches()) == 4
assert q4(c=context(B=1, V=8, M=2, cap=0, d=24)) == 0     # (the width does not matter)
clean()
""")


def test_clip_refusals(without_a_device):
    without_a_device("""
h = context(B=1, V=8, M=2, cap=0, d=8)
N = P + (1 << 50)
inf, nan = float("inf"), float("nan")
def clip(*tensors, max_norm=1.0, norm=N, c=h, n=None):
    arr = (api.GradientDesc * max(len(tensors), 1))()
    for a, t in zip(arr, tensors):
        a.data, a.out, a.n, a.dtype, a.reserved = (*t, 0, 0, 0)[:5] if len(t) < 5 else t
    return lib.z2z_clip_gradients(c, arr, len(tensors) if n is None else n, max_norm, norm, None)
A, B, O = P + (1 << 32), P + (2 << 32), P + (3 << 32)
f, b = api.F32, api.BF16
good = (A, A, 1000, f)
assert clip(good, c=None) == api.E_INVAL and clip(good, norm=None) == api.E_INVAL and clip(good, norm=N + 2) == api.E_INVAL and clip(good, n=-1) == api.E_INVAL
assert lib.z2z_clip_gradients(h, None, 1, 1.0, N, None) == api.E_INVAL
for m in (-1.0, nan, -inf):
    assert clip(good, max_norm=m) == api.E_INVAL
for t in ((None, None, 10, f), (A, A, -1, f), (A, A, 10, 2), (A + 2, A + 2, 10, f), (A + 1, A + 1, 10, b), (A, O + 2, 10, f), (A, A, 10, f, 1)):
    assert clip(good[:0] + t) == api.E_INVAL, t
assert clip((A, A, (1 << 44) + 1, b)) == api.E_UNSUPPORTED
arr = (api.GradientDesc * 5000)()
assert lib.z2z_clip_gradients(h, arr, 5000, 1.0, N, None) == api.E_UNSUPPORTED
# what is written overlaps nothing else
for ts in ((good, good), (good, (A + 3996, A + 3996, 4, f)), ((A, O, 1000, f), (B, O + 2000, 1000, b)), ((A, O, 1000, f), (O + 400, None, 10, f)), ((A, A + 16, 1000, f),),
           ((A, None, 1000, b), (A + 1998, A + 1998, 4, b))):
    assert clip(*ts) == api.E_INVAL, ts
assert clip((A, A, 1000, f), norm=A + 3996) == api.E_INVAL and clip((A, None, 1000, f), norm=A) == api.E_INVAL and clip((A, O, 1000, f), norm=O - 4) == api.E_INVAL
assert launches() == []
assert clip((A, A, 1000, f), (A + 4000, A + 4000, 4, f)) == 0 and clip((A, None, 1000, f), (A, None, 1000, f)) == 0 and clip((A, O, 1000, f), (A, O + 4000, 1000, f)) == 0
assert clip((A, A, 1000, f), norm=A + 4000) == 0 and clip((A, A, 1000, f), (A, A, 0, f), (None, None, 0, b)) == 0
assert clip() == 0 and clip(good, max_norm=inf) == 0 and clip(good, max_norm=0.0) == 0 and clip((A + 2, A + 2, 7, b)) == 0
launches()
# launches: lists of 96 tensors, workgroups by what there is; one where nothing is written
assert clip(*[(A + (i << 16), A + (i << 16), 16, b) for i in range(97)]) == 0
assert [g for _, g in launches()] == [96, 1, 96, 1]
assert clip((A, A, 1 << 30, b)) == 0 and [g for _, g in launches()] == [1024, 1024]
assert clip((A, None, 1 << 30, b)) == 0 and [g for _, g in launches()] == [1024, 1]
many = [(A + (i << 30), A + (i << 30), 1 << 28, b) for i in range(500)]
assert clip(*many) == 0
log = launches()
assert len(named(log, "clip_squares")) == 6 and len(named(log, "clip_total")) == 1 and len(named(log, "clip_scale")) == 6
clean()
stub.stub_capturing(1)
fresh = context(B=1, V=8, M=2, cap=0, d=8)
stub.stub_capturing(1)
assert clip(good, c=fresh) == api.E_CAPTURE and launches() == []
stub.stub_capturing(0)
assert clip(good, c=fresh) == 0
stub.stub_capturing(1)
assert clip(good, c=fresh) == 0
""")


def test_encoder_refusals(without_a_device):
    without_a_device(BLOCK + """
def gated(d=512, layers=2, **kw):
    e = encoder(d, layers)
    g = api.GatedEncoderDesc()
    g.encoder = e
    g.encoder.attention_only = api.ENC_GATED
    g.encoder.d_ff = -5                                   # (not read)
    arr = (api.FfnDesc * layers)(*[block(**kw) for _ in range(layers)])
    g.ffn = ctypes.cast(arr, ctypes.POINTER(api.FfnDesc))
    for lay in e.keep:
        lay.w_1 = lay.b_1 = lay.w_2 = lay.b_2 = None
    g.keep = (e, arr)
    return g
c = context(B=2, V=100, M=3, cap=50, d=512)
enc = lambda g: lib.z2z_hyper_encode(c, P, ctypes.byref(g.encoder), P, None, 1, None)
back = lambda g, q: lib.z2z_hyper_encode_backward(c, P, ctypes.byref(g.encoder), P, ctypes.byref(q.encoder), P, 0, None)
assert enc(gated()) == 0 and back(gated(), gated()) == 0
launches()
for kw in (dict(act=3), dict(w_1=None), dict(w_2=W2 + 8), dict(d_ff=0), dict(reserved=2), dict(group=64)):
    assert enc(gated(**kw)) == api.E_INVAL, kw
assert enc(gated(d_ff=96)) == api.E_UNSUPPORTED
g = gated()
g.ffn[1].d_ff = 320
assert enc(g) == api.E_INVAL
g = gated()
g.ffn = None
assert enc(g) == api.E_INVAL
g = gated()
g.keep[0].keep[0].ln2_g = None
assert enc(g) == api.E_INVAL
q = gated(group=64, scale_1=S1, scale_2=S2)
assert back(q, gated()) == api.E_UNSUPPORTED and lib.z2z_hyper_encode_keep(c, P, ctypes.byref(q.encoder), P, None) == api.E_UNSUPPORTED
plain = encoder(512)
assert lib.z2z_hyper_encode_backward(c, P, ctypes.byref(gated().encoder), P, ctypes.byref(plain), P, 0, None) == api.E_INVAL
assert launches() == []
assert enc(q) == 0
clean()
""")
