"""What the lookup's, the beam search's and their neighbours' entry points refuse, and what they launch: without a GPU, against a HIP runtime that
launches nothing (stub_hip.cpp)."""
import pytest

from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


def test_lookup_refusals(without_a_device):
    without_a_device("""
h = context(B=4, V=1000, M=3, cap=100, d=128)
Q = P + 8                                                 # not 16-byte aligned
inf, nan = float("inf"), float("nan")
fwd = lambda c=h, codes=P, n=P, stride=7, E=P, W=P, scale=1.0, X=P, st=P + 64: lib.z2z_embed_codes(c, codes, n, stride, E, W, scale, X, st, None)
bwd = lambda c=h, codes=P, n=P, stride=7, scale=1.0, dX=P, flags=0, dE=P, dW=P: lib.z2z_embed_codes_backward(c, codes, n, stride, scale, dX, flags, dE, dW, None)
for bad in (dict(c=None), dict(codes=None), dict(E=None), dict(W=None), dict(X=None), dict(st=None), dict(stride=-1), dict(scale=inf), dict(scale=nan),
            dict(E=Q), dict(W=Q), dict(X=Q), dict(st=P)):             # (the last: the lengths' buffer)
    assert fwd(**bad) == api.E_INVAL, bad
for bad in (dict(c=None), dict(codes=None), dict(dX=None), dict(dE=None), dict(dW=None), dict(stride=-1), dict(scale=-inf), dict(flags=2), dict(flags=-1),
            dict(dX=Q), dict(dE=Q), dict(dW=Q)):
    assert bwd(**bad) == api.E_INVAL, bad
assert launches() == []
assert fwd(n=None) == 0 and len(launches()) == 1
assert fwd(stride=0, codes=None, X=None) == 0             # the statuses alone
assert len(launches()) == 1
assert bwd(stride=0, codes=None, dX=None) == 0            # zeros alone
log = launches()
assert len(log) == 1 and named(log, "reduce_kernel") == [(1000 + 400 + 63) // 64], log
assert bwd(stride=0, codes=None, dX=None, flags=api.GRAD_ADD) == 0 and launches() == []
no_book = context(B=4, V=1000, M=3, cap=0, d=128)
assert fwd(c=no_book, W=None) == 0 and bwd(c=no_book, dW=None) == 0
clean()
# positions and rows of the joint table are 32-bit numbers
assert bwd(stride=(1 << 29)) == api.E_UNSUPPORTED
assert bwd(c=context(B=33000, V=1000, M=2, cap=65535, d=8), stride=1) == api.E_UNSUPPORTED
clean()
""")


def test_gradient_work_space(without_a_device):
    without_a_device("""
h = context(B=4, V=1000, M=3, cap=100, d=128)
bwd = lambda stride: lib.z2z_embed_codes_backward(h, P, P, stride, 1.0, P, 0, P, P, None)
stub.stub_capacity(stub.stub_used())
assert bwd(100) == api.E_NOMEM
clean()
assert launches() == []
stub.stub_capacity(1 << 40)
stub.stub_capturing(1)
assert bwd(100) == api.E_CAPTURE and launches() == []     # nothing grows under capture
stub.stub_capturing(0)
assert bwd(1000) == 0
log = launches()
assert [len(named(log, k)) for k in ("sort_small", "sort_count", "reduce_kernel", "join_kernel")] == [1, 0, 1, 1], log
before = stub.stub_used()
assert bwd(5000) == 0                                     # the first buffer has gone back
log = launches()
assert [len(named(log, k)) for k in ("sort_small", "sort_count", "sort_place", "reduce_kernel", "join_kernel")] == [0, 2, 2, 1, 1], log
grown = stub.stub_used()
stub.stub_capturing(1)
assert bwd(5000) == 0                                     # a graph names the buffer from here on
stub.stub_capturing(0)
assert bwd(20000) == 0
assert stub.stub_used() > grown + (20000 - 5000) * 4 * 16 # the graph's buffer is still there
assert lib.z2z_destroy(h) == 0
assert stub.stub_used() == 0
clean()
""")


def test_beam_refusals(without_a_device):
    without_a_device("""
h = context(B=12, V=1000, M=3, cap=100, d=128)
Q = P + 8
pick = lambda c=h, H=P, rows=12, beams=4, Wb=P, Wh=P, score=P, n=8, parent=P, code=P, picked=P + 64: lib.z2z_extended_beam(c, H, rows, beams, Wb, Wh, score, n, parent, code, picked, None)
for bad in (dict(c=None), dict(H=None), dict(Wb=None), dict(Wh=None), dict(score=None), dict(parent=None), dict(code=None), dict(picked=None),
            dict(rows=11), dict(rows=24), dict(beams=0), dict(beams=-4), dict(beams=5), dict(n=0), dict(n=-1), dict(H=Q), dict(Wb=Q), dict(Wh=Q),
            dict(picked=P), dict(picked=P, n=3)):                         # (in place of the scores, but of another length)
    assert pick(**bad) == api.E_INVAL, bad
assert pick(n=65) == api.E_UNSUPPORTED
wide = context(B=66, V=1000, M=3, cap=100, d=128)
assert pick(c=wide, rows=66, beams=33) == api.E_UNSUPPORTED
assert launches() == []
assert pick() == 0 and pick(beams=12, n=64) == 0 and pick(beams=1, n=1) == 0 and pick(picked=P, n=4) == 0
assert named(launches(), "beam_pick") == [3, 1, 12, 3]
move = lambda c=h, beams=4, source=P, W=P: lib.z2z_codebook_reorder(c, beams, source, W, None)
for bad in (dict(c=None), dict(source=None), dict(beams=0), dict(beams=7), dict(W=Q)):
    assert move(**bad) == api.E_INVAL, bad
assert move(c=wide, beams=33) == api.E_UNSUPPORTED and launches() == []
assert move(W=None) == 0 and move() == 0 and len(launches()) == 2
clean()
fresh = context(B=12, V=1000, M=3, cap=100, d=128)
stub.stub_capturing(1)
assert pick(c=fresh) == api.E_CAPTURE and launches() == []
assert move(c=fresh) == 0                                 # (it has no work buffers)
stub.stub_capturing(0)
stub.stub_capacity(stub.stub_used())
assert pick(c=fresh) == api.E_NOMEM
clean()
""")


def test_distill_refusals(without_a_device):
    without_a_device("""
h = context(B=4, V=1000, M=3, cap=100, d=128)
Q = P + 8
fwd = lambda c=h, H=P, rows=40, rps=10, Wb=P, Wh=P, K=8, ids=P, t=P, T=2.0, kl=P, lse=P, st=P + 64: lib.z2z_extended_distill(c, H, rows, rps, Wb, Wh, K, ids, t, T, kl, lse, st, None)
bwd = lambda c=h, H=P, rows=40, rps=10, Wb=P, Wh=P, K=8, ids=P, t=P, T=2.0, lse=P, st=P, g=P, dH=P, dWb=P, dWh=P: lib.z2z_extended_distill_backward(c, H, rows, rps, Wb, Wh, K, ids, t, T, lse, st, g, dH, dWb, dWh, None)
common = [dict(c=None), dict(H=None), dict(Wb=None), dict(Wh=None), dict(ids=None), dict(t=None), dict(lse=None), dict(st=None), dict(rows=0), dict(rows=41),
          dict(rps=0), dict(K=0), dict(K=-3), dict(T=0.0), dict(T=-1.0), dict(T=0.06), dict(T=1025.0), dict(T=float("nan")), dict(T=float("inf")),
          dict(H=Q), dict(Wb=Q), dict(Wh=Q)]
for bad in common + [dict(kl=None), dict(st=P)]:          # (the last: the teacher's buffer)
    assert fwd(**bad) == api.E_INVAL, bad
for bad in common + [dict(dH=None), dict(dWb=None), dict(dWh=None), dict(dH=Q), dict(dWb=Q), dict(dWh=Q)]:
    assert bwd(**bad) == api.E_INVAL, bad
assert fwd(K=257) == api.E_UNSUPPORTED and bwd(K=257) == api.E_UNSUPPORTED
f32 = context(B=4, V=1000, M=3, cap=100, d=128, dtype=api.F32)
assert bwd(c=f32) == api.E_UNSUPPORTED and bwd(c=context(B=4, V=1000, M=3, cap=100, d=72)) == api.E_UNSUPPORTED
assert launches() == []
assert fwd() == 0 and fwd(K=256) == 0 and fwd(c=f32) == 0 and bwd() == 0 and bwd(g=None) == 0
log = launches()
assert len(named(log, "teacher_loss")) == 3 and len(named(log, "teacher_dz")) == 2 and not named(log, "row_grad"), log
clean()
fresh = context(B=4, V=1000, M=3, cap=100, d=128)
stub.stub_capturing(1)
assert fwd(c=fresh) == api.E_CAPTURE and bwd(c=fresh) == api.E_CAPTURE and launches() == []
stub.stub_capturing(0)
stub.stub_capacity(stub.stub_used())
assert fwd(c=fresh) == api.E_NOMEM and bwd(c=fresh) == api.E_NOMEM
clean()
""")


def test_a_temperature_leaves_the_decode_kernels(without_a_device):
    """At T = 1 the logits' parts come from the kernels that extended_nll takes (merged in the loss's own launch), at another T from those whose folds
    take one."""
    without_a_device("""
for rps in (1, 5, 100):
    h = context(B=8, V=40000, M=3, cap=1024, d=256)
    fwd = lambda T: lib.z2z_extended_distill(h, P, 8 * rps, rps, P, P, 4, P, P, T, P, P, P + 64, None)
    assert lib.z2z_extended_nll(h, P, 8 * rps, rps, P, P, P, P, P, None) == 0
    parts = lambda log: [n for n, _ in log if "logits_" in n and "combine" not in n]
    nll = parts(launches())
    assert fwd(1.0) == 0
    log = launches()
    assert parts(log) == nll and len(named(log, "combine")) == 0
    assert lib.z2z_extended_distill(h, P, 8 * rps, rps, P, P, 64, P, P, 1.0, P, P, P + 64, None) == 0
    assert len(named(launches(), "combine")) == (rps == 100)              # (800 rows of 64 columns)
    assert fwd(2.0) == 0
    assert not named(launches(), "logits_decode")
""")


def test_buffers_of_captured_calls_stay(without_a_device):
    """Calls that were captured into a graph, each with the buffers that it names, and larger calls of others behind it: nothing is given back
    before the context goes."""
    without_a_device("""
V, cap, d = 4096, 100, 128
enc = encoder(d)
calls = dict(
    logits=lambda h, n: lib.z2z_extended_logits(h, P, 4 * n, n, P, P, P, P, P, None, None),
    sample=lambda h, n: lib.z2z_extended_sample(h, P, 4, 1, P, P, 1.0, 50, 0.9, 1, 2, P, P, None),
    nll=lambda h, n: lib.z2z_extended_nll(h, P, 4 * n, n, P, P, P, P, P, None),
    nll_backward=lambda h, n: nll_backward(h, 4, n),
    encode=lambda h, n: lib.z2z_hyper_encode(h, P, ctypes.byref(enc), P, None, n, None),
    distill=lambda h, n: lib.z2z_extended_distill(h, P, 4 * n, n, P, P, 8, P, P, 2.0, P, P, P + 64, None),
    distill_backward=lambda h, n: lib.z2z_extended_distill_backward(h, P, 4 * n, n, P, P, 8, P, P, 2.0, P, P, P, P, P, P, None),
    lookup_backward=lambda h, n: lib.z2z_embed_codes_backward(h, P, P, n, 1.0, P, 0, P, P, None),
    beam=lambda h, n: lib.z2z_extended_beam(h, P, 4, 2, P, P, P, 3, P, P, P + 64, None))
none = stub.stub_used()
for name, call in calls.items():
    h = context(B=4, V=V, M=3, cap=cap, d=d)
    fixed = stub.stub_used()
    assert call(h, 50) == 0, name
    held = stub.stub_used()
    assert held > fixed, name
    stub.stub_capturing(1)
    assert call(h, 50) == 0, name
    stub.stub_capturing(0)
    launches()
    for other, larger in calls.items():
        before = stub.stub_used()
        stub.stub_capacity(before)                        # (no room: what the call gives back first is gone)
        larger(h, 90)
        assert stub.stub_used() == before, (name, other)
        stub.stub_capacity(1 << 40)
        assert larger(h, 90) == 0, (name, other)
    assert lib.z2z_destroy(h) == 0 and stub.stub_used() == none
clean()
""")
