"""Outputs that lie in inputs which other workgroups still read: refused, without a GPU, against a HIP runtime that launches nothing (stub_hip.cpp)."""
from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


def test_overlapping_buffers_are_refused(without_a_device):
    without_a_device("""
h = context(B=12, V=1000, M=3, cap=100, d=128)
Q = P + 4096
pick = lambda picked, beams=4, n=8: lib.z2z_extended_beam(h, P, 12, beams, P, P, Q, n, P, P, picked, None)
for n in (1, 3, 4, 8):
    size = 12 // 4 * n * 4                                # bytes of the picks; the scores are 48
    for at in (Q - size, Q + 48):
        assert pick(at, n=n) == 0, (n, at)                # beside them
    for at in (Q - size + 4, Q + 4, Q + 44) + ((Q,) if n != 4 else ()):
        assert pick(at, n=n) == api.E_INVAL, (n, at)
assert pick(Q, n=4) == 0 and pick(Q, beams=12, n=12) == 0 and pick(Q, beams=1, n=1) == 0
look = lambda st, n: lib.z2z_embed_codes(h, P, n, 7, P, P, 1.0, P, st, None)
for at in (Q - 44, Q - 4, Q, Q + 4, Q + 44):
    assert look(at, Q) == api.E_INVAL, at
assert look(Q - 48, Q) == 0 and look(Q + 48, Q) == 0 and look(Q, None) == 0
loss = lambda ids, t, st: lib.z2z_extended_distill(h, P, 12, 1, P, P, 8, ids, t, 2.0, P, P, st, None)
launches()
assert loss(Q, P, Q) == api.E_INVAL and loss(P, Q, Q) == api.E_INVAL and launches() == []
assert loss(P, P, Q) == 0
clean()
""")
