"""Calls of more threads than a launch can count (2^32): several launches or a refusal, without a GPU, against a HIP runtime that launches nothing
(stub_hip.cpp)."""
from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


def test_no_launch_has_more_threads_than_it_can_count(without_a_device):
    without_a_device("""
LIMIT = (1 << 32) - 1
h = context(B=3, V=100, M=2, cap=10, d=8)
look = lambda stride: lib.z2z_embed_codes(h, P, None, stride, P, P, 1.0, P, P, None)
for positions in (3, 3 << 20, (1 << 26) - 13, (1 << 26) - 12, 1 << 26, 3 << 25, (1 << 31) - 2):
    stride = positions // 3
    assert look(stride) == 0
    grids = named(launches(), "embed_codes")
    assert sum(grids) - 3 >= (3 * stride + 3) // 4 and all(g * 256 <= LIMIT for g in grids), (positions, grids)
    assert len(grids) == -(-(3 + (3 * stride + 3) // 4) // (LIMIT // 256)), (positions, grids)
many = context(B=(1 << 24) - 1, V=100, M=2, cap=0, d=8)   # a workgroup each for the statuses
assert lib.z2z_embed_codes(many, P, None, 1, P, None, 1.0, P, P, None) == api.E_UNSUPPORTED and launches() == []
assert lib.z2z_destroy(many) == 0
back = lambda c, stride: lib.z2z_embed_codes_backward(c, P, None, stride, 1.0, P, 0, P, P, None)
wide = context(B=1, V=100, M=2, cap=10, d=4096)
for c, B, slices, stride in ((h, 3, 1, 1000), (h, 3, 1, 600 << 20), (h, 3, 1, 670 << 20), (wide, 1, 8, 100 << 20), (wide, 1, 8, 500 << 20)):
    rc, log = back(c, stride), launches()
    fits = 4 * (100 + B * 10) + 2 * B * stride * slices < (1 << 32) - (1 << 27)
    assert rc == (0 if fits else api.E_UNSUPPORTED), (B, stride, rc)
    assert all(g * (1024 if "sort" in n else 256) <= LIMIT for n, g in log) and (log or rc), log
clean()
""")


def test_moves_of_many_entries(without_a_device):
    without_a_device("""
LIMIT = (1 << 32) - 1
for B, cap, beams, n in ((64, 65535, 2, 1), (2048, 65535, 2, 2), (2100, 65535, 1, 3), (1024, 65535, 1, 2)):
    h = context(B=B, V=1000, M=2, cap=cap, d=8)
    assert lib.z2z_codebook_reorder(h, beams, P, P, None) == 0
    grids = named(launches(), "reorder")
    assert len(grids) == n and all(g * 256 <= LIMIT for g in grids), grids
    assert sum(grids) > (B // beams * cap + 3) // 4
    assert lib.z2z_destroy(h) == 0
clean()
""")


def test_rows_beyond_a_launch_are_refused(without_a_device):
    without_a_device("""
h = context(B=1, V=100, M=2, cap=10, d=64)
fwd = lambda rows, K: lib.z2z_extended_distill(h, P, rows, rows, P, P, K, P, P, 2.0, P, P, P + 64, None)
bwd = lambda rows, K: lib.z2z_extended_distill_backward(h, P, rows, rows, P, P, K, P, P, 2.0, P, P, P, P, P, P, None)
assert fwd((1 << 26) // 12 + 1, 64) == api.E_UNSUPPORTED and fwd((1 << 26) // 5 + 1, 1) == api.E_UNSUPPORTED
assert bwd(1 << 26, 1) == api.E_UNSUPPORTED and bwd(1 << 26, 64) == api.E_UNSUPPORTED
assert launches() == []
assert fwd((1 << 26) // 12 - 1, 64) == 0
clean()
many = context(B=40000, V=7000000, M=2, cap=1, d=4, dtype=api.F32)
assert lib.z2z_extended_beam(many, P, 40000, 1, P, P, P, 1, P, P, P + (1 << 20), None) == api.E_UNSUPPORTED and launches() == []
""")
