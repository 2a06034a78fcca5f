"""The library's work buffers without a GPU, against a HIP runtime that launches nothing (stub_hip.cpp): how large they are, and when they are given back."""
import pytest

from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


@pytest.mark.parametrize("d,dtype", [(4096, "BF16"), (64, "BF16"), (1000, "BF16"), (2048, "F32")])
def test_a_call_makes_room_for_every_smaller_one(without_a_device, d, dtype):
    """After one eager call at the largest shape the smaller ones need nothing more, so that they can be captured; at the lengths around those where the
    sort goes over to tiles and the sums to longer pieces."""
    without_a_device(f"""
d, dtype = {d}, api.{dtype}
slices = -(-d // (512 if dtype == api.BF16 else 256))
def turns(piece):
    first = -(-4096 * piece // slices)
    return [1, 7, 8, 9, 4095, 4096, 4097, 8192, first - 1, first, first + 1, first + 4096]
h = context(B=1, V=1000, M=3, cap=10, d=d, dtype=dtype)
lookup = lambda n: lib.z2z_embed_codes_backward(h, P, None, n, 1.0, P, 0, P, P, None)
assert lookup(2 * turns(32)[-1]) == 0
used = stub.stub_used()
stub.stub_capturing(1)
for n in turns(32):
    assert lookup(n) == 0, n
stub.stub_capturing(0)
assert stub.stub_used() == used
if dtype == api.BF16 and d % 64 == 0:
    K = 32
    h = context(B=1, V=1000, M=3, cap=10, d=d)
    distill = lambda rows: lib.z2z_extended_distill_backward(h, P, rows, rows, P, P, K, P, P, 2.0, P, P, P, P, P, P, None)
    assert distill(2 * turns(64)[-1] // K) == 0
    used = stub.stub_used()
    stub.stub_capturing(1)
    for n in turns(64):
        assert distill(max(n // K, 1)) == 0, n
    stub.stub_capturing(0)
    assert stub.stub_used() == used
clean()
""")


def test_the_work_space_is_what_the_header_says(without_a_device):
    without_a_device("""
for B, V, cap, d, dtype in ((1, 1000, 10, 4096, api.BF16), (4, 50000, 100, 64, api.BF16), (3, 5000, 300, 1000, api.BF16), (1, 1000, 10, 2048, api.F32)):
    slices = -(-d // (512 if dtype == api.BF16 else 256))
    for n in (1, 100, 5000, 100000, 1000000):
        h = context(B=B, V=V, M=3, cap=cap, d=d, dtype=dtype)
        before = stub.stub_used()
        assert lib.z2z_embed_codes_backward(h, P, None, n, 1.0, P, 0, P, P, None) == 0
        positions = B * n
        got = stub.stub_used() - before
        sums = max(positions * d / 4, min(positions, 131072 / slices) * d)
        assert got <= 18 * positions + sums + 8 * d + 4096, (B, d, n, got)
        assert lib.z2z_destroy(h) == 0
clean()
""")
