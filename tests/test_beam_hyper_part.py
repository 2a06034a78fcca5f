"""Where a beam step's hyper part shares the streaming kernel's launch: without a GPU, against a HIP runtime that launches nothing (stub_hip.cpp; 256
CUs)."""
import pytest

from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


@pytest.mark.parametrize("V,d,cap,rows,along", [
    (16000, 4096, 256, 64, True),        # 125 and 128 tiles: one round instead of two
    (16000, 2048, 1024, 16, True),
    (49000, 2048, 1024, 16, True),       # 192 and 64: exactly one
    (49000, 2048, 1024, 64, False),      # 192 and 256: two either way
    (65000, 4096, 256, 4, False),        # 254 and 4
    (65500, 2048, 512, 4, False),        # 256 and 8
    (66000, 1024, 512, 4, True),         # 258 and 8: two instead of three
    (16000, 4096, 1024, 80, False),      # 125 and 640: 765 of three rounds' 768
    (16000, 4096, 1000, 72, True),       # 125 and 576: three instead of four
    (8000, 1024, 65535, 32, True),       # short workgroups, two to a CU
    (8000, 1024, 0, 32, False),
])
def test_the_launches_of_a_beam_step(without_a_device, V, d, cap, rows, along):
    without_a_device(f"""
h = context(B={rows}, V={V}, M=3, cap={cap}, d={d})
assert lib.z2z_extended_beam(h, P, {rows}, 4, P, P, P, 8, P, P, P + 4096, None) == 0
log = launches()
assert len(named(log, "logits_mid")) == 1 and len(named(log, "logits_decode")) == {int(not along and cap > 0)}, log
""")
