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
for B, V, cap, d, K in ((1, 1000, 10, 4096, 64), (4, 50000, 100, 64, 3), (2, 5000, 300, 1024, 200)):
    for rows in (1, 61, 1000, 20000):
        nll, h = context(B=B, V=V, M=3, cap=cap, d=d), context(B=B, V=V, M=3, cap=cap, d=d)
        before = stub.stub_used()
        assert nll_backward(nll, B, rows) == 0
        middle = stub.stub_used()
        assert lib.z2z_extended_distill_backward(h, P, B * rows, rows, P, P, K, P, P, 2.0, P, P, P, P, P, P, None) == 0
        got = (stub.stub_used() - middle) - (middle - before)
        n, tables = B * rows * K, V + B * cap
        sums = max(n * d / 8, min(n, 262144 / -(-d // 512)) * d)
        assert got <= B * rows * (4 * d + 8) + min(n, tables) * 4 * d + 4 * tables + 22 * n + sums + 8 * d + 8192, (B, d, rows, got)
        assert lib.z2z_destroy(nll) == 0 and lib.z2z_destroy(h) == 0
clean()
""")


CALLS = """
V, cap, d = 4096, 100, 128
enc = encoder(d)
calls = dict(
    logits=lambda h, n: lib.z2z_extended_logits(h, P, 4 * n, n, P, P, P, P, P, None, None),
    nll_backward=lambda h, n: nll_backward(h, 4, n),
    encode=lambda h, n: lib.z2z_hyper_encode(h, P, ctypes.byref(enc), P, None, n, None),
    distill_backward=lambda h, n: lib.z2z_extended_distill_backward(h, P, 4 * n, n, P, P, 8, P, P, 2.0, P, P, P, P, P, P, None),
    lookup_backward=lambda h, n: lib.z2z_embed_codes_backward(h, P, P, n, 1.0, P, 0, P, P, None))
def make():
    return context(B=4, V=V, M=3, cap=cap, d=d)
def captured(call, h, n):
    stub.stub_capturing(1)
    rc = call(h, n)
    stub.stub_capturing(0)
    return rc
"""


def test_what_no_graph_names_is_given_back(without_a_device):
    """A context with one captured step and eager calls of slowly growing length holds the step's buffers and the last lengths', not every length's."""
    without_a_device(CALLS + """
step = lambda h: lib.z2z_extended_logits(h, P, 4, 1, P, P, P, P, P, None, None)
for name, call in calls.items():
    h = make()
    assert step(h) == 0 and captured(lambda h, n: step(h), h, 0) == 0
    fixed = stub.stub_used()
    for n in range(30, 100):
        assert call(h, n) == 0, name
    held = stub.stub_used() - fixed
    fresh = make()
    before = stub.stub_used()
    assert call(fresh, 99) == 0
    alone = stub.stub_used() - before
    assert held <= 1.5 * alone, (name, held, alone)       # (a half more where the step's own buffer had to grow)
clean()
""")


def test_a_refused_growth_leaves_what_there_was(without_a_device):
    """... to the shape that fitted, eager and captured, however often the growth is refused; named by a graph or not."""
    without_a_device(CALLS + """
for name, call in calls.items():
    for graph in (False, True):
        h = make()
        assert call(h, 40) == 0
        if graph:
            assert captured(call, h, 40) == 0
        used = stub.stub_used()
        stub.stub_capacity(used)
        for _ in range(5):
            rc = call(h, 90)
            assert rc in (0, api.E_NOMEM), (name, rc)     # (0: the encoder's shorter passes, or nothing had to grow)
            assert stub.stub_used() == used, (name, graph)
            assert captured(call, h, 40) == 0, (name, graph)
        stub.stub_capacity(1 << 40)
        assert call(h, 90) == 0
        clean()
""")


def test_graphs_of_every_length_keep_a_bounded_sum(without_a_device):
    without_a_device(CALLS + """
for name, call in calls.items():
    h = make()
    fixed = stub.stub_used()
    for n in range(30, 100):                              # every length captured before the next one needs more
        assert call(h, n) == 0 and captured(call, h, n) == 0, name
    held = stub.stub_used() - fixed
    fresh = make()
    before = stub.stub_used()
    assert call(fresh, 99) == 0
    assert held <= 4.5 * (stub.stub_used() - before), name        # 1.5 of it, and twice that kept
    assert lib.z2z_destroy(h) == 0
clean()
""")
