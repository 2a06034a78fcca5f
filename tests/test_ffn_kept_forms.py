"""What a gated block's calls keep in 16 bits: sizes, launches and refusals, without a GPU (stub_hip.cpp); and the code of the kernel that keeps it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_01084_amd import api
from test_wait_states import OBJDUMP
from test_ffn_clip_refusals import BLOCK
from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


def test_sizes_launches_and_refusals(without_a_device):
    without_a_device(BLOCK + """
def packed(**kw):
    f = block(**kw)
    f.kept = api.KEPT_16
    return f
keep = 24 * 256 * 4                                       # half of what the other form takes
assert fwd(h, packed(), kept=K) == 0 and bwd(h, packed(), kept=K) == 0
launches()
for rows in (1, 24, 700, 5000):
    assert fwd(h, packed(), rows=rows, kept=K) == 0
    first = launches()
    assert fwd(h, block(), rows=rows, kept=K) == 0
    alike = lambda log: [(n.replace("Lb0ELi3EEEvN10z2z_logits", "Lb0ELi1EEEvN10z2z_logits"), g) for n, g in log]      # (the tile kernel's instance)
    assert alike(launches()) == alike(first)
    assert bwd(h, packed(), rows=rows) == 0
    first = launches()
    assert bwd(h, block(), rows=rows) == 0 and launches() == first[1:] and "kept_pairs" in first[0][0]
assert fwd(h, packed(), kept=X - keep) == 0 and fwd(h, packed(), kept=X - keep + 16) == api.E_INVAL and fwd(h, block(), kept=X - keep) == api.E_INVAL
assert bwd(h, packed(), dX=K + keep) == 0 and bwd(h, packed(), dX=K + keep - 16) == api.E_INVAL and bwd(h, block(), dX=K + keep) == api.E_INVAL
launches()
for form in (1, 2, 8, 32, -16):
    f = block()
    f.kept = form
    assert fwd(h, f, kept=K) == api.E_INVAL and fwd(h, f) == api.E_INVAL and bwd(h, f) == api.E_INVAL
f = four()
f.kept = api.KEPT_16
assert fwd(h, f, kept=K) == api.E_UNSUPPORTED and fwd(h, f) == 0
launches()
# work space: the two gradients, and the matrices that 16 bits are turned into
fresh = context(B=1, V=8, M=2, cap=0, d=512)
used = stub.stub_used()
assert bwd(fresh, packed(), rows=4000) == 0 and stub.stub_used() >= used + 4000 * 256 * 12
launches()
assert bwd(fresh, packed(), rows=0, X=None, kept=None, dY=None, dX=None) == 0
clean()
""")


def test_encoder_blocks_keep_32_bits(without_a_device):
    without_a_device(BLOCK + """
c = context(B=2, V=100, M=3, cap=50, d=512)
g = api.GatedEncoderDesc()
g.encoder = e = encoder(512, 1)
g.encoder.attention_only = api.ENC_GATED
one = (api.FfnDesc * 1)(block())
g.ffn = ctypes.cast(one, ctypes.POINTER(api.FfnDesc))
enc = lambda: lib.z2z_hyper_encode(c, P, ctypes.byref(g.encoder), P, None, 1, None)
assert enc() == 0
launches()
one[0].kept = api.KEPT_16
assert enc() == api.E_INVAL and lib.z2z_hyper_encode_keep(c, P, ctypes.byref(g.encoder), P, None) == api.E_INVAL and launches() == []
""")


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_the_tile_kernel_spills_nothing(tmp_path):
    """Its matrix instructions and their waits are inline assembly: accumulators that the compiler moves to memory are read before they are there."""
    lib = str(tmp_path / "libz2z.so")
    shutil.copy(api.LIB_PATH, lib)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True)
    seen = 0
    for obj in sorted(p for p in tmp_path.iterdir() if "amdgcn" in p.name and "gfx950" in p.name):
        notes = subprocess.run([os.path.join(os.path.dirname(OBJDUMP), "llvm-readelf"), "--notes", str(obj)], check=True, capture_output=True, text=True).stdout
        for name, scratch in re.findall(r"\.name:\s+(\S*logits_fast_kernel\S*)\n(?:.*\n)*?\s+\.private_segment_fixed_size: (\d+)", notes):
            seen += 1
            assert int(scratch) == 0, name
    assert seen >= 20


def test_a_call_that_keeps_its_hidden_layer_takes_no_work_space(without_a_device):
    without_a_device(BLOCK + """
used = stub.stub_used()
stub.stub_capturing(1)
for rows in (1, 16, 64, 200):                             # (no parts either)
    assert fwd(h, block(), rows=rows, kept=K) == 0 and len(launches()) == 2, rows
assert fwd(h, block(), rows=16) == api.E_CAPTURE and launches() == []
f = block()
f.kept = api.KEPT_16
assert fwd(h, f, rows=16, kept=K) == api.E_CAPTURE and launches() == []
stub.stub_capturing(0)
assert stub.stub_used() == used
assert fwd(h, f, rows=16, kept=K) == 0 and stub.stub_used() == used + 16 * 256 * 2
launches()
assert fwd(h, block(), rows=200) == 0 and stub.stub_used() == used + 200 * 256 * 2
clean()
""")
