"""GPU parity of the streaming kernel's builds for 65 to 96 and 129 to 160 hidden rows (section 2.3, steps 7-9): both tile widths, few and many
slabs of K, every row against the oracle as in test_gpu_logits_mid.py."""
import pytest

from test_gpu_logits_mid import test_streaming_kernel_every_row_ragged as check
from test_gpu_logits_mid import test_streaming_kernel_planted_rows_pin_every_base_column as check_planted

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,rows_per_seq,V,d,M,cap,pool", [
    (66, 1, 777, 192, 3, 0, "mean"),             # three slabs: fewer than the stages of half tiles
    (96, 1, 1000, 128, 3, 300, "mean"),          # every row of the 96-row build, two slabs
    (1, 65, 300, 64, 3, 100, "mean"),            # one slab
    (3, 27, 513, 576, 3, 70, "weighted"),        # 81 rows, nine slabs
    (2, 47, 33000, 704, 3, 200, "mean"),         # tiles of 256 columns, eleven slabs, hyper tiles along
    (80, 1, 32900, 192, 3, 0, "mean"),           # three slabs, the ring exactly
    (4, 24, 16500, 4096, 3, 40, "mean"),         # past the caches, half of the waves ask twice
    (129, 1, 1300, 256, 3, 60, "mean"),
    (160, 1, 513, 192, 3, 0, "mean"),            # every row of the 160-row build
    (1, 131, 300, 64, 3, 130, "mean"),
    (2, 79, 33300, 448, 4, 256, "weighted"),
    (5, 30, 32800, 320, 3, 20, "mean"),
    (6, 26, 16500, 4096, 3, 40, "mean"),
])
def test_every_row(B, rows_per_seq, V, d, M, cap, pool):
    check(B, rows_per_seq, V, d, M, cap, pool)


@pytest.mark.parametrize("rows_per_call,d", [(66, 192), (96, 320), (130, 256), (160, 448)])
def test_planted_rows_pin_every_base_column(rows_per_call, d):
    check_planted(rows_per_call, d)
