"""Products of more rows than the tiles' 32-bit offsets reach are launched in parts by one plan
(host only): it has to fit every part, the last and smallest one too."""
import os
import random

import pytest

import qint_reference as ref
from paper_2606_29094_amd import dlm

pytestmark = pytest.mark.skipif(not os.path.exists(dlm.LIB_PATH), reason="libdlm.so not built")
MAX_ROWS = 524288


def part_rows(k):
    """Rows of a part: what 32-bit offsets of 2-byte units reach, in whole 256s."""
    return ((1 << 32) // (ref.row_bytes(k) // 2) - 1) & ~255


@pytest.mark.parametrize("m,n,k,epilogue", [
    (349441, 4, 24576, 0), (349441, 4, 24576, 1), (349441, 4, 24576, 2), (299521, 8192, 28672, 1),
    (300032, 8192, 28672, 1), (65281, 6, 131071, 0), (65536, 2000, 131071, 2)])
def test_no_sub_tiles_in_parts(m, n, k, epilogue):
    assert m > part_rows(k)
    cfg, slices, sub, _ = dlm.debug_qint_linear_plan(m, n, k, epilogue)
    assert cfg >= 0 and slices == 1 and sub == 0


def test_no_sub_tiles_in_parts_of_any_size():
    rng, seen = random.Random(11), 0
    while seen < 4000:
        k = rng.randint(16385, ref.MAX_K)
        m = part_rows(k) + rng.choice([1, 255, 256, 257, rng.randint(1, 100000)])
        n = 2 * int(30000 ** rng.random())
        if m > MAX_ROWS or n * ref.row_bytes(k) >= 1 << 33:
            continue
        seen += 1
        for epilogue in range(3):
            cfg, slices, sub, _ = dlm.debug_qint_linear_plan(m, n, k, epilogue, rng.choice([80, 256, 304]))
            assert cfg >= 0 and slices == 1 and sub == 0, (m, n, k, epilogue)
