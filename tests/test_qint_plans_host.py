"""Plans of products of 8-bit matrices (host only): tiles that exist for them, row tiles in groups
where there are several."""
import os
import random

import pytest

from paper_2606_29094_amd import dlm

pytestmark = pytest.mark.skipif(not os.path.exists(dlm.LIB_PATH), reason="libdlm.so not built")


def test_groups_take_several_row_tiles():
    rng, alone, several = random.Random(5), 0, 0
    for _ in range(4000):
        n, k = rng.choice([(37888, 3584), (28672, 8192), (24576, 4096), (2 * int(30000 ** rng.random()), 16384)])
        m, epilogue = int(524288 ** rng.random()), rng.randrange(3)
        cfg, slices, _, group = dlm.debug_qint_linear_plan(m, n, k, epilogue)
        if cfg < 0 or slices > 1:
            continue
        if m <= dlm.debug_gemm_info(cfg)[0]:
            assert group == 0, (m, n, k, epilogue)
            alone += 1
        else:
            several += group > 0
    assert alone > 500 and several > 500


def test_tiles_exist_for_8_bit_operands():
    """Those of the vocabulary head alone, of 32 x 32 matrix instructions and 82 do not."""
    rng = random.Random(6)
    size = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    for _ in range(10000):
        n, k = 2 * size(1, 30000), size(1, 131071)
        cfg = dlm.debug_qint_linear_plan(size(1, 20000), n, k, rng.randrange(3), rng.choice([8, 80, 256, 304]))[0]
        assert cfg not in (1, 10, 11, 62, 65, 82)
