"""Plans of products of 8-bit matrices (host only): row tiles go in groups where there are
several."""
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
