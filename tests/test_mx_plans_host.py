"""Host-side checks of the planners of the 4-bit calls (no GPU needed): the way taken at sizes on
both sides of each line, and the refusals of their test hooks."""
import os

import pytest
import torch

from paper_2606_29094_amd import dlm

pytestmark = pytest.mark.skipif(not os.path.exists(dlm.LIB_PATH), reason="libdlm.so not built")
BF16, F32 = torch.bfloat16, torch.float32
FEW, TILE32, TILE64, TILE128, UNPACKED = range(5)
STORE, ADD, SWIGLU = dlm.DLM_MX_STORE, dlm.DLM_MX_ADD, dlm.DLM_MX_SWIGLU


@pytest.mark.parametrize("dtype,m,n,k,epilogue,way", [
    (BF16, 1, 4096, 4096, STORE, FEW), (BF16, 32, 4096, 4096, STORE, FEW), (BF16, 64, 4096, 4096, STORE, TILE32),
    (BF16, 12, 24576, 4096, SWIGLU, FEW), (BF16, 32, 24576, 4096, SWIGLU, TILE32),
    (BF16, 4, 4096, 12288, ADD, FEW), (BF16, 16, 4096, 12288, ADD, TILE32), (BF16, 64, 3584, 18944, ADD, TILE64),
    (BF16, 256, 4096, 4096, STORE, TILE32), (BF16, 512, 37888, 3584, SWIGLU, TILE64),
    (BF16, 1000, 37888, 3584, SWIGLU, TILE128), (BF16, 2047, 12288, 4096, STORE, TILE128),
    (BF16, 2048, 12288, 4096, STORE, UNPACKED), (F32, 1, 4096, 4096, STORE, FEW),
    (F32, 4096, 24576, 4096, SWIGLU, TILE128)])
def test_way(dtype, m, n, k, epilogue, way):
    assert dlm.debug_mx_linear_plan(dtype, m, n, k, epilogue)[0] == way


def test_operands_of_32_bits_are_unpacked_others_not():
    """The GEMM kernels take operands of fewer than 2^32 elements."""
    plan = lambda m, n, k, **kw: dlm.debug_mx_linear_plan(BF16, m, n, k, **kw)[0]
    assert plan(2048, 131008, 32768) == UNPACKED and plan(2048, 131072, 32768) != UNPACKED
    assert plan(2048, 4096, 4096, ldx=(1 << 21) - 8) == UNPACKED
    assert plan(2048, 4096, 4096, ldx=1 << 21) != UNPACKED


def test_unpacked_where_the_gemm_kernels_are_faster():
    """Both sides of each line, at the sizes that were measured."""
    for n, k, epilogue in [(24576, 4096, SWIGLU), (4096, 12288, ADD), (4608, 3584, STORE), (4096, 4096, STORE)]:
        for m in (3000, 4096):
            assert dlm.debug_mx_linear_plan(BF16, m, n, k, epilogue)[0] == UNPACKED
            # k no multiple of 64: those kernels stage such operands through registers
            for odd in (k - 8, k - 32, k + 8):
                assert dlm.debug_mx_linear_plan(BF16, m, n, odd, epilogue)[0] != UNPACKED
    for m in (2048, 4096):                  # small matrices
        for n, k in [(2048, 2048), (1088, 1024), (1040, 1032), (512, 18944)]:
            assert dlm.debug_mx_linear_plan(BF16, m, n, k)[0] != UNPACKED


def test_buffers_that_vector_accesses_cannot_take():
    for aligned in (0, 2):                  # rows of x: copied first, straight from the codes
        way, _, staged = dlm.debug_mx_linear_plan(BF16, 4096, 4096, 4096, aligned=aligned)
        assert way != UNPACKED and staged
    assert dlm.debug_mx_linear_plan(BF16, 4096, 4096, 4096, aligned=1)[0] != UNPACKED
    assert not dlm.debug_mx_linear_plan(BF16, 70, 4096, 4096)[2]
    assert dlm.debug_mx_linear_plan(BF16, 70, 4096, 4100)[2] and dlm.debug_mx_linear_plan(F32, 70, 4096, 4096)[2]


def test_slices_left_to_the_reader_cost_less():
    for m in (16, 64, 200, 1000):
        joined = dlm.debug_mx_linear_plan(BF16, m, 3584, 18944)[1]
        assert dlm.debug_mx_linear_plan(BF16, m, 3584, 18944, join=False)[1] >= joined


@pytest.mark.parametrize("heads,batch,kernel,splits", [
    # few rows: waves that split the keys, whole; few blocks: the keys split over blocks as well
    ((32, 32, 128), (8, 32, 1280), 0, 1), ((32, 32, 128), (1, 32, 4256), 0, 8), ((32, 32, 128), (1, 32, 517), 1, 4),
    ((28, 4, 128), (8, 32, 1024), 0, 1), ((28, 4, 128), (16, 64, 1024), 1, 1), ((28, 4, 128), (64, 64, 1024), 2, 1),
    ((28, 4, 128), (3, 700, 700), 2, 1), ((32, 32, 128), (8, 1280, 1280), 2, 1), ((32, 32, 128), (1, 300, 300), 1, 1),
    ((12, 2, 64), (16, 64, 2000), 0, 1), ((12, 2, 64), (64, 64, 1000), 1, 1)])
def test_attention_kernel(heads, batch, kernel, splits):
    n, rows, keys = batch
    assert dlm.debug_mx_attention_plan(BF16, *heads, [rows] * n, [keys] * n) == (kernel, splits)
    assert dlm.debug_mx_attention_plan(F32, *heads, [rows] * n, [keys] * n)[0] == 0


def test_attention_plan_stays_within_the_scratch():
    one = 32 * 32 * (128 + 2) * 4
    for splits in (1, 2, 4, 8):
        assert dlm.debug_mx_attention_plan(BF16, 32, 32, 128, [32], [4256], splits * one)[1] <= splits
    assert dlm.debug_mx_attention_plan(BF16, 32, 32, 128, [32], [4256], 0)[1] == 1
    assert dlm.debug_mx_attention_plan(BF16, 32, 32, 128, [32], [4256], 8 * one)[1] == 8


def test_plan_hooks_refused():
    L = dlm.lib()
    out, k, s = (dlm.c_int32 * 3)(), dlm.c_int32(), dlm.c_int32()
    good = [1, 4, 64, 64, 64, 0, 3, 1, 256]
    assert L.dlm_debug_mx_linear_plan(*good, out) == dlm.DLM_OK
    for at, bad in [(0, 2), (1, 0), (1, -1), (1, 1 << 30), (2, 0), (3, 0), (4, 63), (5, 3), (5, -1), (8, 0)]:
        assert L.dlm_debug_mx_linear_plan(*good[:at], bad, *good[at + 1:], out) == dlm.DLM_EINVAL
    assert L.dlm_debug_mx_linear_plan(*good, None) == dlm.DLM_EINVAL
    assert L.dlm_debug_mx_linear_plan(1, 4, 64, 64, 64, 1, 3, 0, 256, out) == dlm.DLM_EINVAL   # add, not joined
    assert L.dlm_debug_mx_linear_plan(1, 4, 63, 64, 64, 2, 3, 1, 256, out) == dlm.DLM_EINVAL   # odd SwiGLU
    rows, lens = (dlm.c_int32 * 2)(4, 0), (dlm.c_int32 * 2)(0, 70)
    good = [1, 4, 2, 64, 2, rows, lens, 0, 256, k, s]
    assert L.dlm_debug_mx_attention_plan(*good) == dlm.DLM_OK
    for at, bad in [(0, 2), (1, 0), (1, 3), (2, 0), (3, 96), (4, 0), (4, 65), (5, None), (6, None), (8, 0), (9, None),
                    (10, None), (5, (dlm.c_int32 * 2)(-1, 4)), (6, (dlm.c_int32 * 2)(8193, 4))]:
        assert L.dlm_debug_mx_attention_plan(*good[:at], bad, *good[at + 1:]) == dlm.DLM_EINVAL
