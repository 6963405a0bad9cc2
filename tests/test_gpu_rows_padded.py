"""Ragged rows under a leading dimension that keeps them 16-byte aligned, as a program pads them: the last vector of a row reaches into the padding,
which must be neither read as values nor written. RMS norm, rows in 8 bits, gradients and dropout, in every kernel shape. Needs a B200. Cases and
bounds of test_gpu_rmsnorm and test_gpu_dropout (padding of NaN or guard bytes)."""
import pytest
import torch

import test_gpu_dropout as drop
import test_gpu_rmsnorm as rms

pytestmark = pytest.mark.gpu

# one warp per row, blocks of a few and of many warps, rows through shared memory by blocks of 256 and 512 threads, 32 values per thread, single
# rows and longer ones; padding to 8 columns (a whole vector in 16 bits, two in binary32)
COLS = [1, 7, 33, 131, 259, 513, 1001, 1027, 2051, 4091, 5001, 8189, 9001, 16379, 17001, 20001]
ROWS = {cols: [1, 5, max(40, min(9001, 1_300_000 // cols)), max(300, min(9001, 4_000_000 // cols))] for cols in COLS}


@pytest.mark.parametrize("dtype", rms.TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_rows_padded_to_whole_vectors(cols, dtype):
    pad = -cols % 8
    for rows in ROWS[cols]:
        at = dict(pad=pad, seed=rows)
        rms.forward(rows, cols, dtype, **at)
        rms.forward(rows, cols, dtype, res=False, keep=False, **at)
        rms.forward8(rows, cols, dtype, **at)
        rms.forward8(rows, cols, dtype, res=False, keep=False, affine=False, **at)
        rms.rows8(rows, cols, dtype, **at)
        rms.backward(rows, cols, dtype, **at)
        rms.backward(rows, cols, dtype, ds=False, affine=False, **at)
        rms.backward(rows, cols, dtype, want=("dgamma",), **at)


@pytest.mark.parametrize("dtype", rms.TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_outputs_in_the_place_of_inputs(cols, dtype):
    pad = -cols % 8 + 8
    for rows in ROWS[cols][1:]:
        for place in ("X", "R"):
            rms.forward(rows, cols, dtype, in_place=place, pad=pad)
            rms.forward8(rows, cols, dtype, in_place=place, pad=pad)
        rms.backward(rows, cols, dtype, in_place=True, pad=pad)


@pytest.mark.parametrize("dtype", drop.TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_dropout(cols, dtype):
    pad = -cols % 8
    for rows in ROWS[cols]:
        drop._case(rows, cols, dtype, pad=pad)
        drop._case(rows, cols, dtype, res=False, pad=pad + 8)
        drop._case(rows, cols, dtype, pad=pad, place="R")


@pytest.mark.parametrize("cols", [259, 4091, 9001])
def test_padding_of_8_bit_outputs_alone(cols):
    """8-bit rows packed while the others are padded, and the other way round."""
    pad = -cols % 8
    for dtype in rms.TYPES:
        for rows in ROWS[cols]:
            rms.forward8(rows, cols, dtype, pad=pad, qpad=0)
            rms.forward8(rows, cols, dtype, pad=0, qpad=pad)
            rms.forward8(rows, cols, dtype, pad=pad, qpad=pad + 8, qoffset=8)
