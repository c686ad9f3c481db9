"""What the loads of the feed-forward block's products may reach: csrc/load_range.h compiled for the host, asked as the kernels ask it, with
the buffer's own check -- an offset counts if it lies below end - from, in 32 bits, which come round."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2104_01981_amd", "csrc")
SOURCE = """
#include "load_range.h"
using namespace ecrm;
static bool counts(uint32_t offset, uint32_t end, uint32_t from) { return offset < (uint32_t)(end - from); }
extern "C" {
// Tiles of `tile` rows of an operand of `count`, whose first rows are every `step`-th up to `to`, all of K (`width` bytes, 128 at a time):
// how many loads of 16 bytes reach memory that is not the operand's, or miss some of it.
uint64_t wrong_rows(uint32_t count, uint32_t to, uint32_t step, uint32_t tile, uint32_t stride, uint32_t width)
{
    uint64_t wrong = 0;
    for (uint32_t first = 0; first < to; first += step) {
        const uint32_t end = rows_end(count, first, tile, stride, width);
        for (uint32_t at = 0; at < width; at += 128) {
            const uint32_t from = rows_from(end, at);
            if (from > end || counts(kOutside, end, from)) ++wrong;
            for (uint32_t row = 0; row < tile; ++row)
                for (uint32_t chunk = 0; chunk < 128 && at + chunk < width; chunk += 16)
                    if (counts(row * stride + chunk, end, from) != (first + row < count)) ++wrong;
        }
    }
    return wrong;
}
// The same for rows across K: a row of K behind `rows` counts nowhere, and of those before it what the operand has of columns.
uint64_t wrong_columns(uint32_t count, uint32_t to, uint32_t step, uint32_t tile, uint32_t stride, uint32_t rows, uint32_t size)
{
    uint64_t wrong = 0;
    for (uint32_t first = 0; first < to; first += step) {
        const uint32_t width = (count > first ? count - first : 0u) * size, end = columns_end(rows, stride, width);
        if (counts(kOutside, end, 0)) ++wrong;
        for (uint32_t row = 0; row < rows + 3; ++row)
            for (uint32_t byte = 0; byte < tile * size; byte += 16) {
                const bool got = counts(row * stride + byte, end, 0), there = row < rows && byte < width;
                if ((there && !got) || (got && (row >= rows || !width))) ++wrong;
            }
    }
    return wrong;
}
}
"""


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("ranges")
    src, out = tmp / "ranges.cpp", tmp / "ranges.so"
    src.write_text(SOURCE)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-I", CSRC, str(src), "-o", str(out)])
    lib = C.CDLL(str(out))
    for f in (lib.wrong_rows, lib.wrong_columns):
        f.argtypes, f.restype = [C.c_uint32] * (6 if f is lib.wrong_rows else 7), C.c_uint64
    return lib


# rows of a tile and how far the begins of a wave's are from each other: kGate's tiles of 256 columns in 16 bits have two halves of 64 of each
# projection, those of 32 in 32 bits two of 16, the others all of a projection at once
@pytest.mark.parametrize("tile,step,size", [(64, 64, 2), (16, 16, 4), (64, 64, 4), (32, 32, 2), (32, 32, 4), (128, 128, 2), (256, 256, 2)])
def test_rows_of_no_operand_are_never_read(ranges, tile, step, size):
    for count in [4, 8, 12, 60, 64, 68, 124, 128, 132, 196, 260, 364, 516, 684, 860, 1028]:
        to = (count + 2 * step - 1) // (2 * step) * 2 * step     # whole tiles of two halves: the second may lie behind the last row
        for K, extra in ((4, 0), (36, 4), (68, 0), (132, 12), (260, 4), (700, 64)):
            assert ranges.wrong_rows(count, to, step, tile, (K + extra) * size, K * size) == 0, (count, K, extra)


@pytest.mark.parametrize("size", [2, 4])
def test_rows_at_the_largest_distance(ranges, size):
    """2^20 elements from row to row, the longest rows: sums of offsets stay below 2^31."""
    assert ranges.wrong_rows(260, 512, 256, 256, size << 20, 65536 * size) == 0


@pytest.mark.parametrize("tile,size", [(256, 2), (128, 2), (64, 2), (128, 4), (64, 4), (32, 4)])
def test_columns_of_no_operand_are_never_read(ranges, tile, size):
    for count in [4, 12, 60, 64, 68, 132, 260, 516, 684]:
        for rows in (1, 3, 31, 32, 64):
            for extra in (0, 4, 1 << 18):
                assert ranges.wrong_columns(count, count + 2 * tile, tile, tile, (count + extra) * size, rows, size) == 0, (count, rows, extra)
