"""The limits of packed matrices and their products, as the header has them: what lies at one is taken, what lies behind it
refused by a message of its own, before any launch.  No GPU is needed, and no address given here is ever read."""
import ctypes

import pytest

from paper_2605_17879_amd.guard import F32, Detector
from test_matrix_refusals import AT, INVALID, OK, h, lib, mat, pk  # noqa: F401  (two of them fixtures)


@pytest.mark.parametrize("rows", [1, 3])
def test_powers_of_two_lie_at_most_2_24_apart(lib, h, rows):  # noqa: F811
    """Of one row too: its blocks' bytes are as far apart as any's."""
    far, next_ = pk(rows, 300, exp_stride=2 ** 24 + 4), pk(rows, 300, exp_stride=2 ** 24)
    for stride in (2 ** 24 + 4, 2 ** 32 + 4, 2 ** 40):
        assert lib.gd_pack(h, mat(rows, 300), 0, pk(rows, 300, exp_stride=stride), None, None) == INVALID
        assert lib.gd_last_error(h) == b"gd_pack: stride above 2^24 elements"
    out, work = mat(rows, rows), ctypes.c_size_t(1 << 40)
    for a, b in ((far, next_), (next_, far)):
        assert lib.gd_packed_product(h, a, b, out, 0, AT, work, None) == INVALID
        assert lib.gd_last_error(h) == b"gd_packed_product: stride above 2^24 elements"


def test_one_block_s_distance_to_the_next_says_nothing(lib, h):  # noqa: F811
    """(of a matrix without a row: nothing is launched)"""
    assert lib.gd_packed_product(h, pk(0, 100, at=None, exp_at=None), pk(1, 100, exp_stride=2 ** 32), mat(0, 1, F32, at=None), 0, None, 0, None) == OK


class Room:
    """What Detector.alloc_packed takes of a detector, on the CPU."""
    import torch as _torch

    @staticmethod
    def _bytes(n):
        return Room._torch.empty(n, dtype=Room._torch.uint8)


@pytest.mark.parametrize("cols", [2 ** 22, 2 ** 22 - 5, 2 ** 22 - 128, 2 ** 22 - 300, 256, 128, 1])
def test_rooms_keep_to_the_limits(lib, h, cols):  # noqa: F811
    """Up to the longest row there is: of a product of what alloc_packed lays out only the result's size is refused."""
    p = Detector.alloc_packed(Room, 2, cols)
    codes, exp = p["codes"], p["exp"]
    assert codes.shape == (2, cols) and codes.stride(0) % 16 == 0 and cols <= codes.stride(0) <= 2 ** 22
    assert (codes.stride(0) % 256 != 0) or cols > 2 ** 22 - 128
    a = pk(2, cols, stride=codes.stride(0), exp_stride=exp.stride(0))
    assert lib.gd_packed_product(h, a, a, mat(2, 3, F32), 0, AT, ctypes.c_size_t(1 << 40), None) == INVALID
    assert lib.gd_last_error(h) == b"gd_packed_product: sizes of the matrices do not fit each other"


def test_columns_of_a_result(lib, h):  # noqa: F811
    """2^22 of them, and 2^24 rows."""
    wide = 2 ** 22 + 1
    assert lib.gd_packed_product(h, pk(1, 64), pk(wide, 64), mat(1, wide), 0, AT, ctypes.c_size_t(1 << 40), None) == INVALID
    assert lib.gd_last_error(h) == b"gd_packed_product: more than 2^24 rows, 2^22 columns or 2^22 of k"
    assert lib.gd_packed_product_work_bytes(1, wide, 64) == 0
    for n, m in ((1, 2 ** 22), (2 ** 24, 8)):                  # (refused for the result's address alone)
        assert lib.gd_packed_product(h, pk(n, 64), pk(m, 64), mat(n, m, F32, at=AT + 1), 0, AT, ctypes.c_size_t(1 << 40), None) == INVALID
        assert lib.gd_last_error(h) == b"gd_packed_product: pointer of a matrix not aligned to its element"


def test_short_sums_refuse_what_products_do_and_results_of_fp32(lib, h):  # noqa: F811
    work = ctypes.c_size_t(1 << 40)
    for args, status in (((None, pk(20, 64), mat(10, 20), 0, AT, work), INVALID), ((pk(10, 64), pk(20, 65), mat(10, 20), 0, AT, work), INVALID),
                         ((pk(10, 64), pk(20, 64), mat(10, 20, F32), 0, AT, work), 4), ((pk(10, 64), pk(20, 64), mat(10, 21), 0, AT, work), INVALID),
                         ((pk(2, 20_000), pk(64, 20_000), mat(2, 64), 0, AT, ctypes.c_size_t(16)), 3)):
        assert lib.gd_packed_product_short(h, *args, None) == status
        assert lib.gd_last_error(h).startswith(b"gd_packed_product_short: ")
    assert lib.gd_packed_product_short(None, pk(10, 64), pk(20, 64), mat(10, 20), 0, AT, work, None) == INVALID
