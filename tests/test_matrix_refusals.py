"""What the operators of a training step's matrices refuse, by status code and before any launch: no GPU is needed, and no
address given here is ever read."""
import ctypes

import pytest

from paper_2605_17879_amd import guard
from paper_2605_17879_amd.guard import (BF16, E4M3, E5M2, F16, F32, I32, U8, _CMatrix, _CMuonConfig, _CMuonTensor, _CPacked)

OK, INVALID, BAD_CONFIG, TOO_SMALL, UNSUPPORTED = 0, 1, 2, 3, 4
AT = 1 << 20                      # an address that is aligned and never touched


@pytest.fixture(scope="module")
def lib():
    return guard.load_library()


@pytest.fixture(scope="module")
def h(lib):
    c = guard.Config(8, 1, 1, 1).to_c()
    out = ctypes.c_void_p()
    assert lib.gd_create(ctypes.byref(c), ctypes.byref(out)) == OK
    yield out
    lib.gd_destroy(out)


def mat(rows, cols, dtype=BF16, stride=None, at=AT, reserved=0):
    return _CMatrix(at, rows, cols, cols if stride is None else stride, dtype, reserved)


def pk(rows, cols, codes=E4M3, stride=None, at=AT, exp_rows=None, exp_cols=None, exp_stride=None, exp_at=AT, exp_type=U8, reserved=0):
    wide = -(-cols // 16) * 16 if stride is None else stride
    blocks = -(-cols // 128) if exp_rows is None else exp_rows
    n = rows if exp_cols is None else exp_cols
    return _CPacked(_CMatrix(at, rows, cols, wide, codes, reserved), _CMatrix(exp_at, blocks, n, -(-n // 4) * 4 if exp_stride is None else exp_stride, exp_type, 0))


def test_structs_have_the_header_s_sizes():
    assert ctypes.sizeof(_CPacked) == 80 and ctypes.sizeof(_CMuonTensor) == 80 and ctypes.sizeof(_CMuonConfig) == 48


@pytest.mark.parametrize("x,along,across,status", [
    (None, pk(10, 64), None, INVALID), (mat(10, 64), None, None, INVALID),
    (mat(10, 64, I32), pk(10, 64), None, UNSUPPORTED), (mat(10, 64, E4M3), pk(10, 64), None, UNSUPPORTED),
    (mat(10, 64), pk(10, 64, codes=U8), None, INVALID), (mat(10, 64), pk(10, 64, codes=BF16), None, INVALID),
    (mat(10, 64), pk(10, 64, exp_type=E4M3), None, INVALID), (mat(10, 64), pk(11, 64), None, INVALID), (mat(10, 64), pk(10, 65), None, INVALID),
    (mat(10, 64), None, pk(10, 64), INVALID), (mat(10, 200), pk(10, 200, exp_rows=1), None, INVALID), (mat(10, 64), pk(10, 64, exp_cols=9), None, INVALID),
    (mat(10, 64), pk(10, 64, at=AT + 8), None, INVALID), (mat(10, 60), pk(10, 60, stride=72), None, INVALID), (mat(10, 64), pk(10, 64, at=None), None, INVALID),
    (mat(10, 64), pk(10, 64, exp_at=AT + 2), None, INVALID), (mat(10, 200), pk(10, 200, exp_stride=10), None, INVALID),
    (mat(10, 64), pk(10, 64, exp_at=None), None, INVALID), (mat(10, 64), pk(10, 64, stride=48), None, INVALID),
    (mat(10, 64), pk(10, 64, reserved=3), None, INVALID), (mat(10, 64), pk(10, 64), pk(64, 10, codes=E5M2), INVALID),
    (mat(10, 64, stride=63), pk(10, 64), None, INVALID), (mat(10, 64, at=AT + 1), pk(10, 64), None, INVALID),
    (mat(2 ** 24 + 1, 64), pk(2 ** 24 + 1, 64), None, INVALID), (mat(10, 2 ** 22 + 1), pk(10, 2 ** 22 + 1), None, INVALID),
    (mat(10, 64), pk(10, 64, stride=2 ** 22 + 16), None, INVALID),
    (mat(2 ** 23, 65_536), pk(2 ** 23, 65_536), None, UNSUPPORTED), (mat(2 ** 24, 8192), pk(2 ** 24, 8192), None, UNSUPPORTED),
])
def test_packing(lib, h, x, along, across, status):
    assert lib.gd_pack(h, x, 0, along, across, None) == status
    assert lib.gd_last_error(h).startswith(b"gd_pack: ")


def test_packing_of_nothing_is_a_no_op(lib, h):
    assert lib.gd_pack(h, mat(0, 64, at=None), 0, pk(0, 64, at=None, exp_at=None), None, None) == OK
    assert lib.gd_pack(None, mat(10, 64), 0, pk(10, 64), None, None) == INVALID


@pytest.mark.parametrize("a,b,out,work,size,status", [
    (None, pk(20, 64), mat(10, 20), AT, 1 << 30, INVALID), (pk(10, 64), None, mat(10, 20), AT, 1 << 30, INVALID),
    (pk(10, 64), pk(20, 64), None, AT, 1 << 30, INVALID), (pk(10, 64), pk(20, 65), mat(10, 20), AT, 1 << 30, INVALID),
    (pk(10, 64), pk(20, 64), mat(10, 21), AT, 1 << 30, INVALID), (pk(10, 64), pk(20, 64), mat(20, 10), AT, 1 << 30, INVALID),
    (pk(10, 64), pk(20, 64), mat(10, 20, I32), AT, 1 << 30, UNSUPPORTED), (pk(10, 64), pk(20, 64), mat(10, 20, E4M3), AT, 1 << 30, UNSUPPORTED),
    (pk(10, 64, codes=F16), pk(20, 64), mat(10, 20), AT, 1 << 30, INVALID), (pk(10, 64), pk(20, 64, at=AT + 4), mat(10, 20), AT, 1 << 30, INVALID),
    (pk(10, 64), pk(20, 64), mat(10, 20, stride=19), AT, 1 << 30, INVALID), (pk(10, 64), pk(20, 64), mat(10, 20, at=AT + 1), AT, 1 << 30, INVALID),
    (pk(10, 64), pk(20, 64), mat(10, 20, at=None), AT, 1 << 30, INVALID),
    (pk(2, 20_000), pk(64, 20_000), mat(2, 64), AT, 16, TOO_SMALL), (pk(2, 20_000), pk(64, 20_000), mat(2, 64), None, 1 << 30, INVALID),
    (pk(2, 20_000), pk(64, 20_000), mat(2, 64), AT + 16, 1 << 30, INVALID),
    (pk(2 ** 24 + 1, 64), pk(20, 64), mat(2 ** 24 + 1, 20), AT, 1 << 40, INVALID),
    (pk(2 ** 21, 64), pk(2 ** 21, 64), mat(2 ** 21, 2 ** 21), AT, 1 << 60, UNSUPPORTED),
])
def test_products(lib, h, a, b, out, work, size, status):
    assert lib.gd_packed_product(h, a, b, out, 0, work, size, None) == status
    assert lib.gd_last_error(h).startswith(b"gd_packed_product: ")


def test_products_of_nothing_and_work_areas(lib, h):
    assert lib.gd_packed_product(h, pk(0, 64, at=None, exp_at=None), pk(20, 64), mat(0, 20, at=None), 0, None, 0, None) == OK
    assert lib.gd_packed_product_work_bytes(0, 20, 64) == 0 and lib.gd_packed_product_work_bytes(2 ** 24 + 1, 1, 1) == 0
    assert lib.gd_packed_product_work_bytes(4, 64, 65_536) > 0                  # (splits of a long sum)
    assert lib.gd_packed_product_work_bytes(8192, 8192, 1000) >= 2 * 8192 * 1024 * 2   # (operands in bf16)


def tensor(rows=10, cols=20, param=AT, grad=2 * AT, m=3 * AT, copy=None, rate=1.0, decay=0.0, types=(F32, F32, BF16), reserved=0):
    return _CMuonTensor(param, grad, m, copy, rows, cols, rate, decay, *types, reserved)


@pytest.mark.parametrize("t", [
    tensor(param=None), tensor(grad=None), tensor(m=None), tensor(param=AT + 2), tensor(grad=2 * AT + 1), tensor(m=3 * AT + 2), tensor(copy=4 * AT + 1),
    tensor(types=(I32, F32, BF16)), tensor(types=(F32, E4M3, BF16)), tensor(copy=4 * AT, types=(F32, F32, F32)), tensor(rows=65_537),
    tensor(cols=65_537), tensor(rate=float("nan")), tensor(decay=float("inf")), tensor(reserved=1),
    tensor(m=AT), tensor(m=AT + 4 * 199), tensor(copy=3 * AT + 8),                # (what is written overlaps)
    tensor(grad=AT), tensor(grad=3 * AT), tensor(grad=3 * AT + 4 * 199), tensor(grad=3 * AT - 4 * 199), tensor(grad=7 * AT),   # (... a gradient)
    tensor(copy=2 * AT + 16), tensor(copy=8 * AT),
])
def test_matrices(lib, h, t):
    lst = (_CMuonTensor * 2)(tensor(param=7 * AT, grad=8 * AT, m=9 * AT), t)
    assert lib.gd_muon_table_bytes(h, lst, 2) == 0
    assert lib.gd_last_error(h).startswith(b"gd_muon_table_bytes: ")
    host = ctypes.create_string_buffer(4096)
    assert lib.gd_muon_fill_table(h, lst, 2, host, 4096) == INVALID


def test_matrices_that_stand_twice(lib, h):
    assert lib.gd_muon_table_bytes(h, (_CMuonTensor * 2)(tensor(), tensor()), 2) == 0
    assert lib.gd_muon_table_bytes(h, (_CMuonTensor * 2)(tensor(), tensor(param=5 * AT, m=6 * AT)), 2) > 0      # (a shared gradient is read twice)
    assert lib.gd_muon_table_bytes(h, None, 2) == 0 and lib.gd_muon_table_bytes(None, (_CMuonTensor * 1)(tensor()), 1) == 0


def table(lib, h, *tensors):
    lst = (_CMuonTensor * max(1, len(tensors)))(*tensors)
    n = lib.gd_muon_table_bytes(h, lst, len(tensors))
    assert n and n % 256 == 0
    host = ctypes.create_string_buffer(n)
    assert lib.gd_muon_fill_table(h, lst, len(tensors), host, n - 1) == TOO_SMALL
    assert lib.gd_muon_fill_table(h, lst, len(tensors), host, n) == OK
    return host, n


def config(products=F32, steps=5, lr=0.02, momentum=0.95, eps=1e-7, size=48, coefficients=None):
    c = _CMuonConfig(size, 1, products, steps, lr, momentum, eps, None)
    if coefficients is not None:
        c.keep = (ctypes.c_double * len(coefficients))(*coefficients)
        c.coefficients = ctypes.addressof(c.keep)
    return c


@pytest.mark.parametrize("kw,status", [
    (dict(products=BF16), BAD_CONFIG), (dict(steps=17), BAD_CONFIG), (dict(lr=float("nan")), BAD_CONFIG), (dict(momentum=1.0), BAD_CONFIG),
    (dict(momentum=-0.1), BAD_CONFIG), (dict(eps=-1.0), BAD_CONFIG), (dict(eps=float("inf")), BAD_CONFIG), (dict(size=40), BAD_CONFIG),
    (dict(steps=1, coefficients=[10.0, 0.0, 0.0]), BAD_CONFIG),                  # (singular values of 10)
    (dict(steps=1, coefficients=[1.0, float("nan"), 0.0]), BAD_CONFIG),
    (dict(steps=2, coefficients=[1.3, 0.0, 0.0, 1.3, 0.0, 0.0]), BAD_CONFIG),    # (1.3, then 1.69)
    (dict(steps=1, coefficients=[3.0, 1.0, -2.9]), BAD_CONFIG),                  # (1.1 at the end, more before it)
])
def test_configurations_of_an_update(lib, h, kw, status):
    host, n = table(lib, h, tensor(300, 300))
    assert lib.gd_muon(h, host, AT, n, config(**kw), None, AT, 1 << 40, None) == status
    assert lib.gd_last_error(h).startswith(b"gd_muon: ")


def test_arguments_of_an_update(lib, h):
    host, n = table(lib, h, tensor(300, 300))
    need = lib.gd_muon_work_bytes(h, host, n, F32)
    assert need > lib.gd_muon_work_bytes(h, host, n, F16) > 0 and lib.gd_muon_work_bytes(h, host, n, BF16) == 0
    assert lib.gd_muon_work_bytes(h, host, n - 256, F32) == 0 and lib.gd_muon_work_bytes(h, None, n, F32) == 0
    c = config()
    for args, status in (((None, AT, n, c, None, AT, need), INVALID), ((host, None, n, c, None, AT, need), INVALID), ((host, AT, n, None, None, AT, need), INVALID),
                         ((host, AT + 128, n, c, None, AT, need), INVALID), ((host, AT, n, c, AT + 2, AT, need), INVALID), ((host, AT, n - 256, c, None, AT, need), INVALID),
                         ((ctypes.create_string_buffer(n), AT, n, c, None, AT, need), INVALID), ((host, AT, n, c, None, None, need), INVALID),
                         ((host, AT, n, c, None, AT + 64, need), INVALID), ((host, AT, n, c, None, AT, need - 1), TOO_SMALL)):
        assert lib.gd_muon(h, *args, None) == status, args
    assert lib.gd_muon(None, host, AT, n, c, None, AT, need, None) == INVALID


def test_a_table_of_nothing(lib, h):
    host, n = table(lib, h)
    assert lib.gd_muon(h, host, AT, n, config(), None, None, 0, None) == OK
    host, n = table(lib, h, tensor(0, 20, None, None, None), tensor(20, 0, None, None, None))
    assert lib.gd_muon(h, host, AT, n, config(), None, None, 0, None) == OK


def test_tiny_matrices_alone_need_no_work_area_beyond_sums(lib, h):
    host, n = table(lib, h, tensor(64, 192), tensor(192, 64, 5 * AT, 6 * AT, 7 * AT))
    assert lib.gd_muon_work_bytes(h, host, n, F32) <= 256
