"""What the operators of a sweep's training step refuse, by status code and before any launch: no GPU is
needed, and no address given here is ever read."""
import ctypes

import pytest

from paper_2605_17879_amd import guard
from paper_2605_17879_amd.guard import BF16, E4M3, F16, F32, I32, I64, _CAdamwConfig, _CAdamwTensor, _CMatrix

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


def toks(n=10, dtype=I64, **kw):
    return mat(n, 1, dtype, **kw)


def test_structs_have_the_header_s_sizes():
    assert ctypes.sizeof(_CMatrix) == 40 and ctypes.sizeof(_CAdamwTensor) == 104 and ctypes.sizeof(_CAdamwConfig) == 48


@pytest.mark.parametrize("w,t,o,status", [
    (None, toks(), mat(10, 64), INVALID), (mat(50, 64), None, mat(10, 64), INVALID), (mat(50, 64), toks(), None, INVALID),
    (mat(50, 64, I32), toks(), mat(10, 64, I32), UNSUPPORTED), (mat(50, 64, E4M3), toks(), mat(10, 64, E4M3), UNSUPPORTED),
    (mat(50, 64, 77), toks(), mat(10, 64, 77), UNSUPPORTED),
    (mat(50, 64), toks(dtype=F32), mat(10, 64), INVALID), (mat(50, 64), mat(10, 2, I64), mat(10, 64), INVALID),
    (mat(50, 64), toks(), mat(10, 64, F16), INVALID), (mat(50, 64), toks(), mat(11, 64), INVALID), (mat(50, 64), toks(), mat(10, 63), INVALID),
    (mat(50, 64, stride=63), toks(), mat(10, 64), INVALID), (mat(50, 64), toks(), mat(10, 64, stride=10), INVALID),
    (mat(50, 64, at=AT + 1), toks(), mat(10, 64), INVALID), (mat(50, 64), toks(at=AT + 4), mat(10, 64), INVALID),
    (mat(50, 64), toks(stride=0), mat(10, 64), INVALID), (mat(50, 64, at=None), toks(), mat(10, 64), INVALID),
    (mat(50, 64), toks(), mat(10, 64, at=None), INVALID), (mat(50, 64, reserved=1), toks(), mat(10, 64), INVALID),
    (mat(2 ** 24 + 1, 64), toks(), mat(10, 64), INVALID), (mat(50, 65537), toks(), mat(10, 65537), INVALID),
    (mat(50, 64), toks(2 ** 24 + 1), mat(2 ** 24 + 1, 64), INVALID), (mat(50, 64, stride=2 ** 22 + 1), toks(), mat(10, 64), INVALID),
])
def test_lookup(lib, h, w, t, o, status):
    assert lib.gd_embed(h, w, t, 1.0, o, None) == status
    assert lib.gd_last_error(h).startswith(b"gd_embed: ")


def test_lookup_of_nothing_is_a_no_op(lib, h):
    assert lib.gd_embed(h, mat(50, 64), toks(0, at=None), 1.0, mat(0, 64, at=None), None) == OK
    assert lib.gd_embed(None, mat(50, 64), toks(0), 1.0, mat(0, 64), None) == INVALID


def test_lookup_grad(lib, h):
    need = lib.gd_embed_grad_work_bytes(10, 50, 64)
    assert need > 0 and need % 256 == 0
    call = lambda g, t, w, work=AT, size=need: lib.gd_embed_grad(h, g, t, 1.0, 0, w, work, size, None)
    good = (mat(10, 64), toks(), mat(50, 64))
    assert call(*good, work=None) == INVALID and call(*good, work=AT + 8) == INVALID
    assert call(*good, size=need - 1) == TOO_SMALL
    assert call(None, toks(), mat(50, 64)) == INVALID and call(mat(10, 64), toks(), None) == INVALID
    assert call(mat(10, 64, F32), toks(), mat(50, 64)) == INVALID
    assert call(mat(10, 64, I64), toks(), mat(50, 64, I64)) == UNSUPPORTED
    assert call(mat(9, 64), toks(), mat(50, 64)) == INVALID and call(mat(10, 64), toks(), mat(50, 65)) == INVALID
    assert call(mat(10, 64), toks(), mat(2 ** 24 + 1, 64)) == INVALID
    assert lib.gd_embed_grad(None, *good[:2], 1.0, 0, good[2], AT, need, None) == INVALID
    assert call(mat(10, 64), toks(), mat(0, 64, at=None)) == OK                # no table: nothing to write
    assert lib.gd_embed_grad_work_bytes(2 ** 24 + 1, 50, 64) == 0


def loss(lib, h, hid, w, t, loss=AT, lse=AT, mean=AT, work=AT, size=None):
    if size is None:
        size = lib.gd_vocab_loss_work_bytes(10, 50, 64, 1)
    return lib.gd_vocab_loss(h, hid, w, t, 1.0, loss, lse, mean, work, size, None)


def test_loss(lib, h):
    need = lib.gd_vocab_loss_work_bytes(10, 50, 64, 0)
    assert 0 < need <= lib.gd_vocab_loss_work_bytes(10, 50, 64, 1)
    good = (mat(10, 64), mat(50, 64), toks())
    assert loss(lib, None, *good) == INVALID
    for kw in (dict(loss=None), dict(lse=None), dict(mean=None), dict(loss=AT + 2), dict(lse=AT + 1), dict(mean=AT + 3), dict(work=None),
               dict(work=AT + 128)):
        assert loss(lib, h, *good, **kw) == INVALID, kw
    assert loss(lib, h, *good, size=need - 1) == TOO_SMALL
    for bad, status in [((None, good[1], good[2]), INVALID), ((good[0], None, good[2]), INVALID), ((good[0], good[1], None), INVALID),
                        ((mat(10, 64, F32), mat(50, 64, F32), toks()), UNSUPPORTED), ((mat(10, 64, F16), mat(50, 64), toks()), INVALID),
                        ((mat(10, 64), mat(50, 72), toks()), INVALID), ((mat(9, 64), mat(50, 64), toks()), INVALID),
                        ((mat(10, 64), mat(0, 64), toks()), INVALID), ((mat(10, 0), mat(50, 0), toks()), INVALID),
                        ((mat(10, 64), mat(2 ** 24 + 1, 64), toks()), INVALID), ((mat(10, 65537), mat(50, 65537), toks()), INVALID),
                        ((mat(10, 64, stride=2 ** 22 + 1), mat(50, 64), toks()), INVALID),
                        ((mat(10, 64), mat(50, 64), toks(dtype=BF16)), INVALID)]:
        assert loss(lib, h, *bad) == status
        assert lib.gd_last_error(h).startswith(b"gd_vocab_loss: ")
    assert lib.gd_vocab_loss_work_bytes(10, 0, 64, 0) == 0 and lib.gd_vocab_loss_work_bytes(10, 50, 0, 1) == 0


def test_loss_grad(lib, h):
    need = lib.gd_vocab_loss_work_bytes(10, 50, 64, 1)
    hid, w, t = mat(10, 64), mat(50, 64), toks()

    def call(gh=mat(10, 64), gw=mat(50, 64), lse=AT, mean=AT, gm=AT, gr=None, work=AT, size=need, dtype=BF16):
        return lib.gd_vocab_loss_grad(h, mat(10, 64, dtype), mat(50, 64, dtype), t, 1.0, lse, mean, gm, gr, gh, gw, work, size, None)

    for kw in (dict(gm=None), dict(lse=None), dict(mean=None), dict(lse=AT + 2), dict(gm=AT + 2), dict(gr=AT + 1), dict(work=None),
               dict(work=AT + 64), dict(gh=mat(9, 64)), dict(gw=mat(50, 63)), dict(gh=mat(10, 64, F16)), dict(gw=mat(50, 64, F32)),
               dict(gh=mat(10, 64, at=None)), dict(gw=mat(50, 64, stride=60))):
        assert call(**kw) == INVALID, kw
        assert lib.gd_last_error(h).startswith(b"gd_vocab_loss_grad: ")
    assert call(size=need - 1) == TOO_SMALL
    assert call(gh=mat(10, 64, F32), gw=mat(50, 64, F32), dtype=F32) == UNSUPPORTED
    assert call(gh=None, gw=None) == OK                                        # nothing asked for
    assert lib.gd_vocab_loss_grad(None, hid, w, t, 1.0, AT, AT, AT, None, hid, w, AT, need, None) == INVALID


def tensor(**kw):
    d = dict(d_param=AT, d_grad=AT, d_m=AT, d_v=AT, d_m_exp=None, d_v_exp=None, d_copy=None, n=1000, first_index=0, lr_scale=1.0,
             weight_decay=0.0, param_type=F32, grad_type=BF16, copy_type=BF16, state_type=F32)
    d.update(kw)
    return _CAdamwTensor(*d.values())


def config(**kw):
    d = dict(struct_size=48, seed=0, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    d.update(kw)
    return _CAdamwConfig(*d.values())


def test_adamw_tables(lib, h):
    rows = (_CAdamwTensor * 2)(tensor(), tensor(n=0, d_param=None, d_grad=None, d_m=None, d_v=None))
    size = lib.gd_adamw_table_bytes(h, rows, 2)
    assert size > 0 and size % 256 == 0
    buf = (ctypes.c_uint64 * (size // 8 + 1))()
    at = ctypes.addressof(buf)
    assert lib.gd_adamw_fill_table(h, rows, 2, at, size) == OK
    assert lib.gd_adamw_fill_table(h, rows, 2, at, size - 256) == TOO_SMALL
    assert lib.gd_adamw_fill_table(h, rows, 2, None, size) == INVALID
    assert lib.gd_adamw_fill_table(h, rows, 2, at + 4, size) == INVALID
    assert lib.gd_adamw_fill_table(None, rows, 2, at, size) == INVALID
    assert lib.gd_adamw_table_bytes(h, None, 0) >= 256                          # an empty list is one
    assert lib.gd_adamw_table_bytes(h, None, 2) == 0
    for kw in (dict(param_type=I32), dict(grad_type=E4M3), dict(state_type=BF16), dict(d_copy=AT, copy_type=F32), dict(d_param=None),
               dict(d_grad=None), dict(d_m=None), dict(d_v=None), dict(state_type=E4M3), dict(state_type=E4M3, d_m_exp=AT),
               dict(lr_scale=float("nan")), dict(weight_decay=float("inf")), dict(d_param=AT + 2), dict(d_grad=AT + 1), dict(d_m=AT + 2),
               dict(d_v=AT + 1), dict(d_copy=AT + 1), dict(n=2 ** 42 + 1)):
        bad = (_CAdamwTensor * 2)(tensor(), tensor(**kw))
        assert lib.gd_adamw_table_bytes(h, bad, 2) == 0, kw
        assert lib.gd_adamw_fill_table(h, bad, 2, at, size) == INVALID, kw


def test_adamw(lib, h):
    call = lambda c, table=AT, size=512, gs=None, handle=h: lib.gd_adamw(handle, table, size, c, gs, None)
    assert call(config(), handle=None) == INVALID and call(None) == INVALID and call(config(), table=None) == INVALID
    assert call(config(), table=AT + 128) == INVALID and call(config(), gs=AT + 2) == INVALID
    assert call(config(), size=0) == INVALID and call(config(), size=300) == INVALID
    for kw in (dict(struct_size=40), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.5),
               dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("inf")), dict(step=0)):
        assert call(config(**kw)) == BAD_CONFIG, kw
