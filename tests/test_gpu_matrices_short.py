"""Products with the short sums of the 8-bit matrix cores, through what is asked of products at all: sizes of every kind of tiles, codes,
accumulation, what lies around, bytes of powers of two, captured and replayed."""
import pytest
import torch

import test_gpu_matrices as all_products
import test_gpu_matrices_bytes as all_bytes
import test_gpu_matrices_edges as edges
from paper_2605_17879_amd import Config, Detector
from paper_2605_17879_amd.guard import GuardError
from test_gpu_matrices import BF16, F16, F32, check_product, packed, randn

pytestmark = pytest.mark.gpu


class Short:
    """A detector whose products have short sums wherever there are such."""

    def __init__(self, det):
        self.det, self.calls = det, 0

    def __getattr__(self, name):
        return getattr(self.det, name)

    def packed_product(self, a, b, out, work, accumulate=False, stream=None):
        short = out.dtype is not F32
        self.calls += short
        self.det.packed_product(a, b, out, work, accumulate, stream=stream, sums="short" if short else "f32")


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


@pytest.fixture
def short(det):
    s = Short(det)
    yield s
    assert s.calls > 0


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,m,k", [(1, 1, 1), (4, 130, 1000), (17, 64, 260), (65, 63, 300), (100, 1000, 72), (2, 40, 20000), (2100, 2100, 136), (4000, 1200, 100),
                                   (2048, 2048, 257), (4097, 3500, 17), (3600, 3700, 128), (4300, 4250, 136)])
def test_products_of_all_tiles(short, n, m, k, dtype):
    check_product(short, n, m, k, dtype)
    check_product(short, n, m, k, dtype, add=True, gap=1)


@pytest.mark.parametrize("ca,cb", [("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("n,m,k", [(5, 70, 300), (70, 130, 300), (2100, 2050, 200), (3600, 3600, 150)])
def test_products_of_other_codes(short, n, m, k, ca, cb):
    check_product(short, n, m, k, F16, ca, cb)


@pytest.mark.parametrize("n,m", [(3, 200), (200, 100), (2100, 2100), (3600, 3600), (4300, 4250)])
def test_products_leave_out_what_is_not_theirs(short, n, m):
    all_products.test_products_leave_out_what_is_not_theirs(short, n, m, BF16)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,m,k", all_bytes.SIZES)
def test_bytes_of_powers_of_two(short, n, m, k, dtype):
    for codes in ("e4m3", "e5m2"):
        all_bytes.test_the_smallest_power_of_two(short, n, m, k, dtype, codes)
    all_bytes.test_a_power_of_two_that_is_none(short, n, m, k, dtype)


def test_elements_beyond_fp32_are_products_like_others(det):
    """448 * 2^127 times 2^-20: 448 * 2^107."""
    for n, m, k in all_bytes.SIZES:
        a, b = all_bytes.coded(torch.zeros(n, k), "e4m3", 254), all_bytes.coded(torch.zeros(m, k), "e4m3", 127 - 20)
        a["codes"].view(torch.uint8)[1, 5] = torch.tensor(448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        b["codes"].view(torch.uint8)[:, 5] = torch.tensor(1.0).to(torch.float8_e4m3fn).view(torch.uint8)
        out = torch.empty((n, m), dtype=BF16, device="cuda")
        det.packed_product(a, b, out, det.alloc_packed_product_work(n, m, k), sums="short")
        assert bool((out[1] == 448 * 2.0 ** 107).all()) and bool((out[0] == 0).all())


def test_captured_on_other_streams_and_of_one_row(short):
    edges.test_a_layer_s_step_captured_and_replayed(short, 300, 200, 136, "f32")
    edges.test_on_another_stream(short)
    edges.test_one_row_against_many(short, BF16)


def test_rows_far_apart(short):
    edges.test_rows_far_apart(short, BF16)


def test_nothing_and_results_of_fp32(det):
    out = torch.full((3, 4), 5.0, dtype=BF16, device="cuda")
    none = all_products.room(3, 0), all_products.room(4, 0)
    work = det.alloc_packed_product_work(3, 4, 0)
    det.packed_product(*none, out, work, accumulate=True, sums="short")
    assert bool((out == 5.0).all())
    det.packed_product(*none, out, work, sums="short")
    assert bool((out == 0.0).all())
    a, b = packed(det, randn((3, 64), 1)), packed(det, randn((4, 64), 2))
    wide = torch.full((3, 4), 5.0, device="cuda")
    with pytest.raises(GuardError, match="gd_packed_product_short: out must be bf16 or f16"):
        det.packed_product(a, b, wide, det.alloc_packed_product_work(3, 4, 64), sums="short")
    assert bool((wide == 5.0).all())
