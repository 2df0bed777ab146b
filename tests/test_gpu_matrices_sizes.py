"""Products of packed matrices at the largest sizes that a card holds, and where the operands' writing in 16 bits takes more than one
pass of the chip."""
import pytest
import torch

import matrix_refs as refs
from paper_2605_17879_amd import Config, Detector
from test_gpu_matrices import BF16, F32, check_product, randn, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


@pytest.mark.parametrize("n,m,k", [(4300, 4250, 1200), (3700, 9000, 700)])
def test_operands_of_more_than_one_pass(det, n, m, k):
    """More than 2^19 pieces of sixteen numbers, which that many lanes write."""
    assert (n + m) * (-(-k // 64) * 4) > 2 ** 19
    check_product(det, n, m, k, F32)


def test_2_36_numbers(det):
    """More pieces of sixteen numbers than a launch has threads: 64 GiB of codes, and twice that of numbers."""
    n, m, k = 2 ** 22, 256, 16400
    assert (n + m) * (-(-k // 64) * 4) >= 2 ** 32
    torch.cuda.empty_cache()
    need = n * k + det.packed_product_work_bytes(n, m, k) + n * m * 4 + 2 ** 32
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip(f"{need / 1e9:.0f} GB of device memory are not free")
    say(f"product {n} x {m} x {k}, {need / 1e9:.0f} GB")
    codes = torch.zeros((n, k), dtype=torch.uint8, device="cuda")
    a = dict(codes=codes.view(torch.float8_e4m3fn), exp=torch.full((-(-k // 128), n), 127, dtype=torch.uint8, device="cuda"))
    b = det.alloc_packed(m, k)
    det.pack(randn((m, k), 1).cuda(), b)
    rows = [0, 1, 255, n // 3, n // 2 + 77, n - 257, n - 2, n - 1]
    some = randn((len(rows), k), 2).to(torch.float8_e4m3fn)
    codes[rows] = some.view(torch.uint8).cuda()
    out = torch.empty((n, m), device="cuda")
    det.packed_product(a, b, out, det.alloc_packed_product_work(n, m, k))
    ref, bound = refs.product(some.float().double(), refs.values(b["codes"], b["exp"].cpu()), F32)
    assert bool(((out[rows].double().cpu() - ref).abs() <= bound).all())
    zero = (out == 0).all(1)
    assert int(zero.sum()) == n - len(rows) and not bool(zero[rows].any())
    del a, codes, out, zero
    torch.cuda.empty_cache()
