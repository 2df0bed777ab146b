"""Packed matrices that were not made by gd_pack: a power of two of byte 0 is 2^-127 whatever its codes are, one of 255 makes
NaN of codes that are none, and what lies beyond fp32 is infinite."""
import pytest
import torch

import matrix_refs as refs
from paper_2605_17879_amd import Config, Detector
from test_gpu_matrices import BF16, F16, F32, randn, room, say

pytestmark = pytest.mark.gpu

# (tiles of few rows, of 128 x 128 where the result has 16 bits, of 256 x 256)
SIZES = [(3, 70, 200), (70, 130, 300), (2100, 2100, 200), (3600, 3600, 200)]


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


def coded(x, codes, exp):
    """x as codes, with one power of two everywhere."""
    p = room(*x.shape, codes)
    p["codes"].view(torch.uint8).copy_(x.to(refs.CODES[codes]).view(torch.uint8))
    p["exp"].fill_(exp)
    return p


@pytest.mark.parametrize("codes", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,m,k", SIZES)
def test_the_smallest_power_of_two(det, n, m, k, dtype, codes):
    """Codes of magnitudes from 2 on, which times 2^-127 are normal numbers, and zeros; the other operand is large."""
    say(f"byte 0: {n} x {m} x {k} {dtype} {codes}")
    x = randn((n, k), n + k, F32, 40.0)
    a = coded(torch.where(x.abs() < 2, torch.zeros(()), x.clamp(-400, 400)), codes, 127 - 120)
    a["exp"][:, 1::2] = 0
    a["exp"][0, 2] = 0
    b = coded(randn((m, k), m + k), "e4m3", 127 + 120)
    va, vb = refs.values(a["codes"], a["exp"].cpu()), refs.values(b["codes"], b["exp"].cpu())
    assert 0 < float(va[1].abs().max()) < 2.0 ** -117
    ref, bound = refs.product(va, vb, dtype)
    for p, q, r, may in ((a, b, ref, bound), (b, a, ref.t(), bound.t())):
        out = torch.empty(r.shape, dtype=dtype, device="cuda")
        det.packed_product(p, q, out, det.alloc_packed_product_work(*r.shape, k))
        off = (out.double().cpu() - r).abs()
        assert bool((off <= may).all()), float((off / may).max())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,m,k", SIZES)
def test_a_power_of_two_that_is_none(det, n, m, k, dtype):
    say(f"byte 255: {n} x {m} x {k} {dtype}")
    x = randn((n, k), 1)
    x[1], x[2, 1:128] = 0, 0                                    # (rows of zeros, and of all but one)
    a, b = coded(x, "e4m3", 127), coded(randn((m, k), 2), "e5m2", 127)
    a["exp"][0, :3] = 255
    b["exp"][1, m - 1] = 255
    for p, q, shape in ((a, b, (n, m)), (b, a, (m, n))):
        out = torch.empty(shape, dtype=dtype, device="cuda")
        det.packed_product(p, q, out, det.alloc_packed_product_work(*shape, k))
        want = torch.zeros((n, m), dtype=torch.bool)
        want[:3], want[:, m - 1] = True, True
        assert torch.equal(torch.isnan(out).cpu(), want if p is a else want.t())


@pytest.mark.parametrize("n,m,k", SIZES)
def test_elements_beyond_fp32(det, n, m, k):
    """448 * 2^127 times 2^-20."""
    a, b = coded(torch.zeros(n, k), "e4m3", 254), coded(torch.zeros(m, k), "e4m3", 127 - 20)
    a["codes"].view(torch.uint8)[1, 5] = torch.tensor(448.0).to(refs.CODES["e4m3"]).view(torch.uint8)
    b["codes"].view(torch.uint8)[:, 5] = torch.tensor(1.0).to(refs.CODES["e4m3"]).view(torch.uint8)
    for dtype in (F32, BF16, F16):
        out = torch.empty((n, m), dtype=dtype, device="cuda")
        det.packed_product(a, b, out, det.alloc_packed_product_work(n, m, k))
        assert bool((out[1] == float("inf")).all()) and bool((out[0] == 0).all()), dtype
