"""An update of a matrix whose forms in the work area end more than 2^32 bytes behind their begin, wide and tall."""
import pytest
import torch

import matrix_refs as refs
from paper_2605_17879_amd import Config, Detector
from test_gpu_matrices import say

pytestmark = pytest.mark.gpu


def steps_of(s, products):
    """The steps for a diagonal X, whose products are of its numbers alone: exact, or with the roundings of the operands."""
    x = s.double()
    for a, b, c in [refs.USUAL] * 5:
        if products is None:
            x = a * x + (b * x * x + c * x ** 4) * x
            continue
        both, one = 2 if products == "f32" else 1, 2.0 ** 15
        x2, xs = refs._digits(x, 2, one), refs._digits(x, both, one)
        aa = refs._digits(xs * xs, both, one)
        x = a * x2 + refs._digits(b * aa + c * aa * aa, both, 2.0 ** 12) * xs
    return x


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("rows,cols", [(65_536, 16_500), (16_500, 65_536)])
def test_matrices_of_more_than_2_32_bytes(rows, cols, products):
    """One number in each row and column of the shorter side, at places from the first to the last: its singular values are the
    numbers' magnitudes over the norm, and every other element of X is 0."""
    a = min(rows, cols)
    assert 65_536 * (4 * 16_500) > 2 ** 32
    det = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    torch.cuda.empty_cache()
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    ends = torch.tensor([0, 65_535], device="cuda")
    long = torch.cat([ends, 1 + torch.randperm(65_534, device="cuda", generator=g)[:a - 2]])
    short = torch.randperm(a, device="cuda", generator=g)
    v = torch.randn(len(long), device="cuda", generator=g)
    i, j = (long, short) if rows > cols else (short, long)
    grad = torch.zeros((rows, cols), device="cuda")
    grad[i, j] = v
    p, m = torch.zeros_like(grad), torch.zeros_like(grad)
    table = det.muon_table([p], [grad], [m])
    work = det.alloc_muon_work(table, products).fill_(0xFF)
    say(f"muon {rows} x {cols} {products}, work {work.nbytes / 1e9:.0f} GB, {len(v)} numbers")
    det.muon(table, work, lr=1.0, momentum=0.0, nesterov=False, eps=0.0, products=products)
    del work
    assert torch.equal(m[i, j], v)
    s = v.double() / torch.linalg.vector_norm(v.double())
    exact, rounded = steps_of(s, None), steps_of(s, products)
    got = -p[i, j].double()
    # (as refs.orthogonal_bound: the operands' roundings four times over, and sums)
    off, may = torch.linalg.vector_norm(got - exact), 4 * torch.linalg.vector_norm(rounded - exact) + 2 ** -20 * torch.linalg.vector_norm(exact)
    say(f"  off {float(off / torch.linalg.vector_norm(exact)):.3g}, bound {float(may / torch.linalg.vector_norm(exact)):.3g}")
    assert float(off) <= float(may)
    p[i, j] = 0
    assert int(torch.count_nonzero(p)) == 0
    det.close()
    del p, m, grad, table
    torch.cuda.empty_cache()
