"""What the sums of packed products keep: those of fp32, whatever the result is, and the short ones that a caller can ask for, of the
8-bit matrix cores, which cut products before they are added: by the rule of packed_sums.py, to the last digit, so that what is
documented of it holds."""
import pytest
import torch

import matrix_refs as refs
from packed_sums import sums
from paper_2605_17879_amd import Config, Detector
from test_gpu_matrices import BF16, F16, F32, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(shape, g):
    return torch.randn(shape, device="cuda", generator=g)


def hidden(shape, g):
    """A few columns twenty times as large as the others."""
    few = torch.rand((1, shape[1]), device="cuda", generator=g) < 0.002
    return normal(shape, g) * torch.exp(0.5 * normal((1, shape[1]), g) + 3.0 * few) * torch.exp(0.3 * normal((shape[0], 1), g))


def wide(shape, g):
    return normal(shape, g) * torch.exp(1.5 * normal(shape, g))


def any_codes(det, n, k, kind, g, small=0.5):
    """Codes of every exponent, half of them below 2^-6 or 2^-14 or zero, with powers of two of all kinds."""
    t = torch.randint(0, 256, (n, k), device="cuda", generator=g)
    few = torch.rand((n, k), device="cuda", generator=g) < small
    t = torch.where(few, t & (0x8F if kind == "e4m3" else 0x87), t)
    none = (t & 0x7F) == 0x7F if kind == "e4m3" else (t & 0x7F) >= 0x7C
    p = det.alloc_packed(n, k, kind)
    p["codes"].view(torch.uint8).copy_(torch.where(none, t & 0x80, t))
    p["exp"].copy_(torch.randint(124, 131, p["exp"].shape, device="cuda", generator=g))
    return p


def from_values(det, values, kind):
    p = det.alloc_packed(*values.shape, kind)
    p["codes"].view(torch.uint8).copy_(values.to(refs.CODES[kind]).view(torch.uint8))
    p["exp"].fill_(127)
    return p


def some_of(p, rows):
    return dict(codes=p["codes"].view(torch.uint8)[rows].contiguous().view(p["codes"].dtype), exp=p["exp"][:, rows])


def sums_of_the_kernel(det, a, b, n, m, k, dtype, rows, cols, exact, how):
    """The sums before they are rounded to `dtype`, as far as that shows them: to a result that is nearly the sum's negative they are
    added, and what is left is rounded by at most half a step of the difference."""
    out = torch.zeros((n, m), dtype=dtype, device="cuda")
    old = (-exact).to(dtype)
    r = torch.arange(n, device="cuda")[rows]
    c = torch.arange(m, device="cuda")[cols]
    out[r[:, None], c[None]] = old
    det.packed_product(a, b, out, det.alloc_packed_product_work(n, m, k), accumulate=True, sums=how)
    left = out[r[:, None], c[None]].double()
    return left - old.double(), refs.u(dtype) * left.abs() + torch.finfo(dtype).smallest_normal * refs.u(dtype)


# (tiles of few rows, of 64 x 64, of 128 x 128, of 256 x 256)
SIZES = [(7, 200), (70, 130), (2100, 2100), (3600, 3700)]


def operands(det, n, m, k, a_kind, b_kind):
    """Of codes of every kind.  (Sums of e5m2 by e5m2 reach 2^30, of which f16 holds nothing: powers of two bring them down.)"""
    g = gen(n + m)
    a, b = any_codes(det, n, k, a_kind, g), any_codes(det, m, k, b_kind, g)
    for p, kind in ((a, a_kind), (b, b_kind)):
        p["exp"] -= {"e4m3": 8, "e5m2": 15}[kind]
    rows, cols = slice(max(0, n - 96), n), slice(0, min(m, 96))
    return a, b, rows, cols, sums(some_of(a, rows), some_of(b, cols), a_kind, b_kind)


KINDS = pytest.mark.parametrize("a_kind,b_kind", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])


@KINDS
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,m", SIZES)
def test_sums_are_those_of_fp32(det, n, m, dtype, a_kind, b_kind):
    """Whatever type the result has: off by what fp32 leaves of (k + 16) additions."""
    k = 300
    a, b, rows, cols, (_, exact, _, mag) = operands(det, n, m, k, a_kind, b_kind)
    got, rounded = sums_of_the_kernel(det, a, b, n, m, k, dtype, rows, cols, exact, "f32")
    off, may = (got - exact).abs(), (k + 16) * refs.U32 * mag + rounded
    assert bool((off <= may).all()), f"off by {float((off / may).max()):.3g} of what may be"


@KINDS
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n,m", SIZES)
def test_short_sums_are_those_of_the_rule(det, n, m, dtype, a_kind, b_kind):
    """The rule's sum is off by what fp32 leaves of (k + 16) additions, and the exact one by the cut besides, at most 7 * 2^-13 of each
    eight's 2^E."""
    k = 300
    a, b, rows, cols, (cut, exact, units, mag) = operands(det, n, m, k, a_kind, b_kind)
    got, rounded = sums_of_the_kernel(det, a, b, n, m, k, dtype, rows, cols, exact, "short")
    may = (k + 16) * refs.U32 * mag + rounded
    off = (got - cut).abs()
    assert bool((off <= may).all()), f"off by {float((off / may).max()):.3g} of what may be"
    assert bool(((got - exact).abs() <= may + 7 * 2.0 ** -13 * units).all())


@pytest.mark.parametrize("n,m", SIZES)
@pytest.mark.parametrize("a_of,b_of,most", [(normal, normal, 2.5e-5), (hidden, normal, 7e-5), (wide, wide, 1.3e-4)])
def test_what_the_cut_costs_in_the_norm(det, n, m, a_of, b_of, most):
    """On packed data, by the rule and by the kernel: the figures of the header, and 1.4 times as much for another draw (of columns or of
    numbers, of which a few are large).  Sums of fp32 have none of it."""
    k = 1024
    g = gen(3 * n + m)
    a, b = det.alloc_packed(n, k), det.alloc_packed(m, k)
    det.pack(a_of((n, k), g), a)
    det.pack(b_of((m, k), g) * 0.1, b)
    rows, cols = slice(0, min(n, 96)), slice(max(0, m - 96), m)
    cut, exact, units, mag = sums(some_of(a, rows), some_of(b, cols), "e4m3", "e4m3")
    size = torch.linalg.matrix_norm(exact)
    by_rule = float(torch.linalg.matrix_norm(cut - exact) / size)
    short, _ = sums_of_the_kernel(det, a, b, n, m, k, F16, rows, cols, exact, "short")
    of_kernel = float(torch.linalg.matrix_norm(short - exact) / size)
    say(f"{n} x {m} {a_of.__name__}: {by_rule:.3g} by the rule, {of_kernel:.3g}")
    assert by_rule <= most and of_kernel <= most
    for dtype in (F32, F16, BF16):
        got, rounded = sums_of_the_kernel(det, a, b, n, m, k, dtype, rows, cols, exact, "f32")
        assert bool(((got - exact).abs() <= (k + 16) * refs.U32 * mag + rounded).all()), dtype


@pytest.mark.parametrize("n,m", SIZES)
def test_one_large_product_among_eight(det, n, m):
    """What the cut does at its worst, in all rows and columns alike: small products beside a large one are lost, what is left of large ones
    that cancel too.  Sums of fp32 have them."""
    one, other, lost = [], [], []
    for a8, b8, kept in (([16.0] + [2.0 ** -6 * 1.875] * 7, [16.0] + [2.0 ** -6] * 7, 256.0),       # seven of 1.875 * 2^-12 beside 2^8
                         ([16.0] + [2.0 ** -3 * 1.875] * 7, [16.0] + [2.0 ** -3] * 7, 256.0),     # of 1.875 * 2^-6: E = 4 + 4, cut at 2^-5; 8.0e-4 of the result
                         ([1.0, -1.0, 2.0 ** -7, 0, 0, 0, 0, 0], [1.0, 1.0, 2.0 ** -7, 0, 0, 0, 0, 0], 0.0),     # 1 - 1 + 2^-14
                         ([1.0, -1.0, 2.0 ** -7, 0, 0, 0, 0, 0], [1.0, 1.0, 2.0 ** -6, 0, 0, 0, 0, 0], 2.0 ** -13),
                         # a subnormal code counts as one of 2^-6: 2^-9 * 2^8 cuts at 2^(2 - 13)
                         ([2.0 ** -9, -2.0 ** -9, 2.0 ** -6, 0, 0, 0, 0, 0], [256.0, 256.0, 2.0 ** -6, 0, 0, 0, 0, 0], 0.0)):
        one.append(a8), other.append(b8), lost.append(kept)
    for a8, b8, kept in zip(one, other, lost):
        va, vb = torch.tensor([a8], dtype=torch.float64).expand(n, 8), torch.tensor([b8], dtype=torch.float64).expand(m, 8)
        a, b = from_values(det, va.cuda().float(), "e4m3"), from_values(det, vb.cuda().float(), "e4m3")
        cut, exact, units, _ = sums(some_of(a, slice(0, 1)), some_of(b, slice(0, 1)), "e4m3", "e4m3")
        assert float(cut) == kept and abs(float(exact) - kept) <= 7 * 2.0 ** -13 * float(units)
        for dtype, how in ((F16, "f32"), (BF16, "f32"), (F32, "f32"), (F16, "short"), (BF16, "short")):
            out = torch.empty((n, m), dtype=dtype, device="cuda")
            det.packed_product(a, b, out, det.alloc_packed_product_work(n, m, 8), sums=how)
            want = (cut if how == "short" else exact).to(dtype)
            assert bool((out == want).all()), (dtype, how, kept, float(out[0, 0]))
