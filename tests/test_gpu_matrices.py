"""The operators of a training step's matrices (packing into 8-bit codes, products of packed matrices, updates by
orthogonalised momentum) against plain implementations in 64 bits, at the sizes, types and values where they can go
wrong; every bound is derived in matrix_refs.py from the roundings that the kernels make."""
import pytest
import torch

import matrix_refs as refs
from paper_2605_17879_amd import Config, Detector

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


def say(text):
    print(text, flush=True)


def randn(shape, seed, dtype=F32, scale=1.0, wide=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * scale
    if wide:
        x = x * torch.exp(wide * torch.randn(shape, generator=g))
    return x.to(dtype)


def spaced(t, gap, at=0):
    """t on the GPU with `gap` elements between the end of a row and the next, `at` elements into its storage."""
    n, d = t.shape
    store = torch.full((n * (d + gap) + at + 16,), float("nan"), dtype=t.dtype, device="cuda")
    view = store[at:at + n * (d + gap)].view(n, d + gap)[:, :d]
    view.copy_(t)
    return view


def room(rows, cols, codes="e4m3", gap=0):
    """A packed matrix in the middle of bytes of 0xA5, and all of its bytes."""
    wide = -(-max(cols, 1) // 16) * 16 + 16 * gap
    tall = -(-max(rows, 1) // 4) * 4 + 4 * gap
    blocks = -(-cols // 128)
    c = torch.full(((rows + 2) * wide,), 0xA5, dtype=torch.uint8, device="cuda")
    e = torch.full(((blocks + 2) * tall,), 0xA5, dtype=torch.uint8, device="cuda")
    return dict(codes=c.view(refs.CODES[codes]).view(rows + 2, wide)[1:rows + 1, :cols], exp=e.view(blocks + 2, tall)[1:blocks + 1, :rows],
                all=(c, e), shapes=((rows + 2, wide), (blocks + 2, tall)))


def untouched(p):
    """Whether the bytes around a packed matrix are as they were."""
    rows, cols = p["codes"].shape
    for t, shape, (r, c) in zip(p["all"], p["shapes"], ((rows, cols), tuple(p["exp"].shape))):
        b = t.view(shape).clone()
        b[1:r + 1, :c] = 0xA5
        if not bool((b == 0xA5).all()):
            return False
    return True


def same_packed(p, x, square, codes, what):
    want_codes, want_exp = refs.pack(x, square, codes)
    got_codes, got_exp = p["codes"].view(torch.uint8).cpu(), p["exp"].cpu()
    assert torch.equal(got_exp, want_exp), f"{what}: powers of two differ"
    assert torch.equal(got_codes, want_codes), f"{what}: codes differ"
    assert untouched(p), f"{what}: bytes outside were written"


# ---- packing -----------------------------------------------------------------------------------

@pytest.mark.parametrize("codes", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,k,gap,at", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 127, 5, 1), (128, 128, 0, 0), (129, 257, 3, 1), (7, 1000, 0, 0), (300, 72, 8, 8)])
def test_packing(det, n, k, gap, at, dtype, codes):
    say(f"pack {n} x {k} {dtype} {codes}")
    x = randn((n, k), n * 1000 + k, dtype, 3.0, wide=2.0 if dtype is not F16 else 0.5)
    xd = spaced(x, gap, at)
    for square in (False, True):
        along, across = room(n, k, codes, gap=1), room(k, n, codes)
        det.pack(xd, along, across, square=square)
        same_packed(along, x, square, codes, "along")
        same_packed(across, x.t().contiguous(), square, codes, "across")
        alone, turned = room(n, k, codes), room(k, n, codes, gap=2)
        det.pack(xd, along=alone, square=square)
        det.pack(xd, across=turned, square=square)
        assert torch.equal(alone["codes"].view(torch.uint8), along["codes"].view(torch.uint8)) and torch.equal(alone["exp"], along["exp"])
        assert torch.equal(turned["codes"].view(torch.uint8), across["codes"].view(torch.uint8)) and torch.equal(turned["exp"], across["exp"])
        assert untouched(alone) and untouched(turned)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_packing_of_rows_that_end_anywhere(det, dtype):
    """Every number of rest behind eights, along and across; what lies behind the rows' ends counts for nothing."""
    for k in (*range(1, 18), *range(127, 138)):
        n = 5 * k % 23 + 1
        x = randn((n, k), 77 + k, dtype, 3.0)
        xd = torch.full((n, k + 9), float("nan"), dtype=dtype, device="cuda")[:, :k]
        xd.copy_(x)
        along, across = room(n, k, "e4m3", gap=1), room(k, n, "e4m3", gap=1)
        det.pack(xd, along, across)
        same_packed(along, x, False, "e4m3", f"along {n} x {k}")
        same_packed(across, x.t().contiguous(), False, "e4m3", f"across {n} x {k}")


@pytest.mark.parametrize("codes", ["e4m3", "e5m2"])
@pytest.mark.parametrize("square", [False, True])
def test_packing_of_values_at_the_borders(det, codes, square):
    """Zeros of both signs, the largest and smallest numbers, powers of two and what lies beside them, blocks that hold an
    infinity or a NaN next to blocks that do not."""
    x = randn((260, 400), 5, F32, 1.0, wide=1.0)
    x[0] = 0.0
    x[1] = -0.0
    x[2, :128], x[2, 128:256] = torch.finfo(F32).max, 2.0 ** -149
    x[3, :128] = 2.0 ** -130
    x[3, 5] = 2.0 ** -126 * 448
    for i in range(20):
        x[4 + i, :128] = torch.linspace(0, 1, 128) * refs.MOST[codes] * 2.0 ** (i - 10)
        x[4 + i, 3] = refs.MOST[codes] * 2.0 ** (i - 10) * (1 + (i % 3 - 1) * 2.0 ** -23)
    x[140, 10], x[141, 200], x[142, 399], x[143, 20] = float("inf"), float("nan"), float("-inf"), -float("nan")
    along, across = room(260, 400, codes), room(400, 260, codes)
    det.pack(x.cuda(), along, across, square=square)
    same_packed(along, x, square, codes, "along")
    same_packed(across, x.t().contiguous(), square, codes, "across")


def test_packing_of_nothing(det):
    for n, k in ((0, 10), (10, 0), (0, 0)):
        along, across = room(n, k), room(k, n)
        det.pack(torch.empty((n, k), device="cuda"), along, across)
        assert untouched(along) and untouched(across)


# ---- products ------------------------------------------------------------------------------------

def packed(det, x, codes="e4m3", square=False, gap=0):
    p = room(*x.shape, codes, gap)
    det.pack(x.cuda(), p, square=square)
    return p


def check_product(det, n, m, k, dtype, ca="e4m3", cb="e4m3", add=False, gap=0, wide=1.0, seed=0):
    say(f"product {n} x {m} x {k} {dtype} {ca} {cb} add {add}")
    a = packed(det, randn((n, k), 3 * n + k + seed, F32, 2.0, wide), ca, gap=gap)
    b = packed(det, randn((m, k), 5 * m + k + seed, F32, 0.1), cb, square=True, gap=gap)
    old = randn((n, m), 7 * n + m, dtype)
    store = torch.full((n + 2, m + 3), 7.0, dtype=dtype, device="cuda")
    out = store[1:n + 1, 1:m + 1]
    out.copy_(old)
    work = det.alloc_packed_product_work(n, m, k).fill_(0xFF)
    det.packed_product(a, b, out, work, accumulate=add)
    ref, bound = refs.product(refs.values(a["codes"], a["exp"].cpu()), refs.values(b["codes"], b["exp"].cpu()), dtype, old if add else None)
    off = (out.double().cpu() - ref).abs()
    assert bool((off <= bound).all()), f"off by {float((off / bound).max()):.3g} of what may be"
    rest = store.clone()
    rest[1:n + 1, 1:m + 1] = 7.0
    assert bool((rest == 7.0).all()), "elements outside were written"
    again = old.cuda()
    det.packed_product(a, b, again, work, accumulate=add)
    assert torch.equal(again.view(torch.uint8), out.contiguous().view(torch.uint8)), "two passes differ"


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,m,k", [
    (1, 1, 1), (1, 64, 128), (1, 1000, 4096), (4, 130, 1000), (16, 65, 129), (17, 64, 260), (32, 200, 127), (33, 100, 2000), (64, 64, 16),
    (65, 63, 300), (100, 1000, 72), (2, 40, 20000),
])
def test_products_of_few_rows_or_tiles(det, n, m, k, dtype):
    check_product(det, n, m, k, dtype)
    check_product(det, n, m, k, dtype, add=True, gap=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m,k", [(2100, 2100, 136), (4000, 1200, 100), (2048, 2048, 257)])
def test_products_of_middling_tiles(det, n, m, k, dtype):
    check_product(det, n, m, k, dtype, add=dtype is BF16)


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("n,m,k", [(4097, 3500, 17), (3600, 3700, 128), (3650, 3850, 264), (3585, 3585, 400), (4300, 4250, 136)])
def test_products_of_large_tiles(det, n, m, k, dtype):
    check_product(det, n, m, k, dtype, gap=1)


@pytest.mark.parametrize("ca,cb", [("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("n,m,k", [(5, 70, 300), (70, 130, 300), (2100, 2050, 200), (3600, 3600, 150)])
def test_products_of_other_codes(det, n, m, k, ca, cb):
    for dtype in (F32, F16):
        check_product(det, n, m, k, dtype, ca, cb)


@pytest.mark.parametrize("n,m", [(3, 200), (200, 100), (2100, 2100), (3600, 3600), (4300, 4250)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_leave_out_what_is_not_theirs(det, n, m, dtype):
    """Bytes behind the rows' ends are codes of NaN, powers of two behind the rows are those of NaN; a NaN in a row stays in it."""
    k = 200
    a, b = packed(det, randn((n, k), 1), gap=1), packed(det, randn((m, k), 2), gap=1)
    for p, rows in ((a, n), (b, m)):
        (c, e), (sc, se) = p["all"], p["shapes"]
        keep_c, keep_e = p["codes"].view(torch.uint8).clone(), p["exp"].clone()
        c.fill_(0x7F)
        e.fill_(0xFF)
        p["codes"].view(torch.uint8).copy_(keep_c)
        p["exp"].copy_(keep_e)
    out = torch.empty((n, m), dtype=dtype, device="cuda")
    work = det.alloc_packed_product_work(n, m, k).fill_(0xFF)
    det.packed_product(a, b, out, work)
    ref, bound = refs.product(refs.values(a["codes"], a["exp"].cpu()), refs.values(b["codes"], b["exp"].cpu()), dtype)
    assert bool(((out.double().cpu() - ref).abs() <= bound).all())
    a["exp"][0, 1] = 255
    a["codes"].view(torch.uint8)[1, :128] = 0x7F
    b["codes"].view(torch.uint8)[m - 1, 130] = 0x7F
    det.packed_product(a, b, out, work)
    bad = torch.isnan(out).cpu()
    want = torch.zeros((n, m), dtype=torch.bool)
    want[1], want[:, m - 1] = True, True
    assert torch.equal(bad, want)


def test_products_of_nothing(det):
    out = torch.full((3, 4), 5.0, device="cuda")
    work = det.alloc_packed_product_work(3, 4, 0)
    none = room(3, 0), room(4, 0)
    det.packed_product(*none, out, work, accumulate=True)
    assert bool((out == 5.0).all())
    det.packed_product(*none, out, work)
    assert bool((out == 0.0).all())
    det.packed_product(room(0, 100), room(4, 100), torch.empty((0, 4), device="cuda"), det.alloc_packed_product_work(0, 4, 100))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_layer_s_gradients_are_those_of_its_packed_numbers(det, dtype):
    """y = x w^T, dx = dy w, dw = dy^T x against the same products of what was packed, and against differences of
    sum(dy * y): linear in x and w, so that a step of any length gives the gradient."""
    n, m, k = 150, 200, 136
    x, w, dy = randn((n, k), 1, dtype), randn((m, k), 2, dtype, 0.1), randn((n, m), 3, dtype, 1e-3, wide=1.0)
    p = {}
    for name, t, square in (("x", x, False), ("w", w, True), ("dy", dy, False)):
        p[name], p[name + "t"] = room(*t.shape), room(*t.t().shape)
        det.pack(t.cuda(), p[name], p[name + "t"], square=square)
    v = {name: refs.values(q["codes"], q["exp"].cpu()) for name, q in p.items()}
    assert torch.equal(v["w"], v["wt"].t())
    outs = {}
    for name, a, b, shape in (("y", "x", "w", (n, m)), ("dx", "dy", "wt", (n, k)), ("dw", "dyt", "xt", (m, k))):
        outs[name] = torch.empty(shape, device="cuda")
        det.packed_product(p[a], p[b], outs[name], det.alloc_packed_product_work(*shape, v[a].shape[1]))
        ref, bound = refs.product(v[a], v[b], F32)
        assert bool(((outs[name].double().cpu() - ref).abs() <= bound).all()), name
    # differences: f(x + s e) - f(x) = s dx[e] for f = sum(dy * (x w^T)), of the packed w and dy
    g = torch.Generator().manual_seed(9)
    f = lambda x_, w_: float((v["dy"] * (x_ @ w_.t().contiguous())).sum())          # noqa: E731
    for _ in range(5):
        i, j = int(torch.randint(n, (1,), generator=g)), int(torch.randint(k, (1,), generator=g))
        x1 = v["x"].clone()
        x1[i, j] += 0.5
        diff = (f(x1, v["w"]) - f(v["x"], v["w"])) / 0.5
        assert abs(diff - float(outs["dx"][i, j])) <= 1e-9 * f(v["x"].abs(), v["w"].abs()) + float(bound.max()) + 1e-6 * abs(diff)


# ---- updates of matrices ---------------------------------------------------------------------------

def low_rank(rows, cols, seed, noise=0.1):
    r = max(1, min(rows, cols) // 16)
    return randn((rows, r), seed) @ randn((r, cols), seed + 1) + noise * randn((rows, cols), seed + 2)


def run_muon(det, mats, products="f32", grad_type=F32, nesterov=True, momentum=0.95, param=None, copies=None, **kw):
    """Update of zeros with rate 1: W = -X.  Returns the parameters and momenta behind it."""
    params = [torch.zeros(g.shape, device="cuda") for g, _ in mats] if param is None else param
    grads, ms = [g.to(grad_type).cuda() for g, _ in mats], [m.cuda() for _, m in mats]
    table = det.muon_table(params, grads, ms, copies=copies, lr_scale=kw.pop("lr_scale", 1.0), weight_decay=kw.pop("weight_decay", 0.0))
    work = det.alloc_muon_work(table, products).fill_(0xFF)
    det.muon(table, work, lr=kw.pop("lr", 1.0), momentum=momentum, nesterov=nesterov, products=products, **kw)
    return params, ms, (table, work)


def update_of(g, m, momentum=0.95, nesterov=True, scale=None):
    """(new momentum, update) rounded as they are kept."""
    g = g.float() if scale is None else g.float() * scale
    mu = torch.tensor(momentum, dtype=torch.float32)
    m = m * mu + g
    return m, g + mu * m if nesterov else m


SIZES = [(1, 1), (1, 5), (7, 1), (16, 16), (33, 65), (64, 64), (65, 64), (100, 333), (333, 100), (128, 512), (200, 200)]


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("noise", [0.1, 10.0])
def test_updates_of_small_matrices_together(det, products, noise):
    mats = [(low_rank(r, c, 10 * i, noise) * 10.0 ** (i % 7 - 4), low_rank(r, c, 10 * i + 5, noise) * 10.0 ** (i % 7 - 4)) for i, (r, c) in enumerate(SIZES)]
    params, ms, _ = run_muon(det, mats, products)
    for (g, m), p, m1 in zip(mats, params, ms):
        say(f"muon {tuple(g.shape)} {products}")
        want_m, up = update_of(g, m)
        assert torch.equal(m1.cpu(), want_m)
        exact, bound = refs.orthogonal_bound(up, products)
        off = float(torch.linalg.matrix_norm(-p.double().cpu() - exact))
        assert off <= bound, (tuple(g.shape), off, bound)


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("rows,cols", [(512, 512), (515, 900), (1000, 600), (2048, 2048), (2050, 2200), (2300, 2060)])
def test_updates_of_larger_matrices(det, rows, cols, products):
    say(f"muon {rows} x {cols} {products}")
    g, m = low_rank(rows, cols, 1) * 1e-3, low_rank(rows, cols, 4) * 1e-2
    (p,), (m1,), _ = run_muon(det, [(g, m)], products)
    want_m, up = update_of(g, m)
    assert torch.equal(m1.cpu(), want_m)
    exact, bound = refs.orthogonal_bound(up.cuda(), products)
    off = float(torch.linalg.matrix_norm(-p.double() - exact))
    say(f"  off {off / float(torch.linalg.matrix_norm(exact)):.3g} of it, bound {bound / float(torch.linalg.matrix_norm(exact)):.3g}")
    assert off <= bound


@pytest.mark.parametrize("grad_type", [F32, BF16, F16])
@pytest.mark.parametrize("param_type,copy_type", [(F32, None), (F32, BF16), (F32, F16), (BF16, None), (F16, BF16)])
def test_types_and_what_an_update_writes(det, grad_type, param_type, copy_type):
    shapes = [(70, 130), (130, 70), (9, 40), (600, 530)]
    mats = [((low_rank(r, c, i) * 1e-2).to(grad_type), low_rank(r, c, i + 50) * 0.1) for i, (r, c) in enumerate(shapes)]
    start = [randn(s, i, param_type, 0.02) for i, s in enumerate(shapes)]
    copies = None if copy_type is None else [torch.full(s, 3.0, dtype=copy_type, device="cuda") for s in shapes]
    rates, decays = [1.0, 0.5, 2.0, 0.25], [0.0, 0.1, 0.2, 0.3]
    params, ms, _ = run_muon(det, mats, grad_type=grad_type, param=[s.cuda() for s in start], copies=copies, lr=0.1, lr_scale=rates, weight_decay=decays)
    for i, ((g, m), p0, p, m1) in enumerate(zip(mats, start, params, ms)):
        want_m, up = update_of(g, m)
        assert torch.equal(m1.cpu(), want_m)
        exact, bound = refs.orthogonal_bound(up, "f32")
        rate = 0.1 * rates[i]
        want = p0.double() * (1 - rate * decays[i]) - rate * exact
        # the factors, two products and a difference in fp32, then the type's rounding
        per = 4 * refs.U32 * (p0.double().abs() + rate * exact.abs()) + rate * bound
        for what, got in (("param", p),) if copies is None else (("param", p), ("copy", copies[i])):
            off = (got.double().cpu() - want).abs()
            may = per + refs.u(got.dtype) * (want.abs() + per) + torch.finfo(got.dtype).smallest_normal * refs.u(got.dtype)
            assert bool((off <= may).all()), (what, i, float((off / may).max()))


def test_variants_of_an_update(det):
    g, m = low_rank(90, 150, 1), low_rank(90, 150, 2)
    for kw, up in (({}, update_of(g, m)[1]), (dict(nesterov=False), update_of(g, m, nesterov=False)[1]), (dict(momentum=0.0), update_of(g, m, 0.0)[1]),
                   (dict(steps=0), update_of(g, m)[1]), (dict(steps=1), update_of(g, m)[1]), (dict(steps=8), update_of(g, m)[1]),
                   (dict(steps=3, coefficients=[(1.5, -0.5, 0.0)] * 3), update_of(g, m)[1]), (dict(steps=2, coefficients=(1.875, -1.25, 0.375)), update_of(g, m)[1])):
        (p,), _, _ = run_muon(det, [(g, m)], **kw)
        coefficients = kw.get("coefficients")
        if coefficients is not None and not isinstance(coefficients, list):
            coefficients = [coefficients] * kw["steps"]
        steps = kw.get("steps", 5)
        exact, bound = refs.orthogonal_bound(up, "f32", steps=steps, coefficients=coefficients if steps else [])
        if steps == 0:
            exact = up.double() / (float(torch.linalg.matrix_norm(up.double())) + 1e-7)
        assert float(torch.linalg.matrix_norm(-p.double().cpu() - exact)) <= bound + 2 ** -20, kw


def test_gradient_scales_and_skipped_updates(det):
    g, m = low_rank(80, 64, 1), low_rank(80, 64, 2)
    scale = torch.tensor([0.25], device="cuda")
    (p,), (m1,), (table, work) = run_muon(det, [(g, m)], grad_scale=scale)
    want_m, up = update_of(g, m, scale=0.25)
    assert torch.equal(m1.cpu(), want_m)
    exact, bound = refs.orthogonal_bound(up, "f32")
    assert float(torch.linalg.matrix_norm(-p.double().cpu() - exact)) <= bound
    before = p.clone(), m1.clone()
    for bad in (float("inf"), float("nan"), -float("inf")):
        scale.fill_(bad)
        det.muon(table, work, lr=1.0, grad_scale=scale)
        assert torch.equal(p, before[0]) and torch.equal(m1, before[1])


def test_zeros_tiny_huge_and_broken_gradients(det):
    """Next to each other in one table: none has a part in another's update."""
    shapes = [(70, 90)] * 6
    base = low_rank(70, 90, 1)
    gs = [torch.zeros(70, 90), base * 1e-30, base * 1e30, base.clone(), base, base * 1e-44]
    gs[3][5, 7] = float("inf")
    mats = [(g, torch.zeros(70, 90)) for g in gs]
    params, ms, _ = run_muon(det, mats, eps=0.0)
    assert bool((params[0] == 0).all()) and bool((ms[0] == 0).all())
    for i in (1, 2, 4):
        exact, bound = refs.orthogonal_bound(update_of(*mats[i])[1], "f32", eps=0.0)
        assert float(torch.linalg.matrix_norm(-params[i].double().cpu() - exact)) <= bound, i
    assert bool(torch.isnan(params[3]).any()) and bool(torch.isfinite(params[5]).all())
    params, _, _ = run_muon(det, mats[:1], eps=1e-7)
    assert bool((params[0] == 0).all())


def test_two_updates_give_the_same_bits_and_an_empty_table_nothing(det):
    mats = [(low_rank(r, c, i), low_rank(r, c, i + 9)) for i, (r, c) in enumerate([(300, 200), (64, 64), (700, 640), (0, 5), (2100, 2049)])]
    first, _, _ = run_muon(det, mats)
    second, _, _ = run_muon(det, mats)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    run_muon(det, [])
    run_muon(det, [(torch.zeros(0, 4), torch.zeros(0, 4))])
