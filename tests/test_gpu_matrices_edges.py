"""The operators of a training step's matrices where calls meet: captured and replayed, on other streams, one behind the
other as a layer's step with its update, with rows far apart, long lists, and tiles that are left over."""
import pytest
import torch

import matrix_refs as refs
from paper_2605_17879_amd import Config, Detector
from test_gpu_matrices import F32, BF16, F16, low_rank, packed, randn, room, run_muon, say, update_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


class Layer:
    """y = x w^T in packed numbers, its gradients, and the update of w."""

    def __init__(self, det, n=300, m=200, k=136, products="f32", dtype=BF16):
        self.det, self.products = det, products
        self.master = randn((m, k), 1, F32, 0.1).cuda()
        self.w = self.master.to(dtype)
        self.x, self.dy = randn((n, k), 2, dtype).cuda(), randn((n, m), 3, dtype, 1e-3).cuda()
        self.y, self.dx = torch.empty((n, m), dtype=dtype, device="cuda"), torch.empty((n, k), dtype=dtype, device="cuda")
        self.dw = torch.empty((m, k), device="cuda")
        self.m = torch.zeros((m, k), device="cuda")
        self.p = {}
        for name, t in (("x", self.x), ("w", self.w), ("dy", self.dy)):
            self.p[name], self.p[name + "t"] = det.alloc_packed(*t.shape), det.alloc_packed(*t.t().shape)
        self.work = [det.alloc_packed_product_work(*s) for s in ((n, m, k), (n, k, m), (m, k, n))]
        self.table = det.muon_table([self.master], [self.dw], [self.m], copies=[self.w], weight_decay=0.1)
        self.muon_work = det.alloc_muon_work(self.table, products)

    def step(self, stream=None):
        d, p = self.det, self.p
        d.pack(self.x, p["x"], p["xt"], stream=stream)
        d.pack(self.w, p["w"], p["wt"], square=True, stream=stream)
        d.packed_product(p["x"], p["w"], self.y, self.work[0], stream=stream)
        d.pack(self.dy, p["dy"], p["dyt"], stream=stream)
        d.packed_product(p["dy"], p["wt"], self.dx, self.work[1], stream=stream)
        d.packed_product(p["dyt"], p["xt"], self.dw, self.work[2], stream=stream)
        d.muon(self.table, self.muon_work, lr=0.02, products=self.products, stream=stream)

    def state(self):
        return [t.clone() for t in (self.y, self.dx, self.dw, self.m, self.master, self.w)]

    def restart(self):
        self.m.zero_()
        self.master.copy_(randn(self.master.shape, 1, F32, 0.1))
        self.w.copy_(self.master)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("n,m,k", [(300, 200, 136), (40, 96, 64), (1000, 700, 600)])
@pytest.mark.parametrize("products", ["f32", "f16"])
def test_a_layer_s_step_captured_and_replayed(det, n, m, k, products):
    say(f"layer {n} x {m} x {k} {products}")
    layer = Layer(det, n, m, k, products)
    eager = []
    for _ in range(4):
        layer.step()
        eager.append(layer.state())
    layer.restart()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step()
    layer.restart()
    other = Layer(det, n + 3, m + 1, k + 5, products)
    for i in range(4):
        graph.replay()
        other.step()                                     # (eager work of its own between the replays)
        torch.cuda.synchronize()
        assert same(layer.state(), eager[i]), f"replay {i}"


def test_two_graphs_one_behind_the_other_share_a_work_area(det):
    a, b = Layer(det, 300, 200, 136), Layer(det, 300, 200, 136)
    b.work, b.muon_work = a.work, a.muon_work
    a.step()
    want = a.state()
    graphs = []
    for layer in (a, b):
        layer.restart()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            layer.step()
        graphs.append(g)
        layer.restart()
    for _ in range(3):
        a.restart()
        b.restart()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert same(a.state(), want) and same(b.state(), want)


def test_on_another_stream(det):
    layer = Layer(det)
    layer.step()
    want = layer.state()
    side = torch.cuda.Stream()
    for how in ("given", "current"):
        layer.restart()
        x = layer.x.clone()
        layer.x.fill_(float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
            layer.x.copy_(x)                             # (late: a call on the wrong stream reads NaN)
            if how == "current":
                layer.step()
        if how == "given":
            layer.step(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert same(layer.state(), want), how


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_far_apart(det, dtype):
    """Codes, powers of two and results that end more than 2^32 bytes behind their begin."""
    n, m, k, apart = 70_000, 70, 150, 65_664
    say(f"{n} rows {apart} bytes apart, {dtype}")
    x = randn((1000, k), 1).repeat(70, 1)
    a = dict(codes=torch.full((n, apart), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :k],
             exp=torch.full((2, 70_016), 0xFF, dtype=torch.uint8, device="cuda")[:, :n])
    det.pack(x.cuda(), a)
    b = packed(det, randn((m, k), 2))
    out = torch.full((n, 40_000), 7.0, dtype=dtype, device="cuda")[:, 5:5 + m]
    det.packed_product(a, b, out, det.alloc_packed_product_work(n, m, k))
    few = packed(det, x[:1000])
    ref, bound = refs.product(refs.values(few["codes"], few["exp"].cpu()), refs.values(b["codes"], b["exp"].cpu()), dtype)
    for i in range(0, n, 1000):
        assert bool(((out[i:i + 1000].double().cpu() - ref).abs() <= bound).all()), i
    back = torch.full((1, 1), 0.0, device="cuda")
    del out
    # the other operand, and the columns of a matrix of such rows
    swapped = torch.empty((m, n), dtype=dtype, device="cuda")
    det.packed_product(b, a, swapped, det.alloc_packed_product_work(m, n, k))
    for i in range(0, n, 1000):
        assert bool(((swapped[:, i:i + 1000].double().cpu() - ref.t()).abs() <= bound.t()).all()), i
    del a, swapped, back
    far = torch.empty((33_000, 70_000), dtype=BF16, device="cuda")[:, :150]
    far.copy_(x[:33_000])
    across = det.alloc_packed(k, 33_000)
    det.pack(far, across=across)
    near = det.alloc_packed(k, 33_000)
    det.pack(far.contiguous(), across=near)
    assert torch.equal(across["exp"], near["exp"]) and torch.equal(across["codes"].view(torch.uint8), near["codes"].view(torch.uint8))


@pytest.mark.parametrize("products", ["f32", "f16"])
def test_long_lists_of_matrices_of_all_kinds(det, products):
    """More than 64 matrices (what a wave looks through at once) of every kind of tiles, tiny ones among them."""
    g = torch.Generator().manual_seed(1)
    shapes = [(int(torch.randint(1, 200, (1,), generator=g)), int(torch.randint(1, 260, (1,), generator=g))) for _ in range(150)]
    shapes += [(300, 520), (4000, 70), (40, 3000), (520, 530)]
    mats = [(low_rank(r, c, 3 * i), low_rank(r, c, 3 * i + 1000)) for i, (r, c) in enumerate(shapes)]
    params, ms, _ = run_muon(det, mats, products)
    for (gr, m), p, m1 in zip(mats, params, ms):
        want_m, up = update_of(gr, m)
        assert torch.equal(m1.cpu(), want_m), tuple(gr.shape)
        exact, bound = refs.orthogonal_bound(up.cuda(), products)
        off = float(torch.linalg.matrix_norm(-p.double() - exact))
        assert off <= bound, (tuple(gr.shape), off, bound)


@pytest.mark.parametrize("count", [64, 65, 4097, 4500])
def test_lists_that_are_looked_through_in_steps(det, count):
    """64 matrices are looked at at once, 64 stretches of more, and stretches of those."""
    shapes = [(66, 70), (70, 9), (5, 200)]
    pairs = [(low_rank(*s, 7), low_rank(*s, 8)) for s in shapes]
    bounds = [refs.orthogonal_bound(update_of(*p)[1].cuda(), "f32") for p in pairs]
    which = [i % 7 % 3 for i in range(count)]
    params, _, _ = run_muon(det, [pairs[w] for w in which])
    for s in range(3):
        all_of = torch.stack([p for p, w in zip(params, which) if w == s]).double()
        off = torch.linalg.matrix_norm(-all_of - bounds[s][0])
        assert float(off.max()) <= bounds[s][1], (shapes[s], int(off.argmax()))


@pytest.mark.parametrize("count,rows,cols", [(4, 2100, 2100), (6, 2100, 2180), (3, 2177, 4400), (2, 2900, 3000)])
def test_tiles_that_are_left_over(det, count, rows, cols):
    """More large tiles than one round of the chip, the last ones taken in parts: of the products (4: 324 tiles in quarters, 2: 288 in
    sixteenths) and of the symmetric ones (6: 270), wide and tall."""
    for shape in ((rows, cols), (cols, rows)):
        say(f"{count} of {shape}")
        g, m = low_rank(*shape, 1) * 1e-3, low_rank(*shape, 4) * 1e-2
        params, _, _ = run_muon(det, [(g * (1 + i), m * (1 + i)) for i in range(count)], "f32", eps=0.0)
        exact, bound = refs.orthogonal_bound(update_of(g, m)[1].cuda(), "f32", eps=0.0)
        for p in params:
            assert float(torch.linalg.matrix_norm(-p.double() - exact)) <= bound


@pytest.mark.parametrize("products", ["f32", "f16"])
def test_matrices_of_many_sizes_in_one_update(det, products):
    """Sizes that share a launch are dealt out to the parts of the chip each by itself: large ones whose symmetric products are taken in
    quarters, some of whose tiles lie outside, and numbers of tiles that no eighth divides."""
    shapes = [(1030, 1100), (2300, 1100), (300, 260), (600, 4200), (130, 70), (2300, 1100), (1030, 1100), (600, 4200), (2300, 1100), (300, 260),
              (2300, 1100), (1100, 2300), (600, 4200), (1025, 1025), (4200, 600), (2300, 1100)]
    pairs = {s: (low_rank(*s, 1) * 1e-3, low_rank(*s, 4) * 1e-2) for s in set(shapes)}
    params, _, _ = run_muon(det, [pairs[s] for s in shapes], products, eps=0.0)
    bounds = {s: refs.orthogonal_bound(update_of(*pairs[s])[1].cuda(), products, eps=0.0) for s in pairs}
    for s, p in zip(shapes, params):
        exact, bound = bounds[s]
        assert float(torch.linalg.matrix_norm(-p.double() - exact)) <= bound, s


def test_an_update_behind_a_table_whose_lists_the_caller_drops(det):
    """The table keeps the memory of its tensors."""
    mats = [(low_rank(70, 90, 1), low_rank(70, 90, 2))]
    (want,), _, _ = run_muon(det, mats)
    p, g, m = torch.zeros((70, 90), device="cuda"), mats[0][0].cuda(), mats[0][1].cuda()
    at = p.untyped_storage()
    table = det.muon_table([p], [g], [m])
    work = det.alloc_muon_work(table)
    del g, m
    junk = [torch.full((70, 90), float("nan"), device="cuda") for _ in range(8)]
    det.muon(table, work, lr=1.0)
    assert torch.equal(p, want) and len(junk) == 8 and at.nbytes()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_row_against_many(det, dtype):
    """One row of a matrix whose distance to the next says nothing, in tiles of every kind."""
    for n, k in ((5, 101), (700, 77), (50_000, 101), (50_000, 300)):
        a, b = packed(det, randn((n, k), 1)), packed(det, randn((1, k), 2))
        ref, bound = refs.product(refs.values(a["codes"], a["exp"].cpu()), refs.values(b["codes"], b["exp"].cpu()), dtype)
        for x, y, t in ((a, b, False), (b, a, True)):
            shape = (1, n) if t else (n, 1)
            out = torch.empty(shape, dtype=dtype, device="cuda")
            det.packed_product(x, y, out, det.alloc_packed_product_work(*shape, k))
            assert bool(((out.double().cpu() - (ref.t() if t else ref)).abs() <= (bound.t() if t else bound)).all()), (n, k, t)


@pytest.mark.parametrize("shape", [(300, 200), (40, 64)])
def test_a_table_that_is_not_the_host_s_writes_nothing(det, shape):
    p, g, m = torch.zeros(shape, device="cuda"), low_rank(*shape, 1).cuda(), low_rank(*shape, 2).cuda()
    table = det.muon_table([p], [g], [m])
    work, before = det.alloc_muon_work(table), m.clone()
    whole = table["bytes"].clone()
    for spoil in (lambda b: b.zero_(), lambda b: b[300:301].add_(1), lambda b: b[-1:].add_(1)):
        b = whole.clone()
        spoil(b)
        same_mark = bool((b[:8] == whole[:8]).all())
        if same_mark:
            b[:8] = 0                                        # (a copy that was not made whole: not the host's mark)
        det.muon(dict(table, bytes=b), work, lr=1.0)
        assert bool((p == 0).all()) and torch.equal(m, before)
    det.muon(table, work, lr=1.0)
    assert bool((p != 0).any())
