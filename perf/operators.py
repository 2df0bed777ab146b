"""What the operators of a training step's vocabulary side are measured on: the work that a
node sweep has a GPU do, through the public entry points of
``paper_2605_17879_amd.Detector`` where ``own`` is true, and as elementary torch operations
where it is false.

A case is a dict of plain values:
  kind  "lookup"       rows of an embedding table, scaled
        "lookup_grad"  the table's gradient, written whole or added to what is there
        "loss"         softmax cross entropy of hidden states projected onto a vocabulary
        "loss_train"   the same with the gradients of the hidden states and of the weights
        "adamw"        an AdamW step over many tensors at once
  lookup*: rows (tokens looked up), vocab, width, dtype ("f32", "bf16", "f16"), padding
           (share of negative tokens), add (gradient added to what is there)
  loss*:   rows, vocab, width, dtype ("bf16", "f16"), ignored (share of rows left out),
           apart (elements between the end of a row and the next)
  adamw:   matrices, matrix (elements of each), vectors, vector, param, grad ("f32", "bf16",
           "f16"), bits (of the states: 32 or 8), copy (a bf16 copy of the parameters is
           written too)
"""
from __future__ import annotations

import math
import random

import torch

DEVICE = "cuda:0"
own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                      # elements of an 8-bit state that share a power of two
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.999, 1e-8, 0.1
FIRST_STEP = 100


def _lookup(name, rows, vocab, width, dtype, padding=0.0):
    return {"name": name, "kind": "lookup", "rows": rows, "vocab": vocab, "width": width, "dtype": dtype,
            "padding": padding}


def _lookup_grad(name, rows, vocab, width, dtype, padding=0.0, add=False):
    return {"name": name, "kind": "lookup_grad", "rows": rows, "vocab": vocab, "width": width, "dtype": dtype,
            "padding": padding, "add": add}


def _loss(name, kind, rows, vocab, width, dtype, ignored=0.0, apart=0):
    return {"name": name, "kind": kind, "rows": rows, "vocab": vocab, "width": width, "dtype": dtype,
            "ignored": ignored, "apart": apart}


def _adamw(name, matrices, matrix, vectors, vector, param, grad, bits, copy):
    return {"name": name, "kind": "adamw", "matrices": matrices, "matrix": matrix, "vectors": vectors,
            "vector": vector, "param": param, "grad": grad, "bits": bits, "copy": copy}


def listed():
    return [
        # the next tokens of a few sequences that are being answered: all latency
        _lookup("lookup-8x4096-bf16", 8, 131072, 4096, "bf16"),
        # a training batch looked up in a table kept in 32 bits, an odd vocabulary
        _lookup("lookup-16384x2048-f32", 16384, 50001, 2048, "f32", padding=0.02),
        # a small batch's gradient, sizes that are no powers of two
        _lookup_grad("lookup_grad-1000x1000-f32", 1000, 5000, 1000, "f32"),
        # a padded training batch's gradient over a large vocabulary
        _lookup_grad("lookup_grad-32768x2048-bf16", 32768, 131072, 2048, "bf16", padding=0.1),
        # tied weights: added to the gradient that the projection's side has left
        _lookup_grad("lookup_grad-16384x4096-bf16-add", 16384, 131072, 4096, "bf16", add=True),
        # the log-probability of a few answered tokens
        _loss("loss-4x131072x4096-bf16", "loss", 4, 131072, 4096, "bf16"),
        # an evaluation batch of odd sizes, fp16
        _loss("loss-1000x50001x1000-f16", "loss", 1000, 50001, 1000, "f16", ignored=0.1),
        # a small model's training step, padded rows left out
        _loss("loss_train-2000x50001x1024-bf16", "loss_train", 2000, 50001, 1024, "bf16", ignored=0.1),
        # a large model's training step
        _loss("loss_train-8192x131072x4096-bf16", "loss_train", 8192, 131072, 4096, "bf16"),
        # the norms and biases of a model on their own: many small tensors of odd sizes
        _adamw("adamw-32bit-160x1000", 0, 1, 160, 1000, "f32", "f32", 32, False),
        # a model's tensors, parameters in 32 bits with a bf16 copy for the next forward pass
        _adamw("adamw-32bit-200M", 48, 4194304, 97, 2048, "f32", "bf16", 32, True),
        # a larger one with states in 8 bits
        _adamw("adamw-8bit-540M", 32, 16777216, 65, 4096, "f32", "bf16", 8, True),
    ]


def _log_between(rng, lo, hi, unit=1):
    """A multiple of `unit`, but not of 1024 unless it is `hi`: round sizes stand in the list."""
    v = unit * max(1, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) // unit)
    return v + unit if v % 1024 == 0 and v + unit <= hi else v


def _share(rng):
    return rng.choice((0.0, 0.0, 0.02, 0.1, 0.5))


def draw(rng: random.Random):
    kind = rng.choice(("lookup", "lookup_grad", "lookup_grad", "loss", "loss_train", "loss_train", "adamw", "adamw"))
    if kind in ("lookup", "lookup_grad"):
        rows, vocab = _log_between(rng, 1, 32768), _log_between(rng, 256, 131072)
        width = _log_between(rng, 64, 4096, 8 if rng.random() < 0.7 else 1)
        case = {"kind": kind, "rows": rows, "vocab": vocab, "width": width,
                "dtype": rng.choice(("f32", "bf16", "f16")), "padding": _share(rng)}
        if kind == "lookup_grad":
            case["add"] = rng.random() < 0.4
            if case["add"]:
                case["dtype"] = rng.choice(("f32", "bf16"))
        return case
    if kind in ("loss", "loss_train"):
        rows, vocab = _log_between(rng, 1, 8192), _log_between(rng, 1000, 131072)
        width = _log_between(rng, 64, 4096, 8 if rng.random() < 0.8 else 1)
        return {"kind": kind, "rows": rows, "vocab": vocab, "width": width, "dtype": rng.choice(("bf16", "bf16", "f16")),
                "ignored": _share(rng), "apart": rng.choice((0, 0, 64, 5))}
    bits = rng.choice((32, 8))
    most = 540_000_000 if bits == 8 else 300_000_000
    matrix = _log_between(rng, 1000, 16777216)
    matrices = max(1, min(_log_between(rng, 1, 400), most // matrix))
    param = rng.choice(("f32", "f32", "bf16"))
    return {"kind": "adamw", "matrices": matrices, "matrix": matrix, "vectors": rng.randint(0, 200),
            "vector": _log_between(rng, 1, 8192), "param": param, "grad": rng.choice(("f32", "bf16")),
            "bits": bits, "copy": param == "f32" and rng.random() < 0.5}


# ---- inputs ----------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _tokens(n, vocab, share, g):
    """Tokens as text has them: the r-th most frequent about 1/r as often as the first;
    a share of them negative (padding)."""
    u = torch.rand(n, device=DEVICE, generator=g, dtype=torch.float64)
    t = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    if share:
        t = torch.where(torch.rand(n, device=DEVICE, generator=g) < share, torch.full_like(t, -1), t)
    return t


def _randn(shape, g, dtype, scale):
    return (torch.randn(shape, device=DEVICE, generator=g, dtype=torch.float32) * scale).to(dtype)


def _spans(case):
    """(first element, elements, weight decay) of each tensor in the flat buffers, and the buffers' length."""
    at, spans = 0, []
    for count, size, decay in ((case["matrices"], case["matrix"], DECAY), (case["vectors"], case["vector"], 0.0)):
        for _ in range(count):
            spans.append((at, size, decay))
            at += -(-size // BLOCK) * BLOCK
    return spans, at


def _inputs_adamw(case, seed):
    g = _generator(seed)
    spans, total = _spans(case)
    used = torch.zeros(total, dtype=torch.bool, device=DEVICE)
    for at, size, _ in spans:
        used[at:at + size] = True
    buf = {"param": _randn(total, g, TYPES[case["param"]], 0.02) * used}
    # a tensor's gradients differ by the element (rows that are seldom used, outliers)
    spread = torch.exp(1.5 * torch.randn(total, device=DEVICE, generator=g))
    buf["grad"] = (torch.randn(total, device=DEVICE, generator=g) * spread * 1e-3 * used).to(TYPES[case["grad"]])
    m = torch.randn(total, device=DEVICE, generator=g) * spread * 3e-4 * used
    r = torch.rand(total, device=DEVICE, generator=g) * spread * 2e-3 * used
    if case["bits"] == 32:
        buf["m"], buf["v"] = m, r * r
    else:
        still = torch.zeros((), dtype=torch.int64, device=DEVICE)
        buf["m"], buf["m_exp"] = _encode(m, still)
        buf["v"], buf["v_exp"] = _encode(r, still)
    if case["copy"]:
        buf["copy"] = torch.zeros(total, dtype=torch.bfloat16, device=DEVICE)
    return buf, spans


def _inputs(case, seed):
    kind = case["kind"]
    if kind == "adamw":
        buf, spans = _inputs_adamw(case, seed)
        return {"buf": buf, "spans": spans, "step": FIRST_STEP}
    g = _generator(seed)
    n, V, d, dt = case["rows"], case["vocab"], case["width"], TYPES[case["dtype"]]
    if kind == "lookup":
        return {"weight": _randn((V, d), g, dt, 0.02), "tokens": _tokens(n, V, case["padding"], g),
                "out": torch.empty((n, d), dtype=dt, device=DEVICE), "scale": math.sqrt(d)}
    if kind == "lookup_grad":
        s = {"tokens": _tokens(n, V, case["padding"], g), "out_grad": _randn((n, d), g, dt, 1e-3), "scale": math.sqrt(d)}
        s["weight_grad"] = _randn((V, d), g, dt, 1e-2) if case["add"] else torch.empty((V, d), dtype=dt, device=DEVICE)
        return s
    hidden = _randn((n, d + case["apart"]), g, dt, 1.0)[:, :d]
    weight = _randn((V, d + case["apart"]), g, dt, 2.0 / math.sqrt(d))[:, :d]
    return {"hidden": hidden, "weight": weight, "targets": _tokens(n, V, case["ignored"], g)}


def _detector():
    from paper_2605_17879_amd import Config, Detector
    return Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1), DEVICE)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if not own:
        return s
    det = s["det"] = _detector()
    kind = case["kind"]
    if kind == "adamw":
        buf = s["buf"]
        part = lambda name: [buf[name][at:at + size] for at, size, _ in s["spans"]]               # noqa: E731
        exps = lambda name: [buf[name][at // BLOCK:-(-(at + size) // BLOCK)] for at, size, _ in s["spans"]]  # noqa: E731
        state = {"m": part("m"), "v": part("v")}
        if case["bits"] == 8:
            state.update(m_exp=exps("m_exp"), v_exp=exps("v_exp"))
        s["table"] = det.adamw_table(part("param"), part("grad"), state, copies=part("copy") if case["copy"] else None,
                                     weight_decay=[w for _, _, w in s["spans"]],
                                     first_index=[at for at, _, _ in s["spans"]])
    elif kind == "lookup_grad":
        s["work"] = det.alloc_embed_grad_work(case["rows"], case["vocab"], case["width"])
    elif kind in ("loss", "loss_train"):
        n, V, d, dt = case["rows"], case["vocab"], case["width"], TYPES[case["dtype"]]
        s["out"] = det.alloc_vocab_loss(n)
        s["work"] = det.alloc_vocab_loss_work(n, V, d, grad=kind == "loss_train")
        if kind == "loss_train":
            s["grad"] = {"hidden": torch.empty((n, d), dtype=dt, device=DEVICE),
                         "weight": torch.empty((V, d), dtype=dt, device=DEVICE)}
            s["one"] = torch.ones(1, device=DEVICE)
    return s


# ---- the framework's operators ---------------------------------------------------------------

def _run_own(s):
    case, det = s["case"], s["det"]
    kind = case["kind"]
    if kind == "lookup":
        det.embed(s["weight"], s["tokens"], s["out"], scale=s["scale"])
        return s["out"]
    if kind == "lookup_grad":
        det.embed_grad(s["out_grad"], s["tokens"], s["weight_grad"], s["work"], scale=s["scale"], accumulate=case["add"])
        return s["weight_grad"]
    if kind == "loss":
        det.vocab_loss(s["hidden"], s["weight"], s["targets"], s["out"], s["work"])
        return s["out"]
    if kind == "loss_train":
        det.vocab_loss(s["hidden"], s["weight"], s["targets"], s["out"], s["work"])
        det.vocab_loss_grad(s["hidden"], s["weight"], s["targets"], s["out"], s["grad"], s["work"], grad_mean=s["one"])
        return {**s["out"], "hidden_grad": s["grad"]["hidden"], "weight_grad": s["grad"]["weight"]}
    det.adamw(s["table"], lr=LR, step=s["step"], beta1=BETA1, beta2=BETA2, eps=EPS)
    s["step"] += 1
    return _adamw_outputs(s["buf"])


def _adamw_outputs(buf):
    out = dict(buf)
    out.pop("grad")
    if out["m"].dtype == torch.uint8:                # the codes as the numbers they stand for, beside their powers of two
        out["m"], out["v"] = out["m"].view(torch.float8_e4m3fn), out["v"].view(torch.float8_e4m3fn)
    return out


# ---- the plain forms ---------------------------------------------------------------------------

def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "lookup":
        t = s["tokens"]
        rows = s["weight"][t.clamp(min=0)].float() * s["scale"]
        s["out"].copy_(torch.where((t >= 0)[:, None], rows, torch.zeros_like(rows)))
        return s["out"]
    if kind == "lookup_grad":
        t, w = s["tokens"], s["weight_grad"]
        keep = t >= 0
        sums = torch.zeros(w.shape, dtype=torch.float32, device=DEVICE)
        sums.index_add_(0, t[keep], s["out_grad"][keep].float())
        sums *= s["scale"]
        w.copy_(sums + w.float() if case["add"] else sums)
        return w
    if kind == "adamw":
        return _plain_adamw(s)
    h, w, t = s["hidden"].float(), s["weight"].float(), s["targets"]
    logits = h @ w.T
    top = logits.max(dim=1, keepdim=True).values
    lse = torch.log(torch.exp(logits - top).sum(dim=1)) + top[:, 0]
    keep = t >= 0
    at = torch.where(keep, t, torch.zeros_like(t))[:, None]
    loss = torch.where(keep, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    count = keep.sum().float()
    out = {"loss": loss, "lse": lse, "mean": torch.stack((loss.sum() / count.clamp(min=1), count))}
    if kind == "loss":
        return out
    g = torch.exp(logits - lse[:, None])
    del logits
    g.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
    g *= (keep / count.clamp(min=1))[:, None]
    dt = s["hidden"].dtype
    return {**out, "hidden_grad": (g @ w).to(dt), "weight_grad": (g.T @ h).to(dt)}


def _decode(codes, exps):
    """Numbers of an 8-bit state: e4m3 codes times a power of two per block."""
    two = (exps.to(torch.int32) << 23).view(torch.float32)
    return (codes.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * two[:, None]).view(-1)


def _encode(x, dither, keep_positive=False):
    """Codes and powers of two of x: the largest magnitude of a block comes to (224, 448]; the
    other digits are dropped after `dither` (0 to 2^20 - 1, in units of 2^-20 of a step) was added."""
    blocks = x.view(-1, BLOCK)
    bits = blocks.abs().max(dim=1).values.view(torch.int32)
    exps = (bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000)
    exps = torch.where(bits == 0, torch.zeros_like(exps), exps.clamp(min=1))
    up = torch.where(bits == 0, torch.zeros_like(exps), 254 - exps) << 23
    q = (blocks.abs() * up.view(torch.float32)[:, None]).view(-1)
    small = q < 2.0 ** -6
    t = torch.where(small, q + 2.0 ** -6, q).view(torch.int32).long() + dither
    y = (t & 0xFFF00000).int().view(torch.float32)
    y = torch.where(small, y - 2.0 ** -6, y)
    if keep_positive:
        y = torch.where((y == 0) & (q > 0), torch.full_like(y, 2.0 ** -9), y)
    return torch.copysign(y, x).to(torch.float8_e4m3fn).view(torch.uint8), exps.to(torch.uint8)


def _dither(total, seed):
    """Two 16-bit numbers for each element from its index and the seed."""
    x = torch.arange(total, dtype=torch.int64, device=DEVICE)
    low = 0xFFFFFFFF
    x = ((x & low) * 0x9E3779B1 + (x >> 32) * 0x7F4A7C15 + ((seed & low) * 0x85157AF5 & low)) & low
    x = (x ^ (x >> 16)) * 0x58F38DED & low
    x = (x ^ (x >> 15)) * 0x1AC2F6EB & low
    x = x ^ (x >> 16)
    return ((x & 0xFFFF) << 4) + 8, ((x >> 16) << 4) + 8


def _plain_adamw(s):
    buf, step = s["buf"], s["step"]
    s["step"] += 1
    g = buf["grad"].float()
    eight = s["case"]["bits"] == 8
    if eight:
        m = _decode(buf["m"], buf["m_exp"])
        r = _decode(buf["v"], buf["v_exp"])
        v = r * r
    else:
        m, v = buf["m"], buf["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * (1 - BETA2)) * g
    r = torch.sqrt(v)
    size = LR / (1 - BETA1 ** step)
    move = (m * size) / (r * (1 / math.sqrt(1 - BETA2 ** step)) + EPS)
    # the tensors with weight decay come first
    split = sum(-(-size // BLOCK) * BLOCK for _, size, decay in s["spans"] if decay)
    p = buf["param"].float()
    p[:split] *= 1 - LR * DECAY
    p -= move
    buf["param"].copy_(p)
    if "copy" in buf:
        buf["copy"].copy_(p)
    if eight:
        first, second = _dither(m.numel(), step)
        for name, x, dither in (("m", m, first), ("v", r, second)):
            codes, exps = _encode(x, dither, keep_positive=name == "v")
            buf[name].copy_(codes)
            buf[name + "_exp"].copy_(exps)
    else:
        buf["m"].copy_(m)
        buf["v"].copy_(v)
    return _adamw_outputs(buf)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- work --------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "adamw":
        n = case["matrices"] * case["matrix"] + case["vectors"] * case["vector"]
        state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK
        return {"bytes": n * (2 * SIZE[case["param"]] + SIZE[case["grad"]] + state + 2 * case["copy"]), "flops": 14 * n}
    n, V, d, size = case["rows"], case["vocab"], case["width"], SIZE[case["dtype"]]
    if kind in ("lookup", "lookup_grad"):
        there = n * (1 - case["padding"])
        # distinct tokens among so many, the r-th most frequent about 1/r as often as the first
        distinct = sum((1 - math.exp(-there / (r * math.log(V + 1)))) * c for r, c in _ranks(V))
        if kind == "lookup":
            return {"bytes": 8 * n + (distinct + n) * d * size, "flops": n * d}
        written = 2 * distinct if case["add"] else V
        return {"bytes": 8 * n + (there + written) * d * size, "flops": there * d}
    there = n * (1 - case["ignored"])
    data = 8 * n + (n + V) * d * size + 8 * n
    if kind == "loss":
        return {"bytes": data, "flops": 2.0 * n * V * d}
    # the logits and the two products with their gradient, each once (rows left out have no gradient)
    return {"bytes": data + (n + V) * d * size, "flops": (2.0 * n + 4.0 * there) * V * d}


def _ranks(V):
    """(a rank, how many it stands for): every rank up to 64, then 64 for each doubling."""
    at = 0
    while at < V:
        count = min(V - at, max(1, at // 64))
        yield at + (count + 1) / 2, count
        at += count


# ---- the definition in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    kind = case["kind"]
    s = _inputs(case, seed)
    if kind == "adamw":
        return _exact_adamw(case, s)
    if kind == "lookup":
        rows = [s["weight"].double()[s["tokens"].clamp_min(0)] * s["scale"]]
        return rows[0] * (s["tokens"] >= 0).double()[:, None]
    if kind == "lookup_grad":
        # sums over each token's stretch of the sorted tokens, as differences of running sums
        sorted_tokens, order = torch.sort(s["tokens"], stable=True)
        width = s["out_grad"].shape[1]
        running = torch.zeros((len(order) + 1, width), dtype=torch.float64, device=DEVICE)
        torch.cumsum(s["out_grad"][order].double(), 0, out=running[1:])
        ends = torch.searchsorted(sorted_tokens, torch.arange(case["vocab"] + 1, device=DEVICE))
        sums = (running[ends[1:]] - running[ends[:-1]]) * s["scale"]
        return sums + s["weight_grad"].double() if case["add"] else sums
    h, w, t = s["hidden"].double(), s["weight"].double(), s["targets"]
    n, V = case["rows"], case["vocab"]
    logits = torch.mm(h, w.t().contiguous())
    lse = torch.logsumexp(logits, 1)
    counted = torch.nonzero(t >= 0)[:, 0]
    loss = torch.zeros(n, dtype=torch.float64, device=DEVICE)
    loss[counted] = lse[counted] - logits[counted, t[counted]]
    count = max(1, len(counted))
    out = {"loss": loss, "lse": lse,
           "mean": torch.tensor([float(loss.sum()) / count, float(len(counted))], dtype=torch.float64, device=DEVICE)}
    if kind == "loss":
        return out
    g = torch.zeros((n, V), dtype=torch.float64, device=DEVICE)
    g[counted] = torch.softmax(logits[counted], 1) / count
    del logits
    g[counted, t[counted]] -= 1.0 / count
    return {**out, "hidden_grad": torch.mm(g, w), "weight_grad": torch.mm(g.t().contiguous(), h)}


def _exact_adamw(case, s):
    buf, b1, b2 = s["buf"], BETA1, BETA2
    g = buf["grad"].double()
    eight = case["bits"] == 8
    if eight:
        numbers = lambda name: (buf[name].view(torch.float8_e4m3fn).double().view(-1, BLOCK)             # noqa: E731
                                * torch.exp2(buf[name + "_exp"].double() - 127)[:, None]).view(-1)
        m, v = numbers("m"), numbers("v") ** 2
    else:
        m, v = buf["m"].double(), buf["v"].double()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    m_hat, v_hat = m / (1 - b1 ** FIRST_STEP), v / (1 - b2 ** FIRST_STEP)
    p = buf["param"].double()
    for at, size, decay in s["spans"]:
        p[at:at + size] *= 1 - LR * decay
    p -= LR * m_hat / (v_hat.sqrt() + EPS)
    out = {"param": p}
    if case["copy"]:
        out["copy"] = p
    if not eight:
        return {**out, "m": m, "v": v}
    for name, x, dither in zip(("m", "v"), (m, v.sqrt()), _dither(m.numel(), FIRST_STEP)):
        most = x.view(-1, BLOCK).abs().amax(1)
        power = torch.ceil(torch.log2(most / 448)).clamp(min=-126)       # the least that brings it to 448 or below
        q = (x.view(-1, BLOCK).abs() / torch.exp2(power)[:, None]).nan_to_num(0.0).view(-1)
        step = torch.exp2(torch.floor(torch.log2(q.clamp(min=2.0 ** -6))) - 3)
        y = torch.floor(q / step + dither.double() / 2 ** 20) * step
        if name == "v":
            y = torch.where((y == 0) & (q > 0), torch.full_like(y, 2.0 ** -9), y)
        out[name] = torch.copysign(y, x)
        out[name + "_exp"] = torch.where(most > 0, power + 127, torch.zeros_like(power)).to(torch.uint8)
    return out
