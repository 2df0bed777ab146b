"""Plain implementations in 64 bits of the operators of a sweep's training step, with the bounds
that the kernels' roundings stay within.

u(t) is the largest relative error of one rounding to type t; sums of k fp32 terms in any order are
off by at most k u(f32) times the sum of their magnitudes.
"""
import numpy as np
import torch

U32 = 2.0 ** -24


def u(dtype):
    return torch.finfo(dtype).eps / 2


def tokens(n, vocab, seed, padding=0.0, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    t = (torch.rand(n, generator=g) ** 3 * vocab).long().clamp_(max=max(vocab - 1, 0))
    t[torch.rand(n, generator=g) < padding] = -1
    return t.to(dtype)


def lookup(weight, t, scale):
    """Exact: the product is rounded to fp32, then to the type."""
    out = torch.zeros((len(t), weight.shape[1]), dtype=torch.float32)
    inside = (t >= 0) & (t < weight.shape[0])
    out[inside] = weight[t[inside].long()].float() * np.float32(scale).item()
    out[t >= weight.shape[0]] = float("nan")
    return out.to(weight.dtype)


def lookup_grad(out_grad, t, scale, vocab, old=None):
    """(gradient, bound on its error) in 64 bits."""
    inside = (t >= 0) & (t < vocab)
    idx, rows = t[inside].long(), out_grad[inside].double()
    z = lambda: torch.zeros((vocab, out_grad.shape[1]), dtype=torch.float64)
    scale = float(np.float32(scale))
    sums = z().index_add_(0, idx, rows) * scale
    mags = z().index_add_(0, idx, rows.abs()) * abs(scale)
    count = torch.bincount(idx, minlength=vocab).double()[:, None]
    ref = sums if old is None else sums + old.double()
    # additions, the scale's product, with an old value one more addition; then the type's rounding
    bound = (count + 2) * U32 * mags + (0 if old is None else U32 * ref.abs())
    tiny = torch.finfo(out_grad.dtype).smallest_normal * u(out_grad.dtype) * 2
    return ref, bound + u(out_grad.dtype) * (ref.abs() + bound) + tiny


class Loss:
    """Loss and gradients of hidden [n][d], weight [V][d] with c = rows' weights, in 64 bits, with bounds."""

    def __init__(self, hidden, weight, t, scale=1.0, grad_mean=None, grad_rows=None):
        h, w = hidden.double(), weight.double()
        n, d = h.shape
        V = w.shape[0]
        s = float(np.float32(scale))
        keep = (t >= 0) & (t < V)
        clean = torch.where(torch.isfinite(h), h, torch.zeros_like(h))
        logits = s * clean @ w.T
        # an element of the product is off by the sum of d exact products' roundings; scaled by
        # s (rounded) and to units of log 2 and back (three roundings more)
        self.logit_err = (d + 4) * U32 * abs(s) * (clean.abs() @ w.abs().T) + 4 * U32 * logits.abs()
        self.lse = torch.logsumexp(logits, 1)
        rows = torch.arange(n)
        at = torch.where(keep, t.long(), torch.zeros_like(t.long()))
        self.loss = torch.where(keep, self.lse - logits[rows, at], torch.zeros(n, dtype=torch.float64))
        self.loss[t >= V] = float("nan")
        self.count = int((t >= 0).sum())
        self.mean = self.loss.sum() / max(1, self.count) if n else torch.zeros((), dtype=torch.float64)
        # sums of V exponentials (1 ulp each) in a tree of at most 64 + V / 8192 levels' terms; logarithm
        # 1 ulp of a value up to log2(V) + the largest logit
        worst = self.logit_err.max(1).values if n else self.logit_err.sum(1)
        top = logits.abs().max(1).values if n else worst
        self.lse_bound = worst + (80 + V / 8192) * U32 * 2 + 6 * U32 * (top + self.lse.abs() + 24)
        self.loss_bound = self.lse_bound + self.logit_err[rows, at] + U32 * (self.lse.abs() + self.loss.nan_to_num().abs())
        self.mean_bound = ((self.loss_bound * keep).sum() + n * U32 * self.loss.nan_to_num().abs().sum()) / max(1, self.count) \
            + 2 * U32 * self.mean.nan_to_num().abs()
        if grad_mean is None and grad_rows is None:
            return
        c = torch.zeros(n, dtype=torch.float64)
        if grad_rows is not None:
            c = c + grad_rows.double()
        if grad_mean is not None:
            c = c + float(grad_mean) / max(1, self.count)
        c = torch.where(keep, c, torch.zeros_like(c))[:, None]
        hot = torch.zeros((n, V), dtype=torch.float64)
        hot[rows, at] = 1.0
        p = torch.exp(logits - self.lse[:, None])
        g = c * (p - hot)
        # the exponent's error, the exponential's, the subtraction's and products', G's rounding; in f16
        # G also underflows by half of the least number, in units of 2^-14 of the largest c's power of two
        t16 = hidden.dtype
        expo = self.logit_err + self.lse_bound[:, None] + 4 * U32 * (logits.abs() + self.lse.abs()[:, None])
        g_err = c.abs() * p * (torch.expm1(expo) + 4 * U32) + (u(t16) + 6 * U32) * g.abs() * (1 + expo)
        if t16 == torch.float16 and n:
            g_err = g_err + c.abs().max() * 2.0 ** -25 * 2.0 ** -13
        g_err = torch.where(c != 0, g_err, torch.zeros_like(g_err))
        self.hidden_grad = s * g @ w
        self.weight_grad = s * g.T @ clean
        low = torch.finfo(t16).smallest_normal * u(t16) * 2
        for name, a, ea, b, k in (("hidden_grad", g, g_err, w, V), ("weight_grad", g.T, g_err.T, clean, n)):
            ref = getattr(self, name)
            e = abs(s) * (ea @ b.abs()) + (k + 66) * U32 * abs(s) * ((a.abs() + ea) @ b.abs())
            setattr(self, name + "_bound", e + u(t16) * (ref.abs() + e) + low)


# ---- AdamW -----------------------------------------------------------------------------------

F = np.float32


def _hash(index, seed):
    low = np.uint64(0xFFFFFFFF)
    i = index.astype(np.uint64)
    with np.errstate(over="ignore"):
        x = ((i & low) * np.uint64(0x9E3779B1) + (i >> np.uint64(32)) * np.uint64(0x7F4A7C15) +
             np.uint64(seed) * np.uint64(0x85157AF5)) & low
        x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x58F38DED)) & low
        x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x1AC2F6EB)) & low
    return (x ^ (x >> np.uint64(16))).astype(np.uint32)


def e4m3_value(code):
    """The number of an e4m3 code, from its bits."""
    code = np.asarray(code, dtype=np.uint8).astype(np.int64)
    e, f = (code >> 3) & 15, code & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((code & 127) == 127, np.nan, v)
    return np.where(code & 128, -v, v)


_VALUES = e4m3_value(np.arange(127))


def decode(codes, exps):
    two = np.where(exps == 0, 0.0, 2.0 ** (exps.astype(np.float64) - 127))
    two = np.where(exps == 255, np.nan, two)
    return (e4m3_value(codes) * np.repeat(two, 256)[:len(codes)]).astype(F)


def encode(x, dither16, root):
    """Codes and exponents of fp32 values x, by the table of e4m3 numbers: the lower neighbour, or the
    upper one where the distance to the lower plus the dither reaches a whole step."""
    n = len(x)
    blocks = np.zeros(-(-n // 256) * 256, dtype=F)
    blocks[:n] = x
    blocks = blocks.reshape(-1, 256).astype(np.float64)
    bad = ~np.isfinite(blocks).all(1)
    most = np.abs(np.where(np.isfinite(blocks), blocks, 0)).max(1)
    exps = np.zeros(len(most), dtype=np.int64)
    some = most > 0
    exps[some] = np.maximum(np.ceil(np.log2(most[some] / 448.0)).astype(np.int64) + 127, 1)
    # (log2 may round across a whole number)
    exps[some & (most > 448.0 * 2.0 ** (exps - 127.0))] += 1
    down = some & (exps > 1) & (most <= 224.0 * 2.0 ** (exps - 127.0))
    exps[down] -= 1
    q = np.abs(np.where(bad[:, None], 0, blocks)) / np.where(some, 2.0 ** (exps - 127.0), 1.0)[:, None]
    q = q.reshape(-1)[:n]
    # below 2^-6 the kernel adds 2^-6 in fp32 first
    small = q < 2.0 ** -6
    q = np.where(small, (q.astype(F) + F(2.0 ** -6)).astype(np.float64) - 2.0 ** -6, q)
    lower = np.searchsorted(_VALUES, q, side="right") - 1
    upper = np.minimum(lower + 1, 126)
    step = np.where(_VALUES[lower] < 2.0 ** -6, 2.0 ** -9, 2.0 ** (np.floor(np.log2(np.maximum(_VALUES[lower], 2.0 ** -6))) - 3))
    # the digits below 2^-20 of a step are dropped with the rest
    part = np.floor((q - _VALUES[lower]) / step * 2.0 ** 20)
    code = np.where(part + dither16.astype(np.int64) * 16 + 8 >= 2 ** 20, upper, lower)
    if root:
        code = np.where((code == 0) & (x > 0), 1, code)
    code = np.where(np.signbit(x), code | 128, code).astype(np.uint8)
    code = np.where(np.repeat(bad, 256)[:n], 0x7F, code).astype(np.uint8)
    exps[bad] = 255
    return code, exps.astype(np.uint8)


def adamw(p, g, m, v, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, lr_scale=1.0, grad_scale=None,
          m_exp=None, v_exp=None, first_index=0, seed=None):
    """One update in fp32, every operation rounded by itself; numpy arrays (p, g as fp32).  Returns
    (p, m, v) or, with 8-bit states, (p, m, v, m_exp, v_exp)."""
    eight = m_exp is not None
    if eight:
        m, r = decode(m, m_exp), decode(v, v_exp)
        v = r * r
    with np.errstate(all="ignore"):
        if grad_scale is not None:
            g = g * F(grad_scale)
        m = m * F(beta1) + g * F(1 - beta1)
        v = v * F(beta2) + (g * F(1 - beta2)) * g
        r = np.sqrt(v)
        move = (m * F(lr * lr_scale / (1 - beta1 ** step))) / (r * F(1 / np.sqrt(1 - beta2 ** step)) + F(eps))
        p = p * F(1 - lr * lr_scale * decay) - move
    if not eight:
        return p, m, v
    h = _hash(np.arange(first_index, first_index + len(p)), step if seed is None else seed)
    cm, em = encode(m, h & 0xFFFF, False)
    cv, ev = encode(r, h >> 16, True)
    return p, cm, cv, em, ev


def adamw64(p, g, m, v, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0):
    p, g, m, v = (np.asarray(x, dtype=np.float64) for x in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps), m, v
