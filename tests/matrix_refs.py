"""Plain implementations in 64 bits of the operators of a training step's matrices (packing, products of packed
matrices, updates by orthogonalised momentum), with the bounds that the kernels' roundings stay within.

u(t) is the largest relative error of one rounding to type t; sums of k fp32 terms in any order are off by at
most k u(f32) times the sum of their magnitudes.
"""
import math

import torch

U32 = 2.0 ** -24
BLOCK = 128
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
MOST = {"e4m3": 448.0, "e5m2": 57344.0}
DIGITS = {"e4m3": 3, "e5m2": 2}
LEAST = {"e4m3": -6, "e5m2": -14}
USUAL = (3.4445, -4.7750, 2.0315)


def u(dtype):
    return torch.finfo(dtype).eps / 2


def pack(x, square=False, codes="e4m3"):
    """(codes as bytes [n][k], exponents [blocks of k][n]) of x on the CPU, from the definition."""
    n, k = x.shape
    x = x.double()
    blocks = -(-k // BLOCK)
    tall = BLOCK if square else 1
    exp = torch.zeros((blocks, n), dtype=torch.uint8)
    out = torch.zeros((n, k), dtype=torch.uint8)
    for i in range(0, n, tall):
        for b in range(blocks):
            part = x[i:i + tall, b * BLOCK:(b + 1) * BLOCK]
            if not bool(torch.isfinite(part).all()):
                e, bytes_ = 255, torch.full(part.shape, 0x7F, dtype=torch.uint8)
            elif float(part.abs().max()) == 0.0:
                e, bytes_ = 0, part.to(CODES[codes]).view(torch.uint8)
            else:
                e = 1
                while float(part.abs().max()) > MOST[codes] * 2.0 ** (e - 127):
                    e += 1
                q = part * 2.0 ** (127 - e)
                step = torch.exp2((torch.frexp(q)[1] - 1).clamp(min=LEAST[codes]).double() - DIGITS[codes])
                bytes_ = (torch.round(q / step) * step).to(CODES[codes]).view(torch.uint8)   # (exact: a number of the type)
            exp[b, i:i + tall] = e
            out[i:i + tall, b * BLOCK:(b + 1) * BLOCK] = bytes_
    return out, exp


def values(codes, exp):
    """What packed numbers stand for, in 64 bits (on the CPU)."""
    n, k = codes.shape
    two = torch.exp2(exp.double() - 127)
    two[exp == 255] = float("nan")
    return codes.cpu().float().double() * two.t().repeat_interleave(BLOCK, 1)[:, :k]


def product(a, b, dtype, old=None):
    """(a b^T, bound on its error) of the values a, b."""
    k = a.shape[1]
    ref, mag = a @ b.t().contiguous(), a.abs() @ b.abs().t().contiguous()
    if old is not None:
        ref, mag = ref + old.double(), mag + old.double().abs()
    bound = (k + 16) * U32 * mag
    if dtype is not torch.float32:
        # sums of eight neighbours by the 8-bit matrix cores: each product is cut below 2^-13 of the largest one
        largest = torch.zeros_like(ref)
        for g in range(0, k, 8):
            largest += (a[:, None, g:g + 8] * b[None, :, g:g + 8]).abs().amax(2)
        bound += 8 * 2.0 ** -13 * largest
    least = torch.finfo(dtype).smallest_normal * 2 * u(dtype)         # a subnormal's step
    return ref, bound + u(dtype) * (ref.abs() + bound) + least / 2 + 1e-44


def _digits(x, kept, one):
    """x rounded as numbers of f16 times 1 / one: hi alone, or hi + lo."""
    x = x * one
    hi = x.to(torch.float16).double()
    if kept == 2:
        hi = hi + (x - hi).to(torch.float16).double()
    return hi / one


def orthogonal(u_, steps=5, coefficients=None, products=None, eps=1e-7):
    """The Newton-Schulz steps in 64 bits; with products "f32" or "f16" its operands are rounded where the kernels
    round them, and sums to fp32."""
    x = u_.double()
    size = float(torch.linalg.matrix_norm(x)) + eps
    x = x / size if size else x
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    coefficients = coefficients or [USUAL] * steps
    f32 = (lambda t: t.float().double()) if products else (lambda t: t)
    one = 2.0 ** 15
    for a, b, c in coefficients:
        if products is None:
            aa = x @ x.t().contiguous()
            x = a * x + (b * aa + c * (aa @ aa)) @ x
            continue
        both = 2 if products == "f32" else 1
        x2, xs = _digits(f32(x), 2, one), _digits(f32(x), both, one)
        aa = _digits(f32(xs @ xs.t().contiguous()), both, one)
        bb = f32(b * aa + c * (aa @ aa))
        most = max(float(bb.abs().max()), 1e-30)
        bb = _digits(bb, both, 2.0 ** math.floor(math.log2(32768.0 / max(most, 4.0))))
        x = a * x2 + bb @ xs
    x = f32(x)
    return x.t().contiguous() if tall else x


def orthogonal_bound(u_, products, **kw):
    """(exact result, bound on the norm of the kernels' difference from it): what the documented roundings of the operands change,
    computed in 64 bits, and as much again three times over for the roundings of sums, which are not modelled and are no larger."""
    exact = orthogonal(u_, **kw)
    rounded = orthogonal(u_, products=products, **kw)
    off = float(torch.linalg.matrix_norm(rounded - exact))
    return exact, 4 * off + 2 ** -20 * float(torch.linalg.matrix_norm(exact))
