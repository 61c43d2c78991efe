"""Plain 64-bit restatements of the operators of a worker's local step, and the rounding of each type.

Every tolerance of the tests is built from these: `unit(dtype)` is half the spacing of a type's numbers
relative to their size (the one rounding of a result), EPS that of fp32 (the sums), and a sum of k
products may be off by (k + 32) EPS times the sum of their magnitudes, whatever its order.
"""
import math

import torch

EPS = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
_TINY = {torch.float32: 2.0 ** -125, torch.bfloat16: 2.0 ** -125, torch.float16: 2.0 ** -25}


def unit(dtype):
    return _UNIT[dtype]


def rounding(ref, dtype):
    """How far the nearest number of a type may be from ref."""
    return unit(dtype) * ref.abs() + _TINY[dtype]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def matrix(rows, cols, dtype, g, scale=1.0, pad=0, offset=0):
    """[rows, cols] with a row stride of cols + pad, starting `offset` elements into its buffer."""
    flat = torch.randn(offset + rows * (cols + pad), generator=g, device="cuda") * scale
    return flat.to(dtype)[offset:].view(rows, cols + pad)[:, :cols]


def empty(rows, cols, dtype, pad=0, offset=0):
    """An output of the same kind, filled with a value that no kernel writes; its buffer comes too."""
    flat = torch.full((offset + rows * (cols + pad) + 8,), -77.0, device="cuda", dtype=dtype)
    return flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], flat


def untouched(out, flat):
    """Whether nothing outside `out` was written in its buffer."""
    probe = flat.clone()
    view = torch.as_strided(probe, out.shape, out.stride(), out.storage_offset())
    view.fill_(-77.0)
    return bool((probe == -77.0).all())


def close(got, ref, tol, what=""):
    got = got.double()
    assert got.shape == ref.shape, what
    same = (got == ref) | (got.isnan() & ref.isnan())
    off = torch.where(same, torch.zeros_like(ref), (got - ref).abs() - tol)
    bad = ~(off <= 0)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: "
                           f"{got[bad][0].item()} for {ref[bad][0].item()}, allowed {tol.expand_as(ref)[bad][0].item()}")


# ---- layer norm

def layernorm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + eps)
    h = c * rstd[:, None]
    y = h * (1.0 if gamma is None else gamma.double()) + (0.0 if beta is None else beta.double())
    return y, mean, rstd, h


def layernorm_grad(dy, x, gamma, mean, rstd):
    dy, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    g = dy * (1.0 if gamma is None else gamma.double())
    a, b = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    return r * (g - a - h * b), (dy * h).sum(0), dy.sum(0), h, g, r


# ---- product

def act(z, name):
    return {"none": lambda v: v, "relu": lambda v: v.clamp_min(0),
            "gelu": lambda v: 0.5 * v * (1 + torch.erf(v / math.sqrt(2))),
            "gelu_tanh": lambda v: 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))),
            "silu": lambda v: v / (1 + torch.exp(-v))}[name](z)


def act_slope(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def product(a, b):
    """a b^T in 64 bits and how far 32-bit sums of its products may be off."""
    a, b = a.double(), b.double()
    return a @ b.t(), (a.shape[1] + 32) * EPS * (a.abs() @ b.abs().t())


# ---- distillation

def distill(logits, idx, teacher, label, weight, T, kd, ce):
    """loss, gradient and the tolerances of both, by the definition, row by row where that is plainest."""
    z = logits.double()
    rows, vocab = z.shape
    w = torch.ones(rows, device=z.device, dtype=torch.float64) if weight is None else weight.double()
    m = z.amax(1, keepdim=True)
    alive = (m != -math.inf)[:, 0]
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    d = z - m
    loss = torch.zeros(rows, device=z.device, dtype=torch.float64)
    loss_tol = torch.zeros_like(loss)
    grad, tol = torch.zeros_like(z), torch.zeros_like(z)
    reach = 1 + torch.where(d == -math.inf, torch.zeros_like(d), d.abs()) / min(T, 1.0)
    acts = torch.zeros(rows, dtype=torch.bool, device=z.device)
    if idx is not None and idx.shape[1] > 0 and kd != 0:
        there = (idx >= 0) & (idx < vocab)
        t = torch.where(there, teacher.double(), torch.tensor(-math.inf, device=z.device, dtype=torch.float64))
        tm = t.amax(1, keepdim=True)
        some = (tm != -math.inf)[:, 0]
        tm = torch.where(tm == -math.inf, torch.zeros_like(tm), tm)
        e = torch.exp((t - tm) / T)
        q = e / e.sum(1, keepdim=True).clamp_min(1e-300)
        logq = (t - tm) / T - torch.log(e.sum(1, keepdim=True).clamp_min(1e-300))
        at = torch.where(there, idx, torch.zeros_like(idx)).long()
        ez = torch.exp(d / T)
        S = ez.sum(1, keepdim=True)
        p = ez / S
        logp = torch.gather(d, 1, at) / T - torch.log(S)
        term = torch.where(q > 0, q * (logq - logp), torch.zeros_like(q))
        size = torch.where(q > 0, q * (2 + logq.abs() + logp.abs()), torch.zeros_like(q))
        qs = torch.zeros_like(z).scatter_add_(1, at, torch.where(there, q, torch.zeros_like(q)))
        on = some & alive
        loss += torch.where(on, kd * T * T * term.sum(1), loss * 0)
        loss_tol += torch.where(on, abs(kd) * T * T * size.sum(1), loss * 0)
        grad += torch.where(on[:, None], kd * T * (p - qs), grad * 0)
        tol += torch.where(on[:, None], abs(kd) * T * (p * reach + qs), grad * 0)
        acts |= some
    if label is not None and ce != 0:
        has = (label >= 0) & (label < vocab)
        y = torch.where(has, label, torch.zeros_like(label)).long()[:, None]
        e = torch.exp(d)
        S = e.sum(1, keepdim=True)
        p = e / S
        hot = torch.zeros_like(z).scatter_(1, y, 1.0)
        logp = (torch.gather(d, 1, y) - torch.log(S))[:, 0]
        on = has & alive
        loss += torch.where(on, -ce * logp, loss * 0)
        loss_tol += torch.where(on, abs(ce) * (2 + logp.abs()), loss * 0)
        grad += torch.where(on[:, None], ce * (p - hot), grad * 0)
        tol += torch.where(on[:, None], abs(ce) * (p * reach + hot), grad * 0)
        acts |= has
    on = acts & (w != 0)
    loss = torch.where(on, w * loss, torch.zeros_like(loss))
    grad = torch.where(on[:, None], w[:, None] * grad, torch.zeros_like(grad))
    # the exponential's argument and value, the two sums, the quotients and products: 32 roundings of fp32 at most
    return loss, 32 * EPS * w.abs() * loss_tol, grad, 32 * EPS * w.abs()[:, None] * tol
