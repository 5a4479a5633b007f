"""What the tests of the operators at the ends of a stage share: buffers with a margin that must stay as it was, and the formulas
in 64 bits."""
import math

import torch

DEV = "cuda:0"
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24, E4M3: 2.0 ** -4}       # half a step, relative to the value


class Guarded:
    """A [rows, cols] matrix at a row pitch and an element offset inside a larger buffer filled with one byte; `untouched()` says
    whether the bytes around it still are that byte."""

    def __init__(self, rows, cols, dtype, pad=0, offset=0, fill=0x5A):
        es = torch.empty(0, dtype=dtype).element_size()
        self.pitch, self.fill = cols + pad, fill
        n = (rows * self.pitch + offset + 64) * es
        self.raw = torch.full((n + (-n) % 16,), fill, dtype=torch.uint8, device=DEV)
        self.m = self.raw[:n].view(dtype)[offset:].as_strided((rows, cols), (self.pitch, 1))
        mask = torch.zeros_like(self.raw, dtype=torch.bool)
        inner = torch.zeros(n // es, es, dtype=torch.bool, device=DEV)
        inner[offset:].as_strided((rows, cols, es), (self.pitch * es, es, 1)).fill_(True)
        mask[:n] = inner.view(-1)
        self.mask = mask

    def set(self, values):
        self.m.copy_(values)
        return self

    def untouched(self):
        return bool((self.raw[~self.mask] == self.fill).all())


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(shape, g, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=g, device=DEV, dtype=F32) * std).to(dtype)


def f64(t):
    return t.to(torch.float64)


def norm_exact(x, r, w, eps):
    h = f64(x) if r is None else f64(x) + f64(r)
    n = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    y = n if w is None else n * f64(w)
    scale = (y.abs().amax(1) / 448.0).clamp_min(2.0 ** -126)
    return h, y, scale


def norm_grad_exact(h, dy, dh, w, eps):
    h, dy = f64(h), f64(dy)
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    n, g = h * rstd, dy if w is None else dy * f64(w)
    mean = (g * n).mean(1, keepdim=True)
    dx = rstd * (g - n * mean)
    size = rstd * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))     # what the terms' roundings go by
    return dx if dh is None else dx + f64(dh), size, (dy * n).sum(0), (dy * n).abs().sum(0)


def act_exact(z, act):
    if act == "relu":
        return torch.where(z > 0, z, z * 0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def act_grad_exact(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def within(got, want, bound, what):
    """Every element of got within bound of want; NaN and infinities where want has them."""
    got, want = f64(got), f64(want)
    bound = bound if isinstance(bound, torch.Tensor) else torch.full_like(want, bound)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaN in other places" % what
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), "%s: other infinities" % what
    off = ((got - want).abs() - bound)[fine]
    if off.numel() and off.max() > 0:
        at = int(torch.where(fine, (got - want).abs() - bound, torch.full_like(want, -1.0)).argmax())
        raise AssertionError("%s: element %d is %r, should be %r +- %g" % (what, at, got.view(-1)[at].item(), want.reshape(-1)[at].item(), bound.reshape(-1)[at].item()))
