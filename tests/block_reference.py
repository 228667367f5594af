"""The feed-forward block and its checkpoints in 64 bits, with bounds of what the kernels' roundings may do.

A `Range` is a value with how far the kernels' one may be off, both in 64 bits, and is carried along the formulas:

* a sum of K products in 32 bits is off by at most (K + 64) 2^-24 of the sum of their magnitudes (64: the rounding of the
  operands' parts in 32-bit types, and of the joined parts' sums),
* a rounding to a type is off by at most half a step, `unit` of the value (2^-8 bf16, 2^-11 f16, 2^-24 f32),
* an activation and its derivative are off by at most `CLOSE` of 1 + |value| (hardware exponentials and reciprocals; for 16-bit
  types a polynomial that is 8.5e-6 off), and have slopes of at most 1.13.
"""
import math

import torch

GROUP = 32
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}   # half of the smallest step, or less
CLOSE = {torch.float32: 2.0 ** -19, torch.float16: 2.0 ** -15, torch.bfloat16: 2.0 ** -15}


class Range:
    def __init__(self, value, off=None, beyond=math.inf):
        self.value = value.double()
        self.off = torch.zeros_like(self.value) if off is None else off
        self.beyond = beyond   # magnitudes from here on are rounded to infinity

    def t(self):
        return Range(self.value.t(), self.off.t())

    def __mul__(self, other):
        return Range(self.value * other.value,
                     self.value.abs() * other.off + other.value.abs() * self.off + self.off * other.off)

    def __add__(self, other):
        return Range(self.value + other.value, self.off + other.off)

    def __matmul__(self, other):   # sums in 32 bits
        k = self.value.shape[1]
        a, b = self.value.abs().contiguous(), other.value.abs().contiguous()
        x, y = self.off.contiguous(), other.off.contiguous()
        part = (k + 64) * 2.0 ** -24
        off = a @ y + x @ b + x @ y + part * ((a + x) @ (b + y))
        return Range(self.value.contiguous() @ other.value.contiguous(), off)

    def rounded(self, dtype):
        # (the largest number is 2^e (2 - eps), the next step would end at 2^(e + 1); half of it, 2^e eps / 2, is where infinity begins)
        most = torch.finfo(dtype).max
        beyond = most + 2.0 ** math.floor(math.log2(most)) * torch.finfo(dtype).eps / 2
        return Range(self.value, self.off + UNIT[dtype] * (self.value.abs() + self.off) + LEAST[dtype], beyond)

    def holds(self, got, name=""):
        d = (got.double() - self.value).abs()
        infinite = torch.isinf(got) & (got.sign() == self.value.sign()) & (self.value.abs() + self.off >= self.beyond)
        bad = ~((d <= self.off) | infinite)
        assert not bad.any(), (name, int(bad.sum()), float((d / self.off.clamp(min=1e-300)).max()), float(self.off.max()))


def activation(kind, a):
    """(act, its derivative) in 64 bits."""
    if kind == "silu":
        p = torch.sigmoid(a)
        return a * p, p + a * p * (1 - p)
    if kind == "gelu":
        p = 0.5 * torch.special.erfc(-a / math.sqrt(2.0))
        return a * p, p + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        u = math.sqrt(2 / math.pi)
        t = torch.tanh(u * (a + 0.044715 * a ** 3))
        return a * (1 + t) / 2, (1 + t) / 2 + a * (1 - t * t) / 2 * u * (1 + 3 * 0.044715 * a * a)
    return a.clamp(min=0), (a > 0).double()


def activated(kind, a, dtype):
    f, df = activation(kind, a.value)
    close = CLOSE[dtype]
    slope = a.off * 1.0   # (second derivatives are at most 0.8)
    if kind == "relu":    # (a derivative that may be the other one where a may have the other sign)
        slope = torch.where(a.value.abs() <= a.off, 1.0, 0.0).double()
    return Range(f, 1.13 * a.off + close * (1 + f.abs())), Range(df, slope + close * (1 + df.abs()))


def scale_of(top, most):
    """The smallest numbers of 8 significant bits, at least 2^-126, `most` times which reach `top`."""
    least = (top.double() / most).clamp(min=2.0 ** -126)
    below = (1 << 45) - 1   # the bits of a 64-bit number below its eight most significant ones
    return ((least.view(torch.int64) + below) & ~below).view(torch.float64)


def checkpoint(x):
    """(codes, scales) of rows, from the definition; elements that are not finite are coded -128."""
    n, w = x.shape
    groups = -(-w // GROUP)
    full = torch.zeros((n, groups * GROUP), dtype=torch.float64, device=x.device)
    full[:, :w] = x.double()
    full = full.view(n, groups, GROUP)
    fine = torch.isfinite(full)
    scales = scale_of(torch.where(fine, full.abs(), 0.0).amax(dim=2), 127.0)
    codes = torch.where(fine, torch.round(torch.where(fine, full, 0.0) / scales[:, :, None]), -128.0)
    return codes.view(n, -1)[:, :w].to(torch.int8), scales


def kept(c):
    """What a Checkpoint (codes of any type) stands for, in 64 bits."""
    if c.scales is None:
        return c.codes.double()
    w = c.codes.shape[1]
    x = c.codes.double() * c.scales.double().repeat_interleave(GROUP, dim=1)[:, :w]
    return torch.where(c.codes.double() == (-128 if c.codes.dtype == torch.int8 else -32768), math.nan, x)


def projections(x, w_gate, w_up):
    x = Range(x)
    return x @ Range(w_gate).t(), x @ Range(w_up).t()


def forward(x, w_gate, w_up, w_down, kind, dtype):
    gate, up = projections(x, w_gate, w_up)
    h = (activated(kind, gate, dtype)[0] * up)
    h = Range(h.value, h.off + 2.0 ** -22 * h.value.abs())
    if dtype != torch.float32:
        h = h.rounded(dtype)
    return (h @ Range(w_down).t()).rounded(dtype), gate, up


def backward(grad_y, x, w_gate, w_up, w_down, kind, dtype, gate, up, largest=None):
    """Of gate and up as Ranges (kept ones have no range); x: what its checkpoint stands for, rounded to the type."""
    grad_y, x, w_gate, w_up, w_down = (Range(t) for t in (grad_y, x, w_gate, w_up, w_down))
    f, df = activated(kind, gate, dtype)
    d = grad_y @ w_down
    d_gate, d_up, h = d * up * df, d * f, f * up
    few = 2.0 ** -21   # (multiplications in 32 bits)
    d_gate, d_up, h = (Range(r.value, r.off * (1 + few) + few * r.value.abs()) for r in (d_gate, d_up, h))
    if dtype != torch.float32:
        tiny = 0.0
        if dtype == torch.float16 and grad_y.value.numel():   # (held times the power of two of grad_y's largest)
            top = float(grad_y.value[torch.isfinite(grad_y.value)].abs().max())
            tiny = 2.0 ** -25 * 2.0 ** math.floor(math.log2(top)) if top > 0 else 0.0
        d_gate, d_up = (Range(r.value, r.off + UNIT[dtype] * (r.value.abs() + r.off) + tiny) for r in (d_gate, d_up))
        h = h.rounded(dtype)
    return [(d_gate @ w_gate + d_up @ w_up).rounded(dtype), (d_gate.t() @ x).rounded(dtype), (d_up.t() @ x).rounded(dtype),
            (grad_y.t() @ h).rounded(dtype)]
