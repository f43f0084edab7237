"""References in 64 bits for the tests of the training operators, and bounds of their errors."""
import math

import torch

EPS32 = 2.0 ** -23
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a step, relative
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def act64(name, z):
    """act(z), act'(z) for a float64 z, from the definitions."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return torch.where(z > 0, z, 0 * z), torch.where(z > 0, torch.ones_like(z), torch.zeros_like(z))
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        a, b = math.sqrt(2 / math.pi), 0.044715
        t = torch.tanh(a * (z + b * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * b * z * z)
    s = torch.sigmoid(z)
    return z * s, s * (1 + z * (1 - s))


def strided(rows, cols, dtype, gen, scale=1.0, pad=0, shift=0):
    """Normal entries in a matrix whose rows are cols + pad apart, `shift` elements behind an aligned address; what lies
    around it in memory is NaN."""
    n = rows * (cols + pad) + shift + 64
    whole = torch.full((n,), float("nan"), dtype=dtype, device="cuda")
    m = whole[shift:shift + max(rows, 1) * (cols + pad)].view(max(rows, 1), cols + pad)[:rows, :cols]
    if rows and cols:
        m.copy_((torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dtype))
    return m


def forward64(x, w, bias, residual, act):
    """y, z and a bound of the error of a forward pass in fp32 that rounds y once."""
    x, w = x.double(), w.double()
    k = x.shape[1]
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    y = act64(act, z)[0]
    # a sum of k + 1 terms in any order; slopes are at most 1.13; the functions are good to a few units of 1 + |z|
    dz = (k + 4) * EPS32 * size
    err = 1.2 * dz + (0 if act in ("none", "relu") else 2.0 ** -19 * (1 + z.abs()))
    if residual is not None:
        y = y + residual.double()
        err = err + EPS32 * y.abs()
    return y, z, err, dz


def check(got, want, err, dtype, what=""):
    """|got - want| <= err + one rounding to dtype."""
    off = (got.double() - want).abs()
    most = err + UNIT[dtype] * (want.abs() + err) + LEAST[dtype]
    assert torch.isfinite(got).all(), what
    assert bool((off <= most).all()), f"{what}: {float((off / most).max()):.3g} times the bound"
