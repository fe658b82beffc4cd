"""Products of a rank's layer in 64 bits, each with a bound on what the kernels may be off by.

How the bounds come about, u = 2^-23 (a float step that may truncate, as the tensor cores' do):
- a sum of K products adds K terms, each addition off by u times the sum S of the terms' magnitudes at most, and a few
  more where parts are joined: (K + 32) u S. The products themselves are exact in float. Scales: two roundings more.
- act(z): |act'| <= 1.13 carries z's error over; its own: exponents are rounded to u/2 times their magnitude, which is
  the relative error of the exponential, and the hardware's exponential, the quotient and the error
  function are within a few steps. The exponent is |z| (silu), z^2 / 2 (gelu), 1.6 |z| + 0.08 |z|^3 (gelu_tanh), each under
  z^2 + |z|^3 / 8 + 2: (z^2 + |z|^3 / 8 + 16) 2^-21 of the value, and nothing below 2^-100.
- act'(z): |act''| <= 1.2 (relu: everything, where z's error reaches 0); each term of it as act itself, with factors up to
  1 + |z| + the exponent's slope: (z^2 + |z|^3 / 8 + 16) 2^-21 (1 + |z|) at most, as the terms with z decay faster than it
  grows: the factors of the exponential are bounded by 1.
- what is rounded to 16 bits: half a step, eps / 2 of the value or half of the subnormals' step.
"""

import math

import torch

U = 2.0**-23
HALF = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25}


def values(x, scale=None):
    """Rows as doubles: 16-bit, or e4m3 codes with their scales."""
    return x.double() if scale is None else x.view(torch.float8_e4m3fn).double() * scale.double()[:, None]


def _phi(z):
    """The normal distribution (torch.special.ndtr loses the lower tail to cancellation: 0 at -9, not 1.1e-19)."""
    return 0.5 * torch.special.erfc(-z / math.sqrt(2))


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * _phi(z)
    if name == "gelu_tanh":
        return z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z**3))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if name == "gelu":
        return _phi(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(8 / math.pi)
        s = torch.sigmoid(c * (z + 0.044715 * z**3))
        return s + z * s * (1 - s) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _own(z):
    return (z * z + z.abs() ** 3 / 8 + 16) * 2.0**-21


def _sum(x, w):
    """x w^T and what a float sum of it may be off by."""
    s = x.abs() @ w.abs().T
    return x @ w.T, (x.shape[1] + 32) * U * s


def _act(z, dz, name):
    a = act(z, name)
    if name in ("none", "relu"):
        return a, dz
    return a, 1.13 * dz + _own(z) * a.abs() + 2.0**-100


def _rounded(y, dy, dtype):
    return y, dy + HALF[dtype] * (y.abs() + dy) + TINY[dtype]


def linear(x, w, dtype, bias=None, residual=None, activation="none", x_scale=None, w_scale=None):
    z, dz = _sum(values(x, x_scale), values(w, w_scale))
    if bias is not None:
        z = z + bias.double()
        dz = dz + U * z.abs()
    y, dy = _act(z, dz, activation)
    if residual is not None:
        y = y + residual.double()
        dy = dy + U * y.abs()
    return _rounded(y, dy, dtype)


def _gate_and_up(x, wg, wu, xs=None, gs=None, us=None):
    x = values(x, xs)
    return _sum(x, values(wg, gs)), _sum(x, values(wu, us))


def gated(x, wg, wu, dtype, activation="silu", x_scale=None, gate_scale=None, up_scale=None):
    (g, dg), (u, du) = _gate_and_up(x, wg, wu, x_scale, gate_scale, up_scale)
    a, da = _act(g, dg, activation)
    y = a * u
    return _rounded(y, da * (u.abs() + du) + a.abs() * du + U * y.abs(), dtype)


def gated_backward(x, wg, wu, dy, activation="silu"):
    """[(dx, bound), (dw_gate, bound), (dw_up, bound)]"""
    dtype = x.dtype
    (g, eg), (u, eu) = _gate_and_up(x, wg, wu)
    x, wg, wu, dy = (t.double() for t in (x, wg, wu, dy))
    a, ea = _act(g, eg, activation)
    s = slope(g, activation)
    if activation == "none":
        es = torch.zeros_like(s)
    elif activation == "relu":
        es = (g.abs() <= eg).double()
    else:
        es = 1.2 * eg + _own(g) * (1 + g.abs()) * torch.clamp(s.abs() + 0.2, max=1.2)
    dg, du = dy * u * s, dy * a
    dg, eg = _rounded(dg, dy.abs() * (eu * (s.abs() + es) + u.abs() * es) + 2 * U * dg.abs(), dtype)
    du, eu = _rounded(du, dy.abs() * ea + U * du.abs(), dtype)

    def product(pairs, n):
        y = sum(p @ q for p, _, q in pairs)
        e = sum(e @ q.abs() for _, e, q in pairs) + (n + 32) * U * sum((p.abs() + e) @ q.abs() for p, e, q in pairs)
        return _rounded(y, e, dtype)

    return [product([(dg, eg, wg), (du, eu, wu)], 2 * g.shape[1]), product([(dg.T, eg.T, x)], x.shape[0]),
            product([(du.T, eu.T, x)], x.shape[0])]


def quantise(x):
    """(codes' values, scales) as doubles, by the definition: ties to even."""
    x = x.double()
    finite = torch.where(x.isfinite(), x, torch.zeros_like(x))
    amax = finite.abs().amax(-1)
    f, e = torch.frexp(amax / 448)
    two = lambda e: ((e.long() + 1023) << 52).view(torch.float64)  # noqa: E731 (powers are not exact)
    s = torch.where(amax > 0, two(torch.where(f > 0.5, e, e - 1).clamp_min(-126)), torch.zeros_like(amax))
    v = finite / torch.where(s > 0, s, torch.ones_like(s))[:, None]
    step = two(torch.frexp(v.abs().clamp_min(2.0**-6))[1] - 4)
    return torch.where(x.isfinite(), torch.round(v / step) * step, torch.full_like(x, math.nan)), s


def near(got, want):
    """Whether every value is within its bound (want: (value, bound))."""
    y, e = want
    off = (got.double() - y).abs()
    worst = (off / e).max() if off.numel() else 0.0
    assert bool((off <= e).all()), f"off by {float(worst):.3g} times the bound"
