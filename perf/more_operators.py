"""The products of a rank's layer, as measurable cases: what a rank of a serving replica
computes beside its attention.

  linear     fs_linear: y = act(x W^T + bias) + residual
  gated      fs_gated_ff: y = act(x Wg^T) * (x Wu^T)
  backward   fs_gated_ff_backward: the gradients of x, Wg and Wu
  quantise   fs_quantise_rows: 16-bit rows become e4m3 codes with a power-of-two scale a row,
             which is what the e4m3 products read

The replica has 64 query heads and 8 key heads of 128, so rows of 8192 (8192 to 10240 for queries,
keys and values), and a gated block of 14336; a rank of TP degree tau in {1, 2, 4, 8} holds a
tau-th of the heads and of the block. x and W are bfloat16 or float16, or both e4m3 codes with a
scale for each row of x and of W.
"""

import math

import torch

own = False

E4M3_MAX = 448.0
HIDDEN, QKV, BLOCK = 8192, 10240, 14336


# ------------------------------------------------------------------ cases

def _case(op, rows, inner, outer, dtype="bfloat16", act="none", bias=False, residual=False):
    return {"op": op, "rows": rows, "in": inner, "out": outer, "dtype": dtype, "act": act, "bias": bias, "residual": residual}


def listed():
    def named(name, c):
        return dict(c, name=name)

    return [
        # one request's next token: queries, keys and values on a rank of TP 8; all latency
        named("linear_one", _case("linear", 1, HIDDEN, QKV // 8, bias=True)),
        # the next token of 64 requests, TP 1, 8-bit weights: bound by reading them
        named("linear_step", _case("linear", 64, HIDDEN, QKV, "e4m3", bias=True)),
        # a ragged chunk through odd sizes
        named("linear_odd", _case("linear", 333, 1001, 777, "float16", "gelu", bias=True, residual=True)),
        # prompts of 8192 tokens in all: queries, keys and values, TP 1
        named("linear_prompt", _case("linear", 8192, HIDDEN, QKV, bias=True)),
        # the gated block's way back to the residual stream, TP 2, 8-bit
        named("linear_down", _case("linear", 4096, BLOCK // 2, HIDDEN, "e4m3", residual=True)),
        # one request's next token, TP 8
        named("gated_one", _case("gated", 1, HIDDEN, BLOCK // 8, act="silu")),
        # the next token of 48 requests, TP 2, 8-bit
        named("gated_step", _case("gated", 48, HIDDEN, BLOCK // 2, "e4m3", "silu")),
        # prompts of 4096 tokens in all, TP 1: the largest
        named("gated_prompt", _case("gated", 4096, HIDDEN, BLOCK, act="silu")),
        # a small block's gradients, odd sizes
        named("backward_odd", _case("backward", 77, 520, 1003, "float16", "gelu_tanh")),
        # a training batch of 4096 tokens through half a block
        named("backward_batch", _case("backward", 4096, HIDDEN // 2, BLOCK // 2, act="silu")),
        # the rows of a decode step, before an 8-bit product
        named("quantise_step", _case("quantise", 64, HIDDEN, 0)),
        # a prompt's rows before the way back from the gated block
        named("quantise_prompt", _case("quantise", 8192, BLOCK, 0)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("linear", "linear", "linear", "gated", "gated", "backward", "quantise"))
    rows = _log_int(rng, 1, 8192)

    def size(lo, hi):
        n = _log_int(rng, lo, hi)
        return n if rng.random() < 0.4 else max(lo, n // 64 * 64)

    inner = size(64, BLOCK)
    if op == "quantise":
        return _case(op, rows, inner, 0, rng.choice(("bfloat16", "float16")))
    outer = size(16, 10240 if op == "linear" else 8192)
    if op == "backward":
        rows, inner, outer = min(rows, 4096), min(inner, 4096), min(outer, 7168)
        return _case(op, rows, inner, outer, rng.choice(("bfloat16", "float16")), rng.choice(("silu", "gelu", "gelu_tanh", "relu")))
    dtype = rng.choice(("bfloat16", "float16", "e4m3"))
    if op == "gated":
        rows = min(rows, 4096)
        return _case(op, rows, inner, outer, dtype, rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu")))
    return _case(op, rows, inner, outer, dtype, rng.choice(("none", "none", "relu", "silu", "gelu", "gelu_tanh")),
                 rng.random() < 0.5, rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

class State:
    pass


def _rows(n, width, dtype):
    """n rows of `width`, each beginning on a multiple of 16 elements."""
    return torch.empty(n, -(-width // 16) * 16, dtype=dtype, device="cuda")[:, :width]


def _filled(x, g, gain=1.0):
    for a in range(0, x.shape[0], 1 << 12):
        b = min(x.shape[0], a + (1 << 12))
        x[a:b] = (torch.randn(b - a, x.shape[1], generator=g, device="cuda") * gain).to(x.dtype)
    return x


def _power(e):
    """2^e in float, -126 <= e <= 127, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _codes(x, whole):
    """Rows x in e4m3: (codes, a scale a row: a power of two, or with `whole` any number)."""
    amax = x.float().abs().amax(-1)
    if whole:
        s = amax / E4M3_MAX
    else:
        m, e = torch.frexp(amax)
        s = _power(e - torch.where(m <= 0.875, 9, 8))
    s = torch.where(amax > 0, s, 1.0)
    c = _rows(x.shape[0], x.shape[1], torch.uint8)
    c.copy_((x.float() / s[:, None]).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8))
    return c.view(torch.float8_e4m3fn), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    T, K, N, op = case["rows"], case["in"], case["out"], case["op"]
    eight = case["dtype"] == "e4m3"
    dt = torch.bfloat16 if eight else getattr(torch, case["dtype"])
    s = State()
    s.case = case
    # activations: some channels far larger than others, tokens differ in magnitude
    gain = torch.exp(0.7 * torch.randn(K, generator=g, device="cuda"))
    x = _filled(_rows(T, K, dt), g, gain)
    x.mul_(torch.exp(0.3 * torch.randn(T, 1, generator=g, device="cuda")).to(dt))
    weight = lambda n: _filled(_rows(n, K, dt), g, K ** -0.5)  # noqa: E731
    s.x_scale = None
    if op == "quantise":
        s.x, s.codes, s.scale = x, _rows(T, K, torch.uint8).view(torch.float8_e4m3fn), torch.empty(T, device="cuda")
        if own:
            from paper_2608_19659_gb300 import fleetsieve as fsb

            s.fsb = fsb
        return s
    s.w = [weight(N) for _ in range(1 if op == "linear" else 2)]
    s.w_scale = [None] * len(s.w)
    if eight:
        x, s.x_scale = _codes(x, False)
        pairs = [_codes(w, True) for w in s.w]
        s.w, s.w_scale = [p[0] for p in pairs], [p[1] for p in pairs]
    s.x = x
    s.bias = (0.2 * torch.randn(N, generator=g, device="cuda")).to(dt) if case["bias"] else None
    s.residual = _filled(_rows(T, N, dt), g) if case["residual"] else None
    s.y = _rows(T, N, dt)
    if op == "backward":
        s.dy = _filled(_rows(T, N, dt), g)
        s.dx, s.dw = _rows(T, K, dt), [_rows(N, K, dt) for _ in range(2)]
    if own:
        from paper_2608_19659_gb300 import fleetsieve as fsb

        s.fsb = fsb
        s.work = fsb.MmWorkspace(T, K, N, backward=op == "backward")
    return s


# ------------------------------------------------------------------ the plain forms

def _act(x, name):
    if name == "relu":
        return x.clamp_min(0.0)
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (x + 0.044715 * x * x * x)))
    return x


def _slope(x, name):
    if name == "relu":
        return (x > 0).to(x.dtype)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-x))
        return s * (1.0 + x * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(x * 0.5 ** 0.5)) + x * torch.exp(-0.5 * x * x) * (2.0 * math.pi) ** -0.5
    c = (2.0 / math.pi) ** 0.5
    t = torch.tanh(c * (x + 0.044715 * x * x * x))
    return 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * x * x)


def _product(s, i):
    p = s.x.float() @ s.w[i].float().T
    if s.x_scale is not None:
        p = p.mul_(s.x_scale[:, None]).mul_(s.w_scale[i])
    return p


def _plain(s):
    c = s.case
    if c["op"] == "linear":
        p = _product(s, 0)
        if s.bias is not None:
            p += s.bias.float()
        p = _act(p, c["act"])
        if s.residual is not None:
            p += s.residual.float()
        s.y.copy_(p)
    elif c["op"] == "gated":
        s.y.copy_(_act(_product(s, 0), c["act"]) * _product(s, 1))
    elif c["op"] == "backward":
        g, u, dy = _product(s, 0), _product(s, 1), s.dy.float()
        du = dy * _act(g, c["act"])
        dg = dy * u * _slope(g, c["act"])
        x, wg, wu = s.x.float(), s.w[0].float(), s.w[1].float()
        s.dx.copy_(dg @ wg + du @ wu)
        s.dw[0].copy_(dg.T @ x)
        s.dw[1].copy_(du.T @ x)
    else:
        x = s.x.float()
        m, e = torch.frexp(x.abs().amax(-1))
        s.scale.copy_(torch.where(m > 0, _power((e - torch.where(m <= 0.875, 9, 8)).clamp_min(-126)), 0.0))
        y = x / torch.where(s.scale > 0, s.scale, 1.0)[:, None]
        s.codes.copy_(y.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn))


# ------------------------------------------------------------------ one pass

def run(s):
    c = s.case
    if not own:
        _plain(s)
    elif c["op"] == "linear":
        s.fsb.fs_linear(s.x, s.w[0], s.y, bias=s.bias, residual=s.residual, activation=c["act"], x_scale=s.x_scale,
                        w_scale=s.w_scale[0], workspace=s.work)
    elif c["op"] == "gated":
        s.fsb.fs_gated_ff(s.x, s.w[0], s.w[1], s.y, activation=c["act"], x_scale=s.x_scale, gate_scale=s.w_scale[0],
                          up_scale=s.w_scale[1], workspace=s.work)
    elif c["op"] == "backward":
        s.fsb.fs_gated_ff_backward(s.x, s.w[0], s.w[1], s.dy, s.dx, s.dw[0], s.dw[1], activation=c["act"], workspace=s.work)
    else:
        s.fsb.fs_quantise_rows(s.x, s.codes, s.scale)
    if c["op"] == "backward":
        return {"dx": s.dx, "dw_gate": s.dw[0], "dw_up": s.dw[1]}
    if c["op"] == "quantise":
        return {"codes": s.codes, "scale": s.scale}
    return {"y": s.y}


def work(case):
    T, K, N = case["rows"], case["in"], case["out"]
    e = 1 if case["dtype"] == "e4m3" else 2
    if case["op"] == "quantise":
        return {"bytes": 3 * T * K + 4 * T, "flops": 3 * T * K}
    if case["op"] == "linear":
        scales = 4 * (T + N) if e == 1 else 0
        return {"bytes": e * (T * K + N * K) + 2 * T * N * (2 if case["residual"] else 1) + (2 * N if case["bias"] else 0) + scales,
                "flops": 2 * T * K * N}
    if case["op"] == "gated":
        return {"bytes": e * (T * K + 2 * N * K) + 2 * T * N + (4 * (T + 2 * N) if e == 1 else 0), "flops": 4 * T * K * N}
    return {"bytes": 2 * (T * K + 2 * N * K + T * N) + 2 * (T * K + 2 * N * K), "flops": 12 * T * K * N}


# ------------------------------------------------------------------ 64 bits

def _code_values():
    """What each e4m3 code stands for, by its definition."""
    v = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if c & 127 == 127 else m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v.append(-x if c & 128 else x)
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s = prepare(case, seed)
    name, op = case["act"], case["op"]
    if work(case)["flops"] > 6e12:
        return None
    if op == "quantise":
        x = s.x.double()
        amax = x.abs().amax(-1)
        two_to = lambda e: ((e.long() + 1023) << 52).view(torch.float64)  # noqa: E731 (logarithms and powers are not exact)
        f, e = torch.frexp(amax / E4M3_MAX)
        scale = torch.where(amax > 0, two_to(torch.where(f > 0.5, e, e - 1).clamp_min(-126)), 0.0)
        v = x / torch.where(scale > 0, scale, 1.0)[:, None]
        step = two_to(torch.frexp(v.abs().clamp_min(2.0 ** -6))[1] - 4)
        return {"codes": torch.round(v / step) * step, "scale": scale}
    values = _code_values()

    def wide(x, scale):
        return x.double() if scale is None else values[x.view(torch.uint8).long()] * scale.double()[:, None]

    x = wide(s.x, s.x_scale)
    ws = [wide(w, sc) for w, sc in zip(s.w, s.w_scale)]

    def value(z):
        if name == "relu":
            return torch.where(z > 0, z, 0.0)
        if name == "silu":
            return z * torch.special.expit(z)
        if name == "gelu":
            return z * torch.special.ndtr(z)
        if name == "gelu_tanh":  # (1 + tanh a) / 2 is the logistic function of 2 a
            return z * torch.special.expit(math.sqrt(8.0 / math.pi) * (z + 0.044715 * z ** 3))
        return z

    if op == "linear":
        z = torch.einsum("tk,nk->tn", x, ws[0])
        if s.bias is not None:
            z = z + s.bias.double()[None]
        z = value(z)
        return {"y": z if s.residual is None else z + s.residual.double()}
    if op == "gated":
        return {"y": value(torch.einsum("tk,nk->tn", x, ws[0])) * torch.einsum("tk,nk->tn", x, ws[1])}
    z = torch.einsum("tk,nk->tn", x, ws[0]).requires_grad_()
    a = value(z)
    slope, = torch.autograd.grad(a, z, torch.ones_like(a))
    z.requires_grad_(False)
    dy = s.dy.double()
    dg = dy * torch.einsum("tk,nk->tn", x, ws[1]) * slope
    du = dy * a.detach()
    return {"dx": torch.einsum("tn,nk->tk", dg, ws[0]) + torch.einsum("tn,nk->tk", du, ws[1]),
            "dw_gate": torch.einsum("tn,tk->nk", dg, x), "dw_up": torch.einsum("tn,tk->nk", du, x)}
