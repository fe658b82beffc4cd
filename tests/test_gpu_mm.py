"""The products of a rank's layer against 64 bits (tests/mm_reference.py has the bounds)."""

import math
import random

import pytest

import mm_reference as ref

pytestmark = pytest.mark.gpu


def rows(torch, n, width, dtype, seed, gain=1.0, extra=0, fill=7.0):
    """n rows of `width` in a buffer of longer rows (and rows behind the last); what lies between holds `fill`."""
    ld = -(-width // 16) * 16 + extra
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((n + 2, ld), fill, device="cuda").to(dtype)
    buf[:n, :width] = (gain * torch.randn(n, width, generator=g, device="cuda")).to(dtype)
    return buf[:n, :width], buf


def codes(torch, n, width, seed, extra=0):
    x, _ = rows(torch, n, width, torch.float32, seed)
    amax = x.abs().amax(-1).clamp_min(1e-30)
    s = amax / 448 * 1.0
    buf = torch.full((n, -(-width // 16) * 16 + extra), 0x7f, dtype=torch.uint8, device="cuda")  # (NaN behind a row's end)
    buf[:, :width] = (x / s[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return buf.view(torch.float8_e4m3fn)[:, :width], s


def untouched(torch, buf, n, width, fill=7.0):
    want = torch.full_like(buf, fill)
    assert bool((buf[n:] == want[n:]).all()) and bool((buf[:n, width:] == want[:n, width:]).all())


def operands(torch, kind, T, K, N, count, seed, extra=0):
    """x, weights, their scales, and the type of the rest."""
    if kind == "e4m3":
        x, xs = codes(torch, T, K, seed, extra)
        ws = [codes(torch, N, K, seed + 1 + i, 16 * i) for i in range(count)]
        return x, [w for w, _ in ws], xs, [s for _, s in ws], torch.bfloat16 if seed % 2 else torch.float16
    dt = getattr(torch, kind)
    x = rows(torch, T, K, dt, seed, extra=extra)[0]
    return x, [rows(torch, N, K, dt, seed + 1 + i, K**-0.5, 8 * i)[0] for i in range(count)], None, [None] * count, dt


# one token and a tile's edges in every size; sums shorter than a block of them; many tiles, and many tiles of one size alone
SHAPES = [(1, 64, 16), (1, 1, 1), (2, 7, 3), (1, 4096, 1280), (3, 1000, 257), (16, 512, 128), (17, 520, 129), (33, 1031, 65),
          (64, 2048, 1024), (65, 320, 800), (100, 72, 1000), (127, 640, 384), (128, 640, 384), (129, 640, 384), (130, 4097, 40),
          (255, 192, 511), (256, 256, 256), (257, 200, 300), (333, 1001, 777), (600, 96, 2050), (1030, 130, 1290), (2048, 256, 2048),
          (4100, 64, 30), (24, 33, 5000), (1500, 8, 300)]
KINDS = ["bfloat16", "float16", "e4m3"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,K,N", SHAPES)
def test_linear(fsb, cuda, T, K, N, kind):
    torch = cuda
    seed = T + 3 * K + 7 * N
    x, (w,), xs, (ws,), dt = operands(torch, kind, T, K, N, 1, seed, 16)
    y, buf = rows(torch, T, N, dt, 0, extra=8)
    work = fsb.MmWorkspace(T, K, N)
    assert fsb.fs_linear(x, w, y, x_scale=xs, w_scale=ws, workspace=work) is y
    ref.near(y, ref.linear(x, w, dt, x_scale=xs, w_scale=ws))
    untouched(torch, buf, T, N)
    act = ("relu", "silu", "gelu", "gelu_tanh")[(T + K + N) % 4]
    b = rows(torch, 1, N, dt, seed + 5)[0][0]
    r = rows(torch, T, N, dt, seed + 6)[0]
    fsb.fs_linear(x, w, y, bias=b, residual=r, activation=act, x_scale=xs, w_scale=ws, workspace=work)
    ref.near(y, ref.linear(x, w, dt, b, r, act, xs, ws))
    untouched(torch, buf, T, N)
    fsb.fs_mm_check(work)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,K,N", SHAPES)
def test_gated(fsb, cuda, T, K, N, kind):
    torch = cuda
    seed = T + 5 * K + 11 * N
    x, w, xs, ws, dt = operands(torch, kind, T, K, N, 2, seed)
    y, buf = rows(torch, T, N, dt, 0, extra=16)
    work = fsb.MmWorkspace(T, K, N)
    act = ("silu", "gelu", "gelu_tanh", "relu", "none")[(T + K + N) % 5]
    assert fsb.fs_gated_ff(x, *w, y, activation=act, x_scale=xs, gate_scale=ws[0], up_scale=ws[1], workspace=work) is y
    ref.near(y, ref.gated(x, *w, dt, act, xs, *ws))
    untouched(torch, buf, T, N)
    fsb.fs_mm_check(work)


@pytest.mark.parametrize("seed", range(24))
def test_sizes_at_random(fsb, cuda, seed):
    """Sizes, types and activations as they come, every value and what lies around them."""
    torch = cuda
    rng = random.Random(seed)
    size = lambda lo, hi: max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi)))) // rng.choice((1, 1, 8, 64)) * rng.choice((1, 8)))  # noqa: E731
    for _ in range(4):
        T, K, N, kind = min(size(1, 1600), 2500), min(size(1, 3000), 4000), min(size(1, 3000), 4000), rng.choice(KINDS)
        act, bias, residual = rng.choice(list(fsb.ACTIVATIONS)), rng.random() < 0.5, rng.random() < 0.5
        x, w, xs, ws, dt = operands(torch, kind, T, K, N, 2, seed, 16)
        y, buf = rows(torch, T, N, dt, 0, extra=8)
        work = fsb.MmWorkspace(T, K, N)
        b = rows(torch, 1, N, dt, 7)[0][0] if bias else None
        r = rows(torch, T, N, dt, 8)[0] if residual else None
        fsb.fs_linear(x, w[0], y, bias=b, residual=r, activation=act, x_scale=xs, w_scale=ws[0], workspace=work)
        ref.near(y, ref.linear(x, w[0], dt, b, r, act, xs, ws[0]))
        untouched(torch, buf, T, N)
        fsb.fs_gated_ff(x, *w, y, activation=act, x_scale=xs, gate_scale=ws[0], up_scale=ws[1], workspace=work)
        ref.near(y, ref.gated(x, *w, dt, act, xs, *ws))
        untouched(torch, buf, T, N)
        fsb.fs_mm_check(work)


def test_another_stream(fsb, cuda):
    """Calls go to the stream that is asked for, or to torch's current one, after what was put there before."""
    torch = cuda
    other = torch.cuda.Stream()
    for T in (3, 500):
        x, (w,), _, _, dt = operands(torch, "bfloat16", T, 300, 200, 1, 3)
        late = rows(torch, T, 300, dt, 9)[0]
        y, z = (rows(torch, T, 200, dt, 0)[0] for _ in range(2))
        work, more = fsb.MmWorkspace(T, 300, 200), fsb.MmWorkspace(T, 300, 200)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            torch.cuda._sleep(20_000_000)
            x.copy_(late)
            fsb.fs_linear(x, w, y, workspace=work)
        fsb.fs_linear(x, w, z, workspace=more, stream=other)
        fsb.fs_mm_check(work, stream=other)
        fsb.fs_mm_check(more, stream=other)
        ref.near(y, ref.linear(late, w, dt))
        assert torch.equal(y, z)


BACK = [(1, 64, 16), (1, 1, 1), (2, 7, 3), (77, 520, 1003), (128, 128, 128), (129, 65, 257), (300, 1000, 64), (513, 264, 520), (64, 2050, 300),
        (1000, 40, 72), (700, 700, 700)]


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu", "none"])
@pytest.mark.parametrize("T,K,N", BACK)
def test_gated_backward(fsb, cuda, T, K, N, act, kind):
    torch = cuda
    x, w, _, _, dt = operands(torch, kind, T, K, N, 2, T + K + N, 8)
    dy = rows(torch, T, N, dt, 99, 0.5)[0]
    outs = [rows(torch, n, K, dt, 0, extra=8 * i) for i, n in enumerate((T, N, N))]
    work = fsb.MmWorkspace(T, K, N, backward=True)
    fsb.fs_gated_ff_backward(x, *w, dy, *(o for o, _ in outs), activation=act, workspace=work)
    for (o, buf), n, want in zip(outs, (T, N, N), ref.gated_backward(x, *w, dy, act)):
        ref.near(o, want)
        untouched(torch, buf, n, K)
    fsb.fs_mm_check(work)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "none"])
def test_gradients_against_differences(fsb, cuda, act):
    """Along random directions: sum(dy y) by central differences of the forward formula in 64 bits. The kernel's gradient g may be off
    by its bound e, which moves <g, v> by <e, |v|> at most; the differences by h^2 / 6 times a third derivative (a sum over all
    terms of |dy| times at most 30 for these inputs: generous at h = 1e-5) and rounding 2^-52 L / h."""
    torch = cuda
    T, K, N = 40, 48, 56
    x, w, _, _, dt = operands(torch, "float16", T, K, N, 2, 5)
    dy = rows(torch, T, N, dt, 99, 0.5)[0]
    outs = [rows(torch, n, K, dt, 0)[0] for n in (T, N, N)]
    fsb.fs_gated_ff_backward(x, *w, dy, *outs, activation=act, workspace=fsb.MmWorkspace(T, K, N, backward=True))
    at = [t.double() for t in (x, *w)]
    bounds = [e for _, e in ref.gated_backward(x, *w, dy, act)]
    terms = lambda p: dy.double() * ref.act(p[0] @ p[1].T, act) * (p[0] @ p[2].T)  # noqa: E731
    h = 1e-5
    size = float(terms(at).abs().sum())
    for i in range(3):
        for seed in range(4):
            v = torch.randn(at[i].shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.float64)
            up, down = ([t + (s * h * v if j == i else 0) for j, t in enumerate(at)] for s in (1, -1))
            by_differences = float((terms(up) - terms(down)).sum() / (2 * h))
            slack = float((bounds[i] * v.abs()).sum()) + h * h * 30 * float(dy.double().abs().sum()) * K + 2.0**-50 * size / h
            assert abs(float((outs[i].double() * v).sum()) - by_differences) <= slack


@pytest.mark.parametrize("T,K,N", [(5, 200, 90), (150, 200, 400), (700, 130, 1000)])
@pytest.mark.parametrize("kind", KINDS)
def test_not_finite_values_stay_in_their_row_and_column(fsb, cuda, T, K, N, kind):
    torch = cuda
    x, (w, u), xs, (ws, us), dt = operands(torch, kind, T, K, N, 2, 3)
    y = rows(torch, T, N, dt, 0)[0]
    work = fsb.MmWorkspace(T, K, N)
    args = dict(x_scale=xs, w_scale=ws, workspace=work)
    fsb.fs_linear(x, w, y, **args)
    before = y.clone()
    nan = float("nan")
    x[T - 1, K - 1] = nan
    w[N - 1, 0] = nan
    fsb.fs_linear(x, w, y, **args)
    assert bool(y[T - 1].isnan().all()) and bool(y[:, N - 1].isnan().all())
    assert torch.equal(y[:T - 1, :N - 1], before[:T - 1, :N - 1])
    for act in ("silu", "relu", "gelu", "gelu_tanh"):  # a NaN is no negative number
        fsb.fs_gated_ff(x, u, w, y, activation=act, x_scale=xs, gate_scale=us, up_scale=ws, workspace=work)
        assert bool(y[T - 1].isnan().all()) and bool(y[:, N - 1].isnan().all()) and bool(y[:T - 1, :N - 1].isfinite().all())
    if kind == "bfloat16":
        x[T - 1, K - 1], w[N - 1, 0] = float("inf"), 0.0
        fsb.fs_linear(x, w, y, workspace=work)
        want = ref.linear(x, w, dt)[0]
        assert torch.equal(y[T - 1].double(), want[T - 1])  # +-infinity by the weight's sign
        assert torch.equal(y[:T - 1, :N - 1], before[:T - 1, :N - 1])


@pytest.mark.parametrize("T", [1, 40, 300, 2000])
def test_large_values_do_not_overflow_on_the_way(fsb, cuda, T):
    """Sums beyond half precision's range that an activation brings back, and activations far out on both sides."""
    torch = cuda
    K, N = 256, 300
    x = rows(torch, T, K, torch.float16, 1, 200.0)[0]
    w = rows(torch, N, K, torch.float16, 2, 20.0)[0]
    y = rows(torch, T, N, torch.float16, 0)[0]
    r = torch.zeros(T, N + 4, dtype=torch.float16, device="cuda")[:, :N]
    work = fsb.MmWorkspace(T, K, N)
    u = rows(torch, N, K, torch.float16, 3, 1e-6)[0]
    for act in ("silu", "gelu", "gelu_tanh", "relu"):
        fsb.fs_gated_ff(x, w, u, y, activation=act, workspace=work)
        ref.near(y, ref.gated(x, w, u, torch.float16, act))
    fsb.fs_linear(x, w, y, residual=r, workspace=work)
    want, e = ref.linear(x, w, torch.float16)
    far = want.abs() > 65520 + e
    assert bool((y[far] == torch.where(want[far] > 0, float("inf"), float("-inf")).half()).all())


def test_y_is_the_residual(fsb, cuda):
    torch = cuda
    for T, K, N in ((1, 4096, 512), (40, 300, 700), (500, 1000, 900), (3000, 64, 1000)):
        x, (w,), _, _, dt = operands(torch, "bfloat16", T, K, N, 1, 4)
        y, buf = rows(torch, T, N, dt, 9)
        want = ref.linear(x, w, dt, residual=y.clone())
        work = fsb.MmWorkspace(T, K, N)
        fsb.fs_linear(x, w, y, residual=y, workspace=work)
        ref.near(y, want)
        untouched(torch, buf, T, N)


@pytest.mark.parametrize("T", [1, 30, 400, 1500])
def test_strides(fsb, cuda, T):
    """Slices of one projection's output, one residual row for all, a single row with a stride that no row could have."""
    torch = cuda
    K, N, dt = 200, 264, torch.bfloat16
    big = torch.randn(T, 1000, device="cuda").to(dt)
    x, y = big[:, 96:96 + K], big[:, 504:504 + N]
    rest = [big[:, :504].clone(), big[:, 504 + N:].clone()]
    w = torch.randn(N, K, device="cuda").to(dt)
    r = torch.randn(1, N, device="cuda").to(dt).expand(T, N)
    work = fsb.MmWorkspace(T, K, N)
    want = ref.linear(x, w, dt, residual=r)
    fsb.fs_linear(x, w, y, residual=r, workspace=work)
    ref.near(y, want)
    assert torch.equal(big[:, :504], rest[0]) and torch.equal(big[:, 504 + N:], rest[1])
    one = torch.randn(777, device="cuda").to(dt)[None]
    v = torch.randn(31, 784, device="cuda").to(dt)[:, :777]
    out = torch.empty(1, 31, dtype=dt, device="cuda")
    fsb.fs_linear(one, v, out, workspace=work)
    ref.near(out, ref.linear(one, v, dt))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("T,K", [(1, 1), (1, 8), (3, 7), (64, 8192), (5, 8193), (300, 257), (2, 16384), (3, 20001), (1000, 128), (7, 70000),
                                 (257, 2049), (300, 8200), (260, 24000), (270, 24001), (256, 8192), (40, 8193)])
def test_quantise(fsb, cuda, T, K, dtype):
    torch = cuda
    dt = getattr(torch, dtype)
    x, _ = rows(torch, T, K, dt, T + K, 3.0, 8)
    x.mul_(torch.exp2(torch.arange(T, device="cuda") % 24 - 12.0)[:, None].to(dt))
    if T > 2:
        x[0] = 0
        x[1] = torch.finfo(dt).max
        x[2] = 0
        x[2, K - 1] = 448 * 2.0**-9  # the largest code exactly
    buf = torch.full((T + 1, -(-K // 16) * 16 + 32), 5, dtype=torch.uint8, device="cuda")
    c, s = buf[:T, :K].view(torch.float8_e4m3fn), torch.full((T + 3,), -1.0, device="cuda")
    fsb.fs_quantise_rows(x, c, s[:T])
    want, scale = ref.quantise(x)
    assert torch.equal(s[:T].double(), scale) and bool((s[T:] == -1).all())
    assert torch.equal(c.double(), want)
    assert bool((buf[T:] == 5).all()) and bool((buf[:T, K:] == 5).all())


@pytest.mark.parametrize("T,K", [(6, 200), (6, 5003), (6, 9001), (6, 25003), (300, 4001)])
def test_quantise_not_finite_and_tiny(fsb, cuda, T, K):
    torch = cuda
    for dt in (torch.bfloat16, torch.float16):
        x = rows(torch, T, K, dt, 1)[0]
        x[0, 3], x[1, K - 1], x[2, 0] = float("nan"), float("inf"), float("-inf")
        x[3] = float("inf")
        x[4] = 0
        x[4, 7] = torch.finfo(dt).smallest_normal / (4 if dt == torch.float16 else 1)
        x[5] *= 2.0**-14
        c, s = torch.empty(T, -(-K // 16) * 16, dtype=torch.uint8, device="cuda")[:, :K], torch.empty(T, device="cuda")
        fsb.fs_quantise_rows(x, c, s)
        want, scale = ref.quantise(x)
        assert torch.equal(s.double(), scale)
        got = c.view(torch.float8_e4m3fn).double()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


def test_nothing_to_do(fsb, cuda):
    torch = cuda
    dt = torch.bfloat16
    x, w = torch.randn(4, 32, device="cuda").to(dt), torch.randn(8, 32, device="cuda").to(dt)
    work = fsb.MmWorkspace(4, 32, 8, backward=True)
    fsb.fs_linear(x[:0], w, torch.empty(0, 8, dtype=dt, device="cuda"), workspace=work)
    fsb.fs_linear(x, w[:0], torch.empty(4, 0, dtype=dt, device="cuda"), workspace=work)
    fsb.fs_gated_ff(x[:0], w, w, torch.empty(0, 8, dtype=dt, device="cuda"), workspace=work)
    fsb.fs_quantise_rows(x[:0], torch.empty(0, 32, dtype=torch.uint8, device="cuda"), torch.empty(0, device="cuda"))
    dw = [torch.full((8, 32), 3.0, device="cuda").to(dt) for _ in range(2)]
    fsb.fs_gated_ff_backward(x[:0], w, w, torch.empty(0, 8, dtype=dt, device="cuda"), torch.empty(0, 32, dtype=dt, device="cuda"), *dw,
                             workspace=work)
    assert not dw[0].any() and not dw[1].any()
    dx = torch.full((4, 32), 3.0, device="cuda").to(dt)
    fsb.fs_gated_ff_backward(x, w[:0], w[:0], torch.empty(4, 0, dtype=dt, device="cuda"), dx, w[:0], w[:0], workspace=work)
    assert not dx.any()
    fsb.fs_mm_check(work)


class Layer:
    """A layer's products in a row, as a rank runs them: 8-bit operands, quantised on the way."""

    def __init__(self, torch, fsb, T, hidden, block, seed):
        self.fsb, dt = fsb, torch.bfloat16
        self.x, self.h, self.y = (rows(torch, T, n, dt, seed)[0] for n in (hidden, block, hidden))
        self.cx, self.ch = (torch.empty(T, n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for n in (hidden, block))
        self.sx, self.sh = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        self.w = [codes(torch, n, k, seed + i) for i, (n, k) in enumerate(((block, hidden), (block, hidden), (hidden, block)))]
        self.work = fsb.MmWorkspace(T, max(hidden, block), max(hidden, block))

    def run(self):
        f = self.fsb
        (g, gs), (u, us), (d, ds) = self.w
        f.fs_quantise_rows(self.x, self.cx, self.sx)
        f.fs_gated_ff(self.cx, g, u, self.h, x_scale=self.sx, gate_scale=gs, up_scale=us, workspace=self.work)
        f.fs_quantise_rows(self.h, self.ch, self.sh)
        f.fs_linear(self.ch, d, self.y, residual=self.x, x_scale=self.sh, w_scale=ds, workspace=self.work)

    def check(self):
        (g, gs), (u, us), (d, ds) = self.w
        want, scale = ref.quantise(self.x)
        assert bool((self.cx.double() == want).all()) and bool((self.sx.double() == scale).all())
        ref.near(self.h, ref.gated(self.cx, g, u, self.h.dtype, "silu", self.sx, gs, us))
        want, scale = ref.quantise(self.h)
        assert bool((self.ch.double() == want).all()) and bool((self.sh.double() == scale).all())
        ref.near(self.y, ref.linear(self.ch, d, self.y.dtype, residual=self.x, x_scale=self.sh, w_scale=ds))


@pytest.mark.parametrize("T", [1, 48, 700])
def test_a_layer_in_a_row(fsb, cuda, T):
    """Each call reads what the one before it wrote, with nothing between them."""
    torch = cuda
    layer = Layer(torch, fsb, T, 512, 1408, 1)
    for seed in range(3):
        layer.x.copy_(rows(torch, T, 512, torch.bfloat16, seed)[0])
        layer.run()
        layer.check()
    fsb.fs_mm_check(layer.work)


@pytest.mark.parametrize("T", [1, 48, 700])
def test_a_captured_layer_follows_its_inputs(fsb, cuda, T):
    torch = cuda
    layer = Layer(torch, fsb, T, 512, 1408, 1)
    layer.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run()
        layer.run()
    for seed in range(3):
        layer.x.copy_(rows(torch, T, 512, torch.bfloat16, 10 + seed)[0])
        for w, s in layer.w:
            w.view(torch.uint8).copy_(w.view(torch.uint8).roll(1, 0))
            s.copy_(s.roll(1))
        graph.replay()
        layer.check()
    fsb.fs_mm_check(layer.work)


def test_results_repeat(fsb, cuda):
    """The same inputs give the same bits, beside other work of the GPU too."""
    torch = cuda
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    layers = [Layer(torch, fsb, T, 640, 1000 // 16 * 16, 2) for T in (5, 300)]
    want = []
    for layer in layers:
        layer.run()
        want.append(layer.y.clone())
    torch.cuda.synchronize()
    for _ in range(10):
        for layer, stream in zip(layers, (a, b)):
            with torch.cuda.stream(stream):
                layer.y.zero_()
                layer.run()
        torch.cuda.synchronize()
        for layer, y in zip(layers, want):
            assert torch.equal(layer.y, y)
    x, w, _, _, dt = operands(torch, "bfloat16", 300, 200, 500, 2, 1)
    dy = rows(torch, 300, 500, dt, 3)[0]
    work = fsb.MmWorkspace(300, 200, 500, backward=True)
    grads = []
    for _ in range(3):
        outs = [rows(torch, n, 200, dt, 0)[0] for n in (300, 500, 500)]
        fsb.fs_gated_ff_backward(x, *w, dy, *outs, workspace=work)
        grads.append(outs)
    assert all(torch.equal(p, q) for other in grads[1:] for p, q in zip(grads[0], other))


def test_a_backward_pass_captured(fsb, cuda):
    torch = cuda
    T, K, N = 200, 136, 300
    x, w, _, _, dt = operands(torch, "bfloat16", T, K, N, 2, 1)
    dy = rows(torch, T, N, dt, 3)[0]
    outs = [rows(torch, n, K, dt, 0)[0] for n in (T, N, N)]
    work = fsb.MmWorkspace(T, K, N, backward=True)
    call = lambda: fsb.fs_gated_ff_backward(x, *w, dy, *outs, workspace=work)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(2):
        x.copy_(rows(torch, T, K, dt, 20 + seed)[0])
        dy.copy_(rows(torch, T, N, dt, 30 + seed)[0])
        graph.replay()
        for o, want in zip(outs, ref.gated_backward(x, *w, dy)):
            ref.near(o, want)


def test_offsets_beyond_32_bits(fsb, cuda):
    """Rows that begin more than 2^31 elements behind the first."""
    torch = cuda
    T, K, N, ld, dt = 6, 96, 40, 1 << 29, torch.bfloat16
    big = torch.empty(T * ld, dtype=dt, device="cuda")
    view = lambda at, width: big.as_strided((T, width), (ld, 1), at)  # noqa: E731
    x, y, r = view(64, K), view(1024, N), view(4096, N)
    x.copy_(rows(torch, T, K, dt, 1)[0])
    r.copy_(rows(torch, T, N, dt, 2)[0])
    w = rows(torch, N, K, dt, 3)[0]
    fsb.fs_linear(x, w, y, residual=r, workspace=fsb.MmWorkspace(T, K, N))
    ref.near(y, ref.linear(x, w, dt, residual=r))
    c, s = big.view(torch.uint8).as_strided((T, K), (2 * ld, 1), 16384), torch.empty(T, device="cuda")
    fsb.fs_quantise_rows(x, c, s)
    assert torch.equal(c.view(torch.float8_e4m3fn).double(), ref.quantise(x)[0])


@pytest.mark.parametrize("T", [90, 2500])
@pytest.mark.parametrize("kind", KINDS[:2])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "gelu_tanh"])
def test_activations_over_their_range(fsb, cuda, act, kind, T):
    """One term a sum, so that z is what x holds and the activation's own bound is all there is but the rounding."""
    torch = cuda
    dt = getattr(torch, kind)
    z = torch.cat([torch.linspace(-16, 16, T // 2), torch.logspace(-7, 4, T - T // 2 - 2) * (1 - 2 * (torch.arange(T - T // 2 - 2) % 2)), torch.zeros(2)])
    x, w = torch.zeros(T, 24, dtype=dt, device="cuda"), torch.zeros(40, 24, dtype=dt, device="cuda")
    x[:, 3], w[:, 3] = z.cuda().to(dt), 1
    y, work = torch.empty(T, 40, dtype=dt, device="cuda"), fsb.MmWorkspace(T, 24, 40)
    fsb.fs_linear(x, w, y, activation=act, workspace=work)
    at = x[:, 3:4].double().expand(T, 40)
    want = ref._rounded(*ref._act(at, torch.zeros_like(at), act), dt)
    ref.near(y, want)
    fsb.fs_gated_ff(x, w, w, y, activation=act, workspace=work)  # act(z) z, where that is in the type's range
    a, e = ref._act(at, torch.zeros_like(at), act)
    a, e = a * at, e * at.abs() + ref.U * (a * at).abs()
    inside = a.abs() < 60000
    assert bool(inside.any())
    got, (v, bound) = y, ref._rounded(a, e, dt)
    ref.near(got[inside], (v[inside], bound[inside]))


@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "gelu_tanh", "none"])
@pytest.mark.parametrize("size", [1e3, 1e19, 1e24])
def test_gradients_of_large_gates(fsb, cuda, act, size):
    """A gate's values far out, where squares and cubes pass a float's range: the slope is 1 or 0 there (none: 1)."""
    torch = cuda
    T, K, N = 40, 8, 24
    dt = torch.bfloat16
    half = size**0.5
    x, wg, wu, dy = (torch.zeros(n, m, dtype=dt, device="cuda") for n, m in ((T, K), (N, K), (N, K), (T, N)))
    x[:, 0], wg[:, 0], wu[:, 0], dy[:] = half, half, 1 / half, 1 / size
    wg[::2, 0] = -half
    outs = [torch.full((n, K), float("nan"), dtype=dt, device="cuda") for n in (T, N, N)]
    fsb.fs_gated_ff_backward(x, wg, wu, dy, *outs, activation=act, workspace=fsb.MmWorkspace(T, K, N, backward=True))
    on = torch.tensor([1.0 if act == "none" or n % 2 else 0.0 for n in range(N)], device="cuda", dtype=torch.float64)
    sign = torch.tensor([1.0 if n % 2 else -1.0 for n in range(N)], device="cuda", dtype=torch.float64)
    # dg = on / size, du = on sign: dx = sum on sign (half / size + 1 / half), dw_gate = T on half / size, dw_up = T on sign half
    want = [(on * sign).sum() * 2 / half, T * on * half / size, T * on * sign * half]
    for o, w in zip(outs, want):
        # half a step, 2^-8, each: half twice (x and w_gate) and once in dx's or dw's other factor, 1 / half and 1 / size or what stands for
        # them, dg or du, the result: six in every product, and their products with each other
        bound = 6.2 * 2.0**-8 * (w.abs() if w.dim() else 2 * N / half)
        assert bool(((o[:, 0].double() - w).abs() <= bound).all()) and not bool(o[:, 1:].any())


@pytest.mark.parametrize("T,K", [(256, 2048), (257, 2048), (258, 1501), (2048, 130), (2049, 2048), (2100, 777), (1536, 2050), (1537, 2049), (1600, 6144),
                                 (1600, 6145), (2500, 8192)])
def test_quantise_many_rows(fsb, cuda, T, K):
    """Around the sizes where rows change hands between registers, warps and shared memory, with values that are not finite."""
    torch = cuda
    x, _ = rows(torch, T, K, torch.bfloat16, T + K, 3.0, 8)
    x.mul_(torch.exp2(torch.arange(T, device="cuda") % 40 - 20.0)[:, None].to(x.dtype))
    x[1, K - 1], x[T // 2, 0], x[T - 1, K // 2], x[2] = float("inf"), float("nan"), float("-inf"), 0
    buf = torch.full((T + 1, -(-K // 16) * 16 + 16), 5, dtype=torch.uint8, device="cuda")
    c, s = buf[:T, :K].view(torch.float8_e4m3fn), torch.full((T + 3,), -1.0, device="cuda")
    fsb.fs_quantise_rows(x, c, s[:T])
    want, scale = ref.quantise(x)
    assert torch.equal(s[:T].double(), scale) and bool((s[T:] == -1).all())
    got = c.double()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())
    assert bool((buf[T:] == 5).all()) and bool((buf[:T, K:] == 5).all())
