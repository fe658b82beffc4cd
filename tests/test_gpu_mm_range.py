"""Products whose values on the way are far larger or smaller than what comes out."""

import pytest

import mm_reference as ref
from test_gpu_mm import operands, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("T", [40, 600])
def test_gradients_where_dy_u_passes_a_floats_range(fsb, cuda, act, T):
    """dy u = 1e40: with a gate far out on the closed side the slope is 0 and so are all gradients; with one nearer it brings
    dg back into range."""
    torch = cuda
    K, N, dt = 8, 24, torch.bfloat16
    x, wg, wu = (torch.zeros(n, K, dtype=dt, device="cuda") for n in (T, N, N))
    dy = torch.full((T, N), 1e20, device="cuda").to(dt)
    work = fsb.MmWorkspace(T, K, N, backward=True)
    outs = [torch.full((n, K), 7.0, dtype=dt, device="cuda") for n in (T, N, N)]
    x[:, 0], wg[:, 0], wu[:, 0] = 1.0, -1000.0, 1e20
    fsb.fs_gated_ff_backward(x, wg, wu, dy, *outs, activation=act, workspace=work)
    assert all(not bool(o.any()) for o in outs)
    # SiLU at -17 to -28.5: slopes of 7e-7 to 1e-11, GELU at -5 to -7.3: 8e-6 to 8e-12
    low, step = {"relu": (17, 0.5), "silu": (17, 0.5)}.get(act, (5, 0.1))
    wg[:, 0] = -(low + step * torch.arange(N, device="cuda")).to(dt)
    fsb.fs_gated_ff_backward(x, wg, wu, dy, *outs, activation=act, workspace=work)
    for o, want in zip(outs, ref.gated_backward(x, wg, wu, dy, act)):
        assert bool(o.isfinite().all())
        ref.near(o, want)
    fsb.fs_mm_check(work)


SCALES = [(2.0**119, 2.0**-126), (2.0**-126, 2.0**119), (2.0**127, 3e-38), (3e-38, 2.0**127), (2.0**-149, 2.0**127), (3.0, 2.0**-120), (1e-30, 1e30),
          (2.0**60, 2.0**-60), (2.0**-60, 2.0**60), (2.0**100, 2.0**-20), (2.0**-100, 2.0**-40), (0.0, 2.0**127)]


@pytest.mark.parametrize("T,K,N", [(3, 300, 200), (100, 5000, 90), (700, 300, 1000)])
@pytest.mark.parametrize("a,b", SCALES)
def test_scales_far_apart(fsb, cuda, T, K, N, a, b):
    """Any finite scales: a row's may carry a sum out of a float's range that a column's brings back, in some rows and columns
    but not in others."""
    torch = cuda
    x, (w, u), xs, (ws, us), dt = operands(torch, "e4m3", T, K, N, 2, 1, 16)
    xs[::2], ws[::3], us[::5] = a, b, b
    xs[1::4], ws[1::3] = -xs[1::4], -ws[1::3]
    y, work = rows(torch, T, N, dt, 0)[0], fsb.MmWorkspace(T, K, N)
    fsb.fs_linear(x, w, y, x_scale=xs, w_scale=ws, workspace=work)
    within(torch, y, *ref.linear(x, w, dt, x_scale=xs, w_scale=ws))
    fsb.fs_gated_ff(x, w, u, y, activation="relu", x_scale=xs, gate_scale=ws, up_scale=us, workspace=work)
    # (gate and up are floats: where both are in a float's range)
    z = [ref.linear(x, t, dt, x_scale=xs, w_scale=s)[0].abs() for t, s in ((w, ws), (u, us))]
    inside = torch.stack([(t == 0) | (t > 2.0**-120) & (t < 2.0**127) for t in z]).all(0)
    assert bool(inside.any())
    want, e = ref.gated(x, w, u, dt, "relu", xs, ws, us)
    within(torch, y[inside], want[inside], e[inside])
    fsb.fs_mm_check(work)


def within(torch, y, want, e):
    """Within the bounds; infinite where the value is beyond the type's range for sure, and only where it may be."""
    top = torch.finfo(y.dtype).max
    surely, maybe = want.abs() - e > top * (1 + 2.0**-8), want.abs() + e > top
    assert not bool(y.isnan().any())
    assert bool((y[surely] == torch.where(want[surely] > 0, float("inf"), float("-inf")).to(y.dtype)).all())
    assert bool((maybe | y.isfinite()).all())
    ref.near(y[~maybe], (want[~maybe], e[~maybe]))


@pytest.mark.parametrize("T", [40, 700])
def test_halves_bound_what_the_gradients_are_made_of(fsb, cuda, T):
    """dg and du beyond 65504: rows that they go into are not finite, all others are right; a smaller dy brings all of them
    back."""
    torch = cuda
    K, N, dt = 48, 320, torch.float16
    x, (wg, wu), _, _, _ = operands(torch, "float16", T, K, N, 2, 3)
    wu *= 64
    dy = rows(torch, T, N, dt, 4, 100.0)[0]
    dy[::3] *= 60
    dy[:, ::5] /= 64
    outs = [rows(torch, n, K, dt, 0)[0] for n in (T, N, N)]
    work = fsb.MmWorkspace(T, K, N, backward=True)
    fsb.fs_gated_ff_backward(x, wg, wu, dy, *outs, workspace=work)
    g, u = x.double() @ wg.double().T, x.double() @ wu.double().T
    dg, du = (dy.double() * u * ref.slope(g, "silu")).abs(), (dy.double() * ref.act(g, "silu")).abs()
    over = lambda v, dim, at: (v > at).any(dim)  # noqa: E731
    want = ref.gated_backward(x, wg, wu, dy)
    spans = [(torch.maximum(dg, du), 1), (dg, 0), (du, 0)]
    for o, w, (v, dim) in zip(outs, want, spans):
        beyond, inside = over(v, dim, 65504 * 1.001), ~over(v, dim, 65504 * 0.999)
        assert not bool(o[beyond].isfinite().any())
        within(torch, o[inside], w[0][inside], w[1][inside])
    assert bool(over(dg, 1, 65504 * 1.001).any()) and not bool(over(dg, 0, 65504 * 0.999).all())
    small = dy / 2**8  # (exact but for halves under 2^-6)
    fsb.fs_gated_ff_backward(x, wg, wu, small, *outs, workspace=work)
    for o, w in zip(outs, ref.gated_backward(x, wg, wu, small)):
        within(torch, o, *w)  # (dw sums 700 rows: some results are beyond the range themselves)
    assert bool(((want[0][0].abs() < 60000) & over(dg, 1, 65504 * 1.001)[:, None]).any())  # (what had been lost)
    fsb.fs_mm_check(work)
