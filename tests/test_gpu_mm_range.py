"""Products whose values on the way are far larger or smaller than what comes out."""

import pytest

import mm_reference as ref

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
