"""Tiles of the widths and numbers that large calls take: every slot of a ring and both sums of a pair again and again."""

import pytest

import mm_plans
import mm_reference as ref
from test_gpu_mm import operands, rows, untouched

pytestmark = pytest.mark.gpu


def sms(torch):
    return torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("kind", ["bfloat16", "float16", "e4m3"])
@pytest.mark.parametrize("T,K,N,act", [(4100, 1100, 5130, "silu"), (4200, 2300, 5200, "gelu_tanh")])
def test_products_in_whole_tiles(fsb, cuda, T, K, N, act, kind):
    """256 columns a tile, more tiles than pairs, more blocks of a sum than the ring has stages (6)."""
    torch, eight = cuda, kind == "e4m3"
    for gated in (False, True):
        tile, tiles = mm_plans.wide(T, K, N, eight, gated, sms(torch))
        assert tile == 256 and tiles > sms(torch) // 2 and mm_plans.blocks(K, eight) > 6
    x, w, xs, ws, dt = operands(torch, kind, T, K, N, 2, 5, 16)
    y, buf = rows(torch, T, N, dt, 0, extra=8)
    work = fsb.MmWorkspace(T, K, N)
    b, r = rows(torch, 1, N, dt, 7)[0][0], rows(torch, T, N, dt, 8)[0]
    fsb.fs_linear(x, w[0], y, bias=b, residual=r, activation=act, x_scale=xs, w_scale=ws[0], workspace=work)
    ref.near(y, ref.linear(x, w[0], dt, b, r, act, xs, ws[0]))
    untouched(torch, buf, T, N)
    fsb.fs_linear(x, w[1], y, x_scale=xs, w_scale=ws[1], workspace=work)
    ref.near(y, ref.linear(x, w[1], dt, x_scale=xs, w_scale=ws[1]))
    fsb.fs_gated_ff(x, *w, y, activation=act, x_scale=xs, gate_scale=ws[0], up_scale=ws[1], workspace=work)
    ref.near(y, ref.gated(x, *w, dt, act, xs, *ws))
    untouched(torch, buf, T, N)
    fsb.fs_mm_check(work)


WIDTHS = {  # by rows, terms and columns: narrower tiles, several a pair
    224: (2600, 1100, 4200), 192: (1500, 700, 4200), 160: (2304, 1100, 2500), 128: (1500, 150, 3200), 96: (2000, 70, 1800)}


@pytest.mark.parametrize("width", WIDTHS)
def test_widths_in_between(fsb, cuda, width):
    torch = cuda
    T, K, N = WIDTHS[width]
    tile, tiles = mm_plans.wide(T, K, N, False, False, sms(torch))
    assert tile == width and tiles > sms(torch) // 2
    x, (w,), _, _, dt = operands(torch, "bfloat16", T, K, N, 1, 5, 16)
    y, buf = rows(torch, T, N, dt, 0, extra=8)
    r, work = rows(torch, T, N, dt, 8)[0], fsb.MmWorkspace(T, K, N)
    fsb.fs_linear(x, w, y, residual=r, activation="relu", workspace=work)
    ref.near(y, ref.linear(x, w, dt, None, r, "relu"))
    untouched(torch, buf, T, N)
    fsb.fs_mm_check(work)


# rows, in, out; the gradients' tile, whether dW is ahead of dx, whether pairs lead, several rounds; the width of dg's and du's tiles
BACK = [
    (3000, 2600, 2200, 256, False, False, False, 256),
    (2600, 1500, 4200, 256, False, True, True, 256),
    (1362, 704, 3848, 128, False, True, True, 128),
    (5000, 1300, 900, 128, True, False, False, 192),
    (4000, 1000, 300, 128, True, True, True, 192),
    (2310, 520, 2500, 128, False, True, True, 256)]


@pytest.mark.parametrize("kind,act", [("bfloat16", "silu"), ("float16", "gelu")])
@pytest.mark.parametrize("T,K,N,tile,dw_first,leads,rounds,back", BACK)
def test_gradients(fsb, cuda, T, K, N, tile, dw_first, leads, rounds, back, kind, act):
    """More tiles than pairs in every order; both sums of a pair under dg and du."""
    torch = cuda
    p = mm_plans.grad(T, K, N, sms(torch))
    assert (p.tile, p.dw_first, p.lead > 0) == (tile, dw_first, leads) and p.tiles > sms(torch) // 2 and (not rounds or p.rounds > 1)
    width, tiles = mm_plans.wide(T, K, N, False, True, sms(torch))
    assert width == back and (width < 256 or tiles > 2 * (sms(torch) // 2))
    x, w, _, _, dt = operands(torch, kind, T, K, N, 2, 1, 8)
    dy = rows(torch, T, N, dt, 99, 0.5)[0]
    outs = [rows(torch, n, K, dt, 0, extra=8 * i) for i, n in enumerate((T, N, N))]
    work = fsb.MmWorkspace(T, K, N, backward=True)
    fsb.fs_gated_ff_backward(x, *w, dy, *(o for o, _ in outs), activation=act, workspace=work)
    for (o, buf), n, want in zip(outs, (T, N, N), ref.gated_backward(x, *w, dy, act)):
        ref.near(o, want)
        untouched(torch, buf, n, K)
    fsb.fs_mm_check(work)


@pytest.mark.parametrize("seed", range(12))
def test_gradients_of_sizes_at_random(fsb, cuda, seed):
    torch = cuda
    import math
    import random

    rng = random.Random(seed)
    size = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi))))  # noqa: E731
    for _ in range(3):
        T, K, N = size(1, 3000), size(1, 2000), size(1, 3000)
        kind, act = rng.choice(("bfloat16", "float16")), rng.choice(list(fsb.ACTIVATIONS))
        x, w, _, _, dt = operands(torch, kind, T, K, N, 2, seed, 8)
        dy = rows(torch, T, N, dt, 99, 0.5)[0]
        outs = [rows(torch, n, K, dt, 0, extra=8 * i) for i, n in enumerate((T, N, N))]
        work = fsb.MmWorkspace(T, K, N, backward=True)
        fsb.fs_gated_ff_backward(x, *w, dy, *(o for o, _ in outs), activation=act, workspace=work)
        for (o, buf), n, want in zip(outs, (T, N, N), ref.gated_backward(x, *w, dy, act)):
            ref.near(o, want)
            untouched(torch, buf, n, K)
        fsb.fs_mm_check(work)
