"""Gradients of few rows or columns: dg and du in two terms, so that results are off by little more than their own rounding."""

import pytest

import mm_reference as ref
from test_gpu_mm import operands, rows, untouched

pytestmark = pytest.mark.gpu

ROWS, COLUMNS = 64, 64  # up to which dW, and dx, are made of two terms


def bounds(torch, x, wg, wu, dy, act, two):
    """As mm_reference.gated_backward, with dg and du in two terms for the results that `two` says: a value's rounding leaves half a step at
    most, which is rounded to half a step of its own: the square of one's relative error, or half of the subnormals' step."""
    dtype = x.dtype
    (g, eg), (u, eu) = ref._gate_and_up(x, wg, wu)
    x, wg, wu, dy = (t.double() for t in (x, wg, wu, dy))
    a, ea = ref._act(g, eg, act)
    s = ref.slope(g, act)
    if act == "relu":
        es = (g.abs() <= eg).double()
    else:
        es = 1.2 * eg + ref._own(g) * (1 + g.abs()) * torch.clamp(s.abs() + 0.2, max=1.2)
    dg, du = dy * u * s, dy * a
    eg, eu = dy.abs() * (eu * (s.abs() + es) + u.abs() * es) + 2 * ref.U * dg.abs(), dy.abs() * ea + ref.U * du.abs()

    def product(pairs, n, two):
        y = sum(p @ q for p, _, q in pairs)
        at = lambda p, e: e + (ref.HALF[dtype] ** 2 if two else ref.HALF[dtype]) * (p.abs() + e) + ref.TINY[dtype]  # noqa: E731
        e = sum(at(p, e) @ q.abs() for p, e, q in pairs) + (n + 32) * ref.U * sum((p.abs() + at(p, e)) @ q.abs() * 1.01 for p, e, q in pairs)
        return ref._rounded(y, e, dtype)

    # (two terms: twice the additions; the second term's are under 2^-8 of the first's, the factor 1.01)
    return [product([(dg, eg, wg), (du, eu, wu)], 4 * g.shape[1], two[0]), product([(dg.T, eg.T, x)], 2 * x.shape[0], two[1]),
            product([(du.T, eu.T, x)], 2 * x.shape[0], two[1])]


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("T,K,N", [(1, 4096, 16), (1, 64, 2000), (3, 1000, 16), (5, 377, 1088), (45, 64, 16), (77, 520, 1003), (200, 300, 64), (300, 130, 65),
                                   (ROWS, 200, 500), (ROWS + 1, 200, 500), (1, 1, 1), (64, 2050, 7), (500, 700, COLUMNS), (2300, 260, 40), (4500, 130, 60)])
def test_two_terms(fsb, cuda, T, K, N, act, kind):
    torch = cuda
    x, w, _, _, dt = operands(torch, kind, T, K, N, 2, T + K + N, 8)
    dy = rows(torch, T, N, dt, 99, 0.5)[0]
    outs = [rows(torch, n, K, dt, 0, extra=8 * i) for i, n in enumerate((T, N, N))]
    work = fsb.MmWorkspace(T, K, N, backward=True)
    fsb.fs_gated_ff_backward(x, *w, dy, *(o for o, _ in outs), activation=act, workspace=work)
    for (o, buf), n, want in zip(outs, (T, N, N), bounds(torch, x, *w, dy, act, (N <= COLUMNS, T <= ROWS))):
        ref.near(o, want)
        untouched(torch, buf, n, K)
    fsb.fs_mm_check(work)


def test_a_workspace_serves_all_smaller_sizes(fsb, cuda):
    """One with and one without second terms, in the memory of the largest, one after the other."""
    torch = cuda
    sizes = [(ROWS + 1, 200, 600), (ROWS, 200, 600), (3, 200, 600), (ROWS + 1, 200, COLUMNS), (ROWS + 1, 64, COLUMNS + 1), (1, 8, 1)]
    work = fsb.MmWorkspace(ROWS + 1, 200, 600, backward=True)
    for T, K, N in sizes:
        x, w, _, _, dt = operands(torch, "bfloat16", T, K, N, 2, T + K + N, 8)
        dy = rows(torch, T, N, dt, 99, 0.5)[0]
        outs = [rows(torch, n, K, dt, 0)[0] for n in (T, N, N)]
        fsb.fs_gated_ff_backward(x, *w, dy, *outs, workspace=work)
        for o, want in zip(outs, bounds(torch, x, *w, dy, "silu", (N <= COLUMNS, T <= ROWS))):
            ref.near(o, want)
    fsb.fs_mm_check(work)


def test_infinite_terms_are_not_finite(fsb, cuda):
    """What a value beyond a half's range leaves is no finite number either."""
    torch = cuda
    T, K, N, dt = 20, 48, 100, torch.float16
    x, (wg, wu), _, _, _ = operands(torch, "float16", T, K, N, 2, 3)
    wu *= 64
    dy = rows(torch, T, N, dt, 4, 100.0)[0]
    dy[3] = 20000.0
    outs = [rows(torch, n, K, dt, 0)[0] for n in (T, N, N)]
    fsb.fs_gated_ff_backward(x, wg, wu, dy, *outs, workspace=fsb.MmWorkspace(T, K, N, backward=True))
    dg = (dy.double() * (x.double() @ wu.double().T) * ref.slope(x.double() @ wg.double().T, "silu")).abs()
    assert bool((dg[3] > 66000).any()) and not bool(outs[0][3].isfinite().any())
    assert not bool(outs[1][dg[3] > 66000].isfinite().any())
