"""Bounds from a rank's attention: what they do to a model's intervals, and one real probe."""

import numpy as np
import pytest

from paper_2608_19659_gb300 import probe, workloads


def test_heads_of_a_rank():
    d = probe.Decoder()
    assert [probe.rank_heads(d, tp) for tp in (1, 2, 4, 8)] == [(64, 8), (32, 4), (16, 2), (8, 1)]
    assert probe.rank_heads(probe.Decoder(kv_heads=2), 8) == (8, 1)
    for bad in (0, 3, 128):
        with pytest.raises(ValueError):
            probe.rank_heads(d, bad)


def test_tighten_moves_only_the_optimistic_ends_of_one_cell():
    w = workloads.make_workload(1)
    b = (w.cap_lo, w.cap_hi, w.tail_lo, w.tail_hi)
    mid_c, mid_l = (float(x[1, 2, 3] + y[1, 2, 3]) / 2 for x, y in ((b[0], b[1]), (b[2], b[3])))
    for cap, tail in ((mid_c, mid_l), (0.0, 1e9), (1e9, 0.0)):
        new = probe.tighten(*b, 1, 4, 3, probe.Probe(4, 8, 0.0, 0.0, cap, tail))
        assert new[0][1, 2, 3] == b[0][1, 2, 3] and new[3][1, 2, 3] == b[3][1, 2, 3]
        assert new[1][1, 2, 3] == np.float32(np.clip(cap, b[0][1, 2, 3], b[1][1, 2, 3]))
        assert new[2][1, 2, 3] == np.float32(np.clip(tail, b[2][1, 2, 3], b[3][1, 2, 3]))
        for x, y in zip(new, b):
            z = x.copy()
            z[1, 2, 3] = y[1, 2, 3]
            assert np.array_equal(z, y)


@pytest.mark.gpu
def test_a_probe_tightens_a_model(fsb, cuda):
    """A rank's step over real pages: times are positive and grow with the requests, the outputs are those of
    attention over what was appended, and the model takes the tightened bounds (Gamma_t does not grow)."""
    torch = cuda
    d = probe.Decoder(layers=2, context=500, output=64, page=32)
    one, many = probe.probe_cell(d, 8, 1), probe.probe_cell(d, 8, 256)
    assert 0 < one.step_seconds < many.step_seconds and one.prompt_seconds > 0
    assert one.cap_hi == pytest.approx(1 / one.tail_lo) and many.cap_hi == pytest.approx(256 / many.tail_lo)

    s = probe.RankStep(d, 4, 3)
    s.layer()
    fsb.fs_kv_check(s.work)
    k, v, ks, vs = s.cache.tensors
    table, length, _ = s.batch.tensors
    L, H = int(length[0]), k.shape[1]
    for b in range(3):
        at = table[b].long()
        kk, vv = ((c[at].view(torch.float8_e4m3fn).double() * sc[at].double()[..., None, None]).transpose(1, 2).reshape(-1, H, d.dim)[:L]
                  for c, sc in ((k, ks), (v, vs)))
        q = s.q[b].double().view(H, -1, d.dim)
        p = torch.softmax(torch.einsum("hgd,lhd->hgl", q, kk) * s.scale, -1)
        want = torch.einsum("hgl,lhd->hgd", p, vv).reshape(-1, d.dim)
        mag = torch.einsum("hgl,lhd->hgd", p, vv.abs()).reshape(-1, d.dim)
        # weights to 2^-11, scores, and the result's rounding
        assert bool(((s.out[b].double() - want).abs() <= 2.0**-9 * mag + 2.0**-8 * want.abs()).all())

    w = workloads.make_workload(1)
    bounds = (w.cap_lo, w.cap_hi, w.tail_lo, w.tail_hi)
    with fsb.fs_load_model(*bounds, w.slo, w.demand * np.float32(3), w.G, w.K, w.B) as m:
        before = fsb.fs_solve_bounds(m)[2]
        for b in range(w.B):
            bounds = probe.tighten(*bounds, 0, 8, b, probe.Probe(8, 1, 0.1, 0.1, 0.05, 40.0))
        fsb.fs_update_bounds(m, *bounds)
        assert fsb.fs_solve_bounds(m)[2] <= before
