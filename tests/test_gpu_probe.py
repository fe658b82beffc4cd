"""The probe's times are the device's, and its bounds, of probes that were run, are ones a model takes."""

import json
import time

import numpy as np
import pytest

from paper_2608_19659_gb300 import probe, workloads

pytestmark = pytest.mark.gpu


def test_the_host_is_not_timed(fsb, cuda, monkeypatch):
    """Calls that keep the host for 3 ms each: a layer of one short request takes microseconds all the same."""
    slow = fsb.fs_kv_append

    def append(*args, **kw):
        time.sleep(3e-3)
        slow(*args, **kw)

    monkeypatch.setattr(fsb, "fs_kv_append", append)
    s = probe.RankStep(probe.Decoder(context=300, output=16), 8, 1)
    per_layer = s.seconds(2) / 2
    assert 1e-6 < per_layer < 3e-4


def test_times_grow_with_the_work(fsb, cuda):
    """256 times the requests over eight times the context: the device's time per layer is several times as long."""
    small = probe.RankStep(probe.Decoder(context=500, output=64), 8, 1).seconds(4)
    large = probe.RankStep(probe.Decoder(context=4000, output=64), 8, 256).seconds(4)
    assert 0 < 3 * small < large


def test_real_probes_of_long_generations_tighten_the_grid(fsb, cuda):
    w = workloads.make_workload(1)
    old = bounds = (w.cap_lo, w.cap_hi, w.tail_lo, w.tail_hi)
    d = probe.Decoder(context=2048, output=32768)
    for tp in (4, 8):
        for b in (0, 2):
            p = probe.probe_cell(d, tp, 1 << b)
            # (attention over 18000 tokens on average, 60 layers: no replica does a step in 60 us)
            assert p.step_seconds > 60e-6 and p.cap_hi == pytest.approx((1 << b) / p.tail_lo)
            bounds = probe.tighten(*bounds, 0, tp, b, p)
    assert np.array_equal(bounds[0], old[0]) and np.array_equal(bounds[3], old[3])
    assert (bounds[1] <= old[1]).all() and (bounds[2] >= old[2]).all()
    assert (bounds[1] < old[1]).any() and (bounds[2] > old[2]).any()
    with fsb.fs_load_model(*old, w.slo, w.demand * np.float32(3), w.G, w.K, w.B) as m:
        before = fsb.fs_solve_bounds(m)[2]
        fsb.fs_update_bounds(m, *bounds)
        assert fsb.fs_solve_bounds(m)[2] <= before


def test_the_command(fsb, cuda, capsys):
    probe.main(["--context", "200", "--output", "32", "--layers", "2"])
    r = json.loads(capsys.readouterr().out)
    assert len(r["probes"]) == 4 * 8 and r["gamma_after"] <= r["gamma_before"] and r["bounds_moved"] >= 0
    assert all(p["step_seconds"] > 0 and p["prompt_seconds"] > 0 for p in r["probes"])


@pytest.mark.parametrize("context", [1, 2, 300])
def test_a_prompt_is_as_long_as_the_context(fsb, cuda, monkeypatch, context):
    """A prompt of one token too: not a step in the middle of the generation."""
    seen = []

    class Step(probe.RankStep):
        def seconds(self, *args):
            seen.append((self.batch.tokens, self.batch.tensors[1].tolist()))
            return 1e-5

    monkeypatch.setattr(probe, "RankStep", Step)
    probe.probe_cell(probe.Decoder(context=context, output=64), 8, 2)
    assert seen == [(2, [context + 32] * 2), (context, [context])]
