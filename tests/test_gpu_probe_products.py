"""A rank's whole layer in the probe: every call's result against its definition, and what the times bound."""

import json

import pytest

import mm_reference as ref
from paper_2608_19659_gb300 import probe

pytestmark = pytest.mark.gpu

SMALL = probe.Decoder(layers=2, q_heads=16, kv_heads=4, context=200, output=40, page=32, hidden=1024, block=1792)


@pytest.mark.parametrize("tp,requests,new", [(1, 3, 1), (4, 5, 1), (2, 1, 200), (4, 2, 150)])
def test_a_layer(fsb, cuda, tp, requests, new):
    torch = cuda
    d = SMALL
    s = probe.RankStep(d, tp, requests, new=new, products=True)
    p = s.products
    assert len(p.sets) * sum(w.numel() for w, _ in p.sets[0]) >= 2 * torch.cuda.get_device_properties(0).L2_cache_size
    p.sets = p.sets[:3]  # (more are for the times)
    for layer in (1, 2, 0):
        s.layer()
        s.check()
        assert p.layer == layer
        (wq, sq), (wo, so), (wg, sg), (wu, su), (wd, sd) = p.sets[layer]
        for rows, codes, scale in zip((p.x, p.attended, p.mid, p.inner), p.codes, p.scales):
            want, sc = ref.quantise(rows)
            assert torch.equal(codes.double(), want) and torch.equal(scale.double(), sc)
        hq, hk = probe.rank_heads(d, tp)
        kv = hq * d.dim  # (queries have been rotated since)
        want, e = ref.linear(p.codes[0], wq, torch.bfloat16, p.bias, x_scale=p.scales[0], w_scale=sq)
        ref.near(p.qkv[:, kv:], (want[:, kv:], e[:, kv:]))
        pos = (s.batch.tensors[1][:, None] - new + torch.arange(new, device="cuda")).reshape(-1)
        turned = want[:, :kv].view(-1, hq, d.dim)
        a, b = turned.split(d.dim // 2, -1)
        c, si = s.cos[pos].double()[:, None], s.sin[pos].double()[:, None]
        off = (s.q.double() - torch.cat((a * c - b * si, b * c + a * si), -1)).abs()
        near = e[:, :kv].view(-1, hq, d.dim)
        near = torch.cat([near.split(d.dim // 2, -1)[0] + near.split(d.dim // 2, -1)[1]] * 2, -1)
        # (the product's rounding on both of a pair, the rotation's own)
        assert bool((off <= near + 2.0**-7 * (turned.abs() + torch.cat((b, a), -1).abs())).all())
        ref.near(p.mid, ref.linear(p.codes[1], wo, torch.bfloat16, residual=p.x, x_scale=p.scales[1], w_scale=so))
        ref.near(p.inner, ref.gated(p.codes[2], wg, wu, torch.bfloat16, "silu", p.scales[2], sg, su))
        ref.near(p.y, ref.linear(p.codes[3], wd, torch.bfloat16, residual=p.mid, x_scale=p.scales[3], w_scale=sd))


def test_a_block_that_does_not_split(fsb, cuda):
    with pytest.raises(ValueError, match="gated block"):
        probe.RankStep(probe.Decoder(q_heads=16, kv_heads=4, context=20, output=4, hidden=256, block=1001), 2, 1, products=True)


def test_layers_take_longer_than_their_attention(fsb, cuda):
    """A rank of TP 8 reads 62.9 MB of weights a layer (1280, 1024 and three times 1792 rows of 8192 codes), 7 us at
    9 TB/s, which no GPU's memory here gives: its step takes at least that much longer."""
    d = probe.Decoder(context=300, output=16)
    alone, layer = (probe.RankStep(d, 8, 4, products=p).seconds(4) / 4 for p in (False, True))
    assert layer > alone + 7e-6


def test_the_command(fsb, cuda, capsys):
    probe.main(["--context", "64", "--output", "16", "--layers", "2", "--products"])
    r = json.loads(capsys.readouterr().out)
    assert r["products"] and len(r["probes"]) == 4 * 8 and r["gamma_after"] <= r["gamma_before"]
