"""Batches whose contents change between replays of a captured call: every row of a sequence is computed, rows that
are no sequence's are reported."""

import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu


def setup(torch, fsb, new, batch, heads, group, dim, page, length, dtype=None):
    rng = np.random.default_rng(41)
    d = ref.make(rng, [(length, new)] * batch, heads, dim, page)
    cache = fsb.KvCache(*(torch.from_numpy(d[n]).cuda() for n in ("k", "v", "k_scale", "v_scale")))
    T = batch * new
    b = fsb.KvBatch(torch.from_numpy(d["table"]).cuda(), torch.from_numpy(d["length"]).cuda(),
                    torch.from_numpy(d["q_start"]).cuda(), T, new, length)
    q = torch.from_numpy(rng.standard_normal((T, heads * group, dim)).astype(np.float32)).to(torch.bfloat16).cuda()
    return d, cache, b, q, fsb.KvWorkspace(cache, b, heads * group)


def check(out, q, d, length, q_start, scale):
    """bf16 outputs against 64 bits: probabilities to 2^-11, scores (float sums), the result's rounding."""
    want, mag, dots = ref.attend(q.float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], d["table"], length,
                                 q_start, scale, 0)
    n = int(q_start[-1])
    tol = (2.0**-10 + 2.0**-19 * dots) * mag + 2.0**-8 * np.abs(want) + 1e-30
    assert (np.abs(out.float().cpu().numpy() - want)[:n] <= tol[:n]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,group", [(128, 8), (12, 8), (40, 1), (9, 8)])
def test_shorter_sequences_in_a_replay(fsb, cuda, dim, new, group):
    """All sequences had max_new new tokens when the call was captured; then some have fewer."""
    torch = cuda
    d, cache, b, q, ws = setup(torch, fsb, new, 40, 2, group, dim, 32, 300)
    out = torch.full_like(q, 7.0)
    fsb.fs_kv_attend(cache, b, q, out, 0.1, workspace=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fsb.fs_kv_attend(cache, b, q, out, 0.1, workspace=ws)
    rng = np.random.default_rng(42)
    counts = rng.integers(0, new + 1, 40)
    counts[:4] = new, 1, 2, 3
    length = np.maximum(counts, rng.integers(0, 301, 40)).astype(np.int32)
    q_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    b.tensors[1].copy_(torch.from_numpy(length))
    b.tensors[2].copy_(torch.from_numpy(q_start))
    out.fill_(7.0)
    g.replay()
    with pytest.raises(fsb.FleetSieveError) as ei:  # (the rest of the rows are no sequence's)
        fsb.fs_kv_check(ws)
    assert ei.value.code == fsb.FS_EDEVICE and "bounds" in str(ei.value)
    check(out, q, d, length, q_start, 0.1)
    assert bool((out[int(q_start[-1]):] == 7).all())
    # back again: nothing of it stays
    b.tensors[1].copy_(torch.from_numpy(d["length"]))
    b.tensors[2].copy_(torch.from_numpy(d["q_start"]))
    g.replay()
    fsb.fs_kv_check(ws)
    check(out, q, d, d["length"], d["q_start"], 0.1)


@pytest.mark.parametrize("new", [1, 5, 100])
def test_rows_left_over_belong_to_a_sequence_without_tokens(fsb, cuda, new):
    """The way for fewer tokens than captured: the last sequence, of length 0, takes the rows that are left."""
    torch = cuda
    d, cache, b, q, ws = setup(torch, fsb, new, 6, 2, 4, 128, 32, 200)
    length, q_start = d["length"].copy(), d["q_start"].copy()
    length[-1] = 0
    b.tensors[1].copy_(torch.from_numpy(length))
    kv = torch.randn(6 * new, 2, 128, device="cuda").to(torch.bfloat16)
    before = [t.clone() for t in cache.tensors]
    fsb.fs_kv_append(cache, b, kv, kv, workspace=ws)
    own = [int(x) for x in d["table"][-1]]
    assert all(torch.equal(t[own], o[own]) for t, o in zip(cache.tensors, before))
    for t, o in zip(cache.tensors, before):
        t.copy_(o)
    out = torch.full_like(q, float("nan"))
    fsb.fs_kv_attend(cache, b, q, out, 0.1, workspace=ws)
    fsb.fs_kv_check(ws)
    assert bool((out[5 * new:] == 0).all())
    check(out, q, d, length, q_start, 0.1)


@pytest.mark.parametrize("new", [1, 5, 100])
@pytest.mark.parametrize("end", ["first", "last"])
def test_rows_of_no_sequence_are_reported(fsb, cuda, new, end):
    torch = cuda
    d, cache, b, q, ws = setup(torch, fsb, new, 3, 2, 4, 128, 32, 200)
    q_start = d["q_start"].copy()
    if end == "first":
        q_start[0] = 1
    else:
        q_start[-1] -= 1
    b.tensors[2].copy_(torch.from_numpy(q_start))
    kv = torch.randn(3 * new, 2, 128, device="cuda").to(torch.bfloat16)
    for call in (lambda: fsb.fs_kv_attend(cache, b, q, torch.empty_like(q), 0.1, workspace=ws),
                 lambda: fsb.fs_kv_append(cache, b, kv, kv, workspace=ws)):
        call()
        with pytest.raises(fsb.FleetSieveError) as ei:
            fsb.fs_kv_check(ws)
        assert ei.value.code == fsb.FS_EDEVICE and "bounds" in str(ei.value)
