"""fs_kv_attend against attention in 64 bits over the same codes.

Tolerance, per element: a row's probabilities are rounded to half precision (2^-11 each) and
carry the rounding of their scores (fp32 sums of dim exact products: 2^-20 of sum |q k| scale, in
nats, also covers the exponential), so the weighted sum is off by at most
(2^-10 + 2^-19 sum |q k| scale) sum p |v|; then the result is rounded once to its type."""

import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": 2.0**-8, "fp16": 2.0**-11}


def on_gpu(torch, fsb, d, hq, dtype, qf, by_token=False):
    """The inputs on the GPU: caches, batch, queries (float32 values of qf rounded to dtype)."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16

    def codes(x):
        t = torch.from_numpy(x).cuda()
        return t.transpose(1, 2).contiguous().transpose(1, 2) if by_token else t

    cache = fsb.KvCache(codes(d["k"]), codes(d["v"]), torch.from_numpy(d["k_scale"]).cuda(),
                        torch.from_numpy(d["v_scale"]).cuda())
    T = int(d["q_start"][-1])
    new = np.diff(d["q_start"])
    batch = fsb.KvBatch(torch.from_numpy(d["table"]).cuda(), torch.from_numpy(d["length"]).cuda(),
                        torch.from_numpy(d["q_start"]).cuda(), T, int(new.max()), int(d["length"].max()))
    q = torch.from_numpy(qf).to(dt).cuda()
    return cache, batch, q, fsb.KvWorkspace(cache, batch, hq)


def check(out, want, mag, dots, eps):
    tol = (2.0**-10 + 2.0**-19 * dots) * mag + eps * np.abs(want) + 1e-30
    err = np.abs(out.float().cpu().numpy() - want)
    assert np.isfinite(out.float().cpu().numpy()).all()
    assert (err <= tol).all(), float((err / tol).max())


def run(torch, fsb, seed, lens, heads, group, dim, page, dtype="bf16", window=0, by_token=False, q_gain=2.0, change=None,
        garbage=True):
    rng = np.random.default_rng(seed)
    d = ref.make(rng, lens, heads, dim, page)
    if garbage:  # slots without a token hold NaN codes
        for b, (l, _) in enumerate(lens):
            if l % page:
                g = d["table"][b, l // page]
                d["k"][g, :, l % page:] = 0x7F
                d["v"][g, :, l % page:] = 0xFF
    if change:
        change(d)
    T, hq = int(d["q_start"][-1]), heads * group
    cache, batch, q, ws = on_gpu(torch, fsb, d, hq, dtype, (q_gain * rng.standard_normal((T, hq, dim))).astype(np.float32),
                                 by_token)
    out = torch.full((T, hq, dim), float("nan"), dtype=q.dtype, device="cuda")
    scale = dim**-0.5
    n0 = fsb.fs_launch_count()
    fsb.fs_kv_attend(cache, batch, q, out, scale, window=window, workspace=ws)
    fsb.fs_kv_check(ws)
    assert fsb.fs_launch_count() > n0
    want, mag, dots = ref.attend(q.float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], d["table"],
                                 d["length"], d["q_start"], scale, window)
    check(out, want, mag, dots, DTYPES[dtype])
    return out, (cache, batch, q, ws)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,page", [(128, 16), (128, 64), (64, 16), (64, 32), (128, 128), (64, 128)])
def test_single_tokens_of_every_length(fsb, cuda, dim, page, dtype):
    """Lengths at the edges of tiles and pages, an empty slot, all in one batch."""
    lens = [(l, 1) for l in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300)] + [(0, 0), (77, 0), (5, 1)]
    run(cuda, fsb, 1, lens, 2, 4, dim, page, dtype)


@pytest.mark.parametrize("group", [1, 3, 5, 8, 16])
def test_groups(fsb, cuda, group):
    run(cuda, fsb, 2, [(200, 1), (1, 1), (513, 1)], 3, group, 128, 32)


@pytest.mark.parametrize("new,group", [(2, 4), (5, 8), (9, 1), (17, 3), (40, 8)])
@pytest.mark.parametrize("window", [0, 1, 7, 100])
def test_several_tokens_and_windows(fsb, cuda, new, group, window):
    lens = [(new, new), (new + 1, new), (333, new), (0, 0), (97, max(1, new - 1)), (64 + new, new)]
    run(cuda, fsb, 3, lens, 2, group, 128, 16, window=window)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,length", [(128, 128), (129, 200), (300, 300), (257, 1000), (64, 700)])
@pytest.mark.parametrize("window", [0, 150])
def test_chunks(fsb, cuda, dim, new, length, window):
    lens = [(length, new), (new // 2 + 3, new // 2 + 3), (5, 1), (0, 0), (400, 0)]
    run(cuda, fsb, 4, lens, 2, 3, dim, 64, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_chunks_over_every_page_size(fsb, cuda, page, dtype):
    run(cuda, fsb, 5, [(391, 211), (1030, 97), (140, 140)], 1, 8, 128, page, dtype)


def test_one_long_sequence(fsb, cuda):
    """Many parts of one sequence's cache axis, joined by the last block."""
    run(cuda, fsb, 6, [(20011, 1)], 1, 8, 128, 64)
    run(cuda, fsb, 7, [(9000, 3), (17, 2)], 2, 4, 64, 16, window=5000)


@pytest.mark.parametrize("dim,window", [(128, 0), (128, 3000), (64, 0)])
def test_chunks_on_long_sequences(fsb, cuda, dim, window):
    """Few rows over long caches: walks in parts, joined by a second kernel; lengths that end a part early."""
    run(cuda, fsb, 16, [(9001, 40), (700, 33), (0, 0), (5120, 70)], 1, 4, dim, 64, window=window)
    run(cuda, fsb, 17, [(20000, 129)], 1, 1, dim, 128, window=window)


@pytest.mark.parametrize("dim,page", [(128, 16), (128, 64), (128, 128), (64, 32)])
@pytest.mark.parametrize("new,group,window", [(5, 7, 0), (5, 8, 150), (16, 8, 0), (9, 8, 1), (128, 1, 129)])
def test_one_tile_of_rows(fsb, cuda, dim, page, new, group, window):
    """33 to 128 rows a key head over walks of no tile of 128 tokens, one, two and more; windows under which
    some rows see nothing of a tile; scales far apart."""
    lens = [(l, new) for l in (128, 129, 256, 257, 300, 384, 385, 512, 640, 641, 1100, 1537)] + [(0, 0), (max(new, 9), 4), (600, 1)]

    def change(d):
        rng = np.random.default_rng(19)
        d["v_scale"] *= np.exp2(rng.integers(-7, 8, d["v_scale"].shape)).astype(np.float32)

    run(cuda, fsb, 18, lens, 8, group, dim, page, window=window, change=change)


@pytest.mark.parametrize("window", [0, 200])
def test_proposals_among_single_tokens(fsb, cuda, window):
    """Most sequences have one new token, some 33 to 64 rows: both kernels work on the batch."""
    lens = [(700, 5), (300, 1), (1, 1), (0, 0), (257, 4), (900, 8), (128, 1), (129, 1), (40, 1), (512, 1), (1000, 5), (64, 1)]
    run(cuda, fsb, 20, lens, 8, 8, 128, 32, window=window)


def test_cache_laid_out_by_token(fsb, cuda):
    run(cuda, fsb, 8, [(200, 1), (70, 3)], 4, 2, 128, 32, by_token=True)
    run(cuda, fsb, 8, [(300, 150), (70, 3)], 4, 2, 64, 32, by_token=True)


@pytest.mark.parametrize("new", [1, 150])
def test_strided_rows(fsb, cuda, new):
    """Queries cut out of a wider projection, results into every other row block."""
    torch = cuda
    rng = np.random.default_rng(9)
    d = ref.make(rng, [(201, new), (new, new)], 2, 128, 32)
    T, hq = int(d["q_start"][-1]), 6
    qf = rng.standard_normal((T, hq, 128)).astype(np.float32)
    cache, batch, q, ws = on_gpu(torch, fsb, d, hq, "bf16", qf)
    wide = torch.randn(T, hq + 4, 128, device="cuda").to(q.dtype)
    wide[:, 2:2 + hq] = q
    held = torch.full((2 * T, hq, 128), 7.0, dtype=q.dtype, device="cuda")
    fsb.fs_kv_attend(cache, batch, wide[:, 2:2 + hq], held[::2], 0.1, workspace=ws)
    plain = torch.empty(T, hq, 128, dtype=q.dtype, device="cuda")
    fsb.fs_kv_attend(cache, batch, q, plain, 0.1, workspace=ws)
    fsb.fs_kv_check(ws)
    assert torch.equal(held[::2], plain) and bool((held[1::2] == 7).all())
    want, mag, dots = ref.attend(q.float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], d["table"],
                                 d["length"], d["q_start"], 0.1, 0)
    check(plain, want, mag, dots, DTYPES["bf16"])


@pytest.mark.parametrize("new", [1, 140])
def test_scales_far_apart(fsb, cuda, new):
    """Pages whose scales differ by 2^14 either way, some of them 0; values of a page with scale 0 are 0."""

    def change(d):
        rng = np.random.default_rng(10)
        for n in ("k_scale", "v_scale"):
            d[n] *= np.exp2(rng.integers(-7, 8, d[n].shape)).astype(np.float32)
            d[n][rng.random(d[n].shape) < 0.1] = 0.0
        d["k_scale"] *= np.float32(2.0**-6)  # (scores that do not pick a single key)

    run(cuda, fsb, 11, [(700, new), (new, new)], 2, 4, 128, 16, change=change)


@pytest.mark.parametrize("new", [1, 140])
@pytest.mark.parametrize("gain", [0.0, 1e-30, 30.0])
def test_query_magnitudes(fsb, cuda, new, gain):
    """Zero queries (the mean of the values), tiny ones, and scores of hundreds (a single key counts)."""
    run(cuda, fsb, 12, [(300, new), (new, new)], 2, 4, 128, 32, q_gain=gain)


def test_rows_before_the_first_token_are_zero(fsb, cuda):
    """More new tokens than length: rows at negative positions see nothing and become 0."""
    torch = cuda
    rng = np.random.default_rng(13)
    for new in (4, 200):
        d = ref.make(rng, [(3, 3), (50, 1)], 2, 128, 16)
        d["q_start"] = np.array([0, new, new + 1], np.int32)  # sequence 0: `new` rows, 3 tokens
        cache, batch, q, ws = on_gpu(torch, fsb, d, 8, "bf16", rng.standard_normal((new + 1, 8, 128)).astype(np.float32))
        out = torch.full_like(q, float("nan"))
        fsb.fs_kv_attend(cache, batch, q, out, 0.1, workspace=ws)
        fsb.fs_kv_check(ws)
        assert bool((out[: new - 3] == 0).all()) and bool(torch.isfinite(out.float()).all())
        assert bool((out[new - 3:].float().abs().amax((1, 2)) > 0).all())


def test_same_bits_every_time_and_under_a_graph(fsb, cuda):
    torch = cuda
    out, (cache, batch, q, ws) = run(torch, fsb, 14, [(5000, 1), (700, 1), (3, 1)], 2, 8, 128, 64)
    again = torch.empty_like(out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fsb.fs_kv_attend(cache, batch, q, again, 128**-0.5, workspace=ws)
    for _ in range(3):
        again.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, again)


def test_another_stream(fsb, cuda):
    torch = cuda
    out, (cache, batch, q, ws) = run(torch, fsb, 15, [(900, 1), (30, 1)], 2, 4, 128, 64)
    s = torch.cuda.Stream()
    q2, out2 = torch.empty_like(q), torch.empty_like(out)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q2.copy_(q)
        fsb.fs_kv_attend(cache, batch, q2, out2, 128**-0.5, workspace=ws)
    fsb.fs_kv_check(ws, s)
    assert torch.equal(out, out2)
    fsb.fs_kv_attend(cache, batch, q2, out2.zero_(), 128**-0.5, workspace=ws, stream=torch.cuda.current_stream())
    fsb.fs_kv_check(ws)
    assert torch.equal(out, out2)


def test_broken_batches_are_reported(fsb, cuda):
    """Device arrays that break the batch's bounds: the sequence is skipped (or page 0 read in the
    place of a page the cache does not have), a status is reported, the next call is right."""
    torch = cuda
    rng = np.random.default_rng(16)
    d = ref.make(rng, [(100, 1), (40, 1)], 2, 128, 16)
    cache, batch, q, ws = on_gpu(torch, fsb, d, 4, "bf16", rng.standard_normal((2, 4, 128)).astype(np.float32))
    table, length, q_start = batch.tensors
    out = torch.zeros_like(q)
    for t, at, bad, word in ((length, 0, 200, "bounds"), (length, 1, -1, "bounds"), (q_start, 1, 7, "bounds"),
                             (table, (0, 2), d["pages"], "page"), (table, (1, 0), -5, "page"),
                             (cache.tensors[2], (int(d["table"][0, 1]), 1), 0.3, "power of two"),
                             (cache.tensors[3], (int(d["table"][1, 0]), 0), -1.0, "power of two")):
        keep = t[at].clone()
        t[at] = bad
        fsb.fs_kv_attend(cache, batch, q, out, 0.1, workspace=ws)
        with pytest.raises(fsb.FleetSieveError) as ei:
            fsb.fs_kv_check(ws)
        assert ei.value.code == fsb.FS_EDEVICE and word in str(ei.value)
        t[at] = keep
    fsb.fs_kv_attend(cache, batch, q, out, 0.1, workspace=ws)
    fsb.fs_kv_check(ws)
    want, mag, dots = ref.attend(q.float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], d["table"],
                                 d["length"], d["q_start"], 0.1, 0)
    check(out, want, mag, dots, DTYPES["bf16"])


def test_a_workspace_serves_smaller_batches(fsb, cuda):
    """A workspace made for the largest batch, cache and queries is enough for any smaller ones (the cut into
    parts differs), and what one call leaves in it does not show in the next."""
    torch = cuda
    rng = np.random.default_rng(18)
    big = ref.make(rng, [(6000, 300)] + [(3000, 40)] * 11, 2, 64, 16)
    cache, batch, q, ws = on_gpu(torch, fsb, big, 8, "bf16", rng.standard_normal((740, 8, 64)).astype(np.float32))
    for lens in ([(6000, 1)], [(2999, 9), (17, 3)], [(6000, 300)], [(1, 1)] * 12, [(4097, 70)] * 3, [(5000, 1)] * 12):
        need = [-(-l // 16) for l, _ in lens]
        table = np.stack([np.resize(big["table"][0], 375) for _ in lens])
        d = dict(big, table=table, length=np.array([l for l, _ in lens], np.int32),
                 q_start=np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int32))
        assert max(need) <= 375
        T = int(d["q_start"][-1])
        b = fsb.KvBatch(torch.from_numpy(table).cuda(), torch.from_numpy(d["length"]).cuda(), torch.from_numpy(d["q_start"]).cuda(),
                        T, max(n for _, n in lens), max(l for l, _ in lens))
        qq = torch.from_numpy(rng.standard_normal((T, 8, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
        out = torch.full_like(qq, float("nan"))
        fsb.fs_kv_attend(cache, b, qq, out, 0.125, workspace=ws)
        fsb.fs_kv_check(ws)
        want, mag, dots = ref.attend(qq.float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], table, d["length"],
                                     d["q_start"], 0.125, 0)
        check(out, want, mag, dots, DTYPES["bf16"])


@pytest.mark.parametrize("new", [1, 20, 200])
def test_negative_and_zero_scales_of_scores(fsb, cuda, new):
    torch = cuda
    rng = np.random.default_rng(19)
    d = ref.make(rng, [(330, new), (new, new)], 2, 128, 32)
    cache, batch, q, ws = on_gpu(torch, fsb, d, 8, "fp16", rng.standard_normal((2 * new, 8, 128)).astype(np.float32))
    for scale in (-0.1, 0.0):
        out = torch.empty_like(q)
        fsb.fs_kv_attend(cache, batch, q, out, scale, workspace=ws)
        fsb.fs_kv_check(ws)
        want, mag, dots = ref.attend(q.float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], d["table"],
                                     d["length"], d["q_start"], scale, 0)
        check(out, want, mag, dots, DTYPES["fp16"])


@pytest.mark.parametrize("new", [1, 100])
def test_windows_as_wide_as_an_int(fsb, cuda, new):
    """A window that holds everything is no window, however wide."""
    torch = cuda
    rng = np.random.default_rng(20)
    d = ref.make(rng, [(330, new), (new, new)], 1, 64, 16)
    cache, batch, q, ws = on_gpu(torch, fsb, d, 4, "bf16", rng.standard_normal((2 * new, 4, 64)).astype(np.float32))
    outs = []
    for window in (0, 330, 2**31 - 1):
        outs.append(fsb.fs_kv_attend(cache, batch, q, torch.empty_like(q), 0.125, window=window, workspace=ws))
    fsb.fs_kv_check(ws)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("new", [1, 40, 300])
def test_nan_queries_stay_in_their_rows(fsb, cuda, new):
    torch = cuda
    rng = np.random.default_rng(21)
    d = ref.make(rng, [(400, new), (new, new)], 2, 128, 64)
    cache, batch, q, ws = on_gpu(torch, fsb, d, 8, "bf16", rng.standard_normal((2 * new, 8, 128)).astype(np.float32))
    clean = fsb.fs_kv_attend(cache, batch, q, torch.empty_like(q), 0.1, workspace=ws).clone()
    bad = q.clone()
    bad[new - 1, 3, 17] = float("nan")
    bad[new, 6, 0] = float("inf")
    out = fsb.fs_kv_attend(cache, batch, bad, torch.empty_like(q), 0.1, workspace=ws)
    fsb.fs_kv_check(ws)
    hit = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    hit[new - 1, 3] = hit[new, 6] = True
    assert bool(torch.isnan(out[hit].float()).all()) and torch.equal(out[~hit], clean[~hit])


def test_a_length_beyond_the_bound_is_reported(fsb, cuda):
    """Room in the page table, but a length beyond max_length, with every kind of walk: skipped and reported."""
    torch = cuda
    rng = np.random.default_rng(22)
    for new, window in ((1, 0), (3, 100), (300, 0), (300, 100), (70, 0)):
        d = ref.make(rng, [(4000, new), (4000, new)], 1, 64, 16)
        cache, _, q, ws = on_gpu(torch, fsb, d, 4, "bf16", rng.standard_normal((2 * new, 4, 64)).astype(np.float32))
        length = torch.tensor([500, 4000], dtype=torch.int32, device="cuda")
        batch = fsb.KvBatch(torch.from_numpy(d["table"]).cuda(), length, torch.from_numpy(d["q_start"]).cuda(), 2 * new, new, 500)
        work = fsb.KvWorkspace(cache, batch, 4)
        out = torch.full_like(q, 7.0)
        fsb.fs_kv_attend(cache, batch, q, out, 0.1, window=window, workspace=work)
        with pytest.raises(fsb.FleetSieveError) as ei:
            fsb.fs_kv_check(work)
        assert ei.value.code == fsb.FS_EDEVICE and "bounds" in str(ei.value)
        assert bool((out[new:] == 7).all())
        want, mag, dots = ref.attend(q[:new].float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], d["table"][:1],
                                     [500], [0, new], 0.1, window)
        check(out[:new], want, mag, dots, DTYPES["bf16"])


def test_chunks_give_the_same_bits_every_time_and_under_a_graph(fsb, cuda):
    torch = cuda
    for lens, heads in (([(700, 300), (130, 130), (90, 2)], 2), ([(6000, 40)], 1)):
        out, (cache, batch, q, ws) = run(torch, fsb, 23, lens, heads, 8, 128, 32)
        again = torch.empty_like(out)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fsb.fs_kv_attend(cache, batch, q, again, 128**-0.5, workspace=ws)
        for _ in range(3):
            again.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, again)


def test_append_and_attend_in_a_row(fsb, cuda):
    """A prompt in chunks, then single tokens, each step's append and attention queued without a wait between
    them: every step's outputs are those of the same step alone."""
    torch = cuda
    rng = np.random.default_rng(24)
    steps, hk, hq, D, P = [130, 1, 1, 64, 1, 257, 2], 2, 8, 128, 32
    total = sum(steps)
    pages = -(-total // P) + 1
    x = torch.from_numpy(rng.standard_normal((total, hq + 2 * hk, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    table = torch.randperm(pages, device="cuda")[None].to(torch.int32).contiguous()

    def go(wait):
        cache = fsb.KvCache(*(torch.full((pages, hk, P, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)),
                            *(torch.full((pages, hk), 3.0, device="cuda") for _ in range(2)))
        outs, at, keep = [], 0, []
        for n in steps:
            batch = fsb.KvBatch(table, torch.tensor([at + n], dtype=torch.int32, device="cuda"),
                                torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n, total)
            ws = fsb.KvWorkspace(cache, batch, hq)
            row = x[at:at + n]
            out = torch.empty(n, hq, D, dtype=x.dtype, device="cuda")
            fsb.fs_kv_append(cache, batch, row[:, hq:hq + hk], row[:, hq + hk:], workspace=ws)
            fsb.fs_kv_attend(cache, batch, row[:, :hq], out, 0.1, workspace=ws)
            if wait:
                fsb.fs_kv_check(ws)
            keep.append(ws)
            outs.append(out)
            at += n
        for ws in keep:
            fsb.fs_kv_check(ws)
        return outs

    a, b = go(True), go(False)
    assert all(torch.equal(p, q) and bool(torch.isfinite(p.float()).all()) for p, q in zip(a, b))


def test_a_chunk_that_rescales_pages_is_attended_to_at_once(fsb, cuda):
    """Prompts in chunks of many rows, each louder than what is cached (its page's codes are rescaled): attention that
    is queued right behind the append gives the bits of attention after a wait."""
    torch = cuda
    rng = np.random.default_rng(32)
    B, hk, hq, D, P, n, steps = 4, 2, 16, 128, 64, 150, 4
    pages = B * -(-n * steps // P)
    table = torch.randperm(pages, device="cuda").view(B, -1).to(torch.int32).contiguous()
    x = torch.from_numpy(rng.standard_normal((steps, B * n, hq + 2 * hk, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    x *= torch.tensor([1, 3, 9, 27], dtype=x.dtype, device="cuda")[:, None, None, None]
    q_start = torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda")
    batches = [fsb.KvBatch(table, torch.full((B,), n * (i + 1), dtype=torch.int32, device="cuda"), q_start, B * n, n, n * steps)
               for i in range(steps)]

    def go(wait):
        cache = fsb.KvCache(*(torch.zeros(pages, hk, P, D, dtype=torch.uint8, device="cuda") for _ in range(2)),
                            *(torch.zeros(pages, hk, device="cuda") for _ in range(2)))
        ws = fsb.KvWorkspace(cache, batches[-1], hq)
        outs = [torch.empty(B * n, hq, D, dtype=x.dtype, device="cuda") for _ in range(steps)]
        torch.cuda.synchronize()
        for i, b in enumerate(batches):
            fsb.fs_kv_append(cache, b, x[i][:, hq:hq + hk], x[i][:, hq + hk:], workspace=ws)
            if wait:
                fsb.fs_kv_check(ws)
            fsb.fs_kv_attend(cache, b, x[i][:, :hq], outs[i], 0.02, workspace=ws)
        fsb.fs_kv_check(ws)
        return outs

    want = go(True)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(want, go(False)))


def test_workspaces_hold_what_a_batch_can_use(fsb, cuda):
    """Room for tokens as halves (up to 1 GiB) only where a batch can have the rows for that, more than 768 a key
    head. Proposals need parts of results alone: nine parts of 16 rows an item at most, a row 130 floats."""
    torch = cuda
    cache = fsb.KvCache(*(torch.zeros(4, 8, 64, 128, dtype=torch.uint8, device="cuda") for _ in range(2)),
                        *(torch.zeros(4, 8, device="cuda") for _ in range(2)))
    table = torch.zeros(256, 512, dtype=torch.int32, device="cuda")
    ends = torch.zeros(257, dtype=torch.int32, device="cuda")

    def size(batch, new):
        return fsb.KvWorkspace(cache, fsb.KvBatch(table[:batch], ends[:batch], ends[:batch + 1], batch * new, new, 32768), 64).bytes

    assert size(16, 5) < 1 << 27
    assert size(256, 5) <= size(256, 96) < 1 << 30
    assert size(64, 97) >= 1 << 30  # 776 rows a key head
    # one prompt of 8192 tokens over 32768: 256 tiles of keys and values of eight heads in halves
    assert 256 * 8 * 2 * 128 * 256 <= size(1, 8192) < 1 << 30


@pytest.mark.parametrize("dim,page", [(128, 16), (64, 16), (128, 32), (128, 64), (64, 32)])
@pytest.mark.parametrize("new,group", [(1, 4), (5, 4), (9, 8), (70, 8), (120, 8)])
@pytest.mark.parametrize("window", [1, 17, 50, 100])
@pytest.mark.parametrize("freed", ["nothing", "another's"])
def test_pages_before_the_window_may_be_freed(fsb, cuda, dim, page, new, group, window, freed):
    """Entries of pages that lie wholly before the windows of all of a sequence's new tokens hold a number that is no
    page, or a page of NaN codes with NaN for a scale: nothing of it shows, and nothing is reported."""
    torch = cuda
    rng = np.random.default_rng(33)
    lens = [(new + x, new) for x in (0, 15, 16, 31, 33, 40, 64, 100, 127, 128, 129, 200, 257, 390, 500)] + [(0, 0), (300, 1)]
    d = ref.make(rng, lens, 2, dim, page)
    for b, (l, _) in enumerate(lens):  # (slots without a token hold NaN codes, as ever)
        if l % page:
            d["k"][d["table"][b, l // page], :, l % page:] = 0x7F
            d["v"][d["table"][b, l // page], :, l % page:] = 0xFF
    bad = next(g for g in range(d["pages"]) if not (d["table"] == g).any())
    dirty = d["table"].copy()
    n_freed = 0
    for b, (l, n) in enumerate(lens):
        free = max(l - n - window + 1, 0) // page if n else -(-l // page)
        dirty[b, :free] = -7 if freed == "nothing" else bad
        n_freed += free
    assert n_freed > 0
    T, hq = int(d["q_start"][-1]), 2 * group
    cache, batch, q, ws = on_gpu(torch, fsb, d, hq, "bf16", rng.standard_normal((T, hq, dim)).astype(np.float32))
    batch.tensors[0].copy_(torch.from_numpy(dirty))
    for t, x in zip(cache.tensors, (0x7F, 0xFF, float("nan"), float("nan"))):
        t[bad] = x
    out = torch.full_like(q, float("nan"))
    fsb.fs_kv_attend(cache, batch, q, out, 0.1, window=window, workspace=ws)
    fsb.fs_kv_check(ws)
    want, mag, dots = ref.attend(q.float().cpu().numpy(), d["k"], d["v"], d["k_scale"], d["v_scale"], d["table"],
                                 d["length"], d["q_start"], 0.1, window)
    check(out, want, mag, dots, DTYPES["bf16"])
