"""fs_kv_append against the same in 64 bits.

A code may differ from the nearest one to the 64-bit value only as far as the rotation's three
float roundings move that value: |code * scale - y| <= half an e4m3 step + 2^-22 (|a| + |b|), a and b the
rotated pair. Scales are powers of two and equal exactly unless the largest magnitude is that near to
a boundary; codes of earlier tokens are rescaled by powers of two, and equal exactly."""

import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu


def setup(torch, fsb, rng, lens, heads, hq, dim, page, dtype="bf16", rot=None, gain=1.0, by_token=False):
    d = ref.make(rng, lens, heads, dim, page)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16

    def codes(x):
        t = torch.from_numpy(x.copy()).cuda()
        return t.transpose(1, 2).contiguous().transpose(1, 2) if by_token else t

    cache = fsb.KvCache(codes(d["k"]), codes(d["v"]), torch.from_numpy(d["k_scale"].copy()).cuda(),
                        torch.from_numpy(d["v_scale"].copy()).cuda())
    T = int(d["q_start"][-1])
    batch = fsb.KvBatch(torch.from_numpy(d["table"]).cuda(), torch.from_numpy(d["length"]).cuda(),
                        torch.from_numpy(d["q_start"]).cuda(), T, int(np.diff(d["q_start"]).max()),
                        int(d["length"].max()))
    x = {n: torch.from_numpy((gain * rng.standard_normal((T, h, dim))).astype(np.float32)).to(dt).cuda()
         for n, h in (("q", hq), ("k", heads), ("v", heads))}
    rot = dim if rot is None else rot
    ang = np.arange(int(d["length"].max()) + 1)[:, None] * 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    return d, cache, batch, x, cos, sin, fsb.KvWorkspace(cache, batch, hq)


def expected(d, x, cos, sin, interleaved, page):
    """Per cache tensor: (64-bit values, pair magnitudes) of the new tokens, new scales, rescaled old codes."""
    out = {}
    pos = np.concatenate([np.arange(l - n, l) for l, n in zip(d["length"], np.diff(d["q_start"]))] or [[]]).astype(int)
    seq = np.repeat(np.arange(len(d["length"])), np.diff(d["q_start"]))
    for n in ("k", "v"):
        y = x[n].astype(np.float64)
        z = ref.rotate(y, pos, cos, sin, interleaved) if n == "k" and cos.shape[1] else y
        mag = np.abs(y)
        if n == "k" and cos.shape[1]:
            half = cos.shape[1]
            i = np.arange(half)
            lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            s = mag[..., lo] + mag[..., hi]
            mag[..., lo] = mag[..., hi] = s
        scale, codes = d[n + "_scale"].astype(np.float64), d[n].copy()
        for b in range(len(d["length"])):
            L, c = int(d["length"][b]), int(d["q_start"][b + 1] - d["q_start"][b])
            for j in range((L - c) // page, -(-L // page)) if c else ():
                lo, hi = max(L - c, j * page), min(L, (j + 1) * page)
                g = d["table"][b, j]
                rows = z[int(d["q_start"][b]) + lo - (L - c): int(d["q_start"][b]) + hi - (L - c)]
                need = ref.scale_for(np.abs(rows).max((0, 2)))
                old = scale[g] if lo > j * page else np.zeros_like(need)
                now = np.maximum(old, need)
                if lo > j * page:
                    f = np.where(now > 0, old / np.where(now > 0, now, 1), 1.0)
                    codes[g, :, :lo - j * page] = ref.nearest_code(ref.VALUES[codes[g, :, :lo - j * page]] * f[:, None, None])
                scale[g] = now
        out[n] = (z, mag, scale, codes)
    return out, pos, seq


def verify(torch, d, cache, x, cos, sin, interleaved, page, q_out=None, q=None):
    want, pos, seq = expected(d, x, cos, sin, interleaved, page)
    k, v, ks, vs = cache.tensors
    written = np.zeros((d["pages"], page), bool)
    written[d["table"][seq, pos // page], pos % page] = True
    kept = np.zeros((d["pages"], page), bool)
    for b in range(len(d["length"])):
        for p in range(int(d["length"][b]) - int(d["q_start"][b + 1] - d["q_start"][b])):
            kept[d["table"][b, p // page], p % page] = True
    for n, codes, scale in (("k", k, ks), ("v", v, vs)):
        z, mag, w_scale, w_codes = want[n]
        got, got_s = codes.cpu().numpy(), scale.cpu().numpy().astype(np.float64)
        assert np.array_equal(got_s, w_scale)
        # earlier tokens, and slots that hold none
        rest = ~written
        m = np.broadcast_to((kept & rest)[:, None, :, None], got.shape)
        assert np.array_equal(got[m], w_codes[m])
        m = np.broadcast_to((~kept & rest)[:, None, :, None], got.shape)
        assert np.array_equal(got[m], d[n][m])
        page_of, slot = d["table"][seq, pos // page], pos % page
        s = got_s[page_of][:, :, None]
        val = ref.VALUES[got[page_of, :, slot]] * s
        step = np.where(s > 0, np.exp2(np.floor(np.log2(np.maximum(np.abs(z) / np.where(s > 0, s, 1), 2.0**-6))) - 3) * s, 0)
        assert (np.abs(val - z) <= step / 2 + 2.0**-22 * mag).all()
    if q is not None:
        w = ref.rotate(q, pos, cos, sin, interleaved) if cos.shape[1] else q
        eps = 2.0**-8 if q_out.dtype == torch.bfloat16 else 2.0**-11
        amp = np.abs(q).max(-1, keepdims=True)
        assert (np.abs(q_out.float().cpu().numpy() - w) <= eps * np.abs(w) + 2.0**-21 * amp + 2.0**-24).all()


def run(torch, fsb, seed, lens, heads=2, hq=6, dim=128, page=16, dtype="bf16", rot=None, interleaved=False, gain=1.0,
        by_token=False):
    rng = np.random.default_rng(seed)
    d, cache, batch, x, cos, sin, ws = setup(torch, fsb, rng, lens, heads, hq, dim, page, dtype, rot, gain, by_token)
    q_out = torch.empty_like(x["q"])
    ct, st = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()) if cos.shape[1] else (None, None)
    fsb.fs_kv_append(cache, batch, x["k"], x["v"], ct, st, q=x["q"], q_out=q_out, interleaved=interleaved, workspace=ws)
    fsb.fs_kv_check(ws)
    h = {n: t.float().cpu().numpy() for n, t in x.items()}
    verify(torch, d, cache, h, cos, sin, interleaved, page, q_out, h["q"])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_single_tokens(fsb, cuda, dim, page, dtype):
    run(cuda, fsb, 1, [(1, 1), (2, 1), (16, 1), (17, 1), (0, 0), (64, 1), (65, 1), (129, 1), (200, 0)], dim=dim,
        page=page, dtype=dtype)


@pytest.mark.parametrize("gain", [0.02, 1.0, 50.0])
def test_scales_that_grow(fsb, cuda, gain):
    """New tokens smaller and larger than the page's: its codes are rescaled where the scale grows."""
    run(cuda, fsb, 2, [(7, 1), (30, 2), (100, 3), (33, 20)], gain=gain)


@pytest.mark.parametrize("rot,interleaved", [(0, False), (8, False), (64, False), (128, False), (64, True), (128, True), (40, True)])
@pytest.mark.parametrize("page", [16, 64])
def test_rotations(fsb, cuda, rot, interleaved, page):
    run(cuda, fsb, 3, [(50, 3), (131, 131), (9, 1)], rot=rot, interleaved=interleaved, page=page)


@pytest.mark.parametrize("dim,page,dtype", [(128, 16, "bf16"), (128, 64, "fp16"), (64, 32, "bf16"), (64, 128, "fp16"),
                                            (128, 128, "bf16"), (64, 16, "bf16")])
def test_chunks(fsb, cuda, dim, page, dtype):
    run(cuda, fsb, 4, [(300, 211), (128, 128), (1, 1), (0, 0), (97, 65), (260, 17)], heads=3, hq=9, dim=dim, page=page,
        dtype=dtype)


def test_cache_laid_out_by_token(fsb, cuda):
    run(cuda, fsb, 5, [(50, 20), (33, 1)], by_token=True)


def test_without_queries_and_with_strides(fsb, cuda):
    """Keys and values cut out of one projection; queries rotated in place, or not given."""
    torch = cuda
    rng = np.random.default_rng(6)
    d, cache, batch, x, cos, sin, ws = setup(torch, fsb, rng, [(40, 9), (77, 30)], 2, 4, 128, 32)
    T = batch.tokens
    qkv = torch.empty(T, 8, 128, dtype=torch.bfloat16, device="cuda")
    qkv[:, :4], qkv[:, 4:6], qkv[:, 6:] = x["q"], x["k"], x["v"]
    ct, st = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    fsb.fs_kv_append(cache, batch, qkv[:, 4:6], qkv[:, 6:], ct, st, q=qkv[:, :4], q_out=qkv[:, :4], workspace=ws)
    fsb.fs_kv_check(ws)
    h = {n: t.float().cpu().numpy() for n, t in x.items()}
    verify(torch, d, cache, h, cos, sin, False, 32, qkv[:, :4], h["q"])
    before = [t.clone() for t in cache.tensors]
    fsb.fs_kv_append(cache, batch, x["k"], x["v"], ct, st, workspace=ws)  # again, the same bytes
    fsb.fs_kv_check(ws)
    assert all(torch.equal(a, b) for a, b in zip(before, cache.tensors))


def test_zeros_infinities_and_nans(fsb, cuda):
    torch = cuda
    rng = np.random.default_rng(7)
    d, cache, batch, x, cos, sin, ws = setup(torch, fsb, rng, [(16, 16), (16, 16), (3, 3)], 1, 1, 128, 16)
    k, v = x["k"], x["v"]
    k[:16] = 0
    v[:16] = 0
    k[16, 0, 3], v[17, 0, 5] = float("inf"), -float("inf")
    fsb.fs_kv_append(cache, batch, k, v, workspace=ws)
    fsb.fs_kv_check(ws)
    kc, vc, ks, vs = cache.tensors
    g0, g1 = int(d["table"][0, 0]), int(d["table"][1, 0])
    assert float(ks[g0, 0]) == 0 and float(vs[g0, 0]) == 0 and bool((kc[g0] == 0).all()) and bool((vc[g0] == 0).all())
    assert int(kc[g1, 0, 0, 3]) == 0x7E and int(vc[g1, 0, 1, 5]) == 0xFE
    finite = k[16:32].float().cpu().numpy()
    finite = finite[np.isfinite(finite)]
    assert float(ks[g1, 0]) == float(ref.scale_for(np.abs(finite).max()))
    v[33, 0, 7] = float("nan")
    fsb.fs_kv_append(cache, batch, k, v, workspace=ws)
    with pytest.raises(fsb.FleetSieveError) as ei:
        fsb.fs_kv_check(ws)
    assert ei.value.code == fsb.FS_EDEVICE and "NaN" in str(ei.value)
    assert int(vc[int(d["table"][2, 0]), 0, 1, 7]) == 0
    assert not bool(torch.isnan(vc.view(torch.float8_e4m3fn)[int(d["table"][2, 0]), 0, :3].float()).any())


def test_tiny_and_huge_values(fsb, cuda):
    torch = cuda
    rng = np.random.default_rng(8)
    for gain in (1e-38, 1e38):
        d, cache, batch, x, cos, sin, ws = setup(torch, fsb, rng, [(20, 20)], 1, 1, 128, 16, gain=gain)
        k = x["k"].clamp(-3e38, 3e38)
        fsb.fs_kv_append(cache, batch, k, k, workspace=ws)
        fsb.fs_kv_check(ws)
        h = k.float().cpu().numpy()
        verify(torch, d, cache, {"k": h, "v": h}, cos[:, :0], sin[:, :0], False, 16)


def test_broken_batches_are_reported(fsb, cuda):
    torch = cuda
    rng = np.random.default_rng(9)
    d, cache, batch, x, cos, sin, ws = setup(torch, fsb, rng, [(40, 2), (17, 3)], 2, 2, 128, 16)
    table, length, q_start = batch.tensors
    ct, st = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    before = [t.clone() for t in cache.tensors]
    for t, at, bad, word in ((length, 0, 500, "bounds"), (q_start, 2, 9, "bounds"), (table, (0, 2), d["pages"], "page")):
        keep = t[at].clone()
        t[at] = bad
        fsb.fs_kv_append(cache, batch, x["k"], x["v"], ct, st, workspace=ws)
        with pytest.raises(fsb.FleetSieveError) as ei:
            fsb.fs_kv_check(ws)
        assert ei.value.code == fsb.FS_EDEVICE and word in str(ei.value)
        t[at] = keep
        for a, b in zip(before, cache.tensors):
            b.copy_(a)
    fsb.fs_kv_append(cache, batch, x["k"], x["v"], ct[:17], st[:17], workspace=ws)
    with pytest.raises(fsb.FleetSieveError) as ei:
        fsb.fs_kv_check(ws)
    assert "cos" in str(ei.value)


def test_cache_beyond_32_bits(fsb, cuda):
    """Pages whose bytes lie more than 4 GiB into the cache: appended to and attended to."""
    torch = cuda
    H, P, D = 8, 64, 128
    pages = (4 << 30) // (H * P * D) + 40
    k, v = (torch.zeros(pages, H, P, D, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(pages, H, device="cuda") for _ in range(2))
    cache = fsb.KvCache(k, v, ks, vs)
    for n in (1, 200):
        L = 200
        table = torch.arange(pages - 4, pages, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
        batch = fsb.KvBatch(table, torch.tensor([L], dtype=torch.int32, device="cuda"),
                            torch.tensor([0, L], dtype=torch.int32, device="cuda"), L, L, L)
        ws = fsb.KvWorkspace(cache, batch, H)
        x = torch.randn(L, H, D, device="cuda").to(torch.bfloat16)
        fsb.fs_kv_append(cache, batch, x, x, workspace=ws)
        fsb.fs_kv_check(ws)
        assert bool((ks[pages - 4:] > 0).all()) and not bool(ks[:pages - 4].any()) and not bool(k[0].any())
        one = fsb.KvBatch(table, torch.tensor([L], dtype=torch.int32, device="cuda"),
                          torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n, L)
        q = torch.randn(n, H, D, device="cuda").to(torch.bfloat16)
        out = torch.empty_like(q)
        fsb.fs_kv_attend(cache, one, q, out, 0.1, workspace=ws)
        fsb.fs_kv_check(ws)
        kk = (k[pages - 4:].flip(0).view(torch.float8_e4m3fn).double() * ks[pages - 4:].flip(0)[..., None, None].double())
        kk = kk.transpose(1, 2).reshape(-1, H, D)[:L]
        s = torch.einsum("thd,lhd->htl", q.double(), kk) * 0.1
        j = torch.arange(L, device="cuda")
        s = s.masked_fill(j[None, None] > (L - n + torch.arange(n, device="cuda"))[None, :, None], float("-inf"))
        vv = (v[pages - 4:].flip(0).view(torch.float8_e4m3fn).double() * vs[pages - 4:].flip(0)[..., None, None].double())
        vv = vv.transpose(1, 2).reshape(-1, H, D)[:L]
        p = torch.softmax(s, -1)
        want = torch.einsum("htl,lhd->thd", p, vv)
        mag = torch.einsum("htl,lhd->thd", p, vv.abs())
        # (2^-9: probabilities 2^-11, scores, and the rest of the tolerance above with room)
        assert bool(((out.double() - want).abs() <= 2.0**-9 * mag + 2.0**-8 * want.abs()).all())


@pytest.mark.parametrize("new", [1, 3, 20, 70])
@pytest.mark.parametrize("bad", [-1, "pages", -(2**31), 2**31 - 1])
@pytest.mark.parametrize("at", ["first", "last"])
def test_a_page_outside_the_cache_is_not_written(fsb, cuda, new, bad, at):
    """One of a sequence's page ids is none of the cache's: what belongs there is not stored anywhere (page 0 is
    no sequence's here, but could be another request's), the rest is as with the right id, and it is reported."""
    torch = cuda
    rng = np.random.default_rng(31)
    lens, page = [(new + 20, new), (45, new if new < 45 else 9), (16, 1)], 16
    d, cache, batch, x, cos, sin, ws = setup(torch, fsb, rng, lens, 2, 4, 128, page)
    table = batch.tensors[0]
    spare = next(g for g in range(d["pages"]) if not (d["table"] == g).any())
    table[table == 0] = spare
    ct, st = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    before = [t.clone() for t in cache.tensors]
    q_good = torch.empty_like(x["q"])
    fsb.fs_kv_append(cache, batch, x["k"], x["v"], ct, st, q=x["q"], q_out=q_good, workspace=ws)
    fsb.fs_kv_check(ws)
    want = [t.clone() for t in cache.tensors]
    for t, b in zip(cache.tensors, before):
        t.copy_(b)
    col = 20 // page if at == "first" else (new + 20 - 1) // page  # of the pages that sequence 0's new tokens go to
    true = int(table[0, col])
    assert not torch.equal(want[2][true], before[2][true]) or not torch.equal(want[0][true], before[0][true])
    table[0, col] = d["pages"] if bad == "pages" else bad
    q_out = torch.empty_like(x["q"])
    fsb.fs_kv_append(cache, batch, x["k"], x["v"], ct, st, q=x["q"], q_out=q_out, workspace=ws)
    with pytest.raises(fsb.FleetSieveError) as ei:
        fsb.fs_kv_check(ws)
    assert ei.value.code == fsb.FS_EDEVICE and "page" in str(ei.value)
    assert torch.equal(q_out, q_good)
    for t, w, b in zip(cache.tensors, want, before):
        w[true] = b[true]
        assert torch.equal(t, w)
