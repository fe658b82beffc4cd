"""The serving-step operators, as measurable cases: a paged 8-bit cache of keys and
values, and the attention that reads it.

What a rank of a serving replica does per layer and step:

  append   fs_kv_append: the new tokens' keys and values, rotated by position, go
           into e4m3 pages with one power-of-two scale per (page, head); their
           queries are rotated too;
  attend   fs_kv_attend: every new token attends to its sequence's cached tokens
           up to its own position (or a window of them);
  step     both, one after the other.

The replica has 64 query heads and 8 key heads; a rank of TP degree tau in
{1, 2, 4, 8} holds 64 / tau and 8 / tau of them. Lengths are a function of the
case, everything else comes from the seed.
"""

import math
import random

import torch

own = False

E4M3_MAX = 448.0


# ------------------------------------------------------------------ cases

def _case(op, batch, new, ctx, tp=1, **more):
    c = {"op": op, "batch": batch, "new": new, "ctx": ctx, "tp": tp, "hq": 64 // tp, "hkv": 8 // tp, "dim": 128,
         "page": 64, "dtype": "bfloat16", "ragged": True, "window": 0, "rot": 128, "interleaved": False}
    c.update(more)
    return c


def listed():
    def named(name, c):
        return dict(c, name=name)

    return [
        # one request's next token on a rank of TP 8: all latency
        named("append_one", _case("append", 1, 1, 1000, tp=8)),
        # the next token of 256 requests of all lengths
        named("append_256", _case("append", 256, 1, 4096)),
        # chunks of ragged prompts, odd sizes, interleaved pairs, part of the dimensions rotated
        named("append_ragged", _case("append", 7, 777, 2500, tp=2, dtype="float16", page=16, rot=64, interleaved=True)),
        # the largest: a batch of prompts at once
        named("append_prompts", _case("append", 8, 4096, 4096)),
        # one request's next token on a rank of TP 8, short context: all latency
        named("attend_one", _case("attend", 1, 1, 1000, tp=8)),
        # a middling load bin of ragged requests, small pages, heads of 64
        named("attend_mid", _case("attend", 33, 1, 5000, tp=2, dim=64, page=16, rot=64, dtype="float16")),
        # a long context alone: the work has to be split along it
        named("attend_long", _case("attend", 1, 1, 131072, tp=8, ragged=False)),
        # the highest load bin: 64 long requests
        named("attend_load", _case("attend", 64, 1, 32768)),
        # five proposed tokens of 16 requests are verified under a sliding window
        named("attend_verify", _case("attend", 16, 5, 9001, tp=4, window=4096, page=32)),
        # ragged prompt chunks on top of what is cached
        named("attend_chunks", _case("attend", 6, 1111, 3001, tp=4)),
        # a long prompt at once
        named("attend_prompt", _case("attend", 1, 8192, 8192, tp=2, ragged=False)),
        # a decode step's two calls together
        named("step_64", _case("step", 64, 1, 8192, tp=2)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "append", "attend", "attend", "attend", "step"))
    tp = rng.choice((1, 2, 4, 8))
    dim = rng.choice((64, 128, 128))
    more = {"dim": dim, "page": rng.choice((16, 32, 64, 128)), "dtype": rng.choice(("bfloat16", "bfloat16", "float16")),
            "ragged": rng.random() < 0.8, "interleaved": rng.random() < 0.3, "rot": rng.choice((dim, dim, dim // 2))}
    kind = rng.choice(("decode", "decode", "verify", "chunk"))
    if kind == "chunk":
        new = _log_int(rng, 16, 4096)
        ctx = new + _log_int(rng, 1, 4096)
        batch = max(1, min(_log_int(rng, 1, 16), 16384 // new, (1 << 31) // (64 // tp * new * ctx)))
    else:
        new = 1 if kind == "decode" else rng.randint(2, 9)
        ctx = _log_int(rng, 16, 65536)
        batch = max(1, min(_log_int(rng, 1, 256), (1 << 21) // ctx))
    if rng.random() < 0.25:
        more["window"] = _log_int(rng, 16, max(17, ctx))
    return _case(op, batch, new, ctx, tp, **more)


def lengths(case):
    """Per sequence (tokens cached after the call, of these new in the call). Ragged: lengths over
    the whole range, one of them the largest; a slot in ten holds no request."""
    B, N, L = case["batch"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [(L, min(N, L))] * B
    rng = random.Random("%d %d %d %d %d" % (B, N, L, case["page"], case["tp"]))
    out = []
    for b in range(B):
        if b == 0:
            out.append((L, min(N, L)))
        elif rng.random() < 0.1:
            out.append((0, 0))
        else:
            n = N if N < 16 else rng.randint(1, N)
            out.append((max(n, rng.randint(1, L)), n))
    rng.shuffle(out)
    return out


# ------------------------------------------------------------------ inputs

class State:
    pass


def _quantise_pages(x, amax):
    """x [n, H, P, D] in e4m3 with a power-of-two scale per (page, head)."""
    m, e = torch.frexp(amax.float())
    s = torch.ldexp(torch.ones_like(m), e - torch.where(m <= 0.875, 9, 8))
    return (x / s[:, :, None, None]).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), s


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(int(seed))
    B, H, Hq, D, P = case["batch"], case["hkv"], case["hq"], case["dim"], case["page"]
    dt = getattr(torch, case["dtype"])
    ls = lengths(case)
    need = [-(-l // P) for l, _ in ls]
    pages = sum(need) + 3
    s = State()
    # which page holds what: any order, as after many requests have come and gone
    perm = torch.randperm(pages, generator=g, device=dev, dtype=torch.int64).to(torch.int32)
    width = max(1, max(need))
    first = torch.tensor([sum(need[:b]) for b in range(B)], device=dev)
    cols = torch.arange(width, device=dev)[None, :]
    held = cols < torch.tensor(need, device=dev)[:, None]
    s.page_table = torch.where(held, perm[(first[:, None] + cols).clamp_max(pages - 1)], 0).to(torch.int32).contiguous()
    s.length = torch.tensor([l for l, _ in ls], dtype=torch.int32, device=dev)
    starts = [0]
    for _, n in ls:
        starts.append(starts[-1] + n)
    s.q_start = torch.tensor(starts, dtype=torch.int32, device=dev)
    s.tokens, s.max_new, s.max_length = starts[-1], max(n for _, n in ls), max(l for l, _ in ls)
    # cached keys (some channels larger than others) and values; pages differ in magnitude
    s.k, s.v = (torch.empty(pages, H, P, D, dtype=torch.float8_e4m3fn, device=dev) for _ in range(2))
    s.k_scale, s.v_scale = (torch.empty(pages, H, device=dev) for _ in range(2))
    gain = torch.exp(0.5 * torch.randn(H, 1, D, generator=g, device=dev))
    piece = max(1, (1 << 27) // (H * P * D))
    for a in range(0, pages, piece):
        b = min(pages, a + piece)
        for to, sc, f in ((s.k, s.k_scale, gain), (s.v, s.v_scale, 1.0)):
            x = torch.randn(b - a, H, P, D, generator=g, device=dev)
            x.mul_(f).mul_(torch.exp(0.2 * torch.randn(b - a, H, 1, 1, generator=g, device=dev)))
            to[a:b], sc[a:b] = _quantise_pages(x, x.abs().amax((2, 3)))
    # one projection's output holds queries, keys and values side by side
    qkv = torch.randn(s.tokens, Hq + 2 * H, D, generator=g, device=dev)
    qkv[:, :Hq] *= 2  # so that some keys count far more than others
    qkv = qkv.to(dt)
    s.q, s.new_k, s.new_v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    rot = case["rot"]
    angle = torch.arange(s.max_length, device=dev).float()[:, None] * (10000.0 ** (-torch.arange(rot // 2, device=dev).float() * 2 / rot))
    s.cos, s.sin = angle.cos(), angle.sin()
    s.q_out, s.out = (torch.empty(s.tokens, Hq, D, dtype=dt, device=dev) for _ in range(2))
    s.scale = D ** -0.5
    s.case = case
    if own:
        from paper_2608_19659_gb300 import fleetsieve as fsb

        s.fsb = fsb
        s.cache = fsb.KvCache(s.k, s.v, s.k_scale, s.v_scale)
        s.batch = fsb.KvBatch(s.page_table, s.length, s.q_start, s.tokens, s.max_new, s.max_length)
        s.work = fsb.KvWorkspace(s.cache, s.batch, Hq)
    return s


# ------------------------------------------------------------------ the plain forms

def _rows(s):
    """Per new token: its sequence and its position."""
    t = torch.arange(s.tokens, device="cuda")
    b = torch.searchsorted(s.q_start[1:].long(), t, right=True)
    return b, (s.length[b] - s.q_start[b + 1]).long() + t


def _rotate(x, c, s, rot, interleaved):
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    c, s = c[:, None], s[:, None]
    y0, y1 = a * c - b * s, b * c + a * s
    y = torch.stack((y0, y1), -1).flatten(-2) if interleaved else torch.cat((y0, y1), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _store(cache, scale, y, s, page, slot, P):
    """New tokens' values y [tokens, H, D] into their pages, whose scales may grow."""
    amax = torch.zeros_like(scale).index_reduce_(0, page, y.abs().amax(-1), "amax")
    m, e = torch.frexp(amax)
    need = torch.where(amax > 0, torch.ldexp(torch.ones_like(m), (e - torch.where(m <= 0.875, 9, 8)).clamp_min(-126)), 0.0)
    begun = torch.zeros_like(scale).index_reduce_(0, page, (slot == 0).float()[:, None].expand(-1, scale.shape[1]), "amax")
    old = torch.where(begun > 0, 0.0, scale)
    new = torch.maximum(old, need)
    # the page that a sequence's first new token goes into holds older tokens before it
    start = (s.length - (s.q_start[1:] - s.q_start[:-1])).long()
    at = s.page_table.gather(1, (start // P)[:, None].clamp_max(s.page_table.shape[1] - 1))[:, 0].long()
    was = cache[at]
    factor = torch.where(new[at] > 0, old[at] / new[at], 1.0)[:, :, None, None]
    kept = (torch.arange(P, device="cuda")[None, :] < (start % P)[:, None]) & (s.q_start[1:] > s.q_start[:-1])[:, None]
    now = (was.float() * factor).to(torch.float8_e4m3fn)
    # sequences without new tokens write nothing: their rows go where another's does, with the same bytes
    some = torch.argmax((s.q_start[1:] > s.q_start[:-1]).int())
    whose = torch.where(s.q_start[1:] > s.q_start[:-1], torch.arange(at.shape[0], device="cuda"), some)
    cache.view(torch.uint8)[at[whose]] = torch.where(kept[:, None, :, None], now.view(torch.uint8), was.view(torch.uint8))[whose]
    touched = torch.zeros_like(scale).index_fill_(0, page, 1.0)
    scale.copy_(torch.where(touched > 0, new, scale))
    inv = torch.where(new > 0, 1.0 / new, 0.0)[page]
    cache.view(torch.uint8)[page, :, slot] = (y * inv[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def _append(s):
    c, P = s.case, s.case["page"]
    b, pos = _rows(s)
    page, slot = s.page_table[b, pos // P].long(), pos % P
    cos, sin = s.cos[pos], s.sin[pos]
    _store(s.k, s.k_scale, _rotate(s.new_k.float(), cos, sin, c["rot"], c["interleaved"]), s, page, slot, P)
    _store(s.v, s.v_scale, s.new_v.float(), s, page, slot, P)
    s.q_out.copy_(_rotate(s.q.float(), cos, sin, c["rot"], c["interleaved"]))


def _attend(s, q):
    c = s.case
    B, H, D, P, N = c["batch"], c["hkv"], c["dim"], c["page"], s.max_new
    G = c["hq"] // H
    at = s.page_table.long()
    L = at.shape[1] * P
    k = (s.k[at].float() * s.k_scale[at][..., None, None]).transpose(1, 2).reshape(B, H, L, D)
    count = (s.q_start[1:] - s.q_start[:-1]).long()
    i = torch.arange(N, device="cuda")
    row = (s.q_start[:-1].long()[:, None] + i).clamp_max(s.tokens - 1)
    qp = q[row].float().view(B, N, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, N * G, D)
    x = (qp @ k.transpose(-1, -2)).mul_(s.scale).view(B, H, N, G, L)
    del k
    pos = (s.length - count.int()).long()[:, None] + i
    j = torch.arange(L, device="cuda")
    seen = j <= pos[..., None]
    if c["window"]:
        seen &= j > pos[..., None] - c["window"]
    x.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = x.sum(-1, keepdim=True)
    v = (s.v[at].float() * s.v_scale[at][..., None, None]).transpose(1, 2).reshape(B, H, L, D)
    o = (x.view(B, H, N * G, L) @ v).view(B, H, N, G, D) / torch.where(total > 0, total, 1.0)
    # every token from its sequence's rows
    t = torch.arange(s.tokens, device="cuda")
    b = torch.searchsorted(s.q_start[1:].long(), t, right=True)
    s.out.copy_(o.permute(0, 2, 1, 3, 4).reshape(B, N, H * G, D)[b, t - s.q_start[b].long()])


# ------------------------------------------------------------------ one pass

def run(s):
    c = s.case
    if c["op"] in ("append", "step"):
        if own:
            s.fsb.fs_kv_append(s.cache, s.batch, s.new_k, s.new_v, s.cos, s.sin, q=s.q, q_out=s.q_out,
                               interleaved=c["interleaved"], workspace=s.work)
        else:
            _append(s)
    if c["op"] in ("attend", "step"):
        q = s.q_out if c["op"] == "step" else s.q
        if own:
            s.fsb.fs_kv_attend(s.cache, s.batch, q, s.out, s.scale, window=c["window"], workspace=s.work)
        else:
            _attend(s, q)
    if c["op"] == "attend":
        return {"out": s.out}
    r = {"k": s.k, "v": s.v, "k_scale": s.k_scale, "v_scale": s.v_scale, "q": s.q_out}
    if c["op"] == "step":
        r["out"] = s.out
    return r


def _seen(case, length, new):
    """(query, key) pairs of a sequence, and the keys that any of its queries sees."""
    w = case["window"] or length + 1
    pairs = sum(min(p + 1, w) for p in range(length - new, length))
    return pairs, length - max(0, length - new - w + 1) if new else 0


def work(case):
    D, H, Hq, P = case["dim"], case["hkv"], case["hq"], case["page"]
    nbytes = flops = 0
    for l, n in lengths(case):
        if case["op"] in ("append", "step"):
            # keys, values and queries in; 8-bit keys and values and queries out; the tables' rows; pages' scales
            nbytes += n * (2 * H * D * 3 + Hq * D * 4 + case["rot"] * 4)
            nbytes += 2 * H * 4 * (-(-l // P) - (l - n) // P if n else 0)
            flops += n * 3 * (H + Hq) * case["rot"] + n * 2 * H * D * 2
        if case["op"] in ("attend", "step"):
            pairs, keys = _seen(case, l, n)
            nbytes += keys * H * D * 2 + n * Hq * D * 4 + 2 * H * 4 * -(-keys // P)
            flops += pairs * Hq * D * 4
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ 64 bits

def _code_values():
    """What each e4m3 code stands for, by its definition."""
    v = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if c & 127 == 127 else m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v.append(-x if c & 128 else x)
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _nearest_code_value(x):
    """x (|x| <= 448) rounded to the nearest e4m3 value, ties to the even code."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(s, case):
    values = _code_values()
    P, D, rot = case["page"], case["dim"], case["rot"]
    out = {"q": torch.empty(s.q_out.shape, dtype=torch.float64, device="cuda")}
    caches = {n: values[getattr(s, n).view(torch.uint8).long()] for n in ("k", "v")}
    scales = {n: getattr(s, n + "_scale").double() for n in ("k", "v")}
    table, first = s.page_table.tolist(), s.q_start.tolist()

    def turned(x, pos):
        y = x.clone()
        c, si = s.cos[pos].double()[:, None, :], s.sin[pos].double()[:, None, :]
        i = torch.arange(rot // 2, device="cuda")
        lo, hi = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
        y[..., lo] = x[..., lo] * c - x[..., hi] * si
        y[..., hi] = x[..., hi] * c + x[..., lo] * si
        return y

    for b, (l, n) in enumerate(lengths(case)):
        if not n:
            continue
        pos = torch.arange(l - n, l, device="cuda")
        new = {"k": turned(s.new_k[first[b]:first[b] + n].double(), pos), "v": s.new_v[first[b]:first[b] + n].double()}
        out["q"][first[b]:first[b] + n] = turned(s.q[first[b]:first[b] + n].double(), pos)
        for j in range((l - n) // P, (l - 1) // P + 1):
            lo, hi = max(l - n, j * P), min(l, (j + 1) * P)
            g = table[b][j]
            for name in ("k", "v"):
                y = new[name][lo - (l - n):hi - (l - n)]
                a = y.abs().amax((0, 2))
                need = torch.where(a > 0, torch.exp2(torch.ceil(torch.log2(a / E4M3_MAX))), 0.0)
                old = scales[name][g] if lo > j * P else torch.zeros_like(need)
                now = torch.maximum(old, need)
                safe = torch.where(now > 0, now, 1.0)
                page = caches[name][g]
                if lo > j * P:
                    page[:, :lo - j * P] = _nearest_code_value(page[:, :lo - j * P] * (old / safe)[:, None, None])
                page[:, lo - j * P:hi - j * P] = _nearest_code_value((y / safe[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)).transpose(0, 1)
                scales[name][g] = now
    out.update(k=caches["k"], v=caches["v"], k_scale=scales["k"], v_scale=scales["v"])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    D, H, Hq, P = case["dim"], case["hkv"], case["hq"], case["page"]
    r = {}
    k, v, ks, vs, q = s.k, s.v, s.k_scale, s.v_scale, s.q
    values = _code_values()
    as_values = lambda x: values[x.view(torch.uint8).long()]  # noqa: E731
    if case["op"] in ("append", "step"):
        if sum(n for _, n in lengths(case)) > 20000 or s.k.numel() > 1 << 30:
            return None
        r = _exact_append(s, case)
        k, v, ks, vs, q = r["k"], r["v"], r["k_scale"], r["v_scale"], r["q"]
        as_values = lambda x: x  # noqa: E731
    if case["op"] in ("attend", "step"):
        if work(dict(case, op="attend"))["flops"] > 4e12:
            return None
        out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
        first = s.q_start.tolist()
        for b, (l, n) in enumerate(lengths(case)):
            if not n:
                continue
            at = s.page_table[b, :-(-l // P)].long()
            pos = torch.arange(l - n, l, device="cuda")
            for h in range(H):
                kk = (as_values(k[at, h]) * ks[at, h].double()[:, None, None]).reshape(-1, D)[:l]
                vv = (as_values(v[at, h]) * vs[at, h].double()[:, None, None]).reshape(-1, D)[:l]
                heads = slice(h * (Hq // H), (h + 1) * (Hq // H))
                x = torch.einsum("thd,ld->htl", q[first[b]:first[b] + n, heads].double(), kk) * s.scale
                j = torch.arange(l, device="cuda")[None, :]
                ok = (j <= pos[:, None]) & ((j > pos[:, None] - case["window"]) if case["window"] else True)
                p = torch.softmax(torch.where(ok[None], x, -math.inf), -1)
                out[first[b]:first[b] + n, heads] = torch.einsum("htl,ld->thd", p, vv)
        r["out"] = out
    return r
