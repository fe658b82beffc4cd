"""A cell's optimistic bounds from the attention of one rank, or from its whole layer, timed on the GPU at hand.

Measuring a cell (class, TP degree, load bin) takes a replica of TP GPUs for 300 s
(Section 5). Before that, its intervals come from a prior (Section 4.1), and the
optimistic ends of them, capacity from above and tail from below, drive the
optimistic allocation A+. What one GPU of the replica does per decode step beside
its matrix products, appending the new tokens to its share of the cache and
attending to it, takes milliseconds to time on a single GPU, and no replica that
attends with these kernels is faster than that: with R requests in flight, contexts of
L tokens and N generated tokens a request,

    capacity <= R / (N t_step + t_prompt)   req/s per replica (R at a time),
    tail     >= N t_step + t_prompt         s,

t_step and t_prompt the rank's append and attention over all layers, on the device alone: the
layers run in CUDA graphs, as a replica may run them, so that no host's call is counted.
(R requests bring R prompts; one is counted, which leaves the capacity's bound on the safe
side.) :func:`tighten`
puts these into a model's bounds (never past the pessimistic ends), which lowers
Gamma_t and the number of measurements wherever attention alone rules a cell out.

With ``products``, what the rank computes beside its attention counts too, in 8 bits as the paper's replica serves:
the projections (fs_linear) and the gated feed-forward block (fs_gated_ff), with the rows that they read brought
to e4m3 (fs_quantise_rows). The times are then those of whole layers but for their norms and the sums over ranks,
and bound replicas that run these kernels.
"""

from __future__ import annotations

import dataclasses

import numpy as np

from . import fleetsieve as fsb
from .workloads import TP_DEGREES


@dataclasses.dataclass(frozen=True)
class Decoder:
    """The attention side of a served decoder, and how its requests look."""

    layers: int = 60
    q_heads: int = 64
    kv_heads: int = 8
    dim: int = 128
    context: int = 4096  # tokens of a request's prompt
    output: int = 256  # tokens it generates
    page: int = 64
    hidden: int = 8192  # width of a token between the layers
    block: int = 14336  # of the gated feed-forward block, over all ranks


def rank_heads(d: Decoder, tp: int) -> tuple[int, int]:
    """(query heads, key heads) of one of tp ranks; key heads are shared by ranks beyond their number."""
    if tp < 1 or d.q_heads % tp or (d.kv_heads % tp and tp % d.kv_heads):
        raise ValueError(f"{d.q_heads} query and {d.kv_heads} key heads do not split over {tp} ranks")
    return d.q_heads // tp, max(1, d.kv_heads // tp)


def rank_block(d: Decoder, tp: int) -> int:
    """Width of the gated block on one of tp ranks."""
    if tp < 1 or d.block % tp:
        raise ValueError(f"a gated block of {d.block} does not split over {tp} ranks")
    return d.block // tp


class RankProducts:
    """The products of one rank's layer beside its attention, for `tokens` tokens: 8-bit weights in as many sets as exceed the
    L2 (a replica's layers have weights of their own), and the buffers between the calls."""

    def __init__(self, d: Decoder, tp: int, tokens: int, qkv, out, g):
        import torch

        heads, block = out.shape[1] * d.dim, rank_block(d, tp)
        sizes = [(qkv[0].numel(), d.hidden), (d.hidden, heads), (block, d.hidden), (block, d.hidden), (d.hidden, block)]
        l2 = torch.cuda.get_device_properties(qkv.device).L2_cache_size
        self.sets = [[self._weight(*size, g) for size in sizes] for _ in range(-(-2 * l2 // sum(n * k for n, k in sizes)))]
        self.bias = (0.1 * torch.randn(qkv[0].numel(), generator=g, device="cuda")).to(torch.bfloat16)
        self.qkv, self.attended = qkv.view(tokens, -1), out.view(tokens, -1)
        self.x = torch.randn(tokens, d.hidden, generator=g, device="cuda").to(torch.bfloat16)  # what the layer is given
        self.mid, self.y = torch.empty_like(self.x), torch.empty_like(self.x)  # after attention, after the block
        self.inner = self._rows(tokens, block, torch.bfloat16)
        self.codes = [self._rows(tokens, n, torch.float8_e4m3fn) for n in (d.hidden, heads, d.hidden, block)]
        self.scales = [torch.empty(tokens, device="cuda") for _ in self.codes]
        most = max(max(size) for size in sizes)
        self.work = fsb.MmWorkspace(tokens, most, most)
        self.layer = 0

    @staticmethod
    def _rows(n, width, dtype):
        import torch

        return torch.empty(n, -(-width // 16) * 16, dtype=dtype, device="cuda")[:, :width]

    @classmethod
    def _weight(cls, n, k, g):
        import torch

        codes, scale = cls._rows(n, k, torch.float8_e4m3fn), torch.empty(n, device="cuda")
        for a in range(0, n, 4096):
            b = min(n, a + 4096)
            w = cls._rows(b - a, k, torch.bfloat16)
            w.copy_(torch.randn(b - a, k, generator=g, device="cuda") * k**-0.5)
            fsb.fs_quantise_rows(w, codes[a:b], scale[a:b])
        return codes, scale

    def _linear(self, i, rows, y, weight, **more):
        codes, scale = fsb.fs_quantise_rows(rows, self.codes[i], self.scales[i])
        w, w_scale = self.sets[self.layer][weight]
        fsb.fs_linear(codes, w, y, x_scale=scale, w_scale=w_scale, workspace=self.work, **more)

    def before(self) -> None:
        """Queries, keys and values of the layer's rows."""
        self.layer = (self.layer + 1) % len(self.sets)
        self._linear(0, self.x, self.qkv, 0, bias=self.bias)

    def after(self) -> None:
        """The rest of the layer, from what attention gave."""
        self._linear(1, self.attended, self.mid, 1, residual=self.x)
        codes, scale = fsb.fs_quantise_rows(self.mid, self.codes[2], self.scales[2])
        (gate, gate_scale), (up, up_scale) = self.sets[self.layer][2:4]
        fsb.fs_gated_ff(codes, gate, up, self.inner, x_scale=scale, gate_scale=gate_scale, up_scale=up_scale, workspace=self.work)
        self._linear(3, self.inner, self.y, 4, residual=self.mid)


class RankStep:
    """One rank's cache and buffers for `requests` requests of a decoder, and the calls of a layer's
    step over them: append and attention, with ``products`` the rest of the layer too. All layers of a step use the same pages here: a cache that fits the L2 is read faster than
    a replica's layers read theirs, and what is timed bounds those from below all the same."""

    def __init__(self, d: Decoder, tp: int, requests: int, new: int = 1, seed: int = 0, length: int | None = None,
                 products: bool = False):
        import torch

        hq, hk = rank_heads(d, tp)
        if length is None:
            length = d.context if new > 1 else d.context + d.output // 2  # a prompt, or a request half way
        g = torch.Generator(device="cuda").manual_seed(seed)
        per = -(-length // d.page)
        pages = requests * per
        shape = (pages, hk, d.page, d.dim)
        self.cache = fsb.KvCache(*(torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2)),
                                 *(torch.zeros(pages, hk, device="cuda") for _ in range(2)))
        table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(requests, per)
        tokens = requests * new
        self.batch = fsb.KvBatch(table, torch.full((requests,), length, dtype=torch.int32, device="cuda"),
                                 torch.arange(0, tokens + 1, new, dtype=torch.int32, device="cuda"), tokens, new, length)
        self.qkv = torch.randn(tokens, hq + 2 * hk, d.dim, generator=g, device="cuda").to(torch.bfloat16)
        self.q, self.k, self.v = self.qkv[:, :hq], self.qkv[:, hq:hq + hk], self.qkv[:, hq + hk:]
        self.out = torch.empty(tokens, hq, d.dim, dtype=torch.bfloat16, device="cuda")
        angle = torch.arange(length, device="cuda").float()[:, None] * 10000.0 ** (
            -torch.arange(d.dim // 2, device="cuda").float() * 2 / d.dim)
        self.cos, self.sin = angle.cos(), angle.sin()
        self.work = fsb.KvWorkspace(self.cache, self.batch, hq)
        self.scale = d.dim**-0.5
        self._fill(d, requests, per, hk, length, g)
        self.products = RankProducts(d, tp, tokens, self.qkv, self.out, g) if products else None

    def _fill(self, d, requests, per, hk, length, g):
        """Keys and values for the tokens already cached, through the cache's own append."""
        import torch

        old = length - self.batch.tokens // requests
        if old == 0:
            return
        batch = fsb.KvBatch(self.batch.tensors[0], torch.full((requests,), old, dtype=torch.int32, device="cuda"),
                            torch.arange(0, requests * old + 1, old, dtype=torch.int32, device="cuda"), requests * old,
                            old, old)
        kv = torch.randn(requests * old, hk, d.dim, generator=g, device="cuda").to(torch.bfloat16)
        fsb.fs_kv_append(self.cache, batch, kv, kv, self.cos, self.sin, workspace=self.work)

    def layer(self) -> None:
        """One layer: the new tokens into the cache (queries rotated in place), and their attention; with products,
        queries, keys and values are made before, and the layer's rows after."""
        if self.products:
            self.products.before()
        fsb.fs_kv_append(self.cache, self.batch, self.k, self.v, self.cos, self.sin, q=self.q, q_out=self.q,
                         workspace=self.work)
        fsb.fs_kv_attend(self.cache, self.batch, self.q, self.out, self.scale, workspace=self.work)
        if self.products:
            self.products.after()

    def check(self) -> None:
        """Waits, and raises what the calls met on the device."""
        fsb.fs_kv_check(self.work)
        if self.products:
            fsb.fs_mm_check(self.products.work)

    def seconds(self, layers: int, repeats: int = 8) -> float:
        """Time of `layers` layers on the device: what a graph of twice n layers takes longer than one of n (the best
        of `repeats` runs of each, after an untimed one), so that neither the host nor a graph's start counts."""
        import torch

        n = -(-16 // layers) * layers
        self.layer()  # (what a first call sets up does not belong into a capture)
        self.check()
        graphs = {n: torch.cuda.CUDAGraph(), 2 * n: torch.cuda.CUDAGraph()}
        for count, graph in graphs.items():
            with torch.cuda.graph(graph):
                for _ in range(count):
                    self.layer()
        best = dict.fromkeys(graphs, float("inf"))
        for i in range(repeats + 1):
            for count, graph in graphs.items():
                begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                begin.record()
                graph.replay()
                end.record()
                end.synchronize()
                if i:
                    best[count] = min(best[count], begin.elapsed_time(end) * 1e-3)
        self.check()
        return (best[2 * n] - best[n]) * layers / n


@dataclasses.dataclass
class Probe:
    """What a rank's attention, or its layers, bound a cell by."""

    tp: int
    requests: int
    step_seconds: float
    prompt_seconds: float
    cap_hi: float  # req/s per replica, no more
    tail_lo: float  # s, no less


def probe_cell(d: Decoder, tp: int, requests: int, layers_timed: int = 4, products: bool = False) -> Probe:
    """Times one rank of TP degree tp with `requests` requests in flight (layers_timed of the decoder's
    layers, the rest counted like them): its attention, or with ``products`` its layers."""
    more = {"products": True} if products else {}
    step = RankStep(d, tp, requests, **more).seconds(layers_timed) * d.layers / layers_timed
    prompt = RankStep(d, tp, 1, new=d.context, length=d.context, **more).seconds(layers_timed) * d.layers / layers_timed
    tail = d.output * step + prompt
    return Probe(tp, requests, step, prompt, requests / (d.output * step + prompt), tail)


def tighten(cap_lo, cap_hi, tail_lo, tail_hi, cls: int, tp: int, b: int, p: Probe):
    """The bounds [K, 4, B] with cell (cls, tp, b) no better than the probe: cap_hi down to, tail_lo up
    to what it found, neither past the other end of its interval. Returns new arrays."""
    j = TP_DEGREES.index(tp)
    out = [np.array(x, np.float32) for x in (cap_lo, cap_hi, tail_lo, tail_hi)]
    at = (cls, j, b)
    out[1][at] = max(out[0][at], min(out[1][at], np.float32(p.cap_hi)))
    out[2][at] = min(out[3][at], max(out[2][at], np.float32(p.tail_lo)))
    return tuple(out)


def main(argv=None) -> None:
    """Probes every (TP degree, load bin) of the paper-scale grid for one class's requests, bin b taken as 2^b
    requests in flight (the grid's bins are ordered by load and say no more), and prints, as one JSON line, the gap
    between the optimistic and the conservative allocation before and after, and how many of the cells' bounds
    moved. With ordinary requests and attention alone none of this grid's do; generations of 16384 tokens and more move some."""
    import argparse
    import json

    import torch

    from . import workloads

    ap = argparse.ArgumentParser(description=main.__doc__)
    ap.add_argument("--context", type=int, default=4096)
    ap.add_argument("--output", type=int, default=256)
    ap.add_argument("--layers", type=int, default=60)
    ap.add_argument("--cls", type=int, default=0, help="class whose cells are probed")
    ap.add_argument("--demand", type=float, default=3.0, help="factor on the workload's demands (1: the fleet is never short)")
    ap.add_argument("--products", action="store_true", help="time whole layers: projections and the gated block too")
    a = ap.parse_args(argv)
    if not torch.cuda.is_available():
        raise SystemExit("the probe times a rank's attention on a CUDA device")
    w = workloads.make_workload(1)
    d = Decoder(context=a.context, output=a.output, layers=a.layers)
    bounds = (w.cap_lo, w.cap_hi, w.tail_lo, w.tail_hi)
    demand = w.demand * np.float32(a.demand)
    probes = []
    with fsb.fs_load_model(*bounds, w.slo, demand, w.G, w.K, w.B) as m:
        before = fsb.fs_solve_bounds(m)
        for tp in workloads.TP_DEGREES:
            for b in range(w.B):
                p = probe_cell(d, tp, 1 << b, products=a.products)
                bounds = tighten(*bounds, a.cls, tp, b, p)
                probes.append(dataclasses.asdict(p) | {"bin": b})
        fsb.fs_update_bounds(m, *bounds)
        after = fsb.fs_solve_bounds(m)
    moved = sum(int((x != y).sum()) for x, y in zip(bounds, (w.cap_lo, w.cap_hi, w.tail_lo, w.tail_hi)))
    print(json.dumps({"class": a.cls, "products": a.products, "decoder": dataclasses.asdict(d), "gamma_before": before[2], "gamma_after": after[2],
                      "bounds_moved": moved, "probes": probes}))


if __name__ == "__main__":
    main()
