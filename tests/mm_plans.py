"""The products' tiles and order (csrc/fs_mm_plan.h) as a test asks for them."""

import ctypes as C
import dataclasses
import functools
import os
import subprocess
import tempfile

from paper_2608_19659_gb300 import _build

HARNESS = r"""
#include "fs_mm_plan.h"
extern "C" int wide(int rows, int cols, int blocks, int gated, int sms) {
  float ns;
  return fs::mm_wide_tile(rows, cols, blocks, gated, sms, &ns);
}
extern "C" int few(int rows, int cols, int blocks, int gated, int sms, int* out) {
  float ns;
  fs::mm_wide_tile(rows, cols, blocks, gated, sms, &ns);
  const fs::MmFewPlan p = fs::mm_few_plan(rows, cols, blocks, gated, sms);
  out[0] = p.w_rows, out[1] = p.tokens, out[2] = p.token_tiles, out[3] = p.w_tiles, out[4] = p.cluster, out[5] = p.stages, out[6] = fs::bars_at(p, rows);
  return p.ns < ns;
}
extern "C" void grad(int rows, int in, int out, int sms, int* p) {
  const fs::MmGradPlan g = fs::mm_grad_plan(rows, in, out, sms);
  p[0] = g.dw_first, p[1] = g.tile, p[2] = g.lead, p[3] = g.rounds;
}
extern "C" long long terms(int rows, int out) { return fs::mm_terms(rows, out); }
extern "C" int next_tile(int i, int k, int first, int step, int lead, int rounds) { return fs::mm_next_tile(i, k, first, step, lead, rounds); }
"""


@functools.cache
def lib():
    with tempfile.TemporaryDirectory() as at:
        src, so = os.path.join(at, "h.cpp"), os.path.join(at, "h.so")
        with open(src, "w") as f:
            f.write(HARNESS)
        subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", _build.CSRC, src, "-o", so], check=True)
        loaded = C.CDLL(so)
        loaded.terms.restype = C.c_longlong
        return loaded


def up(a, b):
    return -(-a // b)


def blocks(inner, eight=False):
    return up(inner, 128 if eight else 64)


def wide(rows, inner, out, eight=False, gated=False, sms=152):
    """(columns of a tile, tiles) of k_mm_wide."""
    tile = lib().wide(rows, out, blocks(inner, eight), gated, sms)
    return tile, up(rows, 256) * up(out, tile // 2 if gated else tile)


@dataclasses.dataclass
class Few:
    w_rows: int
    tokens: int
    token_tiles: int
    w_tiles: int
    cluster: int
    stages: int
    bytes: int
    taken: bool  # rather than k_mm_wide


def few(rows, inner, out, eight=False, gated=False, sms=152):
    p = (C.c_int * 7)()
    taken = lib().few(rows, out, blocks(inner, eight), gated, sms, p)
    return Few(*p, bool(taken))


@dataclasses.dataclass
class Grad:
    dw_first: bool
    tile: int
    lead: int
    rounds: int
    tiles: int


def grad(rows, inner, out, sms=152):
    p = (C.c_int * 4)()
    lib().grad(rows, inner, out, sms, p)
    return Grad(bool(p[0]), *p[1:], (up(rows, 256) + 2 * up(out, 256)) * up(inner, p[1]))
