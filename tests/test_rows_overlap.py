"""Operands that share bytes are refused (csrc/fs_rows_overlap.h): the rule against every pair of rows, and through the calls."""

import ctypes as C
import random
import subprocess

import pytest

from paper_2608_19659_gb300 import _build
from test_mm_refusals import P16, call, good, refused

HARNESS = r"""
#include "fs_rows_overlap.h"
extern "C" int meet(const int64_t* a, const int64_t* b) {
  return fs::rows_overlap({a[0], a[1], a[2], a[3]}, {b[0], b[1], b[2], b[3]});
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    at = tmp_path_factory.mktemp("overlap")
    (at / "h.cpp").write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC",
                    "-static-libubsan", "-I", _build.CSRC, str(at / "h.cpp"), "-o", str(at / "h.so")], check=True)
    f = C.CDLL(str(at / "h.so")).meet
    return lambda a, b: bool(f((C.c_int64 * 4)(*a), (C.c_int64 * 4)(*b)))


def pairs(a, b):
    """(first byte, rows, width, step) each: every row of one against every row of the other."""
    return any(a[0] + i * a[3] < b[0] + j * b[3] + b[2] and b[0] + j * b[3] < a[0] + i * a[3] + a[2]
               for i in range(a[1]) for j in range(b[1]))


def test_every_pair_of_rows(meet):
    rng, seen = random.Random(1), {True: 0, False: 0}
    for _ in range(60000):
        a, b = ((rng.randint(0, 60), rng.choice((1, 2, 3, 4, 9)), w, rng.randint(w, w + rng.choice((0, 2, 9, 30)))) for w in
                (rng.randint(1, 9) for _ in range(2)))
        want = pairs(a, b)
        seen[want] += 1
        assert meet(a, b) == meet(b, a) == want, (a, b)
    assert min(seen.values()) > 5000


def test_many_rows_far_apart(meet):
    """Rows beyond what can be gone through one by one, and what no memory holds."""
    n, far = 1 << 24, (1 << 39) - 16
    assert not meet((0, n, 64, 256), (64, n, 64, 256)) and not meet((0, n, 64, 256), (64, n // 2, 64, 512))
    assert meet((0, n, 64, 256), (64, n, 193, 256)) and meet((0, n, 64, 256), (64, n, 64, 272))
    # 1008 and 1024 bytes apart: row j of one is 16 j bytes further in a row of the other
    assert not meet((0, 31, 16, 1008), (512, 31, 16, 1024)) and meet((0, 33, 16, 1008), (512, 33, 16, 1024))
    assert not meet((0, n, 64, far), (64, n, 64, far)) and meet((0, n, 64, far), (far - 63, n, 64, far))
    assert not meet((0, 1, 1 << 41, 1 << 41), (1 << 41, n, 64, far)) and meet((0, 1, (1 << 41) + 1, 0), (1 << 41, n, 64, far))
    assert not meet((1 << 47, n, 64, far), (64, 1, 64, 64))


def test_quantise(fsb):
    """Three rows of 20, 64 bytes apart, with codes 32 bytes apart from the first row's 16th byte on."""
    x, c = fsb.fs_mm_rows(P16, 32, None), fsb.fs_mm_rows(P16 + 16, 32, None)
    refused(fsb, fsb.lib().fs_quantise_rows(3, 20, 0, C.byref(x), C.byref(c), 1 << 20, None))
    assert b"overlap" in fsb.lib().fs_last_error()


@pytest.mark.parametrize("name,out,others", [("fs_linear", "y", ("x", "w", "residual")), ("fs_gated_ff", "y", ("x", "w_gate", "w_up")),
                                             ("fs_gated_ff_backward", "dx", ("x", "w_gate", "dy", "dw_up")),
                                             ("fs_gated_ff_backward", "dw_gate", ("x", "w_up", "dy"))])
def test_rows_of_different_strides(fsb, name, out, others):
    for other in others:
        for off in (16, 48, -16):  # (rows of 64 bytes, 20 to 40 of them used, against rows 80 bytes apart)
            a = good(fsb)[name]
            getattr(a, out).data = getattr(a, other).data + off
            getattr(a, out).stride = 40
            refused(fsb, call(fsb, name, a))
            assert b"overlap" in fsb.lib().fs_last_error()
