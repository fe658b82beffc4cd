"""The products' plans on the CPU: what a launch may be given, and that every tile is taken once."""

import math
import random

import pytest

import mm_plans


def sizes(seed, n, *most):
    rng = random.Random(seed)
    for _ in range(n):
        yield tuple(max(1, round(math.exp(rng.uniform(0, math.log(m))))) for m in most)


@pytest.mark.parametrize("sms", [2, 20, 152])
def test_few_rows_fit_an_sm(sms):
    """Stages, clusters and shared memory within what a block may have, two blocks' where two are meant for an SM."""
    for rows, inner, out in sizes(sms, 4000, 1024, 20000, 20000):
        for eight in (False, True):
            for gated in (False, True):
                p, blocks = mm_plans.few(rows, inner, out, eight, gated, sms), mm_plans.blocks(inner, eight)
                assert p.w_rows in (32, 64, 128) and p.tokens % 16 == 0 and 16 <= p.tokens <= 128
                assert 1 <= p.cluster <= min(8, blocks) and 2 <= p.stages <= 12
                assert p.tokens * p.token_tiles >= rows > (p.token_tiles - 1) * p.tokens
                assert p.w_tiles * (p.w_rows // 2 if gated else p.w_rows) >= out
                assert p.stages * (p.w_rows + p.tokens) * 128 <= p.bytes <= 216 * 1024


@pytest.mark.parametrize("sms", [2, 20, 152])
def test_every_gradient_tile_is_taken_once(sms):
    pairs, led = sms // 2, 0
    for rows, inner, out in sizes(sms, 1500, 9000, 5000, 9000):
        p = mm_plans.grad(rows, inner, out, sms)
        assert p.tile in (128, 256) and p.rounds >= 1 and 0 <= p.lead < pairs
        step, led = min(p.tiles, pairs), led + (p.lead > 0)
        assert not p.lead or step == pairs
        seen = []
        for first in range(step):
            i, k = first, 0
            while i < p.tiles:
                seen.append(i)
                k += 1
                then = mm_plans.lib().next_tile(i, k, first, step, p.lead, p.rounds)
                assert then > i
                i = then
        assert sorted(seen) == list(range(p.tiles)), (rows, inner, out, p)
    assert sms == 2 or led > 20


def test_the_terms_of_smaller_sizes_fit():
    """A workspace's room for dg, du and their second terms: never less for a larger size, and enough for its own."""
    lib = mm_plans.lib()
    for rows, out in sizes(3, 4000, 9000, 9000):
        most = lib.terms(rows, out)
        two = rows <= 64 or out <= 64
        assert most >= (4 if two else 2) * rows * mm_plans.up(out, 64) * 64
        for r, o in sizes(rows + out, 6, rows, out):
            assert lib.terms(r, o) <= most
    assert [lib.terms(*s) for s in ((64, 64), (65, 64), (65, 256), (10000, 64), (10000, 65), (0, 5), (5, 0))] == [
        4 * 64 * 64, 4 * 65 * 64, 4 * 64 * 256, 4 * 10000 * 64, 4 * 10000 * 64, 0, 0]
