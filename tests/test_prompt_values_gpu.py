"""Prompt attention where one form of the division could give other results than another."""
from __future__ import annotations

import math

import pytest
import torch

from test_cache_ops_gpu import F32
from test_prompt_gpu import INF, NAN, Case, _exact, _put

pytestmark = pytest.mark.gpu


def _say(msg):
    print(f"[values] {msg}", flush=True)


def _quiet(c, r, tokens, head):
    """The first tokens of request r: their scores lie far below the others': weights of zero in any type."""
    pool = c.kv.k.view(torch.uint8) if c.kind == "q8" else c.kv.k
    t = torch.arange(tokens)
    pool[c.table[r, t // 16].long(), head, t % 16, 0] = 0xfe if c.kind == "q8" else -3000.0     # (8 bits: -448 times the page's scale)
    if c.kind == "q8":
        c.kv.k_scale[c.table[r, :(tokens + 15) // 16].long(), head] = 4.0


# the request that is looked at, and others that change how it is divided: alone it is split (or its waves have blocks of
# their own), beside longer ones it is not, among many it goes out with its request
BATCHES = [[], [(30000, 1876, 3)] * 4, [(0, 126, 2000)] * 12, [(5, 2, 1)] * 70]
SEEN = [((2500, 160, 2), 700), ((2500, 176, 300), 700), ((60, 5, 3), 32), ((3, 160, 2500), 1100), ((700, 60, 200), 256)]


@pytest.mark.parametrize("kind,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 4, 2, 64), ("f32", 4, 2, 64), ("f32", 2, 1, 128), ("q8", 8, 2, 128),
                                           ("q8", 4, 2, 64)])
def test_seen_values_that_are_not_finite(kind, hq, hkv, d):
    """A value that is infinite or NaN leaves no row that sees it finite in its dim, whatever its weight and however
    the batch is divided; all other outputs are as they would be without it."""
    for (m, P, n), quiet in SEEN:
        for others in BATCHES:
            _say(f"{kind} {hq}/{hkv} d {d} {n} tokens behind {m}, {len(others)} others")
            h = hkv - 1
            G = hq // hkv
            c = Case(kind, [(m, P, n), *others], hq, hkv, d, 3)
            c.q[:n, :, 0] = 8.0
            k = c.kv.k.view(torch.uint8) if kind == "q8" else c.kv.k
            t = torch.arange(m + n)
            k[c.table[0, t // 16].long(), h, t % 16, 0] = 0
            _quiet(c, 0, quiet, h)
            c.call()
            torch.cuda.synchronize()
            want = c.out[:n].clone()
            assert bool(want.isfinite().all())
            marks = [(quiet // 2, 5, INF), (quiet // 2 + 1, 6, -INF), (quiet // 3, 7, NAN)]
            for i, dim, x in marks:
                _put(c, 0, i, h, dim, x, 1)
            c.out.fill_(7.0)
            c.call()
            torch.cuda.synchronize()
            got = c.out[:n]
            assert torch.equal(got[:, :h * G], want[:, :h * G])
            rest = torch.ones(d, dtype=torch.bool)
            for i, dim, _ in marks:
                rest[dim] = False
                first = max(i - m, 0)                          # the first row that sees it
                assert not bool(got[first:, h * G:, dim].isfinite().any()), (others, dim)
                assert torch.equal(got[:first, h * G:, dim], want[:first, h * G:, dim])
            assert torch.equal(got[:, h * G:, rest], want[:, h * G:, rest])
@pytest.mark.parametrize("m,P,n", [(200, 13, 1), (700, 45, 1), (3, 14, 200)])
def test_scales_of_which_the_lag_is_no_number(m, P, n):
    """A scale so small that 2^8 of its units is past float32, and blocks in which one head's scores are all -inf, another's
    not: the mean of the values that have weights."""
    _say(f"lag {n} tokens behind {m}")
    c = Case("f32", [(m, P, n)], 2, 1, 64, 3)
    c.scale = 1e-39
    total = m + n
    V = c.tokens(1, 0, total)[0]
    pages, slots = c.table[0, torch.arange(total) // 16].long(), torch.arange(total) % 16
    c.kv.k[pages, 0, slots, 0] = torch.where(torch.arange(total) < 32, -1e30, 0.0).to(c.kv.k)
    c.q[:, 0, 0], c.q[:, 1, 0] = 1e30, 0.0
    c.call()
    torch.cuda.synchronize()
    for j in range(n):
        sees = m + j + 1
        for g, first in ((0, 32), (1, 0)):
            want = V[first:sees].mean(0) if sees > first else torch.zeros_like(V[0])
            # the sums of weights next to one: a step of 2^-24 for each token, twice, and the quotient's
            assert bool(((c.out[j, g].double() - want).abs() <= V.abs().amax() * (2 * sees + 2) * 2.0 ** -24).all()), (j, g)


@pytest.mark.parametrize("m,P,n", [(200, 13, 1), (40, 3, 1), (3, 14, 200)])
def test_scores_further_apart_than_float32_reaches(m, P, n):
    """Scores of -3e38 and, from token 32 on, 3e38 under a scale that brings them next to each other."""
    _say(f"far scores, {n} tokens behind {m}")
    c = Case("f32", [(m, P, n)], 1, 1, 64, 3)
    c.scale = 1e-38
    total = m + n
    V = c.tokens(1, 0, total)[0]
    t = torch.arange(total)
    c.kv.k[c.table[0, t // 16].long(), 0, t % 16] = 0.0
    c.kv.k[c.table[0, t // 16].long(), 0, t % 16, 0] = torch.where(t < 32, -3e19, 3e19).to(c.kv.k)
    c.q[:, :, 0] = 1e19
    c.call()
    torch.cuda.synchronize()
    w = torch.where(t < 32, math.exp(-3.0), math.exp(3.0)).double().to(V)
    for j in range(n):
        sees = m + j + 1
        want = (w[:sees, None] * V[:sees]).sum(0) / w[:sees].sum()
        # the weights by the rounding of the scale (a denormal number of 23 bits and fewer: 2^-20), of scores of 4.4
        # in log2 and of the exponential, twice, and the sums' steps
        tol = V.abs().amax() * (2 * 3.0 * (2.0 ** -20 + 3 * 2.0 ** -23) + 2.0 ** -21 + (2 * sees + 2) * 2.0 ** -24)
        assert bool(((c.out[j, 0].double() - want).abs() <= tol).all()), j


def _tol_few(out, size, dots, d, m):
    """As _tol, with the weights in two terms: half a step of half a step, 2^-16."""
    score = 2 * ((d + 4) * 2.0 ** -24 * dots + 2.0 ** -22)
    return out.abs() * 2.0 ** -8 + size * (2.0 ** -16 + score + 2 * m * 2.0 ** -24) + 1e-37


@pytest.mark.parametrize("kind,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 2, 2, 64), ("bf16", 8, 1, 64), ("bf16", 4, 2, 128), ("q8", 8, 2, 128),
                                           ("q8", 2, 2, 64), ("q8", 8, 1, 128)])
def test_few_rows_are_as_exact_as_the_decode_step(kind, hq, hkv, d):
    """Values that nearly cancel show the weights' rounding: single and drafted tokens have them in two terms, as
    the decode calls do."""
    reqs = [(3, 1, 1), (9, 1, 2), (40, 4, 3), (200, 13, 1), (1500, 96, 4), (7000, 440, 1), (0, 1, 1), (33, 5, 32 // (hq // hkv))]
    for rs in (reqs, [reqs[5]], [reqs[4]], [(m, P, 1) for m, P, _ in reqs * 10]):
        _say(f"exact {kind} {hq}/{hkv} d {d}, {len(rs)} requests")
        c = Case(kind, rs, hq, hkv, d, 4, heavy=0.3)
        v = c.kv.v.view(torch.uint8) if kind == "q8" else c.kv.v
        v[:, :, 1::2] = torch.where(torch.isnan(c.kv.v[:, :, 1::2].float()), v[:, :, 1::2], v[:, :, ::2] ^ 0x80 if kind == "q8" else -v[:, :, ::2])
        c.call()
        torch.cuda.synchronize()
        scale = float(torch.tensor(c.scale, dtype=F32))
        for r, (m, P, n) in enumerate(rs):
            got = c.out[c.starts[r]:c.starts[r + 1]].double()
            want, size, dots = _exact(c.q[c.starts[r]:c.starts[r + 1]].double(), c.tokens(0, r, m + n), c.tokens(1, r, m + n), m, scale)
            far = (got - want).abs() - _tol_few(want, size, dots, d, m + n)
            assert bool((far <= 0).all()), (r, (m, P, n), float(far.max()), float((size * 2.0 ** -16).max()))
