"""Prompt attention where one form of the division could give other results than another."""
from __future__ import annotations

import pytest
import torch

from test_prompt_gpu import INF, NAN, Case, _put

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
