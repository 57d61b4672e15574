"""The division of prompt attention batches against the room that its workspace has for them: the library's own rule
(split_of, share_of) over batches of all kinds, on the host."""
import ctypes
import math
import os
import random
import subprocess

import pytest

from paper_2609_03494_amd import build

SOURCE = r"""
#include "gp_internal.h"
using namespace gp;
// Request r: n[r] new tokens behind before[r].  -> pieces, split items, units of 32 rows of their parts; the room for each; the
// items' tokens that no piece has.
extern "C" void division(int R, const int *before, const int *n, int hq, int hkv, int d, int direct, long long *out) {
    const int G = hq / hkv, tokens = kPromptRows / G;
    long long T = 0;
    unsigned long long cost = 0;
    for (int r = 0; r < R; ++r) {
        T += n[r];
        for (int j = 0; j < n[r]; j += tokens) cost += std::max(before[r] + j + std::min(tokens, n[r] - j), 0);
    }
    const PromptWs w = prompt_ws(R, T, hq, hkv, d, direct);
    const int share = share_of(cost, w.slots);
    long long pieces = 0, merges = 0, units = 0, missed = 0;
    for (int r = 0; r < R; ++r)
        for (int j = 0; j < n[r]; j += tokens) {
            const int m = std::min(tokens, n[r] - j), seen = std::max(before[r] + j + m, 0), rows = m * G;
            const Split x = split_of(seen, rows, share, w.fine);
            pieces += x.parts;
            if (x.parts > 1) {
                ++merges;
                units += x.parts * (rows <= 32 ? 1 : w.part_rows / 32);
                if (x.per % 64) missed = 1 << 30;
            }
            // the last piece is the one that ends the item, and has tokens
            missed += std::max(seen - x.parts * x.per, 0) + (x.parts > 1 && (x.parts - 1) * x.per >= seen);
        }
    const long long to[] = {pieces, merges, units, w.max_pieces, w.max_merges, w.units, missed,
                            (long long)(w.total - w.partial) / (4LL * hkv * 32 * (d + 2))};
    std::copy(to, to + 8, out);
}
"""


@pytest.fixture(scope="module")
def division(tmp_path_factory):
    to = tmp_path_factory.mktemp("division")
    (to / "division.cpp").write_text(SOURCE)
    subprocess.run([build.hipcc(), "-x", "hip", "--cuda-host-only", *build.flags(), "-shared", str(to / "division.cpp"), "-o",
                    str(to / "division.so")], check=True, capture_output=True)
    fn = ctypes.CDLL(os.path.join(str(to), "division.so")).division
    fn.restype = None

    def call(before, n, hq, hkv, d, direct):
        R, out = len(n), (ctypes.c_longlong * 8)()
        fn(R, (ctypes.c_int * R)(*before), (ctypes.c_int * R)(*n), hq, hkv, d, int(direct), out)
        return list(out)
    return call


def _fits(division, before, n, g, hkv, d=64):
    """-> the largest part of the units that is taken.  Calls of few items once more without a list (see prompt_call)."""
    tokens, T, R = 128 // g, sum(n), len(n)
    forms = [False] + ([True] if R <= 64 and (T <= tokens or T // tokens + R <= 64) else [])
    most = 0.0
    for direct in forms:
        pieces, merges, units, max_pieces, max_merges, max_units, missed, room = division(before, n, g * hkv, hkv, d, direct)
        what = (before[:8], n[:8], R, g, hkv, direct)
        assert pieces <= max_pieces and merges <= max_merges and units <= max_units <= room and missed == 0, what
        most = max(most, units / max_units)
    return most


def test_random_batches_fit(division):
    rng = random.Random(0)
    most = 0.0
    for _ in range(6000):
        g, hkv = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 8, 12, 40, 64, 300, 8192])
        R = int(math.exp(rng.uniform(0, math.log(300))))
        top, new = math.exp(rng.uniform(0, math.log(131072))), math.exp(rng.uniform(0, math.log(3000)))
        kind = rng.randrange(4)
        n = [1 if kind == 0 or (kind == 1 and rng.random() < 0.8) else rng.randint(0, int(new)) for _ in range(R)]
        if sum(n) == 0:
            n[0] = 1
        before = [max(0, min(131072 - k, int(top * rng.random() ** rng.choice([1, 4])))) for k in n]
        if kind == 3:                                          # tokens that see nothing: lengths less than the new tokens
            before = [b - rng.choice([0, 0, k, k // 2]) for b, k in zip(before, n)]
        most = max(most, _fits(division, before, n, g, hkv))
    assert most > 0.4                                          # (the batches do come near)


@pytest.mark.parametrize("g", [1, 8])
@pytest.mark.parametrize("rows", [8, 32, 40, 128])
def test_batches_at_the_borders_of_the_rule_fit(division, g, rows):
    """Items alike, alone or beside one long one, as many and as long as makes each of them just long enough to be split."""
    n = max(rows // g, 1)
    for hkv in (1, 5, 64):
        slots = -(-512 // hkv)
        for R in sorted({1, 2, 3, slots // 3, slots // 2, slots - 1, slots, *(int(slots * x) for x in (0.55, 0.57, 0.58, 0.79, 0.8, 0.81, 1.2))}):
            if R < 1:
                continue
            for seen in (319, 320, 321, 385, 639, 640, 641, 700, 1000, 1281, 5000, 40001, 131072):
                _fits(division, [max(seen - n, 0)] * R, [n] * R, g, hkv)
                for long in (1.0, 1.26, 1.76, 3.0, 20.0):
                    _fits(division, [max(seen - n, 0)] * R + [min(int(seen * long), 131000)], [n] * (R + 1), g, hkv)
