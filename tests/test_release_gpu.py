"""gp_pages_release of many rows, which takes two launches (rows times table width past 32768): several workgroups at once
drop references to the same pages, rows of more pages than a workgroup takes at a time, a pool that fills the marks."""
from __future__ import annotations

import random

import pytest
import torch

import paper_2609_03494_amd as gp
from test_pages_gpu import PAGE, Book, _book, _i32

pytestmark = pytest.mark.gpu


def _release(b, reqs, what):
    assert len(reqs) * b.width > 32768 and b.pool <= 1 << 20   # (two launches)
    gp.gp_pages_release(b.ps, _i32(reqs))
    b.release(reqs)
    b.same(what)


@pytest.mark.parametrize("R,hi,width,spare,shared", [(64, 9000, 600, 500, 20), (300, 3000, 190, 40, 100), (9, 70000, 4400, 33, 700),
                                                     (2000, 600, 40, 900, 5)])
def test_rows_that_share_pages(R, hi, width, spare, shared):
    """Some rows leave, listed twice, held or out of range among them, then more, then all: a shared page goes with its last row."""
    for seed in range(3):
        print(f"[release] {R} rows of up to {hi} tokens, seed {seed}", flush=True)
        rng = random.Random(100 * R + seed)
        b = _book(rng, R, hi, width, spare, shared=shared)
        b.device()
        for round_ in range(3):
            reqs = [rng.randint(-2, R + 1) for _ in range(max(R // 2, 32768 // width + 1))]
            _release(b, reqs, (R, seed, round_))
        _release(b, list(range(R)) * max(1, -(-32769 // (R * width))), (R, seed, "all"))
        assert b.P.count(0) >= sum(m >= 0 for m in b.m)


def test_rows_alike():
    """300 rows of the same 200 pages, one of them held: its release in the end pushes them, each once."""
    print("[release] rows alike", flush=True)
    rng = random.Random(1)
    b = Book([list(range(200)) for _ in range(300)], [200 * PAGE - r for r in range(10)] * 30, 220, 1000, rng)
    b.m[17] = -b.m[17] - 1
    b.device()
    _release(b, list(range(300)) * 2, "all but one")
    assert b.height == 800 and max(b.refs) == 1
    b.ps.seq_lens[17] = 5
    b.m[17] = 5
    _release(b, [17] * 200, "the last")
    assert b.height == 1000 and max(b.refs) == 0


def test_pool_that_fills_the_marks():
    """2^20 pages, the first and the last of them among those that go and among those that stay."""
    print("[release] 2^20 pages", flush=True)
    for keep in (False, True):
        rng = random.Random(2 + keep)
        b = _book(rng, 120, 6000, 400, 50, empty=0.0, shared=30)
        more = (1 << 20) - b.pool
        b.refs += [0] * more
        b.stack += [5] * more
        b.pool = 1 << 20
        rows = [r for r in range(120) if b.P[r] > 40 and b.m[r] >= 0][:3]
        for i, r in enumerate(rows):                           # the last page of the pool is three rows'
            b.refs[b.table[r][35]] -= 1
            b.table[r][35] = (1 << 20) - 1
            b.refs[(1 << 20) - 1] += 1
        b.device()
        reqs = [r for r in range(120) if not keep or r != rows[1]]
        _release(b, reqs, keep)
        assert (b.refs[(1 << 20) - 1] == 1) == keep


def test_captured_with_eager_rounds_between():
    """The two launches in a graph, the state set back before each replay."""
    print("[release] captured", flush=True)
    rng = random.Random(5)
    b = _book(rng, 128, 5000, 330, 70, shared=12)
    b.device()
    first = {k: v.clone() for k, v in vars(b.ps).items()}
    reqs = [r for r in range(128) if r % 5] + [3, 3, -1, 128]
    assert len(reqs) * 330 > 32768
    on = _i32(reqs)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        gp.gp_pages_release(b.ps, on)
    b.release(reqs)
    for k in range(4):
        for name, t in first.items():
            getattr(b.ps, name).copy_(t)
        torch.cuda.synchronize()
        if k % 2:
            gp.gp_pages_release(b.ps, on)
        else:
            graph.replay()
        torch.cuda.synchronize()
        b.same(k)
