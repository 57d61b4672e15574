"""Pages reserved, forked and released on the device against the same rules kept in
Python lists: every array of the page state, the copied rows, flags and positions."""
from __future__ import annotations

import random

import pytest
import torch

import paper_2609_03494_amd as gp

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
PAGE = 16


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32).to(DEV)


class Book:
    """The page state in lists, and the three calls on it."""

    def __init__(self, rows, lens, width, pool, rng, positions=None):
        ids = list(range(pool))
        rng.shuffle(ids)
        self.pool, self.width = pool, width
        self.table = [[ids[p] for p in row] + [-1] * (width - len(row)) for row in rows]
        self.P, self.m = [len(row) for row in rows], list(lens)
        self.refs = [0] * pool
        for row, P in zip(self.table, self.P):
            for p in row[:P]:
                self.refs[p] += 1
        left = [p for p in ids if self.refs[p] == 0]
        self.height, self.stack = len(left), left + [7] * (pool - len(left))
        self.pos = positions or [3 * m + 11 for m in lens]

    def device(self):
        self.ps = gp.PageState(_i32(self.table), _i32(self.P), _i32(self.m), _i32(self.refs), _i32(self.stack), _i32([self.height]))
        self.positions = _i32(self.pos)
        return self.ps

    def same(self, what=""):
        ps = self.ps
        for name, want in (("num_pages", self.P), ("seq_lens", self.m), ("page_table", self.table), ("refcount", self.refs),
                           ("free_count", [self.height]), ("free_list", self.stack)):
            got = getattr(ps, name).cpu()
            assert torch.equal(got, torch.tensor(want, dtype=torch.int32)), (what, name)
        assert self.positions.tolist() == self.pos, (what, "positions")

    def release(self, reqs):
        gone = []
        for r in reqs:
            if not 0 <= r < len(self.P) or self.m[r] < 0:
                continue
            for p in self.table[r][:self.P[r]]:
                self.refs[p] -= 1
                if self.refs[p] == 0:
                    gone.append(p)
            self.P[r] = self.m[r] = 0
        for p in sorted(gone):
            self.stack[self.height] = p
            self.height += 1

    def reserve(self, tokens, keep=0):
        left, granted = self.height - keep, []
        blocked = False
        for r, t in enumerate(tokens):
            want = -(-(self.m[r] + max(t, 0)) // PAGE)
            need = max(0, want - self.P[r])
            if self.m[r] < 0 or want > self.width:
                granted.append(0)
                continue
            if need and (blocked or need > left):
                blocked = True
                granted.append(0)
                continue
            for _ in range(need):
                self.height -= 1
                left -= 1
                p = self.table[r][self.P[r]] = self.stack[self.height]
                self.refs[p] = 1
                self.P[r] += 1
            granted.append(1)
        return granted

    def fork(self, parents, children, lengths=None, positions=True):
        """-> forked, and (parent page, child page, rows) of each copy."""
        P0, m0, pos0 = list(self.P), list(self.m), list(self.pos)
        seen, forked, copies, out = set(), [], [], False
        for i, (p, c) in enumerate(zip(parents, children)):
            ok = 0 <= p < len(P0) and 0 <= c < len(P0) and c not in seen and P0[c] == 0 and m0[c] == 0 and m0[p] >= 0
            seen.add(c)
            L = 0
            if ok:
                L = min(m0[p], P0[p] * PAGE) if lengths is None else min(m0[p], P0[p] * PAGE, max(lengths[i], 0))
                if L % PAGE and (out or self.height == 0):
                    ok, out = False, True
            forked.append(int(ok))
            if not ok:
                continue
            full = L // PAGE
            for j in range(full):
                q = self.table[c][j] = self.table[p][j]
                self.refs[q] += 1
            if L % PAGE:
                self.height -= 1
                q = self.table[c][full] = self.stack[self.height]
                self.refs[q] = 1
                copies.append((self.table[p][full], q, L % PAGE))
            self.P[c], self.m[c] = -(-L // PAGE), L
            if positions:
                self.pos[c] = pos0[p] - (m0[p] - L)
        return forked, copies


def _book(rng, R, hi, width, spare, empty=0.2, held=0.1, shared=0):
    """R rows of up to hi tokens, some empty, some held, some with pages to spare, the first `shared` pages of the longer ones in common."""
    rows, lens, at = [], [], shared
    for _ in range(R):
        m = 0 if rng.random() < empty else rng.choice([rng.randint(1, hi), PAGE * rng.randint(1, max(1, hi // PAGE))])
        P = -(-m // PAGE) + (rng.randint(0, 2) if m else 0)
        P = min(P, width)
        m = min(m, P * PAGE)
        k = shared if shared and P > shared else 0
        rows.append(list(range(k)) + list(range(at, at + P - k)))
        at += P - k
        lens.append(-m - 1 if m and rng.random() < held else m)
    return Book(rows, lens, width, at + spare, rng)


@pytest.mark.parametrize("R,hi,width,spare,shared", [(1, 40, 4, 3, 0), (7, 200, 16, 40, 3), (64, 900, 64, 500, 10), (300, 100, 10, 90, 2),
                                                     (2500, 60, 6, 4000, 1), (3, 20000, 1400, 2000, 0)])
def test_release_and_reserve(R, hi, width, spare, shared):
    for seed in range(4):
        rng = random.Random(1000 * R + seed)
        b = _book(rng, R, hi, width, spare, shared=shared)
        b.device()
        for round_ in range(3):
            reqs = [rng.randint(-2, R + 1) for _ in range(rng.randint(1, 2 * R))]     # some twice, some out of range
            gp.gp_pages_release(b.ps, _i32(reqs))
            b.release(reqs)
            b.same((R, seed, round_, "release"))
            tokens = [rng.choice([0, -5, 1, rng.randint(0, hi), rng.randint(0, 2 * hi)]) for _ in range(R)]
            keep = rng.choice([0, 0, 1, spare // 2, b.pool + 5])
            granted = torch.full((R,), 9, dtype=torch.int32, device=DEV)
            gp.gp_pages_reserve(b.ps, _i32(tokens), granted, keep_free=keep)
            want = b.reserve(tokens, keep)
            assert granted.tolist() == want
            b.same((R, seed, round_, "reserve"))


def test_release_of_long_lists_and_large_pools():
    """More rows than one pass over the list takes, all twice; pools whose pages are marked in their counts."""
    rng = random.Random(5)
    b = _book(rng, 5000, 50, 5, 100, held=0.02)
    b.device()
    reqs = [r for r in range(5000) if r % 9] * 2
    rng.shuffle(reqs)
    gp.gp_pages_release(b.ps, _i32(reqs))
    b.release(reqs)
    b.same("long list")
    for pool in (1 << 20, (1 << 20) + 1, 3000001):
        b = _book(rng, 40, 4000, 300, 17, shared=20)
        more = pool - b.pool                                   # spare ids above all others, and one table entry up there
        b.refs += [0] * more
        b.stack += [5] * more
        b.pool = pool
        r = next(i for i in range(40) if b.P[i] > 25 and b.m[i] >= 0)
        b.refs[b.table[r][22]] -= 1
        b.table[r][22] = pool - 1
        b.refs[pool - 1] = 1
        b.device()
        reqs = list(range(0, 40, 2)) + [r]
        gp.gp_pages_release(b.ps, _i32(reqs))
        b.release(reqs)
        b.same(pool)


def _pools(kind, L, pool, hkv, d, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if kind == "q8":
        codes = torch.randint(0, 256, (L, 2, pool, hkv, PAGE, d), generator=gen, device=DEV, dtype=torch.uint8)
        scales = torch.rand(L, 2, pool, hkv, generator=gen, device=DEV)
        return codes, scales, [gp.KV8Layer(codes[i, 0], codes[i, 1], scales[i, 0], scales[i, 1]) for i in range(L)]
    x = torch.randn(L, 2, pool, hkv, PAGE, d, generator=gen, device=DEV, dtype=BF16 if kind == "bf16" else F32)
    return x, None, [gp.KVLayer(x[i, 0], x[i, 1]) for i in range(L)]


def _copied(x, scales, copies):
    want, ws = x.clone(), None if scales is None else scales.clone()
    for src, dst, rows in copies:
        want[:, :, dst, :, :rows] = x[:, :, src, :, :rows]
        if scales is not None:
            ws[:, :, dst] = scales[:, :, src]
    return want, ws


@pytest.mark.parametrize("kind,L,hkv,d", [("bf16", 1, 8, 128), ("bf16", 3, 2, 64), ("f32", 2, 3, 128), ("q8", 2, 8, 128), ("q8", 70, 1, 64),
                                          ("bf16", 65, 1, 64)])
@pytest.mark.parametrize("whole", [True, False])
def test_fork(kind, L, hkv, d, whole):
    for seed in range(3):
        rng = random.Random(77 * L + 10 * hkv + seed)
        R = rng.choice([5, 30])
        b = _book(rng, R, 300, 24, rng.choice([0, 2, 40]), empty=0.5, shared=2)
        b.device()
        x, scales, layers = _pools(kind, L, b.pool, hkv, d, seed)
        n = rng.randint(1, 2 * R)
        parents = [rng.randint(-1, R) for _ in range(n)]
        children = [rng.choice([rng.randint(-1, R), rng.choice([r for r in range(R) if b.P[r] == 0] or [0])]) for _ in range(n)]
        lengths = None if whole else [rng.choice([-3, 0, 16, 32, rng.randint(0, 320)]) for _ in range(n)]
        forked, copies = b.fork(parents, children, lengths)
        want, ws = _copied(x, scales, copies)
        got = torch.full((n,), 9, dtype=torch.int32, device=DEV)
        (gp.gp_pages_fork_q8 if kind == "q8" else gp.gp_pages_fork)(
            gp.Layers(layers) if seed else layers, b.ps, _i32(parents), _i32(children), got,
            lengths=None if whole else _i32(lengths), positions=b.positions)
        assert got.tolist() == forked
        b.same((kind, L, seed))
        assert torch.equal(x.view(torch.uint8), want.view(torch.uint8))
        assert scales is None or torch.equal(scales, ws)


def test_fork_many():
    """2048 forks of a few parents, with fewer pages on the stack than they ask for; rows 8192 pages long."""
    rng = random.Random(3)
    rows = [list(range(0, 40)), list(range(40, 47)), list(range(47, 8239))] + [[]] * 2100
    lens = [40 * PAGE - 3, 7 * PAGE, 8192 * PAGE - 1] + [0] * 2100
    b = Book(rows, lens, 8192, 8239 + 1000, rng)
    b.device()
    x, _, layers = _pools("bf16", 1, b.pool, 1, 64, 1)
    parents = [rng.choice([0, 0, 1]) for _ in range(2046)] + [2, 2]
    children = list(range(3, 2051))
    rng.shuffle(children)
    children[100] = children[50]
    lengths = [min(b.m[p], rng.randint(1, 700)) if p < 2 else b.m[p] - k for k, p in enumerate(parents)]
    forked, copies = b.fork(parents, children, lengths)
    assert 0 in forked[200:] and 1 in forked[1500:]
    want, _ = _copied(x, None, copies)
    got = torch.zeros(2048, dtype=torch.int32, device=DEV)
    gp.gp_pages_fork(layers, b.ps, _i32(parents), _i32(children), got, lengths=_i32(lengths), positions=b.positions)
    assert got.tolist() == forked
    b.same()
    assert torch.equal(x, want)


def test_life_captured():
    """Rounds of release, fork and reserve in a graph, replayed with eager rounds between."""
    rng = random.Random(9)
    b = _book(rng, 24, 300, 40, 400, empty=0.0, held=0.0)
    kids = list(range(8, 24))
    b.device()
    x, _, layers = _pools("bf16", 3, b.pool, 2, 64, 4)
    handle = gp.Layers(layers)
    par = _i32([k % 8 for k in range(16)])
    chi, ask = _i32(kids), _i32([17] * 24)
    forked, granted = torch.zeros(16, dtype=torch.int32, device=DEV), torch.zeros(24, dtype=torch.int32, device=DEV)

    def step():
        gp.gp_pages_release(b.ps, chi)
        gp.gp_pages_fork(handle, b.ps, par, chi, forked, positions=b.positions)
        gp.gp_pages_reserve(b.ps, ask, granted)

    def book():
        b.release(kids)
        _, copies = b.fork(par.tolist(), kids)
        return copies, b.reserve([17] * 24)

    def check(want, copies, what):
        want, _ = _copied(want, None, copies)
        b.same(what)
        assert torch.equal(x, want), what

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    before = x.clone()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    copies, g = book()
    check(before, copies, "eager")
    assert granted.tolist() == g
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for k in range(4):
        before = x.clone()
        if k % 2:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        copies, g = book()
        check(before, copies, k)
        assert granted.tolist() == g
