"""Attention of new tokens over the paged cache against float64: ragged batches of prompts, chunks, drafted and
single tokens, borders that hold infinities and NaN, and a prompt's whole way from its pages to the decode step."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_03494_amd as gp
from test_cache_ops_gpu import BF16, DEV, F32, NAN, _i32, _offset, _paged, _state

pytestmark = pytest.mark.gpu
INF = float("inf")


def _say(msg):
    print(f"[prompt] {msg}", flush=True)


def _exact(q, K, V, before, scale):
    """q [n][Hq][d], K and V [Hkv][m][d] float64 on the device: outputs, and the bounds of their errors' parts:
    sum of w |v|, the largest sum of |q k| and |z| of each row."""
    n, hq, d = q.shape
    hkv, m = K.shape[:2]
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    dots = torch.zeros(n, hq, 1, dtype=torch.float64, device=q.device)
    for h in range(hkv):
        G = hq // hkv
        x = q[:, h * G:(h + 1) * G].reshape(n * G, d)
        see = (torch.arange(m, device=q.device)[None] <= before + torch.arange(n, device=q.device)[:, None]).repeat_interleave(G, 0)
        z = scale * (x @ K[h].T)
        z = torch.where(see, z, -INF)
        top = z.amax(-1, keepdim=True)
        w = torch.where(see, (z - top).exp(), 0.0)
        w = w / w.sum(-1, keepdim=True)
        # a row that sees an infinite value of weight zero sees 0 * inf; a row that does not see it does not
        out[:, h * G:(h + 1) * G] = (w @ V[h]).view(n, G, d)
        size[:, h * G:(h + 1) * G] = (w @ V[h].abs()).view(n, G, d)
        dots[:, h * G:(h + 1) * G] = scale * torch.where(see, x.abs() @ K[h].abs().T, 0.0).amax(-1).view(n, G, 1)
    return out, size, dots


def _tol(dt, out, size, dots, d, m):
    """Half a step of the output; the weights' rounding to bfloat16 (half a step each, 2^-8); a score is a chain of d
    products and sums and three more roundings (scale, factor, difference), each 2^-24 of sum |q k|, its weight off by that much and the
    exponential's 2^-22; the sums over m tokens 2^-24 a step each, twice (weights, outputs).  Score errors count
    twice, in the weight and in the sum that divides it."""
    score = 2 * ((d + 4) * 2.0 ** -24 * dots + 2.0 ** -22)
    sums = 2 * m * 2.0 ** -24
    if dt == F32:
        return out.abs() * 2.0 ** -24 + size * (score + sums) + 1e-37
    return out.abs() * 2.0 ** -8 + size * (2.0 ** -8 + score + sums) + 1e-37


class Case:
    """A cache of `kind` that holds the tokens of reqs = [(before, pages, new)], before < 0: held (-before - 1 tokens)."""

    def __init__(self, kind, reqs, hq, hkv, d, seed, advanced=False, single=False, fused=False, offset=0, heavy=1.0, spare=2):
        gen = torch.Generator().manual_seed(seed)
        self.kind, self.reqs, self.hq, self.hkv, self.d, self.advanced = kind, reqs, hq, hkv, d, advanced
        self.dt = F32 if kind == "f32" else BF16
        npages = [P for _, P, _ in reqs]
        pool, self.table = _paged(npages, max(max(npages), 1) + spare, gen)
        self.scale = 1.0 / math.sqrt(d)
        T = sum(n for _, _, n in reqs)
        self.starts = [0]
        for _, _, n in reqs:
            self.starts.append(self.starts[-1] + n)
        self.start = None if single else _i32(self.starts)
        rows = torch.randn(T, hq, d, generator=gen).to(self.dt)
        if fused:                                             # queries within wider rows
            buf = torch.full((T, (hq + 3) * d + offset), NAN, dtype=self.dt, device=DEV)
            self.q = buf[:, offset:offset + hq * d].unflatten(1, (hq, d))
            self.q.copy_(rows)
        else:
            self.q = _offset(rows.to(DEV), offset)
        k = torch.randn(pool, hkv, 16, d, generator=gen) * heavy + 0.5 * torch.randn(1, hkv, 1, d, generator=gen)
        k[torch.rand(pool, hkv, 16, generator=gen) < 0.02] *= 4
        v = torch.randn(pool, hkv, 16, d, generator=gen)
        if kind == "q8":
            scale = torch.exp2(torch.randint(-10, -6, (2, pool, hkv), generator=gen).float()) * (0.75 + 0.5 * torch.rand(2, pool, hkv, generator=gen))
            codes = [(x / s[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn) for x, s in ((k, scale[0]), (v, scale[1]))]
            self.kv = gp.KV8Layer(codes[0].to(DEV), codes[1].to(DEV), scale[0].to(DEV), scale[1].to(DEV))
        else:
            self.kv = gp.KVLayer(k.to(self.dt).to(DEV), v.to(self.dt).to(DEV))
        # whatever is no token of a request's
        inside = torch.zeros(pool, 16, dtype=torch.bool)
        for r, (m, P, n) in enumerate(reqs):
            total = (-m - 1 if m < 0 else m) + (n if m >= 0 and m + n <= 16 * P else 0)
            ids = self.table[r, :P].long()
            inside[ids] = (torch.arange(16 * P) < total).view(P, 16)
        out = (~inside).to(DEV)
        for t in (self.kv.k, self.kv.v):
            if kind == "q8":
                t.view(torch.uint8).masked_fill_(out[:, None, :, None], 0x7f)
            else:
                t.masked_fill_(out[:, None, :, None], NAN)
        lens = [m + (n if advanced and m >= 0 and m + n <= 16 * P else 0) for m, P, n in reqs]
        self.ps = _state(self.table, npages, lens, pool)
        self.out = torch.full((T, hq, d), 7.0, dtype=self.dt, device=DEV)
        self.ws = gp.workspace(gp.GP_OP_PROMPT, len(reqs), T, hq, hkv, d, self.table.shape[1], self.dt)

    def tokens(self, which, r, m):
        pool = self.kv.k if which == 0 else self.kv.v
        ids = self.table[r, :-(-m // 16)].long().to(DEV)
        x = pool.view(torch.uint8)[ids].view(pool.dtype).double() if self.kind == "q8" else pool[ids].double()
        if self.kind == "q8":
            x = x * (self.kv.k_scale if which == 0 else self.kv.v_scale)[ids].double()[..., None, None]
        return x.transpose(0, 1).flatten(1, 2)[:, :m]

    def call(self, **kw):
        fn = gp.gp_prompt_attention_q8 if self.kind == "q8" else gp.gp_prompt_attention
        a = dict(tok_start=self.start, advanced=self.advanced)
        a.update(kw)
        fn(self.kv, self.ps, self.q, self.scale, self.out, self.ws, **a)

    def check(self, what=""):
        scale = float(torch.tensor(self.scale, dtype=F32))
        for r, (m, P, n) in enumerate(self.reqs):
            got = self.out[self.starts[r]:self.starts[r + 1]].double()
            if n == 0:
                continue
            if m < 0:
                assert bool((got == 7.0).all()), (what, r, "held")
                continue
            if m + n > 16 * P:                                # without room: not in the cache
                if not self.advanced:
                    assert bool((got == 0.0).all()), (what, r, "no room")
                continue
            q = self.q[self.starts[r]:self.starts[r + 1]].double()
            want, size, dots = _exact(q, self.tokens(0, r, m + n), self.tokens(1, r, m + n), m, scale)
            far = (got - want).abs() - _tol(self.dt, want, size, dots, self.d, m + n)
            assert bool((far <= 0).all()), (what, r, (m, P, n), float(far.max()))


RAGGED = [(0, 3, 40), (5, 2, 1), (16, 4, 33), (15, 2, 17), (7, 1, 0), (10, 1, 7), (-20, 4, 3), (31, 2, 1), (16, 1, 1), (0, 1, 16),
          (3, 9, 120), (0, 1, 1), (40, 3, 8), (100, 40, 513), (700, 60, 129), (0, 9, 128), (63, 8, 65), (64, 8, 64), (200, 13, 5)]
SINGLE = [(m, P, 1) for m, P, _ in RAGGED] + [(0, 0, 1), (17, 1, 1), (1000, 63, 1)]
SHAPES = [("bf16", 8, 2, 128), ("bf16", 3, 3, 64), ("bf16", 16, 2, 64), ("bf16", 4, 2, 128), ("bf16", 8, 1, 128), ("f32", 8, 1, 64),
          ("f32", 4, 2, 128), ("f32", 4, 1, 128), ("f32", 2, 2, 64), ("q8", 32, 8, 128), ("q8", 5, 5, 64), ("q8", 16, 2, 64), ("q8", 4, 2, 128),
          ("q8", 8, 1, 128)]


@pytest.mark.parametrize("kind,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("form", ["ragged", "advanced", "single", "fused"])
def test_prompt_attention(kind, hq, hkv, d, form):
    _say(f"{kind} {hq}/{hkv} d {d} {form}")
    c = Case(kind, SINGLE if form == "single" else RAGGED, hq, hkv, d, 5 + hq, form == "advanced", form == "single", form == "fused",
             3 if form == "fused" else 0)
    c.call()
    torch.cuda.synchronize()
    c.check(form)


@pytest.mark.parametrize("kind,hq,hkv,d", [("bf16", 8, 2, 128), ("f32", 4, 2, 64), ("q8", 8, 1, 128)])
def test_prompt_long_contexts(kind, hq, hkv, d):
    """Few tokens behind long contexts, beside short requests and a prompt."""
    _say(f"long contexts {kind}")
    reqs = [(9000, 570, 5), (20, 2, 1), (0, 63, 1000), (5000, 313, 8), (3, 1, 2), (2999, 188, 1), (4000, 260, 70)]
    for advanced in (False, True):
        c = Case(kind, reqs, hq, hkv, d, 2, advanced)
        c.call()
        torch.cuda.synchronize()
        c.check("long")
    c = Case(kind, [(30011, 1880, 3)], hq, hkv, d, 2)
    c.call()
    torch.cuda.synchronize()
    c.check("one")


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_prompt_many_requests(kind):
    _say(f"many requests {kind}")
    reqs = [((7 * r) % 333, 24, (r * r) % 23 if r % 5 else 0) for r in range(700)]
    c = Case(kind, reqs, 2, 1, 64, 5)
    c.call()
    torch.cuda.synchronize()
    c.check("many")


@pytest.mark.parametrize("kind,hq,hkv,d", [("bf16", 4, 2, 128), ("f32", 4, 1, 64), ("q8", 2, 2, 64)])
def test_prompt_sharp_scores(kind, hq, hkv, d):
    """Scores of hundreds: weights next to one and zero, maxima that move from tile to tile."""
    _say(f"sharp {kind}")
    c = Case(kind, [(100, 40, 300), (0, 10, 150)], hq, hkv, d, 9, heavy=30.0)
    c.call()
    torch.cuda.synchronize()
    c.check("sharp")


def _put(c, r, i, h, dim, x, which):
    """Element `dim` of token i of request r, head h, becomes x (8-bit: NaN for any)."""
    pool = c.kv.k if which == 0 else c.kv.v
    if c.kind == "q8":
        pool.view(torch.uint8)[int(c.table[r, i // 16]), h, i % 16, dim] = 0x7f
    else:
        pool[int(c.table[r, i // 16]), h, i % 16, dim] = x


@pytest.mark.parametrize("kind,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 2, 2, 64), ("f32", 4, 2, 64), ("f32", 2, 2, 128), ("q8", 8, 2, 128),
                                           ("q8", 2, 2, 64)])
def test_prompt_values_that_rows_do_not_see(kind, hq, hkv, d):
    """Infinite and NaN values and keys of later tokens leave the rows before them as they are; rows that see them get
    what the formula says."""
    _say(f"unseen {kind} {hq}/{hkv} d {d}")
    reqs = [(37, 16, 180), (0, 6, 90), (500, 40, 3)]
    marks = [(0, 37 + 60, 5, INF), (0, 37 + 60, 6, -INF), (0, 37 + 70, 5, -INF), (0, 37 + 100, 40, NAN), (1, 20, 3, INF), (1, 89, 7, NAN),
             (2, 501, 9, INF), (2, 502, 10, -INF)]
    plain = Case(kind, reqs, hq, hkv, d, 4)
    plain.call()
    c = Case(kind, reqs, hq, hkv, d, 4)
    for r, i, dim, x in marks:
        _put(c, r, i, 1, dim, x, 1)
    c.call()
    torch.cuda.synchronize()
    G = hq // hkv
    for r, (m, _, n) in enumerate(reqs):
        for j in range(n):
            want = plain.out[c.starts[r] + j].clone()
            got = c.out[c.starts[r] + j]
            seen = {}
            for rr, i, dim, x in marks:
                if rr == r and i <= m + j:
                    seen[dim] = seen.get(dim, 0.0) + (NAN if kind == "q8" else x)
            assert torch.equal(got[:G], want[:G])                       # the other KV head
            for dim, x in seen.items():
                y = got[G:, dim].float()
                assert bool((y.isnan() if math.isnan(x) else y == x).all()), (r, j, dim, x, y)
            rest = [k for k in range(d) if k not in seen]
            a, b = got[G:, rest].float(), want[G:, rest].float()
            assert bool(((a - b).abs() <= b.abs() * 2.0 ** -7 + 1e-6).all()), (r, j)
    # keys: the scores of rows that see a NaN are NaN, their outputs zero
    c = Case(kind, reqs, hq, hkv, d, 4)
    for r, i in ((0, 37 + 60), (1, 20), (2, 501)):
        _put(c, r, i, 1, 11, NAN, 0)
    c.call()
    torch.cuda.synchronize()
    for r, (m, _, n), i in ((0, reqs[0], 97), (1, reqs[1], 20), (2, reqs[2], 501)):
        a, b = c.out[c.starts[r]:c.starts[r + 1]], plain.out[c.starts[r]:c.starts[r + 1]]
        unseen = i - m
        assert torch.equal(a[:, :G], b[:, :G])
        assert bool(((a[:unseen, G:].float() - b[:unseen, G:].float()).abs() <= b[:unseen, G:].float().abs() * 2.0 ** -7 + 1e-6).all())
        assert bool((a[unseen:, G:] == 0).all())


def test_prompt_infinite_scores():
    """Keys and queries whose scores are infinite, by the rules of decode attention: +inf is no number, -inf no weight."""
    _say("infinite scores")
    c = Case("bf16", [(5, 4, 50)], 2, 1, 64, 3)
    c.q[:, :, 0] = 1.0
    page, slot = int(c.table[0, 20 // 16]), 20 % 16
    c.kv.k[page, 0, slot] = 0.0
    c.kv.k[page, 0, slot, 0] = -INF                                     # token 20 has no weight
    c.call()
    torch.cuda.synchronize()
    got = c.out.clone()
    want, size, dots = _exact(c.q.double(), torch.where(c.tokens(0, 0, 55).isfinite(), c.tokens(0, 0, 55), -1e30), c.tokens(1, 0, 55), 5, c.scale)
    assert bool(((got.double() - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -7 + 1e-6).all())
    c.kv.k[page, 0, slot, 0] = INF
    c.call()
    torch.cuda.synchronize()
    assert torch.equal(c.out[:15], got[:15]) and bool((c.out[15:] == 0).all())


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_prompt_rows_of_nobody(kind):
    """Rows outside the requests' keep what they hold; starts and page states that break the contract end the call
    with every access in its buffers."""
    _say(f"rows of nobody {kind}")
    c = Case(kind, [(30, 8, 60), (0, 4, 33), (9, 2, 4)], 4, 2, 64, 8)
    c.call()
    want = c.out.clone()
    T = c.q.shape[0]
    q = torch.cat([torch.full_like(c.q[:5], NAN), c.q, torch.full_like(c.q[:9], NAN)])
    c.out = torch.full_like(q, 7.0)
    c.q, keep = q, c.q
    c.ws = gp.workspace(gp.GP_OP_PROMPT, 3, T + 14, 4, 2, 64, c.table.shape[1], c.dt)
    c.call(tok_start=c.start + 5)
    torch.cuda.synchronize()
    assert torch.equal(c.out[5:5 + T], want) and bool((c.out[:5] == 7).all()) and bool((c.out[5 + T:] == 7).all())
    for starts in ([0, -5, 30, 10], [-2 ** 31, 2 ** 31 - 1, -7, 2 ** 31 - 1], [40, 3, 2, 1], [T + 100, T + 101, T + 102, T + 103],
                   [5, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1]):
        c.call(tok_start=_i32(starts))
        torch.cuda.synchronize()
    c.ps.page_table[0, 1], c.ps.page_table[0, 2], c.ps.page_table[1, 0] = -3, c.ps.refcount.numel(), 2 ** 30
    c.ps.num_pages[2], c.ps.seq_lens[2] = 5000, 2 ** 31 - 1
    for advanced in (False, True):
        c.call(tok_start=c.start + 5, advanced=advanced)
        torch.cuda.synchronize()


def test_prompt_before_zero():
    """advanced with lengths that do not hold all new tokens: those that see nothing get zeros."""
    _say("before zero")
    c = Case("bf16", [(0, 4, 50), (0, 4, 7)], 4, 2, 64, 8, advanced=True)
    c.ps.seq_lens.copy_(_i32([20, 0]))
    c.call()
    torch.cuda.synchronize()
    assert bool((c.out[:30] == 0).all()) and bool((c.out[50:] == 0).all())
    want, size, dots = _exact(c.q[30:50].double(), c.tokens(0, 0, 20), c.tokens(1, 0, 20), 0, c.scale)
    assert bool(((c.out[30:50].double() - want).abs() <= _tol(BF16, want, size, dots, 64, 20)).all())


@pytest.mark.parametrize("kind", ["bf16", "q8"])
def test_prompt_captured_and_on_streams(kind):
    """Replays with eager calls and other lengths between; two calls at once with a workspace each."""
    _say(f"captured {kind}")
    reqs = [(300, 40, 100), (5, 1, 3), (2000, 130, 4), (0, 20, 300)]
    c, e = Case(kind, reqs, 8, 2, 128, 6), Case(kind, reqs, 8, 2, 128, 6)
    other = Case(kind, [(10, 30, 400), (3000, 200, 17)], 8, 2, 128, 7)
    e.call()
    torch.cuda.synchronize()
    e.check()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.call()
    for k in range(4):
        for t in (c, e):
            t.ps.seq_lens.copy_(_i32([300 - k, 5, 2000 - 31 * k, 17 * k]))
        c.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        e.call()
        torch.cuda.synchronize()
        assert torch.equal(c.out, e.out), k
    other.call()
    torch.cuda.synchronize()
    want = other.out.clone()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        e.out.fill_(7.0)
        other.out.fill_(7.0)
        torch.cuda.synchronize()
        e.call(stream=one)
        other.call(stream=two)
        torch.cuda.synchronize()
        assert torch.equal(c.out, e.out) and torch.equal(other.out, want)


def test_prompt_more_requests_than_the_planner_has_threads():
    """Long prompts before and behind the first thousand of requests, single tokens, and starts that are not given."""
    _say("1500 requests")
    reqs = [((5 * r) % 90, 26, 300 if r in (3, 1023, 1024, 1499) else r % 3) for r in range(1500)]
    c = Case("bf16", reqs, 4, 2, 64, 7)
    c.call()
    torch.cuda.synchronize()
    c.check("1500")
    c = Case("q8", [((11 * r) % 700, 45, 1) for r in range(300)], 4, 2, 64, 7, single=True)
    c.call()
    torch.cuda.synchronize()
    c.check("300 singles")


@pytest.mark.parametrize("kind,hq,hkv,d,reqs", [("bf16", 8, 1, 128, [(100000, 6260, 70)]), ("f32", 1, 1, 64, [(70000, 4380, 2), (30, 4, 9)]),
                                                ("q8", 4, 1, 64, [(60000, 3800, 1)] * 3), ("bf16", 64, 64, 64, [(900, 70, 130), (5, 2, 20)]),
                                                ("f32", 80, 40, 64, [(300, 30, 33)]), ("q8", 40, 40, 128, [(40, 9, 90), (2000, 130, 3)]), ("bf16", 16, 4, 64, [(12000, 783, 512)]),
                                                ("q8", 8, 2, 128, [(6000, 440, 1000), (9000, 628, 1030)])])
def test_prompt_few_and_many_heads(kind, hq, hkv, d, reqs):
    """One KV head: an item in as many pieces as there are places for them; many heads: hardly any."""
    _say(f"heads {kind} {hq}/{hkv}")
    c = Case(kind, reqs, hq, hkv, d, 12)
    c.call()
    torch.cuda.synchronize()
    c.check("heads")


def test_prompt_one_workspace_for_calls_of_all_sizes():
    """The workspace of the largest call serves smaller ones, whatever was left in it."""
    _say("one workspace")
    big = Case("bf16", [(500, 120, 900), (7, 40, 300), (3000, 200, 9)], 8, 2, 64, 1)
    big.ws.random_(0, 256)
    for reqs in ([(500, 120, 900), (7, 40, 300), (3000, 200, 9)], [(3000, 200, 1), (5, 1, 1), (100, 20, 6)], [(0, 9, 100), (0, 9, 0), (4, 1, 2)]):
        c = Case("bf16", reqs, 8, 2, 64, 1)
        assert c.ws.numel() <= big.ws.numel()
        c.ws = big.ws
        for _ in range(2):
            c.out.fill_(7.0)
            c.call()
            torch.cuda.synchronize()
            c.check("workspace")


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_prompt_pools_past_32_bits(kind):
    """Pages whose bytes lie past 2^32 of the pool's start."""
    _say(f"large pool {kind}")
    hkv, d = 16, 128
    c = Case(kind, [(200, 20, 90), (70, 6, 1)], 2 * hkv, hkv, d, 3)
    page = hkv * 16 * d * c.kv.k.element_size()
    pool, small = 2 ** 32 // page + 300, c.kv.k.shape[0]
    ids = torch.randperm(pool - 2 ** 31 // page, generator=torch.Generator().manual_seed(0))[:small] + 2 ** 31 // page
    ids[::2] = pool - 1 - torch.arange(len(ids[::2]))
    made = []
    for x in vars(c.kv).values():
        y = torch.zeros((pool, *x.shape[1:]), dtype=torch.uint8 if kind == "q8" and x.dim() == 4 else x.dtype, device=DEV)
        y[ids.to(DEV)] = x.view(torch.uint8) if y.dtype == torch.uint8 else x
        made.append(y.view(x.dtype))
    want = c.tokens(0, 0, 290).clone()
    c.kv = type(c.kv)(*made)
    c.table = torch.where(c.table >= 0, ids[c.table.clamp(min=0).long()].int(), -1)
    c.ps = _state(c.table, [P for _, P, _ in c.reqs], [m for m, _, _ in c.reqs], pool)
    assert torch.equal(c.tokens(0, 0, 290), want) and int(c.table.max()) * page > 2 ** 32
    c.call()
    torch.cuda.synchronize()
    c.check("large pool")


def test_prompt_scales_at_the_ends_of_their_range():
    """Scales whose product with log2(e) is as small or as large as float32 holds: the mean, and the first of the largest scores."""
    _say("scales")
    c = Case("f32", [(40, 4, 9)], 2, 1, 64, 3)
    V = c.tokens(1, 0, 49)[0]
    c.scale = 1e-38
    c.call()
    torch.cuda.synchronize()
    for j in range(9):
        mean = V[:41 + j].mean(0)
        assert bool(((c.out[j].double() - mean).abs() <= V.abs().mean() * 49 * 2.0 ** -20).all())
    c.scale = 1.6e38                                            # below 2^127
    c.q.zero_()
    c.q[:, :, 0] = 2.0 ** -126
    c.kv.k.masked_fill_(c.kv.k == c.kv.k, 0.0)                  # (the NaN of nobody's slots stay)
    _put(c, 0, 7, 0, 0, 1000.0, 0)
    c.call()
    torch.cuda.synchronize()
    # token 7 is ahead by 1000 * 1.6e38 * 2^-126 = 1880
    assert torch.equal(c.out.double(), V[7].expand(9, 2, 64))


@pytest.mark.parametrize("kind", ["bf16", "q8"])
def test_prompt_requests_kept_together(kind):
    """Items enough for pieces to go out request by request: prompts, a chunk, one long context that is split, short ones."""
    _say(f"together {kind}")
    reqs = [(3000, 270, 1300), (60000, 3760, 1), (0, 90, 1400), (9000, 600, 500), (100, 10, 3), (0, 1, 0), (-30, 4, 20), (7000, 440, 33), (40, 3, 60)]
    for advanced in (False, True):
        c = Case(kind, reqs, 64, 8, 64, 3, advanced)
        c.call()
        torch.cuda.synchronize()
        c.check("together")
