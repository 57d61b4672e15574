"""Pages, rotations, prompt and decode attention, boundary steps and forks as a serving program runs them one after
the other, against a plain record of every request's tokens; decode steps that take their own pages, captured."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_03494_amd as gp
from test_cache_ops_gpu import BF16, DEV, F32, _i32
from test_prompt_gpu import _exact, _tol
from test_rotary_gpu import HALF, SIDE, _turned

pytestmark = pytest.mark.gpu


def _say(msg):
    print(f"[run] {msg}", flush=True)


class Server:
    """Two layers of a cache, all of its pages on the stack, and beside it what each request holds: hist[l][r] = (K, V)
    [tokens][Hkv][d] float64, as they lay in the pool when they went in; pos[r] the index of the last token."""

    def __init__(self, kind, rope, R=6, width=24, pool=90, hq=8, hkv=2, d=64, layers=2, seed=0):
        self.kind, self.rope, self.hq, self.hkv, self.d = kind, rope, hq, hkv, d
        self.dt, self.R, self.pool = (F32 if kind == "f32" else BF16), R, pool
        self.gen = torch.Generator().manual_seed(seed)
        shape = (pool, hkv, 16, d)
        if kind == "q8":
            e4 = torch.float8_e4m3fn
            self.layers = [gp.KV8Layer(*[torch.full(shape, 0x7f, dtype=torch.uint8, device=DEV).view(e4) for _ in range(2)],
                                       *[torch.ones(pool, hkv, device=DEV) for _ in range(2)]) for _ in range(layers)]
        else:
            self.layers = [gp.KVLayer(*[torch.full(shape, float("nan"), dtype=self.dt, device=DEV) for _ in range(2)]) for _ in range(layers)]
        self.handle = gp.Layers(self.layers)
        zero = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
        self.ps = gp.PageState(torch.full((R, width), -1, dtype=torch.int32, device=DEV), zero(R), zero(R), zero(pool),
                               torch.randperm(pool, generator=self.gen).to(torch.int32).to(DEV), _i32([pool]))
        self.positions = _i32([-1] * R)
        self.pos = [-1] * R
        none = torch.zeros(0, hkv, d, dtype=torch.float64, device=DEV)
        self.hist = [[(none, none)] * R for _ in range(layers)]
        self.scale = float(torch.tensor(1.0 / math.sqrt(d), dtype=F32))
        self.ws = gp.workspace(gp.GP_OP_PROMPT, R, 256, hq, hkv, d, width, self.dt)
        self.ws_decode = gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, width, self.dt)
        self.qstate = torch.zeros(R, 2, hq, d, device=DEV)

    def held(self, r):
        return self.hist[0][r][0].shape[0]

    def stored(self, l, which, r, m):
        """The first m tokens of row r of the pool [m][Hkv][d]."""
        kv = self.layers[l]
        pool = kv.k if which == 0 else kv.v
        ids = self.ps.page_table[r, :-(-m // 16)].long()
        x = pool.view(torch.uint8)[ids].view(pool.dtype).double() if self.kind == "q8" else pool[ids].double()
        if self.kind == "q8":
            x = x * (kv.k_scale if which == 0 else kv.v_scale)[ids].double()[..., None, None]
        return x.permute(0, 2, 1, 3).flatten(0, 1)[:m]

    def check_pages(self):
        """Counts are the references of the tables; the stack and the tables have every page once."""
        torch.cuda.synchronize()
        table, pages, lens = self.ps.page_table.cpu(), self.ps.num_pages.cpu(), self.ps.seq_lens.cpu()
        refs = torch.zeros(self.pool, dtype=torch.int32)
        for r in range(self.R):
            assert int(lens[r]) == self.held(r), (r, int(lens[r]), self.held(r))
            assert int(pages[r]) * 16 >= int(lens[r])
            refs.index_add_(0, table[r, :int(pages[r])].long(), torch.ones(int(pages[r]), dtype=torch.int32))
        assert torch.equal(refs, self.ps.refcount.cpu())
        free = self.ps.free_list[:int(self.ps.free_count)].cpu().sort().values
        assert torch.equal(free, (refs == 0).nonzero()[:, 0].to(torch.int32))

    def reserve(self, ns):
        granted = _i32([-1] * self.R)
        gp.gp_pages_reserve(self.ps, _i32(ns), granted)
        assert granted.tolist() == [1] * self.R

    def step(self, ns, single=False):
        """ns[r] new tokens of each request through both layers."""
        self.reserve(ns)
        starts = [0]
        for n in ns:
            starts.append(starts[-1] + n)
        T = starts[-1]
        start = None if single else _i32(starts)
        q8 = self.kind == "q8"
        outs = []
        for l, kv in enumerate(self.layers):
            rows = torch.randn(T, self.hq + 2 * self.hkv, self.d, generator=self.gen).to(self.dt).to(DEV)
            q, k, v = rows[:, :self.hq], rows[:, self.hq:self.hq + self.hkv], rows[:, self.hq + self.hkv:]
            q_out = torch.full((T, self.hq, self.d), 5.0, dtype=self.dt, device=DEV)
            last = l == len(self.layers) - 1
            (gp.gp_append_rotary_q8 if q8 else gp.gp_append_rotary)(kv, self.ps, self.positions, k, v, self.rope, q=q, q_out=q_out,
                                                                    tok_start=start, advance=last)
            out = torch.full((T, self.hq, self.d), 7.0, dtype=self.dt, device=DEV)
            (gp.gp_prompt_attention_q8 if q8 else gp.gp_prompt_attention)(kv, self.ps, q_out, self.scale, out, self.ws, tok_start=start,
                                                                          advanced=last)
            torch.cuda.synchronize()
            for r in range(self.R):
                self.took(l, r, slice(starts[r], starts[r + 1]), q, q_out, k, v, out)
            outs.append((q, q_out, out))
        for r in range(self.R):
            self.pos[r] += ns[r]
        assert self.positions.tolist() == self.pos
        self.check_pages()
        return outs

    def took(self, l, r, s, q, q_out, k, v, out):
        n = s.stop - s.start
        if n == 0:
            return
        K, V = self.hist[l][r]
        m = K.shape[0]
        pos = self.pos[r] + 1 + torch.arange(n)
        # half a step of the type, and of float32 for cosine, sine, two products and their sum; 8 bits: 2^-4
        # of the value, or half of the smallest step, 2^-10 scales
        step = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "q8": 2.0 ** -8}[self.kind]
        turned, size = (x.to(DEV) for x in _turned(q[s].double().cpu(), pos, self.rope))
        assert bool(((q_out[s].double() - turned).abs() <= turned.abs() * step + size * 4 * 2.0 ** -24).all())
        newK, newV = self.stored(l, 0, r, m + n), self.stored(l, 1, r, m + n)
        turned, size = (x.to(DEV) for x in _turned(k[s].double().cpu(), pos, self.rope))
        for got, want, err, scales in ((newK[m:], turned, size * 4 * 2.0 ** -24, 0), (newV[m:], v[s].double(), 0.0, 1)):
            if self.kind == "q8":
                kv = self.layers[l]
                sc = (kv.v_scale if scales else kv.k_scale)[self.ps.page_table[r, :-(-(m + n) // 16)].long()].double()
                sc = sc.repeat_interleave(16, 0)[m:m + n, :, None]
                tol = want.abs() * 2.0 ** -4 + sc * 2.0 ** -10 + 2 * err
            else:
                tol = want.abs() * (step if scales == 0 else 0.0) + err
            assert bool(((got - want).abs() <= tol).all()), (l, r, scales)
        # older tokens as they were: 8-bit codes of the page that went on may have been rounded again
        whole = m if self.kind != "q8" else m // 16 * 16
        assert torch.equal(newK[:whole], K[:whole]) and torch.equal(newV[:whole], V[:whole]), (l, r)
        self.hist[l][r] = newK, newV
        self.check(l, r, q_out[s].double(), out[s], m, "prompt")

    def check(self, l, r, q, out, m, what):
        K, V = (x.transpose(0, 1).contiguous() for x in self.hist[l][r])
        want, size, dots = _exact(q, K, V, m, self.scale)
        far = (out.double() - want).abs() - _tol(self.dt, want, size, dots, self.d, K.shape[1])
        assert bool((far <= 0).all()), (what, l, r, m, float(far.max()))

    def decode(self, outs):
        """The decode step's attention of the tokens that went in last: the same outputs."""
        for l, kv in enumerate(self.layers):
            _, q_out, _ = outs[l]
            out = torch.full_like(q_out, 7.0)
            (gp.gp_decode_attention_q8 if self.kind == "q8" else gp.gp_decode_attention)(kv, self.ps, q_out, self.scale, out, self.ws_decode)
            torch.cuda.synchronize()
            for r in range(self.R):
                self.check(l, r, q_out[r:r + 1].double(), out[r:r + 1], self.held(r) - 1, "decode")

    def fork(self, parents, children, lengths):
        forked = _i32([-1] * len(parents))
        (gp.gp_pages_fork_q8 if self.kind == "q8" else gp.gp_pages_fork)(self.handle, self.ps, _i32(parents), _i32(children), forked,
                                                                         lengths=_i32(lengths), positions=self.positions)
        assert forked.tolist() == [1] * len(parents)
        for p, c, n in zip(parents, children, lengths):
            L = min(n, self.held(p))
            self.pos[c] = self.pos[p] - (self.held(p) - L)
            for h in self.hist:
                h[c] = tuple(x[:L].clone() for x in h[p])
        self.check_pages()
        for l in range(len(self.layers)):
            for c in children:
                for which in (0, 1):
                    assert torch.equal(self.stored(l, which, c, self.held(c)), self.hist[l][c][which])

    def release(self, rows):
        gp.gp_pages_release(self.ps, _i32(rows))
        for r in rows:
            self.pos[r] = -1
            self.positions[r] = -1
            for h in self.hist:
                h[r] = tuple(x[:0] for x in h[r])
        self.check_pages()

    def boundary(self, r, q_pre):
        """Row r, whose pages are full, gives up one page of tokens."""
        P, m = int(self.ps.num_pages[r]), self.held(r)
        assert m == 16 * P
        params = gp.Params(scale=self.scale, policy=gp.GP_POLICY_FIXED, fixed_pages=1)
        slots, bnd, cand = _i32(range(self.R)), _i32([r]), 16 * (self.ps.page_table.shape[1] - 1)
        n = len(self.layers)
        gp.gp_update_summaries(q_pre, slots, torch.ones(self.R, dtype=torch.uint8, device=DEV), self.qstate, 0.9, 0.999)
        counts = torch.zeros(n, 1, self.hkv, 2, dtype=torch.int32, device=DEV)
        scores = torch.zeros(n, 1, self.hkv, cand, device=DEV)
        ws = gp.workspace(gp.GP_OP_SCORE, self.R, 1, self.hq, self.hkv, self.d, self.ps.page_table.shape[1], self.dt)
        for l, kv in enumerate(self.layers):
            gp.gp_boundary_score_rotary(kv, self.ps, q_pre, self.qstate, slots, self.positions, bnd, params, self.rope, counts[l], scores[l], ws)
        ws = gp.workspace(gp.GP_OP_APPLY, self.R, 1, self.hq, self.hkv, self.d, self.ps.page_table.shape[1], self.dt, n)
        dec, delta = _i32([-1]), torch.zeros(1, device=DEV)
        gp.gp_boundary_apply(self.layers, self.ps, bnd, counts, scores, params, dec, delta, torch.zeros(4, dtype=torch.int64, device=DEV), ws)
        assert dec.tolist() == [gp.GP_COMPRESS]
        for l in range(n):
            K, V = self.hist[l][r]
            new = self.stored(l, 0, r, m - 16), self.stored(l, 1, r, m - 16)
            for h in range(self.hkv):
                # every token that stayed is one of before, key and value together, in order, the last page whole
                same = (new[0][:, None, h] == K[None, :, h]).all(-1) & (new[1][:, None, h] == V[None, :, h]).all(-1)
                at = same.int().argmax(1)
                assert bool(same.any(1).all()) and bool((at[1:] > at[:-1]).all()) and at[-16:].tolist() == list(range(m - 16, m))
            self.hist[l][r] = new
        self.check_pages()


ROPES = [(HALF, 32, True), (SIDE, 64, False)]


@pytest.mark.parametrize("layout,n,scaled", ROPES)
@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_requests_come_fork_decode_and_leave(kind, layout, n, scaled):
    _say(f"{kind} {layout} {n}")
    rope = (gp.Rope(layout, gp.gp_rope_frequencies(n, 1.0e4, 8.0, 1.0, 4.0, 8192), 1.2) if scaled else
            gp.Rope(layout, gp.gp_rope_frequencies(n, 1.0e6)))
    s = Server(kind, rope)
    s.step([37, 60, 16, 0, 0, 0])                             # prompts
    s.step([0, 43, 3, 0, 0, 0])                               # a chunk, and drafted tokens behind a full page
    s.fork([0, 0, 1], [3, 4, 5], [1000, 21, 96])              # replies to one prompt, a prompt that begins like another
    s.step([2, 0, 1, 5, 1, 30])                               # all go on, each on pages of its own
    s.decode(s.step([1] * 6, single=True))
    s.release([4, 0])
    s.step([100, 0, 0, 0, 7, 0])                              # new requests in their rows
    fill = [-s.held(r) % 16 for r in range(6)]
    s.step(fill)
    outs = s.step([16, 16, 0, 16, 0, 16])
    if kind != "q8":                                          # (boundary steps are for bfloat16 and float32 caches)
        q_pre = torch.randn(6, 8, 64, generator=s.gen).to(s.dt).to(DEV)
        s.boundary(5, q_pre)                                  # shares six pages with row 1, which keeps them
        s.boundary(0, q_pre)
    outs = s.step([1] * 6, single=True)
    s.decode(outs)
    s.release([1, 5, 5, 0, 2, 3, 4])
    assert int(s.ps.free_count) == s.pool and s.ps.refcount.tolist() == [0] * s.pool


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_decode_steps_that_take_their_pages_captured(kind):
    """Reserve, append and attend for one token each, captured and replayed over several pages, two graphs with one
    workspace in turn, against eager calls on a second cache of the same contents."""
    _say(f"captured {kind}")
    rope = gp.Rope(SIDE, gp.gp_rope_frequencies(64, 1.0e6))
    pair = []
    for _ in range(2):
        s = Server(kind, rope, seed=3)
        s.step([37, 60, 16, 1, 9, 0])
        s.release([3])
        s.fork([1], [3], [50])
        pair.append(s)
    c, e = pair
    R, q8 = c.R, kind == "q8"
    gen = torch.Generator().manual_seed(1)
    rows = torch.zeros(2, R, c.hq + 2 * c.hkv, c.d, dtype=c.dt, device=DEV)

    def one(s, outs):
        gp.gp_pages_reserve(s.ps, s.want, s.granted, keep_free=3)
        for l, kv in enumerate(s.layers):
            q, k, v = rows[l, :, :s.hq], rows[l, :, s.hq:s.hq + s.hkv], rows[l, :, s.hq + s.hkv:]
            q_out = outs[2 * l]
            last = l == 1
            (gp.gp_append_rotary_q8 if q8 else gp.gp_append_rotary)(kv, s.ps, s.positions, k, v, rope, q=q, q_out=q_out, advance=last)
            (gp.gp_prompt_attention_q8 if q8 else gp.gp_prompt_attention)(kv, s.ps, q_out, s.scale, outs[2 * l + 1], s.ws, advanced=last)

    for s in pair:
        s.want, s.granted = _i32([1] * R), _i32([-1] * R)
        s.outs = [[torch.zeros(R, s.hq, s.d, dtype=s.dt, device=DEV) for _ in range(4)] for _ in range(2)]
    graphs, stream = [], torch.cuda.Stream()
    for g in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            one(c, c.outs[g])
        graphs.append(graph)
    for t in range(40):
        rows.copy_(torch.randn(rows.shape, generator=gen))
        graphs[t % 2].replay()
        torch.cuda.synchronize()
        one(e, e.outs[t % 2])
        torch.cuda.synchronize()
        for x, y in zip(c.outs[t % 2], e.outs[t % 2]):
            assert torch.equal(x, y), t
        assert torch.equal(c.ps.page_table, e.ps.page_table) and torch.equal(c.ps.seq_lens, e.ps.seq_lens)
        assert torch.equal(c.granted, e.granted) and torch.equal(c.ps.free_count, e.ps.free_count)
    assert c.ps.seq_lens.tolist() == [77, 100, 56, 90, 49, 40]
    for x, y in zip(c.layers, e.layers):
        for a, b in zip(vars(x).values(), vars(y).values()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
