"""The cache operators' forms for large calls against float64: 8-bit attention whose runs pass 64 pages, rows
past the caches, selection waves of two steps; and the page bounds of a cache that a compaction rearranged."""
from __future__ import annotations

import math

import pytest
import torch

import oracle as O
import paper_2609_03494_amd as gp
import workloads as W
from _harness import DeviceCase
from test_cache_ops_gpu import (BF16, DEV, F32, HALF, NAN, ROT, _attention, _attention_tol, _bounds64, _i32, _offset,
                                _rotated, _select64, _state, _tokens, _values)

pytestmark = pytest.mark.gpu


def _say(msg):
    print(f"[cache ops, large] {msg}", flush=True)


# ------------------------------------------- 8-bit attention, runs past 64 pages --

def _shared_q8(lens, hkv, d, gen, spare, common=1500):
    """Requests over `common` pages that all of them read (each in an order of its own), and a last page of their
    own, NaN past the length; scales that differ from page to page, NaN where nothing is."""
    R, npages = len(lens), [-(-m // 16) for m in lens]
    pool = common + R
    codes = torch.full((2, pool, hkv, 16, d), 0x7f, dtype=torch.uint8)
    scale = torch.full((2, pool, hkv), NAN)
    x = torch.randn(2, common, hkv, 16, d, generator=gen)
    s = torch.exp2(torch.randint(-8, -5, (2, common, hkv), generator=gen).float()) * (0.75 + 0.5 * torch.rand(2, common, hkv, generator=gen))
    codes[:, :common] = (x / s[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    scale[:, :common] = s
    table = torch.full((R, max(npages) + spare), -1, dtype=torch.int32)
    for r, m in enumerate(lens):
        if m == 0:
            continue
        P, t, pid = npages[r], m - 16 * (npages[r] - 1), common + r
        table[r, :P - 1] = torch.randint(0, common, (P - 1,), generator=gen).int()
        table[r, P - 1] = pid
        codes[:, pid, :, :t] = (torch.randn(2, hkv, t, d, generator=gen) * 64).to(torch.float8_e4m3fn).view(torch.uint8)
        scale[:, pid] = 2.0 ** -6 * (0.75 + 0.5 * torch.rand(2, hkv, generator=gen))
    kv = gp.KV8Layer(codes[0].to(DEV), codes[1].to(DEV), scale[0].to(DEV), scale[1].to(DEV))
    return kv, pool, table, npages


def _sample(lens, n):
    """The longest requests, those of no and few tokens, and some between."""
    order = sorted(range(len(lens)), key=lambda r: lens[r])
    return sorted(set(order[:4] + order[-6:] + order[::max(1, len(order) // n)]))


@pytest.mark.parametrize("hq,d", [(8, 64), (32, 128)])
def test_decode_q8_long_runs(hq, d):
    """300 requests, 8 KV heads, about 21 thousand pairs of pages per head: runs of 41 pairs, so that a wave
    fetches ids and scales again in the middle of a request, and begins and ends requests anywhere."""
    hkv = 8
    _say(f"decode q8 long runs heads {hq}/{hkv} d {d}")
    gen = torch.Generator().manual_seed(d)
    lens = [int(x) for x in torch.randint(1500, 3001, (300,), generator=gen)]
    lens[7], lens[8], lens[9], lens[150], lens[299] = 0, 1, 17, 9001, 5000
    pairs = sum(-(-m // 32) for m in lens)
    assert pairs > 64 * 8 * 33                            # (64 workgroups of 8 waves per KV head hold the batch at once)
    kv, pool, table, npages = _shared_q8(lens, hkv, d, gen, 400)
    R, width = table.shape
    q = torch.randn(R, hq, d, generator=gen).to(BF16)
    out = torch.full((R, hq, d), NAN, dtype=BF16, device=DEV)
    scale = d ** -0.5
    gp.gp_decode_attention_q8(kv, _state(table, npages, lens, pool), q.to(DEV), scale, out,
                              gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, width, BF16))
    torch.cuda.synchronize()
    got, k64, v64 = out.cpu().double(), _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    assert bool(got.isfinite().all())
    for r in _sample(lens, 40):
        if lens[r] == 0:
            assert bool((got[r] == 0).all())
            continue
        want, mag, size = _attention(_tokens(k64, table, r, lens[r]), _tokens(v64, table, r, lens[r]), q[r].double(), scale)
        assert bool(((got[r] - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), r


@pytest.mark.parametrize("hq,d", [(8, 64), (32, 128)])
def test_decode_pages_q8_long_runs(hq, d):
    """Lists of 400 pages for 120 requests and 8 KV heads, another one for each head, some with entries that are
    no pages: runs of up to 48 pairs."""
    hkv, budget = 8, 400
    _say(f"decode pages q8 long runs heads {hq}/{hkv} d {d}")
    gen = torch.Generator().manual_seed(d + 1)
    lens = [int(x) for x in torch.randint(5000, 8001, (120,), generator=gen)]
    lens[3], lens[4], lens[5] = 0, 40, 3000
    kv, pool, table, npages = _shared_q8(lens, hkv, d, gen, 5)
    R = len(lens)
    assert sum(min(budget, P) // 2 for P in npages) > 64 * 8 * 33
    sel = torch.full((R, hkv, budget), -1, dtype=torch.int32)
    for r, n in enumerate(npages):
        for h in range(hkv):
            row = torch.randperm(n, generator=gen)[:budget].int()
            if (r + h) % 3 == 0 and n > 100:
                row[torch.randint(0, len(row), (9,), generator=gen)] = torch.tensor([-1, n, 2 ** 30] * 3, dtype=torch.int32)
            sel[r, h, :len(row)] = row
    q = torch.randn(R, hq, d, generator=gen).to(BF16)
    out = torch.full((R, hq, d), NAN, dtype=BF16, device=DEV)
    scale, G = d ** -0.5, hq // hkv
    gp.gp_decode_attention_pages_q8(kv, _state(table, npages, lens, pool), sel.to(DEV), q.to(DEV), scale, out,
                                    gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, budget, BF16))
    torch.cuda.synchronize()
    got, k64, v64 = out.cpu().double(), _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    assert bool(got.isfinite().all())
    for r in _sample(lens, 15):
        n, m = npages[r], lens[r]
        for h in range(hkv):
            mine = got[r, h * G:(h + 1) * G]
            p = sel[r, h, :min(n, budget)].long()
            tok = (p[(p >= 0) & (p < n)][:, None] * 16 + torch.arange(16)).flatten()
            tok = tok[tok < m]
            if len(tok) == 0:
                assert bool((mine == 0).all()), (r, h)
                continue
            want, mag, size = _attention(_tokens(k64[:, h:h + 1], table, r, m)[:, tok], _tokens(v64[:, h:h + 1], table, r, m)[:, tok],
                                         q[r, h * G:(h + 1) * G].double(), scale)
            assert bool(((mine - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), (r, h)


# ------------------------------------------------------- rows past the caches --

@pytest.mark.parametrize("cache,hq,hkv,d", [("bf16", 8, 8, 128), ("bf16", 16, 4, 64), ("f32", 8, 8, 64), ("f32", 4, 4, 128),
                                            ("q8", 8, 8, 128), ("q8", 16, 4, 64)])
@pytest.mark.parametrize("offset", [0, 3])
def test_append_rope_large(cache, hq, hkv, d, offset):
    """Prompts of more than 256 MB of rows, also off 16 bytes: sampled tokens against float64, and every byte as
    smaller calls of a few requests each leave it."""
    dt, q8 = F32 if cache == "f32" else BF16, cache == "q8"
    per = d * (4 if cache == "f32" else 2) * (2 * hq + 3 * hkv)
    T = (300 << 20) // per
    _say(f"append large {cache} heads {hq}/{hkv} d {d} offset {offset}: {T} tokens")
    gen = torch.Generator().manual_seed(T)
    R = 9
    cut = sorted(torch.randperm(T - 1, generator=gen)[:R - 1].tolist())
    new = [b - a for a, b in zip([0] + [c + 1 for c in cut], [c + 1 for c in cut] + [T])]
    held = [int(x) for x in torch.randint(0, 40, (R,), generator=gen)]
    npages = [-(-(m + n) // 16) for m, n in zip(held, new)]
    pool = sum(npages) + 2
    perm, table, at = torch.randperm(pool, generator=gen).int(), torch.full((R, max(npages) + 1), -1, dtype=torch.int32), 0
    for r, P in enumerate(npages):
        table[r, :P] = perm[at:at + P]
        at += P
    dev = torch.Generator(device=DEV).manual_seed(T)
    rand = lambda h: _offset(torch.randn(T, h, d, generator=dev, device=DEV).to(dt), offset)  # noqa: E731
    q, k, v = rand(hq), rand(hkv), rand(hkv)
    starts = [sum(new[:r]) for r in range(R + 1)]
    theta = 1.0e6
    fn = gp.gp_append_rope_q8 if q8 else gp.gp_append_rope

    def fresh():
        if q8:
            code = torch.arange(pool * hkv * 16 * d, device=DEV).view(pool, hkv, 16, d).remainder(120).to(torch.uint8)
            return gp.KV8Layer(code, code.clone(), torch.full((pool, hkv), 2.0 ** -7, device=DEV), torch.full((pool, hkv), 2.0 ** -7, device=DEV))
        return gp.KVLayer(*(_offset(torch.full((pool, hkv, 16, d), 9.0, dtype=dt, device=DEV), offset) for _ in range(2)))

    whole, parts = fresh(), fresh()
    outs = [torch.full((T, hq, d), 7.0, dtype=dt, device=DEV) for _ in range(2)]
    states = [_state(table, npages, held, pool) for _ in range(2)]
    positions = [_i32([m - 1 for m in held]) for _ in range(2)]
    fn(whole, states[0], positions[0], k, v, theta, q=q, q_out=outs[0], tok_start=_i32(starts))
    for r0 in range(0, R, 3):                             # three requests at a time: 100 MB
        a, b = starts[r0], starts[r0 + 3]
        fn(parts, states[1], positions[1], k[a:b], v[a:b], theta, q=q[a:b], q_out=outs[1][a:b],
           tok_start=_i32([min(max(s - a, 0), b - a) for s in starts]))
    torch.cuda.synchronize()
    raw = lambda t: t.view(torch.uint8 if q8 and t.dtype == torch.uint8 else torch.int16 if t.dtype == BF16 else torch.int32)  # noqa: E731
    assert torch.equal(raw(outs[0]), raw(outs[1]))
    for x, y in zip(vars(whole).values(), vars(parts).values()):
        assert torch.equal(raw(x), raw(y))
    for ps, pos in zip(states, positions):
        assert ps.seq_lens.cpu().tolist() == [m + n for m, n in zip(held, new)]
        assert pos.cpu().tolist() == [m + n - 1 for m, n in zip(held, new)]
    # sampled tokens, the first and the last of each request among them
    pick = sorted(set(torch.randint(0, T, (150,), generator=gen).tolist() + [s for s in starts[:-1]] + [s - 1 for s in starts[1:]]))
    req = [max(r for r in range(R) if starts[r] <= t) for t in pick]
    logical = torch.tensor([held[r] + t - starts[r] for r, t in zip(req, pick)])
    ids = torch.tensor(pick, device=DEV)
    page = table[torch.tensor(req), logical // 16].long()
    slot = logical % 16
    want_q, mag = _rotated(q[ids].cpu().double(), logical, theta)
    assert bool(((outs[0][ids].cpu().double() - want_q).abs() <= want_q.abs() * HALF[dt] + ROT * mag).all())
    want_k, mag = _rotated(k[ids].cpu().double(), logical, theta)
    want_v = v[ids].cpu().double()
    for pool_t, scales, want, off in ((whole.k, "k_scale", want_k, ROT * mag), (whole.v, "v_scale", want_v, 0 * mag)):
        got = pool_t[page.to(DEV)].cpu()[torch.arange(len(pick)), :, slot]
        if q8:
            per_page = getattr(whole, scales)[page.to(DEV)].cpu().double().unsqueeze(-1)
            got = got.view(torch.float8_e4m3fn).double() * per_page
            assert bool(((got - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, per_page * 2.0 ** -10) + off).all())
        else:
            assert bool(((got.double() - want).abs() <= want.abs() * HALF[dt] + off).all())


# ------------------------------------------------- selection, two steps a wave --

def _select_by_sum(bounds, table, n, q, budget, first, last, r, h, hkv):
    """_select64 for one KV head, where a query value of zero adds nothing whatever the bound."""
    d = q.shape[-1]
    box = bounds[table[r, :n].long(), h].double()
    x = q[r].double().view(hkv, -1, 1, d)[h]
    term = torch.where(x == 0, torch.zeros(()).double(), torch.maximum(x * box[:, 0], x * box[:, 1]))
    score = term.sum((0, 2)).float()
    middle = torch.arange(first, n - last)
    best = middle[score[middle].sort(dim=0, descending=True, stable=True)[1]][:budget - first - last]
    return torch.cat([torch.arange(first), best, torch.arange(n - last, n)]).sort()[0].int()


@pytest.mark.parametrize("dtype,d,G", [(BF16, 128, 4), (BF16, 64, 8), (F32, 128, 1), (F32, 64, 2)])
def test_select_two_steps(dtype, d, G):
    """64 requests of 8 KV heads in a table of 640 pages: more waves than the chip holds at one step each, so that
    a wave takes two.  Lengths end anywhere in either step; infinite bounds lie in both, some against a zero."""
    R, hkv, width, budget, first, last = 64, 8, 640, 50, 1, 2
    _say(f"select two steps {dtype} d {d} G {G}")
    gen = torch.Generator().manual_seed(d + G)
    npages = [int(x) for x in torch.randint(60, width + 1, (R,), generator=gen)]
    npages[:5] = [640, 608, 609, 625, 50]
    lens = [16 * n - int(x) for n, x in zip(npages, torch.randint(0, 16, (R,), generator=gen))]
    pool = 3000
    table = torch.full((R, width), -1, dtype=torch.int32)
    for r, n in enumerate(npages):
        table[r, :n] = torch.randperm(pool, generator=gen)[:n].int()
    centre = torch.randn(pool, hkv, 1, d, generator=gen)
    half = torch.rand(pool, hkv, 1, d, generator=gen)
    bounds = torch.cat([centre - half, centre + half], 2).to(dtype)
    far = torch.randperm(pool, generator=gen)
    bounds[far[:120], :, 1, 5] = math.inf
    bounds[far[60:180], :, 0, 5] = -math.inf
    q = torch.randn(R, hkv * G, d, generator=gen).to(dtype)
    q[::2, :, 5] = 0.0                                    # (the other requests: infinite scores, tied)
    sel = torch.full((R, hkv, budget), -9, dtype=torch.int32, device=DEV)
    ws = gp.workspace(gp.GP_OP_SELECT, R, 0, hkv * G, hkv, d, width, dtype)
    gp.gp_select_pages(bounds.to(DEV), _state(table, npages, lens, pool), q.to(DEV), first, last, sel, ws)
    torch.cuda.synchronize()
    got = sel.cpu()
    for r in list(range(12)) + list(range(12, R, 7)):
        for h in range(hkv):
            if npages[r] <= budget:
                assert got[r, h].tolist() == list(range(npages[r])) + [-1] * (budget - npages[r])
            else:
                assert torch.equal(got[r, h], _select_by_sum(bounds, table, npages[r], q, budget, first, last, r, h, hkv)), (r, h)


# --------------------------------------------------- after a capacity boundary --

def test_bounds_after_a_compaction():
    """A boundary that compacts some requests and grows others; the bounds of all pages made again; pages
    selected and read: those of the cache as the boundary left it."""
    _say("bounds, selection and attention after a compaction")
    w = W.qwen3_8b(seed=19, num_reqs=8, len_lo=300, len_hi=2500, budget_choices=(8, 60, 150), boundary_frac=0.75, free_pages=30)
    dc = DeviceCase(w)
    hq, hkv, d, R, budget = w.num_q_heads, w.num_kv_heads, w.head_dim, w.num_reqs, 6
    pool = w.pool_pages
    bounds = torch.full((pool, hkv, 2, d), NAN, dtype=BF16, device=DEV)
    gp.gp_page_bounds(dc.layers[0], dc.ps, bounds)
    before = dc.ps.seq_lens.cpu().tolist()
    res = dc.boundary(O.Params(tau=math.inf))
    assert (res["decisions"] == O.COMPRESS).any()
    lens = dc.ps.seq_lens.cpu().tolist()
    assert any(0 < a < b for a, b in zip(lens, before))
    gp.gp_page_bounds(dc.layers[0], dc.ps, bounds)
    sel = torch.full((R, hkv, budget), -9, dtype=torch.int32, device=DEV)
    out = torch.full((R, hq, d), 7.0, dtype=BF16, device=DEV)
    gp.gp_select_pages(bounds, dc.ps, dc.q_post, 1, 1, sel, gp.workspace(gp.GP_OP_SELECT, R, 0, hq, hkv, d, w.max_pages, BF16))
    gp.gp_decode_attention_pages(dc.layers[0], dc.ps, sel, dc.q_post, 0.09, out, gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, budget, BF16))
    torch.cuda.synchronize()
    table, q, box, chosen, got = dc.ps.page_table.cpu(), dc.q_post.cpu(), bounds.cpu(), sel.cpu(), out.cpu().double()
    k64, v64 = dc.layers[0].k.cpu().double(), dc.layers[0].v.cpu().double()
    G = hq // hkv
    for r, m in enumerate(lens):
        if m < 0:                                         # held: neither lists nor output
            assert bool((chosen[r] == -9).all()) and bool((got[r] == 7.0).all())
            continue
        n = -(-m // 16)
        for p in range(n):
            assert torch.equal(box[table[r, p].long()].double(), _bounds64(k64, table, lens, r, p)), (r, p)
        want_sel = _select64(box, table, n, q, hkv, budget, 1, 1, r)
        assert torch.equal(chosen[r], want_sel), r
        for h in range(hkv):
            tok = [16 * p + j for p in want_sel[h].tolist() if p >= 0 for j in range(min(16, m - 16 * p))]
            g = slice(h * G, (h + 1) * G)
            want, mag, size = _attention(_tokens(k64, table, r, m)[h:h + 1, tok], _tokens(v64, table, r, m)[h:h + 1, tok], q[r, g].double(), 0.09)
            assert bool(((got[r, g] - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), (r, h)


# ------------------------------------------------------------- the ends of the ranges --

@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_small_buffers_off_16_bytes(kind):
    """Queries, outputs, bounds, lists and scales at any multiple of their element, float32 pools too: the bytes
    of the aligned calls."""
    _say(f"buffers off 16 bytes {kind}")
    hq, hkv, d, budget = 8, 2, 128, 5
    dt, q8 = F32 if kind == "f32" else BF16, kind == "q8"
    gen = torch.Generator().manual_seed(31)
    lens = [300, 17, 1, 0, 160]
    npages = [-(-m // 16) for m in lens]
    R, width, pool = len(lens), 24, sum(npages)
    table = torch.full((R, width), -1, dtype=torch.int32)
    perm, at = torch.randperm(pool, generator=gen).int(), 0
    for r, P in enumerate(npages):
        table[r, :P] = perm[at:at + P]
        at += P
    if q8:
        pools = [torch.randint(0, 120, (pool, hkv, 16, d), generator=gen).to(torch.uint8).to(DEV) for _ in range(2)]
        scales = [torch.rand(pool, hkv, generator=gen).add(0.5).to(DEV) for _ in range(2)]
    else:
        pools = [torch.randn(pool, hkv, 16, d, generator=gen).to(dt).to(DEV) for _ in range(2)]
    q = torch.randn(R, hq, d, generator=gen).to(dt).to(DEV)
    results = []
    for off in (0, 1, 3):
        if q8:
            kv = gp.KV8Layer(*pools, *(_offset(s, off) for s in scales))
        else:
            kv = gp.KVLayer(*(_offset(p, off) if kind == "f32" else p for p in pools))
        to = lambda t: _offset(t, off)  # noqa: E731
        ps = gp.PageState(to(table.to(DEV)), to(_i32(npages)), to(_i32(lens)), _i32([1] * pool), _i32([0] * pool), _i32([0]))
        bounds, out = to(torch.zeros(pool, hkv, 2, d, dtype=dt, device=DEV)), [to(torch.full_like(q, NAN)) for _ in range(2)]
        sel, mine = to(torch.zeros(R, hkv, budget, dtype=torch.int32, device=DEV)), to(q)
        (gp.gp_page_bounds_q8 if q8 else gp.gp_page_bounds)(kv, ps, bounds)
        gp.gp_select_pages(bounds, ps, mine, 1, 1, sel, gp.workspace(gp.GP_OP_SELECT, R, 0, hq, hkv, d, width, dt))
        (gp.gp_decode_attention_pages_q8 if q8 else gp.gp_decode_attention_pages)(
            kv, ps, sel, mine, 0.1, out[0], gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, budget, dt))
        (gp.gp_decode_attention_q8 if q8 else gp.gp_decode_attention)(
            kv, ps, mine, 0.1, out[1], gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, width, dt))
        torch.cuda.synchronize()
        results.append([t.clone() for t in (bounds, sel, *out)])
        assert bool(out[0].isfinite().all()) and bool(out[1].isfinite().all())
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "q8"])
def test_most_requests(kind):
    """65535 requests of up to three pages, one KV head: prompts and a token each, bounds, selection, attention."""
    R, hq, hkv, d, width, budget = 65535, 1, 1, 64, 3, 2
    _say(f"most requests {kind}")
    q8 = kind == "q8"
    gen = torch.Generator().manual_seed(65)
    new = torch.randint(0, 46, (R,), generator=gen)
    new[:4] = torch.tensor([0, 45, 1, 16])
    lens = (new + 1).tolist()
    table = torch.randperm(width * R, generator=gen).int().view(R, width)
    pool = width * R
    if q8:
        kv = gp.KV8Layer(*(torch.full((pool, hkv, 16, d), 0x7f, dtype=torch.uint8, device=DEV) for _ in range(2)),
                         *(torch.full((pool, hkv), NAN, device=DEV) for _ in range(2)))
    else:
        kv = gp.KVLayer(*(torch.full((pool, hkv, 16, d), NAN, dtype=BF16, device=DEV) for _ in range(2)))
    append, bound, attend, whole = ((gp.gp_append_rope_q8, gp.gp_page_bounds_q8, gp.gp_decode_attention_pages_q8, gp.gp_decode_attention_q8)
                                    if q8 else (gp.gp_append_rope, gp.gp_page_bounds, gp.gp_decode_attention_pages, gp.gp_decode_attention))
    ps, pos = _state(table, [width] * R, [0] * R, pool), _i32([-1] * R)
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
    T = int(starts[-1])
    k, v = (torch.randn(T, hkv, d, generator=gen).to(BF16) for _ in range(2))
    k1, v1, q = (torch.randn(R, hkv, d, generator=gen).to(BF16) for _ in range(3))
    append(kv, ps, pos, k.to(DEV), v.to(DEV), 1e4, tok_start=_i32(starts))
    q_out = torch.zeros(R, hq, d, dtype=BF16, device=DEV)
    append(kv, ps, pos, k1.to(DEV), v1.to(DEV), 1e4, q=q.to(DEV), q_out=q_out)
    bounds = torch.zeros(pool, hkv, 2, d, dtype=BF16, device=DEV)
    bound(kv, ps, bounds)
    sel = torch.zeros(R, hkv, budget, dtype=torch.int32, device=DEV)
    gp.gp_select_pages(bounds, ps, q_out, 0, 1, sel, gp.workspace(gp.GP_OP_SELECT, R, 0, hq, hkv, d, width, BF16))
    out = [torch.full((R, hq, d), NAN, dtype=BF16, device=DEV) for _ in range(2)]
    attend(kv, ps, sel, q_out, 0.125, out[0], gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, budget, BF16))
    whole(kv, ps, q_out, 0.125, out[1], gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, width, BF16))
    torch.cuda.synchronize()
    assert ps.seq_lens.cpu().tolist() == lens and pos.cpu().tolist() == [m - 1 for m in lens]
    assert all(bool(o.isfinite().all()) for o in out)
    k64, v64 = (_values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)) if q8 else (kv.k.cpu().double(), kv.v.cpu().double())
    box, chosen, qr, got = bounds.cpu(), sel.cpu(), q_out.cpu(), [o.cpu().double() for o in out]
    for r in [0, 1, 2, 3, R - 1] + torch.randint(0, R, (200,), generator=gen).tolist():
        m, n = lens[r], -(-lens[r] // 16)
        rows = torch.cat([k[starts[r]:starts[r + 1]], k1[r:r + 1]]).double()
        want, mag = _rotated(rows, torch.arange(m), 1e4)
        K, V = _tokens(k64, table, r, m), _tokens(v64, table, r, m)
        floor = 2.0 ** -10 * float(kv.k_scale[table[r, :n].long().to(DEV)].max()) if q8 else 0.0
        # (the last page's older codes may have been rounded again under the token's scale: half its lowest step)
        assert bool(((K.transpose(0, 1) - want).abs() <= want.abs() * (2.0 ** -4 if q8 else 2.0 ** -8) + ROT * mag + 2 * floor).all()), r
        for p in range(n):
            assert torch.equal(box[int(table[r, p])].double(), _bounds64(k64, table, lens, r, p)), (r, p)
        want_sel = _select64(box, table, n, qr, hkv, budget, 0, 1, r)
        assert torch.equal(chosen[r], want_sel), r
        tok = [16 * p + j for p in want_sel[0].tolist() if p >= 0 for j in range(min(16, m - 16 * p))]
        for o, pick in ((got[0], tok), (got[1], list(range(m)))):
            want, mag, size = _attention(K[:, pick], V[:, pick], qr[r].double(), 0.125)
            assert bool(((o[r] - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), r


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_widest_tables(kind):
    """Tables and lists of 8192 pages: every page listed, in an order of its own, against the whole cache."""
    R, hq, hkv, d, width = 2, 4, 1, 64, 8192
    _say(f"widest tables {kind}")
    dt, q8 = F32 if kind == "f32" else BF16, kind == "q8"
    gen = torch.Generator().manual_seed(8192)
    lens, npages, pool = [16 * width, 16 * width - 9], [width, width], 2 * width
    table = torch.randperm(pool, generator=gen).int().view(R, width)
    if q8:
        kv = gp.KV8Layer(*(torch.randint(0, 100, (pool, hkv, 16, d), generator=gen).to(torch.uint8).to(DEV) for _ in range(2)),
                         *(torch.rand(pool, hkv, generator=gen).add(0.5).mul(2.0 ** -5).to(DEV) for _ in range(2)))
        k64, v64 = _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    else:
        kv = gp.KVLayer(*(torch.randn(pool, hkv, 16, d, generator=gen).to(dt).to(DEV) for _ in range(2)))
        k64, v64 = kv.k.cpu().double(), kv.v.cpu().double()
    sel = torch.stack([torch.randperm(width, generator=gen) for _ in range(R)]).int().view(R, hkv, width).to(DEV)
    q = torch.randn(R, hq, d, generator=gen).to(dt)
    ps, out = _state(table, npages, lens, pool), [torch.full((R, hq, d), NAN, dtype=dt, device=DEV) for _ in range(2)]
    ws = gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, width, dt)
    (gp.gp_decode_attention_pages_q8 if q8 else gp.gp_decode_attention_pages)(kv, ps, sel, q.to(DEV), 0.125, out[0], ws)
    (gp.gp_decode_attention_q8 if q8 else gp.gp_decode_attention)(kv, ps, q.to(DEV), 0.125, out[1], ws)
    torch.cuda.synchronize()
    for r, m in enumerate(lens):
        want, mag, size = _attention(_tokens(k64, table, r, m), _tokens(v64, table, r, m), q[r].double(), 0.125)
        for o in out:
            assert bool(((o[r].cpu().double() - want).abs() <= _attention_tol(want, mag, size, d, dt)).all()), r


def test_rows_past_32_bits():
    """2^26 + 13 new tokens, whose rows and pages lie past 2^32 bytes: the last of them where they belong."""
    T, R, hkv, d = 2 ** 26 + 13, 600, 1, 64
    _say(f"rows past 32 bits, {T} tokens")
    per = -(-T // R)
    new = [per] * (R - 1) + [T - per * (R - 1)]
    npages = [-(-n // 16) for n in new]
    pool, width = sum(npages), max(npages)
    assert width <= 8192 and T * d * 2 > 2 ** 32
    first = torch.tensor([0] + npages[:-1]).cumsum(0)
    table = (first[:, None] + torch.arange(width)).int()
    for r, P in enumerate(npages):
        table[r, P:] = -1
    table = torch.where(table >= 0, pool - 1 - table, table)              # the last request's pages first
    table = torch.cat([table[R // 2:], table[:R // 2]])                   # (and halfway round)
    counts = npages[R // 2:] + npages[:R // 2]
    sizes = new[R // 2:] + new[:R // 2]
    gen = torch.Generator(device=DEV).manual_seed(26)
    k = torch.randn(T, hkv, d, generator=gen, device=DEV, dtype=BF16)
    v = torch.randn(T, hkv, d, generator=gen, device=DEV, dtype=BF16)
    kv = gp.KVLayer(*(torch.zeros(pool, hkv, 16, d, dtype=BF16, device=DEV) for _ in range(2)))
    ps, pos = _state(table, counts, [0] * R, pool), _i32([-1] * R)
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + n)
    gp.gp_append_rope(kv, ps, pos, k, v, 1e6, tok_start=_i32(starts))
    torch.cuda.synchronize()
    assert ps.seq_lens.cpu().tolist() == sizes
    for r in (0, 1, R // 2 - 1, R // 2, R - 2, R - 1):
        n = sizes[r]
        ids = table[r, :counts[r]].long().to(DEV)
        got = kv.v[ids].transpose(1, 2).reshape(-1, hkv, d)
        assert torch.equal(got[:n], v[starts[r]:starts[r + 1]]) and bool((got[n:] == 0).all()), r
        at = torch.tensor([0, 1, n // 2, n - 2, n - 1])
        want, mag = _rotated(k[starts[r] + at.to(DEV)].cpu().double(), at, 1e6)
        turned = kv.k[ids].transpose(1, 2).reshape(-1, hkv, d)[at.to(DEV)].cpu().double()
        assert bool(((turned - want).abs() <= want.abs() * HALF[BF16] + ROT * mag).all()), r
