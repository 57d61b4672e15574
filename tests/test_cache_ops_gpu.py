"""The operators around the paged cache against plain float64 evaluations of their
definitions: rotated appends, the 8-bit cache and its attention, page bounds,
page selection, attention over listed pages, and a run of them together."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_03494_amd as gp

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


def _say(msg):
    print(f"[cache ops] {msg}", flush=True)


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32).to(DEV)


def _paged(npages, width, gen, spare=3):
    """A table of npages[r] distinct pages per request in random order, -1 behind them."""
    pool = sum(npages) + spare
    perm = torch.randperm(pool, generator=gen).to(torch.int32)
    table = torch.full((len(npages), width), -1, dtype=torch.int32)
    at = 0
    for r, P in enumerate(npages):
        table[r, :P] = perm[at:at + P]
        at += P
    return pool, table


def _state(table, npages, lens, pool):
    return gp.PageState(table.to(DEV), _i32(npages), _i32(lens), torch.ones(pool, dtype=torch.int32, device=DEV),
                        torch.zeros(pool, dtype=torch.int32, device=DEV), _i32([0]))


def _values(codes, scale):
    """What e4m3 codes [pool][head][16][d] stand for, float64 on the CPU."""
    return codes.cpu().view(torch.float8_e4m3fn).double() * scale.cpu().double()[..., None, None]


def _offset(t, elems):
    """A contiguous copy of t whose first element lies `elems` elements into its allocation."""
    buf = torch.empty(t.numel() + elems, dtype=t.dtype, device=t.device)
    buf[elems:].copy_(t.reshape(-1))
    return buf[elems:].view(t.shape)


def _rotated(x, pos, theta):
    """x [tokens][heads][d] float64, positions [tokens]: rotated, and |a| + |b| of each element's pair."""
    d = x.shape[-1]
    ang = pos.double()[:, None, None] * theta ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    mag = (a.abs() + b.abs()).repeat(1, 1, 2)
    return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1), mag


# a float32 cosine or sine is off by 2^-25, each product by 2^-24 of it and the sum by
# 2^-24 of |a| + |b|: less than 2^-22 (|a| + |b|); then half a step of the type
ROT = 2.0 ** -22
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


# ------------------------------------------------------------------- append --

# (resident, pages, new tokens): fresh, mid-page, page edges, none, no room, held (< 0), filling the last slot
RAGGED = [(0, 3, 40), (5, 2, 1), (16, 4, 33), (15, 2, 17), (7, 1, 0), (10, 1, 7), (-20, 4, 3), (31, 2, 1), (16, 1, 1),
          (0, 1, 16), (3, 9, 120), (0, 1, 1), (40, 3, 8)]
SINGLE = [(m, P, 1) for m, P, _ in RAGGED] + [(0, 0, 1), (17, 1, 1)]


def _append_case(cache, reqs, hq, hkv, d, seed, fused, offset, single):
    gen = torch.Generator().manual_seed(seed)
    dt = F32 if cache == "f32" else BF16
    npages = [P for _, P, _ in reqs]
    pool, table = _paged(npages, max(max(npages), 1) + 2, gen)
    T = sum(n for _, _, n in reqs)
    rows = torch.randn(T, hq + 2 * hkv, d, generator=gen)
    rows[..., 3] *= 30.0
    rows = rows.to(dt)
    if fused:                                             # one projection's output, a gap behind every row
        buf = torch.zeros(T, (hq + 2 * hkv) * d + offset + 5, dtype=dt, device=DEV)
        view = buf[:, offset:offset + (hq + 2 * hkv) * d].unflatten(1, (hq + 2 * hkv, d))
        view.copy_(rows)
        q, k, v = view.split([hq, hkv, hkv], 1)
    else:
        q, k, v = (_offset(t.to(DEV), offset) for t in rows.split([hq, hkv, hkv], 1))
    s = dict(gen=gen, dt=dt, pool=pool, table=table, q=q, k=k, v=v, rows=rows.double())
    s["ps"] = _state(table, npages, [m for m, _, _ in reqs], pool)
    s["pos"] = [1000003 * (r % 5) + 7 * r - 1 for r in range(len(reqs))]
    starts = [0]
    for _, _, n in reqs:
        starts.append(starts[-1] + n)
    s["start"], s["starts"] = None if single else _i32(starts), starts
    if cache == "q8":
        codes = torch.randint(0, 127, (2, pool, hkv, 16, d), generator=gen).to(torch.uint8)     # finite, either sign
        codes |= (torch.randint(0, 2, codes.shape, generator=gen) * 128).to(torch.uint8)
        scale = torch.exp2(torch.randint(-12, 2, (2, pool, hkv), generator=gen).float())
        s["kv"] = gp.KV8Layer(codes[0].to(DEV), codes[1].to(DEV), scale[0].to(DEV), scale[1].to(DEV))
        s["before"] = [t.clone() for t in (s["kv"].k, s["kv"].v, s["kv"].k_scale, s["kv"].v_scale)]
    else:
        pools = [_offset(torch.randn(pool, hkv, 16, d, generator=gen).to(dt).to(DEV), offset) for _ in range(2)]
        s["kv"] = gp.KVLayer(*pools)
        s["before"] = [t.clone() for t in pools]
    return s


def _takes(m, P, n):
    return m >= 0 and P > 0 and m + n <= 16 * P


def _check_append(s, cache, reqs, hq, hkv, d, theta, q_out, advanced):
    """Every output of an append, and every byte that it must leave alone."""
    kv, table = s["kv"], s["table"]
    got_q = q_out.cpu().double()
    want_q, mag = _rotated(s["rows"][:, :hq], torch.cat([s["pos"][r] + 1 + torch.arange(n) for r, (_, _, n) in enumerate(reqs)]), theta)
    want_k, mag_k = _rotated(s["rows"][:, hq:hq + hkv], torch.cat([s["pos"][r] + 1 + torch.arange(n) for r, (_, _, n) in enumerate(reqs)]), theta)
    new_v = s["rows"][:, hq + hkv:]
    live = torch.zeros(len(got_q), dtype=torch.bool)
    for r, (m, _, n) in enumerate(reqs):
        live[s["starts"][r]:s["starts"][r + 1]] = m >= 0
    tol = want_q.abs() * HALF[s["dt"]] + ROT * mag
    assert bool(((got_q - want_q).abs() <= tol)[live].all()), float(((got_q - want_q).abs() - tol)[live].max())
    assert bool((got_q[~live] == 7.0).all()), "queries of held requests"
    lens, pos = [m for m, _, _ in reqs], list(s["pos"])
    untouched = torch.ones(s["pool"], 16, dtype=torch.bool)             # (page, slot)
    pages = torch.zeros(s["pool"], dtype=torch.bool)
    for r, (m, P, n) in enumerate(reqs):
        if not _takes(m, P, n) or n == 0:
            continue
        lens[r], pos[r] = m + n, pos[r] + n
        ids = table[r, m // 16:(m + n - 1) // 16 + 1].long()
        pages[ids] = True
        at = torch.arange(m, m + n)
        page, slot = table[r, at // 16].long(), at % 16
        untouched[page, slot] = False
        rows = slice(s["starts"][r], s["starts"][r + 1])
        if cache != "q8":
            k, v = kv.k.cpu()[page, :, slot].double(), kv.v.cpu()[page, :, slot].double()
            assert bool(((k - want_k[rows]).abs() <= want_k[rows].abs() * HALF[s["dt"]] + ROT * mag_k[rows]).all()), f"keys of request {r}"
            assert torch.equal(v, new_v[rows]), f"values of request {r}"
            continue
        for which, want, off in ((0, want_k[rows], ROT * mag_k[rows]), (1, new_v[rows], 0 * mag_k[rows])):
            codes, scale = (kv.k, kv.k_scale) if which == 0 else (kv.v, kv.v_scale)
            new = scale.cpu().double()[ids]
            for i, p in enumerate(ids.tolist()):
                old = s["before"][2 + which].cpu().double()[p]                       # [hkv]
                mine = page == p
                amax = want[mine].abs().amax((0, 2))
                slack = off[mine].amax((0, 2))
                had = i == 0 and m % 16 > 0
                assert bool((torch.frexp(new[i])[0] == 0.5).all()), "a scale that is no power of two"
                assert bool((amax - slack <= 448 * new[i]).all()), "a scale too small"
                if had:
                    assert bool((new[i] >= old).all())
                # no larger than it has to be (the least power of two, or the older one)
                free = ~((new[i] == old) & had)
                assert bool(((amax + slack > 224 * new[i]) | (new[i] == 2.0 ** -100) | ~free).all()), "a scale too large"
                if had:                                                              # the older rows
                    a, b = _values(codes[p:p + 1], scale[p:p + 1])[0][:, :m % 16], _values(s["before"][which][p:p + 1], s["before"][2 + which][p:p + 1])[0][:, :m % 16]
                    assert bool(((a - b).abs() <= new[i][:, None, None] * 2.0 ** -10).all()), "older rows"
                    same = new[i] == old
                    assert torch.equal(codes[p].cpu().view(torch.uint8)[same, :m % 16], s["before"][which][p].cpu().view(torch.uint8)[same, :m % 16])
            got = _values(codes, scale)[page, :, slot]
            per = scale.cpu().double()[page].unsqueeze(-1)
            # half a step of e4m3: 2^-4 of the value, 2^-10 below the normal range
            assert bool(((got - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, per * 2.0 ** -10) + off).all()), f"codes of request {r}"
    older = torch.zeros_like(untouched)
    for r, (m, P, n) in enumerate(reqs):
        if cache == "q8" and _takes(m, P, n) and n and m % 16:
            older[table[r, m // 16].long(), :m % 16] = True             # re-rounded, checked above
    keep = (untouched & ~older)[:, None, :, None].expand(-1, hkv, -1, d)
    raw = torch.uint8 if cache == "q8" else torch.int32 if s["dt"] == F32 else torch.int16
    for t, t0 in ((kv.k, s["before"][0]), (kv.v, s["before"][1])):
        assert torch.equal(t.view(raw).cpu()[keep], t0.view(raw).cpu()[keep]), "slots that nothing was written to"
    if cache == "q8":
        for t, t0 in ((kv.k_scale, s["before"][2]), (kv.v_scale, s["before"][3])):
            assert torch.equal(t.cpu()[~pages], t0.cpu()[~pages]), "scales of pages that nothing was written to"
    if not advanced:
        lens, pos = [m for m, _, _ in reqs], s["pos"]
    assert s["ps"].seq_lens.cpu().tolist() == lens
    assert s["position_tensor"].cpu().tolist() == pos


@pytest.mark.parametrize("cache,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 3, 3, 64), ("f32", 8, 1, 64), ("f32", 4, 2, 128),
                                            ("q8", 32, 8, 128), ("q8", 5, 5, 64), ("q8", 16, 2, 64), ("q8", 4, 2, 128)])
@pytest.mark.parametrize("form", ["ragged", "single", "fused", "no_advance"])
def test_append_rope(cache, hq, hkv, d, form):
    _say(f"append {cache} heads {hq}/{hkv} d {d} {form}")
    reqs = SINGLE if form == "single" else RAGGED
    offset = 0 if form == "ragged" else 3                 # rows (and pools of their type) off 16 bytes
    s = _append_case(cache, reqs, hq, hkv, d, 11 + hq, form == "fused", offset, form == "single")
    q_out = torch.full((s["q"].shape[0], hq, d), 7.0, dtype=s["dt"], device=DEV)
    s["position_tensor"] = _i32(s["pos"])
    fn = gp.gp_append_rope_q8 if cache == "q8" else gp.gp_append_rope
    advance = form != "no_advance"
    theta = 1.0e4 if d == 64 else 1.0e6
    fn(s["kv"], s["ps"], s["position_tensor"], s["k"], s["v"], theta, q=s["q"], q_out=q_out, tok_start=s["start"], advance=advance)
    torch.cuda.synchronize()
    _check_append(s, cache, reqs, hq, hkv, d, theta, q_out, advance)


@pytest.mark.parametrize("cache", ["bf16", "f32", "q8"])
def test_append_rope_many_requests(cache):
    """More requests than a search step covers, most of them short, with and without queries."""
    _say(f"append many requests {cache}")
    reqs = [((7 * r) % 33, 4, (r * r) % 23 if r % 5 else 0) for r in range(300)]
    hq, hkv, d = 2, 2, 64
    s = _append_case(cache, reqs, hq, hkv, d, 5, False, 0, False)
    q_out = torch.full((s["q"].shape[0], hq, d), 7.0, dtype=s["dt"], device=DEV)
    s["position_tensor"] = _i32(s["pos"])
    fn = gp.gp_append_rope_q8 if cache == "q8" else gp.gp_append_rope
    fn(s["kv"], s["ps"], s["position_tensor"], s["k"], s["v"], 1e4, q=s["q"], q_out=q_out, tok_start=s["start"])
    torch.cuda.synchronize()
    _check_append(s, cache, reqs, hq, hkv, d, 1e4, q_out, True)
    # without queries: the same cache
    again = _append_case(cache, reqs, hq, hkv, d, 5, False, 0, False)
    fn(again["kv"], again["ps"], _i32(s["pos"]), again["k"], again["v"], 1e4, tok_start=again["start"])
    torch.cuda.synchronize()
    for x, y in zip(vars(again["kv"]).values(), vars(s["kv"]).values()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_rope_in_place(dtype):
    """q_out may be q: the same rotated queries."""
    _say(f"append in place {dtype}")
    s = _append_case("f32" if dtype == F32 else "bf16", RAGGED, 8, 2, 128, 3, False, 0, False)
    outs = []
    for place in (False, True):
        q = s["q"].clone()
        out = q if place else q.clone()
        gp.gp_append_rope(s["kv"], s["ps"], _i32(s["pos"]), s["k"], s["v"], 1e4, q=q, q_out=out, tok_start=s["start"], advance=False)
        torch.cuda.synchronize()
        outs.append(out.clone())
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("cache", ["bf16", "q8"])
def test_append_rope_starts(cache):
    """Rows before the first request's and behind the last one's are nobody's: their queries are left as they
    were.  Starts that decrease or leave the rows end the call without a write outside the requests' pages."""
    _say(f"append starts {cache}")
    reqs = [(0, 2, 9), (3, 3, 20), (0, 1, 4)]
    s = _append_case(cache, reqs, 2, 2, 64, 17, False, 0, False)
    fn = gp.gp_append_rope_q8 if cache == "q8" else gp.gp_append_rope
    T = s["q"].shape[0]
    pad = lambda t: torch.cat([t[:4], t, t[:7]]).contiguous()  # noqa: E731
    q, k, v = pad(s["q"]), pad(s["k"]), pad(s["v"])
    s["position_tensor"] = _i32(s["pos"])
    q_out = torch.full_like(q, 7.0)
    fn(s["kv"], s["ps"], s["position_tensor"], k, v, 1e4, q=q, q_out=q_out, tok_start=s["start"] + 4)
    torch.cuda.synchronize()
    assert bool((q_out[:4] == 7.0).all()) and bool((q_out[4 + T:] == 7.0).all())
    _check_append(s, cache, reqs, 2, 2, 64, 1e4, q_out[4:4 + T], True)
    owned = torch.zeros(s["pool"], dtype=torch.bool)
    owned[s["table"][s["table"] >= 0].long()] = True
    for starts in ([0, -5, 30, 10], [-2 ** 31, 2 ** 31 - 1, -7, 2 ** 31 - 1], [40, 3, 2, 1], [T + 100, T + 101, T + 102, T + 103]):
        fn(s["kv"], s["ps"], s["position_tensor"], s["k"], s["v"], 1e4, q=s["q"], q_out=torch.empty_like(s["q"]),
           tok_start=_i32(starts), advance=False)
        torch.cuda.synchronize()
        for t, t0 in zip(vars(s["kv"]).values(), s["before"]):
            assert torch.equal(t.view(torch.uint8)[~owned.to(DEV)], t0.view(torch.uint8)[~owned.to(DEV)])


def test_append_rope_bad_pages():
    """Page ids outside the pool and pages beyond the table write nothing."""
    _say("append bad pages")
    for cache in ("bf16", "q8"):
        s = _append_case(cache, [(0, 2, 20), (4, 1, 5), (0, 50, 30)], 2, 2, 64, 9, False, 0, False)
        s["ps"].page_table[0, 0], s["ps"].page_table[0, 1], s["ps"].page_table[1, 0] = -3, s["pool"], 2 ** 30
        s["ps"].num_pages[2] = 500                        # more than the table is wide
        fn = gp.gp_append_rope_q8 if cache == "q8" else gp.gp_append_rope
        fn(s["kv"], s["ps"], _i32(s["pos"]), s["k"], s["v"], 1e4, tok_start=s["start"], advance=False)
        torch.cuda.synchronize()
        for t, t0 in zip(vars(s["kv"]).values(), s["before"]):
            assert torch.equal(t.view(torch.uint8), t0.view(torch.uint8)), cache


def test_append_rope_q8_extremes():
    """Scales of tiny, huge, zero and non-finite rows; older rows under a grown scale, token by token."""
    _say("append q8 extremes")
    hkv, d, R = 2, 64, 6
    pool, table = _paged([1] * R, 1, torch.Generator().manual_seed(0))
    ps = _state(table, [1] * R, [0] * R, pool)
    zero = torch.zeros(pool, hkv, 16, d, dtype=torch.uint8, device=DEV)
    kv = gp.KV8Layer(zero.clone(), zero.clone(), torch.full((pool, hkv), 5.0, device=DEV), torch.full((pool, hkv), NAN, device=DEV))
    pos = _i32([-1] * R)
    ids = table[:, 0].long()
    sizes = torch.tensor([0.0, 2.0 ** -126, 1.0, 3.0e38, 448.0, 1.0])
    gen = torch.Generator().manual_seed(4)
    history = []
    for step in range(16):
        grow = 1.0 if step < 8 else 256.0
        v = (torch.rand(R, hkv, d, generator=gen) - 0.5) * 2
        v[:, :, 0] = 1.0
        v = (v * sizes[:, None, None] * (1.0 if step == 0 else 0.5 * min(grow, 1.0)))
        v[5] *= grow
        v = v.to(BF16)
        if step == 3:
            v[4, 0, 5], v[4, 1, 6], v[4, 1, 7] = float("inf"), -float("inf"), NAN
        history.append(v.double())
        gp.gp_append_rope_q8(kv, ps, pos, torch.zeros_like(v).to(DEV), v.to(DEV), 1e4)
    torch.cuda.synchronize()
    scale = kv.v_scale.cpu()[ids]
    want = torch.stack(history, 2)                                       # [R][hkv][16][d]
    finite = torch.where(want.isfinite(), want, torch.zeros_like(want))
    amax = finite.abs().amax((2, 3))
    for r in range(R):
        for h in range(hkv):
            e = max(-100, math.ceil(math.log2(amax[r, h] / 448))) if amax[r, h] > 0 else -100
            assert float(scale[r, h]) == 2.0 ** e, (r, h, float(scale[r, h]), e)
    assert bool((kv.k_scale.cpu()[ids] == 2.0 ** -100).all())            # keys of zeros
    got = _values(kv.v, kv.v_scale)[ids]
    assert torch.equal(got.isnan(), ~want.isfinite())
    # rounded once under the first scale and once more, below its normal range only, under each larger one
    step = scale.double()[..., None, None] * 2.0 ** -10
    ok = (got - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, 2 * step)
    assert bool((ok | ~want.isfinite()).all())


# ------------------------------------------------------------ 8-bit attention --

def _attention(K, V, q, scale):
    """K, V [Hkv][tokens][d], q [Hq][d], float64: the output, sum_i a_i |v_i|, and the largest sum_d |q_d k_d| scale."""
    Hkv, _, d = K.shape
    z = q.view(Hkv, -1, d) @ K.transpose(1, 2)
    a = torch.softmax(scale * z, -1)
    size = scale * float((q.abs().view(Hkv, -1, d) @ K.abs().transpose(1, 2)).max())
    return (a @ V).reshape(q.shape), (a @ V.abs()).reshape(q.shape), size


def _attention_tol(want, mag, size, d, dtype):
    """Half a step of the output; a score summed in float32 is off by d 2^-24 of its terms' size, which moves each
    weight, and the weights' sum, by as much again; weights of 17 bits; sums of the output as elsewhere in
    float32 (2^-18 of its terms)."""
    return want.abs() * HALF[dtype] + mag * (2 * d * 2.0 ** -24 * size + 2.0 ** -17 + 2.0 ** -18) + 1e-30


def _q8_cache(lens, npages, hkv, d, gen, width, pow2=True):
    """An 8-bit cache whose unowned pages, slots past a length and scales of unowned pages are NaN."""
    pool, table = _paged(npages, width, gen)
    codes = torch.full((2, pool, hkv, 16, d), 0x7f, dtype=torch.uint8)
    scale = torch.full((2, pool, hkv), NAN)
    for r, m in enumerate(lens):
        for p in range(-(-max(m, 0) // 16)):
            t, pid = min(16, m - 16 * p), int(table[r, p])
            x = torch.randn(2, hkv, t, d, generator=gen)
            s = torch.exp2(torch.randint(-9, -5, (2, hkv), generator=gen).float())
            if not pow2:
                s = s * (0.75 + 0.5 * torch.rand(2, hkv, generator=gen))
            codes[:, pid, :, :t] = (x / s[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            scale[:, pid] = s
    kv = gp.KV8Layer(codes[0].to(DEV), codes[1].to(DEV), scale[0].to(DEV), scale[1].to(DEV))
    return kv, pool, table


def _tokens(pool64, table, r, m):
    ids = table[r, :-(-m // 16)].long()
    return pool64[ids].transpose(0, 1).flatten(1, 2)[:, :m]


LENGTHS = {
    "one_token": [1],
    "page_edges": [15, 16, 17, 0, 1, 33, 32],
    "one_long": [4099],
    "mixed": [0, 700, 3, 0, 2500, 16, 48, 1, 1600, 0],
    "many_short": [(r * 37) % 60 for r in range(600)],
    "short_in_wide_table": [0, 768, 5, 384, 17, 383, 1],
    "a_page_too_long": [769, 385, 40, 0, 3],
}


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("spare", [2, 70, 130])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (2, 2, 128), (3, 3, 64), (8, 4, 64), (16, 2, 64), (8, 1, 128)])
def test_decode_q8(name, spare, hq, hkv, d):
    lens = LENGTHS[name]
    _say(f"decode q8 {name} heads {hq}/{hkv} d {d} spare {spare}")
    gen = torch.Generator().manual_seed(hq * 100 + spare)
    npages = [-(-m // 16) + (r % 3 == 1) for r, m in enumerate(lens)]
    width = max(max(npages), 1) + spare
    kv, pool, table = _q8_cache(lens, npages, hkv, d, gen, width, pow2=spare != 70)
    q = torch.randn(len(lens), hq, d, generator=gen).to(BF16)
    ps = _state(table, npages, lens, pool)
    ws = gp.workspace(gp.GP_OP_DECODE, len(lens), 0, hq, hkv, d, width, BF16)
    scale = d ** -0.5
    out = torch.full((len(lens), hq, d), NAN, dtype=BF16, device=DEV)
    gp.gp_decode_attention_q8(kv, ps, q.to(DEV), scale, out, ws)
    torch.cuda.synchronize()
    got, k64, v64 = out.cpu().double(), _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    for r, m in enumerate(lens):
        if m == 0:
            assert bool((got[r] == 0).all())
            continue
        want, mag, size = _attention(_tokens(k64, table, r, m), _tokens(v64, table, r, m), q[r].double(), scale)
        assert bool(((got[r] - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), f"request {r}"
    # the same call again: the same bytes; held requests keep their place and their rows
    held = [r for r in range(0, len(lens), 3) if lens[r] > 0]
    for r in held:
        ps.seq_lens[r] = -lens[r] - 1
    again = torch.full_like(out, 7.0)
    gp.gp_decode_attention_q8(kv, ps, q.to(DEV), scale, again, ws)
    torch.cuda.synchronize()
    keep = torch.tensor([r not in held for r in range(len(lens))], device=DEV)
    assert torch.equal(again[keep], out[keep]) and bool((again[~keep] == 7.0).all())


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (3, 3, 64)])
def test_decode_q8_every_code(hq, hkv, d):
    """Each finite code as a value, met by a weight of one: the value it stands for, times the scale."""
    _say(f"decode q8 every code heads {hq}/{hkv} d {d}")
    finite = [c for c in range(256) if c & 0x7f != 0x7f]
    lens = [1] * 16
    pool, table = _paged([1] * 16, 4, torch.Generator().manual_seed(1))
    codes = torch.full((pool, hkv, 16, d), 0x7f, dtype=torch.uint8)
    for r in range(16):
        codes[table[r, 0], :, 0] = torch.tensor([[finite[(d * (hkv * r + h) + i) % len(finite)] for i in range(d)] for h in range(hkv)], dtype=torch.uint8)
    scale = torch.full((pool, hkv), 0.5)
    kv = gp.KV8Layer(torch.zeros_like(codes).to(DEV), codes.to(DEV), scale.to(DEV), scale.to(DEV))
    ps = _state(table, [1] * 16, lens, pool)
    q = torch.randn(16, hq, d).to(BF16).to(DEV)
    out = torch.empty_like(q)
    gp.gp_decode_attention_q8(kv, ps, q, 0.1, out, gp.workspace(gp.GP_OP_DECODE, 16, 0, hq, hkv, d, 4, BF16))
    torch.cuda.synchronize()
    want = _values(kv.v, kv.v_scale)[table[:, 0].long()][:, :, 0].repeat_interleave(hq // hkv, 1)
    assert torch.equal(out.cpu().double(), want)


def test_decode_q8_nan_and_bad_pages():
    """A NaN key gives a zero output, a NaN value a NaN in its dim only; bad page ids add nothing."""
    _say("decode q8 NaN and bad pages")
    hq, hkv, d = 4, 2, 64
    lens = [40, 40, 40, 900]
    npages = [3, 3, 3, 57]
    gen = torch.Generator().manual_seed(2)
    kv, pool, table = _q8_cache(lens, npages, hkv, d, gen, 200)
    kv.k[int(table[0, 1]), 0, 5, 9] = 0x7f
    kv.v[int(table[1, 1]), 1, 6, 11] = 0xff
    ps = _state(table, npages, lens, pool)
    ps.page_table[2, 1] = pool + 5
    ps.page_table[3, 20] = -7
    q = torch.randn(4, hq, d, generator=gen).to(BF16)
    out = torch.empty(4, hq, d, dtype=BF16, device=DEV)
    gp.gp_decode_attention_q8(kv, ps, q.to(DEV), 0.2, out, gp.workspace(gp.GP_OP_DECODE, 4, 0, hq, hkv, d, 200, BF16))
    torch.cuda.synchronize()
    got = out.cpu().double()
    assert bool((got[0, :2] == 0).all()) and bool(got[0, 2:].isfinite().all())
    nan = torch.zeros(hq, d, dtype=torch.bool)
    nan[2:, 11] = True
    assert torch.equal(got[1].isnan(), nan)
    k64, v64 = _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    for r, gone in ((2, 1), (3, 20)):
        keep = [i for i in range(lens[r]) if i // 16 != gone]
        want, mag, size = _attention(_tokens(k64, table, r, lens[r])[:, keep], _tokens(v64, table, r, lens[r])[:, keep], q[r].double(), 0.2)
        assert bool(((got[r] - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), r


@pytest.mark.parametrize("spare", [2, 130])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (3, 3, 64)])
def test_decode_q8_pages_gone(hq, hkv, d, spare):
    """Page ids outside the pool, two or more in a row, at a request's ends and all of one's: they add
    nothing, whatever page 0 and its scales hold."""
    _say(f"decode q8 pages gone heads {hq}/{hkv} d {d} spare {spare}")
    gen = torch.Generator().manual_seed(6 + spare)
    lens = [200, 33, 64, 1500, 16]
    npages = [-(-m // 16) for m in lens]
    width = max(npages) + spare
    kv, pool, table = _q8_cache(lens, npages, hkv, d, gen, width, pow2=False)
    k64, v64 = _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    gone = {0: [0, 1, 2, 5, 12], 1: [2], 2: [0, 1, 2, 3], 3: list(range(40, 71)) + [93], 4: []}
    ps = _state(table, npages, lens, pool)
    owner = (table == 0).nonzero()
    if len(owner):                                        # page 0 belongs to nobody in what follows
        gone[int(owner[0, 0])].append(int(owner[0, 1]))
    for r, ps_ in gone.items():
        for i, p in enumerate(ps_):
            ps.page_table[r, p] = (-1, pool, -2 ** 31, 2 ** 31 - 1)[i % 4]
    kv.k[0], kv.v[0], kv.k_scale[0], kv.v_scale[0] = 0x7f, 0xff, NAN, NAN
    q = torch.randn(len(lens), hq, d, generator=gen).to(BF16)
    out = torch.empty(len(lens), hq, d, dtype=BF16, device=DEV)
    gp.gp_decode_attention_q8(kv, ps, q.to(DEV), 0.2, out, gp.workspace(gp.GP_OP_DECODE, len(lens), 0, hq, hkv, d, width, BF16))
    torch.cuda.synchronize()
    got = out.cpu().double()
    for r, m in enumerate(lens):
        keep = [i for i in range(m) if i // 16 not in gone[r]]
        if not keep:
            assert bool((got[r] == 0).all()), r
            continue
        want, mag, size = _attention(_tokens(k64, table, r, m)[:, keep], _tokens(v64, table, r, m)[:, keep], q[r].double(), 0.2)
        assert bool(((got[r] - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), r


@pytest.mark.parametrize("spare", [2, 130])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (3, 3, 64)])
def test_decode_q8_small_weights(hq, hkv, d, spare):
    """A weight of 2^-128 beside one of 1 whose value is zero: the result is that weight times its value, to the
    2^-150 that a subnormal weight is off (2^-22 of the result), the tokens in one page, in a pair and in two."""
    _say(f"decode q8 small weights heads {hq}/{hkv} d {d} spare {spare}")
    lens, gen = [2, 17, 33], torch.Generator().manual_seed(1)
    npages = [1, 2, 3]
    kv, pool, table = _q8_cache(lens, npages, hkv, d, gen, 3 + spare)
    code = lambda x: int(torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8))  # noqa: E731
    for r, m in enumerate(lens):
        for p in range(npages[r]):
            pid, t = int(table[r, p]), min(16, m - 16 * p)
            kv.k[pid, :, :t], kv.v[pid, :, :t] = 0, 0
            kv.k[pid, :, :t, 0] = code(-384.0)
            kv.k_scale[pid], kv.v_scale[pid] = 2.0, 2.0 ** 93
        kv.k[int(table[r, 0]), :, 0, 0] = 0
        kv.k[int(table[r, (m - 1) // 16]), :, (m - 1) % 16, 0] = code(-64.0)
        kv.v[int(table[r, (m - 1) // 16]), :, (m - 1) % 16] = code(128.0)
    q = torch.zeros(3, hq, d, dtype=BF16, device=DEV)
    q[..., 0] = 1.0
    out = torch.empty_like(q)
    gp.gp_decode_attention_q8(kv, _state(table, npages, lens, pool), q, 1.0 / 1.4426950408889634, out,
                              gp.workspace(gp.GP_OP_DECODE, 3, 0, hq, hkv, d, 3 + spare, BF16))
    torch.cuda.synchronize()
    # the float32 scale moves 2^-128 by 128 of its roundings at most, and the result is rounded to bfloat16
    assert bool(((out.cpu().double() / 2.0 ** -28 - 1).abs() <= 2.0 ** -8).all()), out.flatten()[:4]


# -------------------------------------------------------------------- bounds --

def _cache(kind, lens, npages, hkv, d, gen, width):
    """A cache of any kind with NaN where nothing is resident: (layer, pool, table, keys, values in float64)."""
    if kind == "q8":
        kv, pool, table = _q8_cache(lens, npages, hkv, d, gen, width)
        return kv, pool, table, _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    dt = F32 if kind == "f32" else BF16
    pool, table = _paged(npages, width, gen)
    kv = torch.full((2, pool, hkv, 16, d), NAN, dtype=dt)
    for r, m in enumerate(lens):
        for p in range(-(-max(m, 0) // 16)):
            t = min(16, m - 16 * p)
            kv[:, table[r, p], :, :t] = torch.randn(2, hkv, t, d, generator=gen).to(dt)
    return gp.KVLayer(kv[0].to(DEV), kv[1].to(DEV)), pool, table, kv[0].double(), kv[1].double()


def _bounds64(k64, table, lens, r, p):
    x = k64[int(table[r, p])][:, :min(16, lens[r] - 16 * p)]
    return torch.stack([x.amin(1), x.amax(1)], 1)


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
@pytest.mark.parametrize("hkv,d", [(1, 64), (3, 128), (8, 128), (5, 64)])
@pytest.mark.parametrize("limit", [0, 1, 2])
def test_page_bounds(kind, hkv, d, limit):
    _say(f"bounds {kind} heads {hkv} d {d} max_update {limit}")
    lens = [0, 1, 16, 17, 500, 33, 47, 64, 2]
    frm = [0, 0, 15, 16, 100, 0, 47, -5, 1]
    npages = [-(-m // 16) + 1 for m in lens]
    kv, pool, table, k64, _ = _cache(kind, lens, npages, hkv, d, torch.Generator().manual_seed(d + hkv), 40)
    bad = (4, 10)
    state_lens = list(lens)
    state_lens[5] = -lens[5] - 1                                          # held
    ps = _state(table, npages, state_lens, pool)
    ps.page_table[bad] = pool
    dt = F32 if kind == "f32" else BF16
    bounds = torch.full((pool, hkv, 2, d), 7.0, dtype=dt, device=DEV)
    want = bounds.cpu().double()
    for given in (True, False):
        (gp.gp_page_bounds_q8 if kind == "q8" else gp.gp_page_bounds)(kv, ps, bounds, from_tokens=_i32(frm) if given else None, max_update=limit)
        torch.cuda.synchronize()
        for r, m in enumerate(lens):
            f = max(0, frm[r]) if given else 0
            pages = range(f // 16, -(-m // 16)) if r != 5 and f < m else ()
            for p in list(pages)[:limit or None]:
                if (r, p) != bad:
                    want[int(table[r, p])] = _bounds64(k64, table, lens, r, p).to(dt).double()
        assert torch.equal(bounds.cpu().double(), want)


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_page_bounds_nan_and_infinities(kind):
    _say(f"bounds NaN {kind}")
    gen = torch.Generator().manual_seed(8)
    kv, pool, table, k64, _ = _cache(kind, [16, 16, 16], [1, 1, 1], 2, 64, gen, 2)
    a, b, c = (int(x) for x in table[:, 0])
    if kind == "q8":
        kv.k[a, 0, 3, 7] = 0x7f
        kv.k[b, 1, 15, 8] = 0xff
    else:
        kv.k[a, 0, 3, 7] = kv.k[b, 1, 15, 8] = NAN
        kv.k[c, 0, 0, 1], kv.k[c, 0, 9, 2] = float("inf"), -float("inf")
        k64[c, 0, 0, 1], k64[c, 0, 9, 2] = float("inf"), -float("inf")
    bounds = torch.zeros(pool, 2, 2, 64, dtype=F32 if kind == "f32" else BF16, device=DEV)
    (gp.gp_page_bounds_q8 if kind == "q8" else gp.gp_page_bounds)(kv, _state(table, [1] * 3, [16] * 3, pool), bounds)
    torch.cuda.synchronize()
    got = bounds.cpu().double()
    nan = torch.zeros(pool, 2, 2, 64, dtype=torch.bool)
    nan[a, 0, :, 7] = nan[b, 1, :, 8] = True
    assert torch.equal(got.isnan(), nan)
    for r, p in enumerate((a, b, c)):
        want = _bounds64(k64, table, [16] * 3, r, 0)
        assert torch.equal(got[p][~nan[p]], want[~nan[p]])


# ----------------------------------------------------------------- selection --

def _select64(bounds, table, n, q, hkv, budget, first, last, r):
    """Selected logical pages of request r, by the definition in float64, [hkv][budget]."""
    d = q.shape[-1]
    out = torch.full((hkv, budget), -1, dtype=torch.int32)
    for h in range(hkv):
        if n <= budget:
            pick = torch.arange(n)
        else:
            box = bounds[table[r, :n].long(), h].double()                 # [n][2][d]
            x = q[r].double().view(hkv, -1, 1, d)[h]
            score = torch.maximum(x * box[:, 0], x * box[:, 1]).sum((0, 2)).float()
            middle = torch.arange(first, n - last)
            # (torch sorts NaN as the greatest)
            best = middle[score[middle].sort(dim=0, descending=True, stable=True)[1]][:budget - first - last]
            pick = torch.cat([torch.arange(first), best, torch.arange(n - last, n)]).sort()[0]
        out[h, :len(pick)] = pick.int()
    return out


SELECT = {                                                # lengths, table width, budget, keep_first, keep_last
    "small": ([0, 1, 16, 17, 100, 160, 161, 400], 30, 10, 1, 2),
    "forced_only": ([400, 1000, 33], 70, 5, 2, 3),
    "one_page": ([400, 16, 5], 30, 1, 0, 0),
    "no_forced": ([1000, 900, 129], 70, 8, 0, 0),
    "middle": ([16 * 1500, 16 * 1024 + 1, 16 * 1023, 5000], 1501, 200, 1, 1),
    "wide": ([16 * 8192, 16 * 4097, 16 * 8191 + 3], 8192, 1000, 4, 9),
    "whole_table": ([16 * 30, 200], 30, 64, 1, 1),
    "all_but_one": ([16 * 300, 16 * 299], 300, 299, 0, 1),
}


@pytest.mark.parametrize("name", list(SELECT))
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF16, 8, 2, 128), (BF16, 8, 1, 64), (F32, 4, 2, 64), (F32, 2, 2, 128), (BF16, 3, 3, 64)])
def test_select_pages(name, dtype, hq, hkv, d):
    lens, width, budget, first, last = SELECT[name]
    _say(f"select {name} {dtype} heads {hq}/{hkv} d {d}")
    gen = torch.Generator().manual_seed(len(name) + d)
    npages = [min(width, -(-m // 16) + 1) for m in lens]
    pool, table = _paged(npages, width, gen)
    centre = torch.randn(pool, hkv, 1, d, generator=gen)
    half = torch.rand(pool, hkv, 1, d, generator=gen) * 2
    bounds = torch.cat([centre - half, centre + half], 2).to(dtype)
    for r, m in enumerate(lens):                          # ties: the same box on several pages
        n = -(-m // 16)
        if n > 20:
            for p in range(7, n, 5):
                bounds[table[r, p].long()] = bounds[table[r, 7].long()]
    q = torch.randn(len(lens), hq, d, generator=gen).to(dtype)
    ps = _state(table, npages, lens, pool)
    ps.seq_lens[1] = -lens[1] - 1                         # held: its lists are not written
    ws = gp.workspace(gp.GP_OP_SELECT, len(lens), 0, hq, hkv, d, width, dtype)
    sel = torch.full((len(lens), hkv, budget), -9, dtype=torch.int32, device=DEV)
    gp.gp_select_pages(bounds.to(DEV), ps, q.to(DEV), first, last, sel, ws)
    torch.cuda.synchronize()
    got = sel.cpu()
    for r, m in enumerate(lens):
        if r == 1:
            assert bool((got[r] == -9).all())
        else:
            want = _select64(bounds, table, -(-m // 16), q, hkv, budget, first, last, r)
            assert torch.equal(got[r], want), (r, m)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_extreme_scores(dtype):
    """NaN above all, infinities, all scores equal, zero queries, negative scores; a bad page id comes last."""
    _say(f"select extremes {dtype}")
    hq, hkv, d, n, budget = 2, 1, 64, 50, 8
    gen = torch.Generator().manual_seed(3)
    pool, table = _paged([n] * 5, n, gen)
    bounds = torch.randn(pool, hkv, 1, d, generator=gen).repeat(1, 1, 2, 1).to(dtype)
    q = torch.ones(5, hq, d).to(dtype)
    at = lambda r, p: table[r, p].long()  # noqa: E731
    bounds[at(0, 30), 0, 1, 3] = NAN
    bounds[at(0, 40), 0, 1, 3] = float("inf")
    bounds[at(0, 41), 0, :, 3] = -float("inf")
    bounds[table[1].long()] = 0.5                                        # all alike
    q[2] = 0.0
    bounds[table[3].long()] -= 20.0                                      # all negative
    ps = _state(table, [n] * 5, [16 * n] * 5, pool)
    ps.page_table[4, 10] = pool
    ps.page_table[4, 11] = -2
    sel = torch.empty(5, hkv, budget, dtype=torch.int32, device=DEV)
    ws = gp.workspace(gp.GP_OP_SELECT, 5, 0, hq, hkv, d, n, dtype)
    gp.gp_select_pages(bounds.to(DEV), ps, q.to(DEV), 1, 1, sel, ws)
    torch.cuda.synchronize()
    got = sel.cpu()
    for r in range(4):
        assert torch.equal(got[r], _select64(bounds, table, n, q, hkv, budget, 1, 1, r)), r
    assert got[0, 0].tolist().count(30) == 1 and got[0, 0].tolist().count(40) == 1 and 41 not in got[0, 0].tolist()
    assert got[1, 0].tolist() == got[2, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, n - 1]
    assert 10 not in got[4, 0].tolist() and 11 not in got[4, 0].tolist()


@pytest.mark.parametrize("n,width,budget", [(2000, 2048, 700), (1000, 1000, 300), (8192, 8192, 4000), (600, 700, 3)])
def test_select_many_alike(n, width, budget):
    """Hundreds of pages of the same score at the border of the selection: the lowest are taken; beside
    them others above and below, or NaN, or nothing else."""
    _say(f"select many alike {n} of {width} budget {budget}")
    hq, hkv, d = 4, 2, 64
    gen = torch.Generator().manual_seed(n)
    pool, table = _paged([n] * 4, width, gen)
    bounds = torch.ones(pool, hkv, 2, d, dtype=BF16)
    some = torch.randperm(n, generator=gen)
    up, down = some[:budget // 3], some[budget // 3:budget // 3 + n // 8]
    bounds[table[1, up].long()] = 3.0
    bounds[table[1, down].long()] = torch.randn(len(down), 1, 1, 1, generator=gen).clamp(-2, 0.9).to(BF16)
    bounds[table[2, some[:n // 2]].long(), :, 1, 5] = NAN
    bounds[table[3, up].long(), :, 1] = float("inf")
    bounds[table[3, down].long(), :, 0] = -float("inf")
    q = torch.ones(4, hq, d, dtype=BF16)
    sel = torch.empty(4, hkv, budget, dtype=torch.int32, device=DEV)
    ws = gp.workspace(gp.GP_OP_SELECT, 4, 0, hq, hkv, d, width, BF16)
    gp.gp_select_pages(bounds.to(DEV), _state(table, [n] * 4, [16 * n - 5] * 4, pool), q.to(DEV), 1, 1, sel, ws)
    torch.cuda.synchronize()
    got = sel.cpu()
    for r in range(4):
        b = bounds.clone()
        if r == 3:                                        # a least value of -inf meets no negative query
            b[..., 0, :] = torch.where(b[..., 0, :].isinf(), torch.zeros(()).to(BF16), b[..., 0, :])
        assert torch.equal(got[r], _select64(b, table, n, q, hkv, budget, 1, 1, r)), r


# --------------------------------------------------------- attention over lists --

@pytest.mark.parametrize("kind,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 3, 3, 64), ("f32", 8, 1, 64), ("f32", 4, 2, 128),
                                           ("q8", 8, 2, 128), ("q8", 8, 1, 64), ("q8", 2, 2, 64)])
@pytest.mark.parametrize("name", ["mixed", "page_edges", "one_long", "short_in_wide_table"])
@pytest.mark.parametrize("budget", [1, 7, 60, 200])
def test_decode_pages(kind, hq, hkv, d, name, budget):
    """Lists of any pages in any order, another one for each head: repeated pages, -1 and pages
    that are not resident among them."""
    lens = LENGTHS[name]
    _say(f"decode pages {kind} {name} heads {hq}/{hkv} d {d} budget {budget}")
    gen = torch.Generator().manual_seed(budget + d)
    npages = [-(-m // 16) + (r % 3 == 1) for r, m in enumerate(lens)]
    width = max(npages) + 3
    kv, pool, table, k64, v64 = _cache(kind, lens, npages, hkv, d, gen, width)
    R, dt = len(lens), F32 if kind == "f32" else BF16
    sel = torch.full((R, hkv, budget), -1, dtype=torch.int32)
    for r, m in enumerate(lens):
        n = -(-m // 16)
        for h in range(hkv):
            row = torch.randint(-1, n + 2, (budget,), generator=gen).int()
            if (r + h) % 2 and n:
                row = torch.randperm(n, generator=gen)[:budget].int()
            sel[r, h, :len(row)] = row
    q = torch.randn(R, hq, d, generator=gen).to(dt)
    ps = _state(table, npages, lens, pool)
    ps.seq_lens[R - 1] = -lens[R - 1] - 1 if R > 1 else lens[0]
    out = torch.full((R, hq, d), 7.0, dtype=dt, device=DEV)
    ws = gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, budget, dt)
    scale, G = d ** -0.5, hq // hkv
    (gp.gp_decode_attention_pages_q8 if kind == "q8" else gp.gp_decode_attention_pages)(kv, ps, sel.to(DEV), q.to(DEV), scale, out, ws)
    torch.cuda.synchronize()
    got = out.cpu().double()
    for r, m in enumerate(lens):
        if r == R - 1 and R > 1:
            assert bool((got[r] == 7.0).all())
            continue
        n = -(-m // 16)
        for h in range(hkv):
            tok = [16 * p + i for p in sel[r, h, :min(n, budget)].tolist() if 0 <= p < n for i in range(min(16, m - 16 * p))]
            mine = got[r, h * G:(h + 1) * G]
            if not tok:
                assert bool((mine == 0).all()), (r, h)
                continue
            want, mag, size = _attention(_tokens(k64, table, r, m)[h:h + 1, tok], _tokens(v64, table, r, m)[h:h + 1, tok],
                                         q[r, h * G:(h + 1) * G].double(), scale)
            tol = _attention_tol(want, mag, size, d, dt)
            assert bool(((mine - want).abs() <= tol).all()), (r, h, float(((mine - want).abs() - tol).max()))


@pytest.mark.parametrize("kind", ["bf16", "q8"])
def test_decode_pages_many_requests(kind):
    """More requests than a block of the split's scan, lists of a few pages."""
    _say(f"decode pages many requests {kind}")
    hq, hkv, d, budget = 4, 2, 64, 5
    gen = torch.Generator().manual_seed(12)
    lens = [(r * 37) % 150 for r in range(1100)]
    npages = [-(-m // 16) for m in lens]
    kv, pool, table, k64, v64 = _cache(kind, lens, npages, hkv, d, gen, max(npages) + 40)
    sel = torch.randint(-1, 10, (len(lens), hkv, budget), generator=gen).int()
    q = torch.randn(len(lens), hq, d, generator=gen).to(BF16)
    for columns in (budget, 80):                          # a workgroup per request, or equal runs of the batch
        wide = torch.cat([sel, torch.full((len(lens), hkv, columns - budget), -1, dtype=torch.int32)], 2)
        out = torch.full((len(lens), hq, d), NAN, dtype=BF16, device=DEV)
        ws = gp.workspace(gp.GP_OP_DECODE, len(lens), 0, hq, hkv, d, columns, BF16)
        (gp.gp_decode_attention_pages_q8 if kind == "q8" else gp.gp_decode_attention_pages)(
            kv, _state(table, npages, lens, pool), wide.to(DEV), q.to(DEV), 0.125, out, ws)
        torch.cuda.synchronize()
        got = out.cpu().double()
        for r, m in enumerate(lens):
            n = -(-m // 16)
            for h in range(hkv):
                tok = [16 * p + i for p in wide[r, h, :min(n, columns)].tolist() if 0 <= p < n for i in range(min(16, m - 16 * p))]
                mine = got[r, 2 * h:2 * h + 2]
                if not tok:
                    assert bool((mine == 0).all()), (r, h)
                    continue
                want, mag, size = _attention(_tokens(k64, table, r, m)[h:h + 1, tok], _tokens(v64, table, r, m)[h:h + 1, tok],
                                             q[r, 2 * h:2 * h + 2].double(), 0.125)
                assert bool(((mine - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), (r, h)


# --------------------------------------------------------------- all together --

@pytest.mark.parametrize("kind", ["bf16", "q8"])
def test_pools_past_32_bits(kind):
    """Pools of more than 2^32 bytes, their last pages used: prompts in, bounds, selection, attention."""
    hkv, d, hq, budget = 8, 128, 16, 6
    dt, size = (torch.uint8, 1) if kind == "q8" else (BF16, 2)
    pool = (2 ** 32 + 2 ** 28) // (hkv * 16 * d * size)
    _say(f"pools past 32 bits {kind}, {pool} pages")
    lens = [200, 37]
    npages = [-(-m // 16) for m in lens]
    table = torch.full((2, 16), -1, dtype=torch.int32)
    table[0, :13], table[1, :3] = pool - 1 - torch.arange(13), pool - 20 - torch.arange(3)
    k, v = (torch.empty(pool, hkv, 16, d, dtype=dt, device=DEV) for _ in range(2))
    if kind == "q8":
        kv = gp.KV8Layer(k, v, torch.zeros(pool, hkv, device=DEV), torch.zeros(pool, hkv, device=DEV))
    else:
        kv = gp.KVLayer(k, v)
    bounds = torch.empty(pool, hkv, 2, d, dtype=BF16, device=DEV)
    ps = _state(table, npages, [0, 0], pool)
    gen = torch.Generator().manual_seed(5)
    T = sum(lens)
    kn, vn = (torch.randn(T, hkv, d, generator=gen).to(BF16) for _ in range(2))
    q = torch.randn(2, hq, d, generator=gen).to(BF16)
    q8 = kind == "q8"
    (gp.gp_append_rope_q8 if q8 else gp.gp_append_rope)(kv, ps, _i32([-1, -1]), kn.to(DEV), vn.to(DEV), 1e4, tok_start=_i32([0, lens[0], T]))
    (gp.gp_page_bounds_q8 if q8 else gp.gp_page_bounds)(kv, ps, bounds)
    sel = torch.zeros(2, hkv, budget, dtype=torch.int32, device=DEV)
    gp.gp_select_pages(bounds, ps, q.to(DEV), 1, 1, sel, gp.workspace(gp.GP_OP_SELECT, 2, 0, hq, hkv, d, 16, BF16))
    outs = [torch.zeros(2, hq, d, dtype=BF16, device=DEV) for _ in range(2)]
    (gp.gp_decode_attention_pages_q8 if q8 else gp.gp_decode_attention_pages)(
        kv, ps, sel, q.to(DEV), 0.1, outs[0], gp.workspace(gp.GP_OP_DECODE, 2, 0, hq, hkv, d, budget, BF16))
    (gp.gp_decode_attention_q8 if q8 else gp.gp_decode_attention)(
        kv, ps, q.to(DEV), 0.1, outs[1], gp.workspace(gp.GP_OP_DECODE, 2, 0, hq, hkv, d, 16, BF16))
    torch.cuda.synchronize()
    start = 0
    for r, m in enumerate(lens):
        ids = table[r, :npages[r]].long().to(DEV)
        K, V = kv.k[ids].cpu(), kv.v[ids].cpu()
        K, V = ((_values(K, kv.k_scale[ids]), _values(V, kv.v_scale[ids])) if q8 else (K.double(), V.double()))
        K, V = (x.transpose(0, 1).flatten(1, 2)[:, :m] for x in (K, V))
        want, mag = _rotated(kn[start:start + m].double(), torch.arange(m), 1e4)
        step = 2.0 ** -4 if q8 else 2.0 ** -8             # (no value of these is below e4m3's normal range by much)
        floor = 2.0 ** -10 * float(kv.k_scale[ids].max()) if q8 else 0.0
        assert bool(((K.transpose(0, 1) - want).abs() <= want.abs() * step + ROT * mag + floor).all())
        start += m
        box, n = bounds[ids].cpu(), npages[r]
        local = torch.arange(n).view(1, n).expand(2, n)
        want_sel = _select64(box, local, n, q, hkv, budget, 1, 1, r)
        assert torch.equal(sel[r].cpu(), want_sel)
        for h in range(hkv):
            g = slice(2 * h, 2 * h + 2)
            tok = [16 * p + i for p in want_sel[h].tolist() if p >= 0 for i in range(min(16, m - 16 * p))]
            for out, pick in ((outs[0], tok), (outs[1], list(range(m)))):
                want, mag, size = _attention(K[h:h + 1, pick], V[h:h + 1, pick], q[r, g].double(), 0.1)
                assert bool(((out[r, g].cpu().double() - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), (r, h)


def test_two_streams_at_once():
    """Two batches on two streams with workspaces of their own: the results of one after the other."""
    _say("two streams at once")
    hq, hkv, d, budget = 32, 8, 128, 20
    gen = torch.Generator().manual_seed(77)
    batches = []
    for b in range(2):
        lens = [700 + 90 * ((r + b) % 11) for r in range(24)]
        npages = [-(-m // 16) for m in lens]
        width = max(npages) + 200
        kv, pool, table = _q8_cache(lens, npages, hkv, d, gen, width)
        batches.append(dict(kv=kv, ps=_state(table, npages, lens, pool), q=torch.randn(24, hq, d, generator=gen).to(BF16).to(DEV),
                            bounds=torch.zeros(pool, hkv, 2, d, dtype=BF16, device=DEV),
                            sel=torch.zeros(24, hkv, budget, dtype=torch.int32, device=DEV),
                            out=[torch.zeros(24, hq, d, dtype=BF16, device=DEV) for _ in range(2)],
                            ws=[gp.workspace(gp.GP_OP_SELECT, 24, 0, hq, hkv, d, width, BF16),
                                gp.workspace(gp.GP_OP_DECODE, 24, 0, hq, hkv, d, budget, BF16),
                                gp.workspace(gp.GP_OP_DECODE, 24, 0, hq, hkv, d, width, BF16)],
                            stream=torch.cuda.Stream()))

    def go(x, stream):
        gp.gp_page_bounds_q8(x["kv"], x["ps"], x["bounds"], stream=stream)
        gp.gp_select_pages(x["bounds"], x["ps"], x["q"], 1, 2, x["sel"], x["ws"][0], stream=stream)
        gp.gp_decode_attention_pages_q8(x["kv"], x["ps"], x["sel"], x["q"], 0.1, x["out"][0], x["ws"][1], stream=stream)
        gp.gp_decode_attention_q8(x["kv"], x["ps"], x["q"], 0.1, x["out"][1], x["ws"][2], stream=stream)

    torch.cuda.synchronize()
    for x in batches:
        go(x, None)
    torch.cuda.synchronize()
    alone = [[t.clone() for t in (x["bounds"], x["sel"], *x["out"])] for x in batches]
    for x in batches:
        for t in (x["bounds"], x["sel"], *x["out"]):
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        for x in batches:
            go(x, x["stream"])
    torch.cuda.synchronize()
    for x, want in zip(batches, alone):
        for t, w in zip((x["bounds"], x["sel"], *x["out"]), want):
            assert torch.equal(t, w)

@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
@pytest.mark.parametrize("captured", [False, True])
def test_a_run_of_them(kind, captured):
    """Prompts of several lengths go in, then decode steps: each appends a token, brings the
    last page's bounds up to date, selects pages and attends over them -- eager on a stream of its own, or
    as a captured step replayed with eager work in between.  Selections and outputs are those
    of the cache as it stands after each step."""
    _say(f"a run of them {kind} captured {captured}")
    hq, hkv, d, budget = 8, 2, 128, 6
    q8, dt = kind == "q8", F32 if kind == "f32" else BF16
    prompts, steps = [1, 70, 16, 200, 95, 33], 20
    R, npages = len(prompts), [-(-(n + 24) // 16) for n in prompts]
    gen = torch.Generator().manual_seed(21)
    pool, table = _paged(npages, max(npages) + 1, gen)
    ps = _state(table, npages, [0] * R, pool)
    if q8:
        codes = torch.full((2, pool, hkv, 16, d), 0x7f, dtype=torch.uint8, device=DEV)
        scales = torch.full((2, pool, hkv), NAN, device=DEV)
        kv = gp.KV8Layer(codes[0], codes[1], scales[0], scales[1])
    else:
        kv = gp.KVLayer(*(torch.full((pool, hkv, 16, d), NAN, dtype=dt, device=DEV) for _ in range(2)))
    append, bound, attend = ((gp.gp_append_rope_q8, gp.gp_page_bounds_q8, gp.gp_decode_attention_pages_q8) if q8 else
                             (gp.gp_append_rope, gp.gp_page_bounds, gp.gp_decode_attention_pages))
    bounds = torch.full((pool, hkv, 2, d), NAN, dtype=dt, device=DEV)
    pos = _i32([-1] * R)
    starts = [0]
    for n in prompts:
        starts.append(starts[-1] + n)
    T, scale = starts[-1], d ** -0.5
    k, v = (torch.randn(T, hkv, d, generator=gen).to(dt).to(DEV) for _ in range(2))
    append(kv, ps, pos, k, v, 1e4, tok_start=_i32(starts))
    bound(kv, ps, bounds)
    qkv = torch.zeros(R, hq + 2 * hkv, d, dtype=dt, device=DEV)
    q_out, out = torch.zeros(R, hq, d, dtype=dt, device=DEV), torch.zeros(R, hq, d, dtype=dt, device=DEV)
    sel = torch.zeros(R, hkv, budget, dtype=torch.int32, device=DEV)
    ws_s = gp.workspace(gp.GP_OP_SELECT, R, 0, hq, hkv, d, table.shape[1], dt)
    ws_d = gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, budget, dt)

    def step():
        q, kn, vn = qkv.split([hq, hkv, hkv], 1)
        append(kv, ps, pos, kn, vn, 1e4, q=q, q_out=q_out)
        bound(kv, ps, bounds, from_tokens=ps.seq_lens - 1, max_update=1)
        gp.gp_select_pages(bounds, ps, q_out, 1, 1, sel, ws_s)
        attend(kv, ps, sel, q_out, scale, out, ws_d)

    stream = torch.cuda.Stream()
    graph = None
    if captured:
        saved = [t.clone() for t in (*vars(kv).values(), ps.seq_lens, pos, bounds)]
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for t, t0 in zip((*vars(kv).values(), ps.seq_lens, pos, bounds), saved):
            t.copy_(t0)
    for i in range(steps):
        qkv.copy_(torch.randn(R, hq + 2 * hkv, d, generator=gen).to(dt))
        if captured:
            graph.replay()
        else:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                step()
        torch.cuda.synchronize()
        lens = [n + i + 1 for n in prompts]
        assert ps.seq_lens.cpu().tolist() == lens and pos.cpu().tolist() == [m - 1 for m in lens]
        k64 = _values(kv.k, kv.k_scale) if q8 else kv.k.cpu().double()
        v64 = _values(kv.v, kv.v_scale) if q8 else kv.v.cpu().double()
        q, got, chosen, box = q_out.cpu(), out.cpu().double(), sel.cpu(), bounds.cpu()
        turned, mag = _rotated(qkv.cpu().double(), torch.tensor([m - 1 for m in lens]), 1e4)
        assert bool(((q.double() - turned[:, :hq]).abs() <= turned[:, :hq].abs() * HALF[dt] + ROT * mag[:, :hq]).all())
        for r, m in enumerate(lens):
            n = -(-m // 16)
            for p in range(n):
                assert torch.equal(box[table[r, p].long()].double(), _bounds64(k64, table, lens, r, p).to(dt).double()), (i, r, p)
            want_sel = _select64(box, table, n, q, hkv, budget, 1, 1, r)
            assert torch.equal(chosen[r], want_sel), (i, r)
            for h in range(hkv):
                tok = [16 * p + j for p in want_sel[h].tolist() if p >= 0 for j in range(min(16, m - 16 * p))]
                g = slice(h * hq // hkv, (h + 1) * hq // hkv)
                want, size_, size = _attention(_tokens(k64, table, r, m)[h:h + 1, tok], _tokens(v64, table, r, m)[h:h + 1, tok],
                                               q[r, g].double(), scale)
                assert bool(((got[r, g] - want).abs() <= _attention_tol(want, size_, size, d, dt)).all()), (i, r, h)


# ----------------------------------------------------- factors at the range's ends --

@pytest.mark.parametrize("spare", [2, 130])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (3, 3, 64)])
def test_decode_q8_scale_products(hq, hkv, d, spare):
    """Page scales and softmax scales whose product rounds to zero or past the largest float, on pages that are
    not full: the weights are those of the scores all the same.  The product of less than 2^-149 may stand for
    2^-149, which moves a score of up to 2^128 by 2^-21 and its weight by as much: within the 2^-17."""
    _say(f"decode q8 scale products heads {hq}/{hkv} d {d} spare {spare}")
    gen = torch.Generator().manual_seed(hq + spare)
    lens = [5, 21, 40, 16, 1]
    npages = [-(-m // 16) for m in lens]
    width = max(npages) + spare
    R = len(lens)
    kv, pool, table = _q8_cache(lens, npages, hkv, d, gen, width)
    ps = _state(table, npages, lens, pool)
    plain = torch.randn(R, hq, d, generator=gen).to(BF16)
    sel = torch.arange(width, dtype=torch.int32).expand(R, hkv, width).contiguous().to(DEV)
    ws = gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, width, BF16)
    zero_keys = (kv.k.to(torch.int32) * 0).to(torch.uint8)
    for keys, k_scale, scale, q in ((zero_keys, 2.0 ** -100, 1e-16, plain), (kv.k, 2.0 ** -149, 0.125, plain),
                                    (kv.k, 2.0 ** -115, 2.0 ** -40, plain * 2.0 ** 115), (kv.k, 2.0 ** 119, 2.0 ** 20, plain * 0.0)):
        layer = gp.KV8Layer(keys, kv.v, torch.full_like(kv.k_scale, k_scale), kv.v_scale)
        outs = [torch.full((R, hq, d), NAN, dtype=BF16, device=DEV) for _ in range(2)]
        gp.gp_decode_attention_q8(layer, ps, q.to(DEV), scale, outs[0], ws)
        gp.gp_decode_attention_pages_q8(layer, ps, sel, q.to(DEV), scale, outs[1], ws)
        torch.cuda.synchronize()
        k64, v64 = _values(layer.k, layer.k_scale), _values(layer.v, layer.v_scale)
        for r, m in enumerate(lens):
            want, mag, size = _attention(_tokens(k64, table, r, m), _tokens(v64, table, r, m), q[r].double(), scale)
            for out in outs:
                assert bool(((out[r].cpu().double() - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), (k_scale, scale, r)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,width,budget", [(40, 40, 12), (700, 700, 200), (3000, 3100, 900)])
def test_select_signed_zero(dtype, n, width, budget):
    """Sums so small that they round to -0: as good as the pages whose sum is 0, the lowest of all first."""
    _say(f"select signed zero {dtype} {n} of {width} budget {budget}")
    hq, hkv, d = 2, 1, 64
    gen = torch.Generator().manual_seed(n)
    pool, table = _paged([n] * 2, width, gen)
    bounds = torch.zeros(pool, hkv, 2, d, dtype=dtype)
    bounds[table[0, 1:n:3].long(), :, :, 7] = 2.0 ** -120                # times -2^-120: -2^-240
    bounds[table[1, :n // 2].long(), :, :, 7] = 2.0 ** -120
    bounds[table[1, 3].long()] = 1.0
    q = torch.zeros(2, hq, d, dtype=dtype)
    q[:, 0, 7] = -(2.0 ** -120)
    sel = torch.empty(2, hkv, budget, dtype=torch.int32, device=DEV)
    ws = gp.workspace(gp.GP_OP_SELECT, 2, 0, hq, hkv, d, width, dtype)
    gp.gp_select_pages(bounds.to(DEV), _state(table, [n] * 2, [16 * n] * 2, pool), q.to(DEV), 1, 1, sel, ws)
    torch.cuda.synchronize()
    for r in range(2):
        assert torch.equal(sel[r].cpu(), _select64(bounds, table, n, q, hkv, budget, 1, 1, r)), r


def _e4m3(x):
    """float64, |x| <= 448: the nearest e4m3 value, ties to even."""
    step = torch.exp2((torch.frexp(x)[1].double() - 4).clamp_min(-9))
    return (x / step).round() * step


@pytest.mark.parametrize("hkv,d", [(2, 128), (1, 64)])
@pytest.mark.parametrize("size", [2.0 ** -6, 300.0])
def test_append_rope_q8_other_scales(hkv, d, size):
    """Pages that hold tokens under scales that are no powers of two, among them scales next to those that bring
    an older code to a tie: the new scale is a power of two, the older codes are rounded once from their
    products' exact values, the new ones from theirs."""
    _say(f"append q8 other scales heads {hkv} d {d} size {size}")
    gen = torch.Generator().manual_seed(d)
    old = [1.0 / 3, 0.7, 1.5, 448.0 / 447, 0.5, 2.0 ** -100, 1.5 * 2.0 ** -120, 3e-42, 3.0 * 2.0 ** 30, 1.9 * 2.0 ** 126]
    for x in range(9, 16):                                # x old is a tie between two codes, but for old's own rounding
        for t in range(17, 32, 2):
            f = torch.tensor(t / (2 * x), dtype=F32)
            old += [float(torch.nextafter(f, f * k)) for k in (0, 1, 2) if 0.5 < f < 1]
    R, m = len(old), 7
    npages = [1] * R
    pool, table = _paged(npages, 1, gen)
    ps = _state(table, npages, [m] * R, pool)
    codes = torch.randint(0, 256, (2, pool, hkv, 16, d), generator=gen).to(torch.uint8)
    scale = torch.full((pool, hkv), 1.0)
    scale[table[:, 0].long()] = torch.tensor(old, dtype=F32)[:, None].expand(-1, hkv)
    kv = gp.KV8Layer(codes[0].to(DEV), codes[1].to(DEV), scale.to(DEV), scale.clone().to(DEV))
    new = (torch.randn(2, R, hkv, d, generator=gen) * size).to(BF16)
    gp.gp_append_rope_q8(kv, ps, _i32([-1] * R), new[0].to(DEV), new[1].to(DEV), 1e4)       # position 0: no turn
    torch.cuda.synchronize()
    ids = table[:, 0].long()
    for which, got_codes, got_scale in ((0, kv.k, kv.k_scale), (1, kv.v, kv.v_scale)):
        x, s0 = new[which].double(), scale.double()[ids]
        least = (torch.frexp(x.abs().amax(-1) / 448)[1] - (torch.frexp(x.abs().amax(-1) / 448)[0] == 0.5).int()).clamp_min(-100)
        kept = torch.frexp(s0)[1] - (torch.frexp(s0)[0] == 0.5).int()
        s = torch.exp2(torch.maximum(least, kept).double())
        assert torch.equal(got_scale.cpu().double()[ids], s)
        got = got_codes.cpu().view(torch.float8_e4m3fn).double()[ids]
        older = codes[which].view(torch.float8_e4m3fn).double()[ids][:, :, :m]
        want = _e4m3(older * (s0 / s)[..., None, None])
        assert torch.equal(got[:, :, :m].isnan(), older.isnan())
        wrong = (got[:, :, :m] != want) & ~older.isnan()
        assert not bool(wrong.any()), (int(wrong.sum()), old[int(wrong.nonzero()[0, 0])])
        assert torch.equal(got[:, :, m], _e4m3(x / s[..., None]))
        assert torch.equal(got_codes.cpu()[ids][:, :, m + 1:], codes[which][ids][:, :, m + 1:])


def _bf16(x):
    """float64 to the nearest bfloat16 value, ties to even, in one rounding."""
    step = torch.exp2(torch.frexp(x)[1].double() - 8)
    return (x / step).round() * step


@pytest.mark.parametrize("hkv,d", [(2, 128), (1, 64)])
def test_page_bounds_q8_other_scales(hkv, d):
    """Scales that are no powers of two, among them those next to the ones that bring a code to a tie: the bounds
    are the codes' values rounded once."""
    _say(f"bounds q8 other scales heads {hkv} d {d}")
    gen = torch.Generator().manual_seed(d)
    scales = [1.0 / 3, 0.7, 2.0 ** -100, 1.9 * 2.0 ** -100, 1.3 * 2.0 ** 90]
    for x in range(9, 16, 2):                             # x scale is a tie between two bfloat16 values, but for the scale's own rounding
        for t in range(257, 512, 10):
            f = torch.tensor(t / x, dtype=F32)
            scales += [float(torch.nextafter(f, f * k)) for k in (0, 1, 2)]
    R = len(scales)
    lens = [1 + 5 * r % 16 for r in range(R)]
    pool, table = _paged([1] * R, 1, gen)
    codes = torch.randint(0, 254, (pool, hkv, 16, d), generator=gen)
    codes = torch.where(codes >= 127, codes + 1, codes).to(torch.uint8)        # every finite code
    scale = torch.ones(pool, hkv)
    scale[table[:, 0].long()] = torch.tensor(scales, dtype=F32)[:, None].expand(-1, hkv)
    kv = gp.KV8Layer(codes.to(DEV), codes.to(DEV), scale.to(DEV), scale.to(DEV))
    bounds = torch.zeros(pool, hkv, 2, d, dtype=BF16, device=DEV)
    gp.gp_page_bounds_q8(kv, _state(table, [1] * R, lens, pool), bounds)
    torch.cuda.synchronize()
    got, v64 = bounds.cpu().double(), _values(kv.k, kv.k_scale)
    for r, m in enumerate(lens):
        want = _bf16(_bounds64(v64, table, lens, r, 0))
        assert torch.equal(got[int(table[r, 0])], want), (r, m, scales[r])


@pytest.mark.parametrize("k_scale,q_size", [(2.0 ** -6, 1.0), (2.0 ** -100, 2.0 ** 94), (2.0 ** 100, 2.0 ** -106)])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (2, 2, 64)])
def test_decode_q8_every_key_code(hq, hkv, d, k_scale, q_size):
    """Each finite code as a key, met by a query of one dim: the weights are those of the values it stands for."""
    _say(f"decode q8 every key code heads {hq}/{hkv} d {d} scale {k_scale}")
    gen = torch.Generator().manual_seed(d)
    finite = torch.tensor([c for c in range(256) if c & 0x7f != 0x7f], dtype=torch.uint8)
    R, lens = 16, [16] * 16
    pool, table = _paged([1] * R, 4, gen)
    codes = torch.zeros(pool, hkv, 16, d, dtype=torch.uint8)
    for r in range(R):                                    # dim 5 + h: 16 codes side by side, other ones in each head
        for h in range(hkv):
            codes[int(table[r, 0]), h, :, 5 + h] = finite[(16 * r + 37 * h + torch.arange(16)) % 254]
    values = torch.randn(pool, hkv, 16, d, generator=gen).to(torch.float8_e4m3fn).view(torch.uint8)
    scale = torch.full((pool, hkv), k_scale)
    kv = gp.KV8Layer(codes.to(DEV), values.to(DEV), scale.to(DEV), torch.ones(pool, hkv, device=DEV))
    q = torch.zeros(R, hq, d)
    for h in range(hkv):
        q[:, h * (hq // hkv):(h + 1) * (hq // hkv), 5 + h] = q_size
    q = q.to(BF16)
    out = torch.full((R, hq, d), NAN, dtype=BF16, device=DEV)
    gp.gp_decode_attention_q8(kv, _state(table, [1] * R, lens, pool), q.to(DEV), 0.5, out,
                              gp.workspace(gp.GP_OP_DECODE, R, 0, hq, hkv, d, 4, BF16))
    torch.cuda.synchronize()
    k64, v64 = _values(kv.k, kv.k_scale), _values(kv.v, kv.v_scale)
    for r in range(R):
        want, mag, size = _attention(_tokens(k64, table, r, 16), _tokens(v64, table, r, 16), q[r].double(), 0.5)
        assert bool(((out[r].cpu().double() - want).abs() <= _attention_tol(want, mag, size, d, BF16)).all()), r
