"""Timed calls of the operators that take a prompt from its arrival to the decode
step: pages, rotary positions in their several forms, and attention.

  prompt    gp_prompt_attention / gp_prompt_attention_q8: the new tokens of each
            request attend over its pages (whole prompts, chunks of them behind a
            context, a few drafted tokens, single tokens among the chunks)
  rotary    gp_append_rotary / gp_append_rotary_q8: new tokens into the cache, keys
            and queries rotated in either pairing, a part of the head, frequencies
            scaled for longer contexts
  fork      gp_pages_release, then gp_pages_fork: the replies of the last round are
            dropped and new ones continue their parents, which share their pages
  turnover  gp_pages_release, then gp_pages_reserve: finished requests leave, and
            those in their places get pages for their prompts

Lengths are drawn from the case alone, so that every seed of a case does the
same work; page placement and all contents come from the seed.  Values follow
the synthetic workloads of this repository: N(0, 1) values and queries, keys
with an offset per head and dim and 1 % heavy ones of four times the norm.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

PAGE = 16
DEV = "cuda"
THETA = 1.0e6
TOP = 448.0                     # the largest e4m3 value
LEAST = -100                    # the smallest exponent of a page's scale
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "q8": torch.bfloat16}     # of queries and new rows

BASE = dict(cache="bf16", q_heads=32, kv_heads=8, head_dim=128, dist="uniform", sigma=0.0, new_lo=0, new_hi=0, singles=0,
            pairs="half", rotary_dim=128, factor=1.0, low=0.0, high=0.0, context=0, layers=1, children=0, prefix=0, done=0,
            spare=3)


def _case(kind, reqs, lo, hi, **kw):
    return dict(BASE, kind=kind, reqs=reqs, len_lo=lo, len_hi=hi, **kw)


def listed():
    return [
        # one user's reply, five drafted tokens to check: the smallest attention call
        dict(_case("prompt", 1, 6001, 6001, new_lo=5, new_hi=5), name="prompt_drafted"),
        # a batch of new prompts of the Qwen3-8B layer, nothing in the cache before (the largest call)
        dict(_case("prompt", 12, 0, 0, new_lo=200, new_hi=6000), name="prompt_fresh"),
        # chunks of long prompts over an 8-bit cache, mid-page
        dict(_case("prompt", 4, 8001, 24001, cache="q8", new_lo=1001, new_hi=1024), name="prompt_chunks_q8"),
        # a serving step: 60 decoding requests and four chunks in one call, eight query heads per KV head, head_dim 64
        dict(_case("prompt", 64, 256, 8192, q_heads=64, head_dim=64, new_lo=400, new_hi=512, singles=60), name="prompt_mixed"),
        # float32, the precision in which the path is checked, heads 2 : 1
        dict(_case("prompt", 6, 0, 700, cache="f32", q_heads=16, head_dim=64, new_lo=100, new_hi=2000), name="prompt_f32"),
        # the decode step of the Qwen3-8B layer batch, pairs side by side, frequencies scaled for eight times the context
        dict(_case("rotary", 64, 1024, 8192, new_lo=1, new_hi=1, pairs="interleaved", factor=8.0, low=1.0, high=4.0, context=8192),
             name="rotary_step"),
        # a batch of new prompts, Qwen3-32B heads, half of the head turns, all frequencies divided by two
        dict(_case("rotary", 12, 0, 0, q_heads=64, new_lo=200, new_hi=6000, rotary_dim=64, factor=2.0), name="rotary_prompts"),
        # chunks of long prompts into an 8-bit cache, mid-page, pairs side by side
        dict(_case("rotary", 24, 1, 6000, cache="q8", new_lo=500, new_hi=2000, pairs="interleaved"), name="rotary_chunks_q8"),
        # one prompt answered four times: one layer of a small cache
        dict(_case("fork", 1, 1500, 1500, children=4, kv_heads=2, q_heads=8), name="fork_one"),
        # a round of a search over replies: eight kept, four continuations each, 36 layers
        dict(_case("fork", 8, 400, 2000, children=4, layers=36), name="fork_round"),
        # one reply ends and one prompt comes
        dict(_case("turnover", 4, 1500, 3000, new_lo=700, new_hi=700, done=1), name="turnover_one"),
        # the pages of a full server: an eighth of the requests leave, new prompts take their places
        dict(_case("turnover", 256, 256, 16384, dist="lognormal", sigma=0.8, new_lo=200, new_hi=6000, done=32, prefix=512,
                   spare=200000), name="turnover_full"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "prompt", "rotary", "rotary", "rotary", "fork", "fork", "turnover"])
    g, d, hkv = rng.choice([1, 2, 4, 4, 8]), rng.choice([64, 128, 128]), rng.choice([2, 4, 8, 8, 12])
    cache = rng.choice(["bf16", "bf16", "q8", "q8", "f32"])
    kw = dict(cache=cache, q_heads=g * hkv, kv_heads=hkv, head_dim=d)
    e = 4 if cache == "f32" else 2
    if kind == "prompt":
        held = rng.choice([0, _log_int(rng, 1, 50000)])
        new = rng.choice([_log_int(rng, 1, 16), _log_int(rng, 16, 6000), _log_int(rng, 16, 6000)])
        most = (1e11 if cache == "f32" else 1e12) / (4 * d * g * hkv)          # pairs of tokens of one call
        new = max(1, min(new, int(math.sqrt(held * held / 4 + most) - held / 2)))
        reqs = max(1, min(_log_int(rng, 1, 64), int(most / (new * (held + new))), int(1.2e9 / (2 * hkv * d * e * (held + new)))))
        singles = rng.choice([0, 0, reqs // 2, reqs - 1])
        return _case(kind, reqs, rng.randint(held // 8, held), held, new_lo=max(1, new // rng.randint(1, 8)), new_hi=new,
                     singles=singles, **kw)
    if kind == "rotary":
        row = (2 * g + 4) * hkv * d * e                        # bytes of one token's queries, keys and values, both ways
        new = rng.choice([1, 1, _log_int(rng, 2, 6000)])
        reqs = max(1, min(_log_int(rng, 1, 256), int(4e8 / (row * new)), int(1.2e9 / (4 * hkv * d * e * (new + 2000)))))
        lo = rng.choice([0, rng.randint(0, 2000)])
        kw.update(pairs=rng.choice(["half", "interleaved"]), rotary_dim=rng.choice([d, d, d // 2, 16 * rng.randint(1, d // 16)]))
        kw.update(rng.choice([{}, dict(factor=rng.uniform(1.0, 8.0)),
                              dict(factor=rng.uniform(2.0, 40.0), low=1.0, high=rng.choice([4.0, 32.0]), context=rng.choice([4096, 8192]))]))
        return _case(kind, reqs, lo, rng.randint(lo, 2000), new_lo=max(1, new // rng.randint(1, 8)), new_hi=new, **kw)
    if kind == "fork":
        layers, reqs, children = _log_int(rng, 1, 36), _log_int(rng, 1, 16), rng.randint(1, 8)
        page = 2 * layers * hkv * d * PAGE * (1 if cache == "q8" else e)
        hi = min(_log_int(rng, 20, 8000), max(20, int(PAGE * (2.0e9 / page - 2 * reqs * (children + 1)) / reqs)))
        lo = rng.randint(1, hi)
        return _case(kind, reqs, lo, hi, layers=layers, children=children, prefix=rng.choice([0, 0, rng.randint(1, lo)]), **kw)
    reqs = _log_int(rng, 1, 512)
    hi = _log_int(rng, 40, 16384)
    return _case(kind, reqs, rng.randint(1, hi), hi, new_lo=1, new_hi=_log_int(rng, 1, 16384), done=rng.randint(1, reqs),
                 prefix=rng.choice([0, rng.randint(0, 2048)]), spare=_log_int(rng, 3, 200000))


# ------------------------------------------------------------------ shapes --

def _lengths(case):
    """Resident tokens before the call, and new ones, of every request (fork: of every parent)."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    R, lo, hi = case["reqs"], case["len_lo"], case["len_hi"]
    if case["dist"] == "lognormal":
        mid = math.sqrt(lo * hi)
        held = [min(hi, max(lo, round(mid * math.exp(case["sigma"] * rng.gauss(0, 1))))) for _ in range(R)]
    else:
        held = [rng.randint(lo, hi) for _ in range(R)]
    return held, [1 if r < case["singles"] else rng.randint(case["new_lo"], case["new_hi"]) for r in range(R)]


def _touched(case):
    """Per request the pages that an append writes: (first, count)."""
    held, new = _lengths(case)
    return [(m // PAGE, (m + n - 1) // PAGE - m // PAGE + 1) for m, n in zip(held, new)]


def _forks(case):
    """(parent before, parent now, tokens taken) of each child; children are the rows behind the parents."""
    held, _ = _lengths(case)
    n = case["reqs"] * case["children"]
    cut = case["prefix"] or max(held)
    now = [c % case["reqs"] for c in range(n)]
    before = [(c * 7 + 3) % case["reqs"] for c in range(n)]
    return before, now, [min(held[p], cut) for p in before], [min(held[p], cut) for p in now]


def _leaving(case):
    """The requests that leave (and whose rows are taken again) and the tokens that each row then asks pages for."""
    _, new = _lengths(case)
    rng = random.Random(case["reqs"] * 1000003 + case["done"])
    done = rng.sample(range(case["reqs"]), case["done"])
    ask = [0] * case["reqs"]
    for r in done:
        ask[r] = new[r]
    return done, ask


def _frequencies(case):
    """Radians per position of each pair: theta^(-2 i / n); with a factor, pairs that turn fewer than `low` times over the
    first context are slowed by it, those of more than `high` turns are left, and in between the two are mixed."""
    n, f = case["rotary_dim"], case["factor"]
    out = []
    for i in range(n // 2):
        w = THETA ** (-2.0 * i / n)
        keep = 0.0
        if case["high"] > 0:
            keep = min(1.0, max(0.0, (case["context"] * w / (2 * math.pi) - case["low"]) / (case["high"] - case["low"])))
        out.append(w * (keep + (1 - keep) / f))
    return out


def _magnitude(case):
    """Rotated keys and queries grow with the scaled context, so that the logits keep their spread."""
    return 0.1 * math.log(case["factor"]) + 1.0 if case["high"] > 0 else 1.0


# ----------------------------------------------------------------- prepare --

def _quantised(x):
    """[pages][heads][16][dim] float32 -> e4m3 codes and a power-of-two scale per page and head."""
    scale = _scale_for(x.abs().amax((-1, -2)))
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn), scale


def _scale_for(amax):
    """The least power of two (from 2^LEAST on) that brings amax to 448 or less."""
    m, x = torch.frexp(amax)                                   # m in [1/2, 1): 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, x - 9, x - 8).clamp_min(LEAST)
    return _power(torch.where(amax > 0, e, torch.full_like(e, LEAST)))


def _power(e):
    """2^e of int32 e in [-126, 127], float32: from its bits (a power function need not be exact)."""
    return ((e + 127) << 23).view(torch.float32)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _paged(rows, pool, gen):
    """A table of the given lists of pages (as indices of a random order of the pool), its spare columns -1."""
    perm = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32).cpu()
    table = torch.full((len(rows), max(map(len, rows)) + 2), -1, dtype=torch.int32)
    for r, ids in enumerate(rows):
        table[r, :len(ids)] = perm[torch.tensor(ids, dtype=torch.long)]
    return table, perm


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=case, gen=gen)
    if case["kind"] in ("fork", "turnover"):
        return _prepare_pages(case, s, gen)
    held, new = _lengths(case)
    Hq, Hkv, d, dt = case["q_heads"], case["kv_heads"], case["head_dim"], TYPES[case["cache"]]
    pages = [-(-(m + n) // PAGE) for m, n in zip(held, new)]
    pool, T = sum(pages) + 3, sum(new)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    ids = iter(range(pool))
    table, perm = _paged([[next(ids) for _ in range(P)] for P in pages], pool, gen)
    refs = torch.zeros(pool, dtype=torch.int32, device=DEV)
    refs[perm[:sum(pages)].to(DEV).long()] = 1
    free = torch.zeros(pool, dtype=torch.int32, device=DEV)
    free[:3] = perm[sum(pages):].to(DEV)
    s["ps"] = SimpleNamespace(page_table=table.to(DEV), num_pages=_i32(pages), seq_lens=_i32(held), refcount=refs,
                              free_list=free, free_count=_i32([3]))
    s["tok_start"], s["positions"] = _i32(starts), _i32([m - 1 for m in held])
    k = torch.randn(pool, Hkv, PAGE, d, generator=gen, device=DEV, dtype=dt)
    if case["kind"] == "prompt":
        # keys with an offset per head and dim, as rotated keys of a model have on their slow pairs; 1 % heavy
        k += 0.5 * torch.randn(1, Hkv, 1, d, generator=gen, device=DEV, dtype=dt)
        k *= 1 + 3 * (torch.rand(pool, Hkv, PAGE, 1, generator=gen, device=DEV) < 0.01).to(dt)
    v = torch.randn(pool, Hkv, PAGE, d, generator=gen, device=DEV, dtype=dt)
    s["kv"] = SimpleNamespace(k=k, v=v)
    if case["cache"] == "q8":
        (k, ks), (v, vs) = _quantised(k.float()), _quantised(v.float())
        s["kv"] = SimpleNamespace(k=k, v=v, k_scale=ks, v_scale=vs)
    if case["kind"] == "prompt":
        s["q"] = torch.randn(T, Hq, d, generator=gen, device=DEV, dtype=dt)
        s["out"] = torch.zeros(T, Hq, d, dtype=dt, device=DEV)
        s["scale"] = 1.0 / math.sqrt(d)
    else:
        # the projection's output as a model has it: queries, keys and values side by side in a row per token
        s["rows"] = torch.randn(T, (Hq + 2 * Hkv) * d, generator=gen, device=DEV, dtype=dt)
        s["q_out"] = torch.zeros(T, Hq, d, dtype=dt, device=DEV)
    if own:
        _handles(s)
    return s


def _prepare_pages(case, s, gen):
    held, _ = _lengths(case)
    R, spare = case["reqs"], case["spare"]
    n_of = [-(-m // PAGE) for m in held]
    if case["kind"] == "fork":
        before, now, taken, take = _forks(case)
        spare += len(now)
        at = sum(n_of)
        first = [sum(n_of[:r]) for r in range(R)]
        rows = [list(range(f, f + n)) for f, n in zip(first, n_of)]
        for p, L in zip(before, taken):
            rows.append(rows[p][:L // PAGE] + ([at] if L % PAGE else []))
            at += L % PAGE > 0
        lens = held + taken
    else:
        shared = case["prefix"] // PAGE                        # pages that all requests of that length share
        at, rows = shared, []
        for n in n_of:
            k = shared if n > shared else 0
            rows.append(list(range(k)) + list(range(at, at + n - k)))
            at += n - k
        spare += sum(-(-a // PAGE) for a in _leaving(case)[1])
        lens = held
    pool = at + spare
    table, perm = _paged(rows, pool, gen)
    if case["kind"] == "turnover":                             # a place may ask for more pages than it held
        wide = max(table.shape[1], -(-max(_leaving(case)[1]) // PAGE) + 2)
        table = torch.cat([table, torch.full((R, wide - table.shape[1]), -1, dtype=torch.int32)], 1)
    refs = torch.zeros(pool, dtype=torch.int32)
    for ids in rows:
        refs[perm[torch.tensor(ids, dtype=torch.long)].long()] += 1
    free = torch.zeros(pool, dtype=torch.int32)
    left = perm[at:].sort()[0]
    if case["kind"] == "turnover" and case["prefix"] // PAGE and not any(n > case["prefix"] // PAGE for n in n_of):
        left = torch.cat([left, perm[:case["prefix"] // PAGE]])          # nobody holds the prefix
    free[:len(left)] = left
    s["ps"] = SimpleNamespace(page_table=table.to(DEV), num_pages=_i32([len(x) for x in rows]), seq_lens=_i32(lens),
                              refcount=refs.to(DEV), free_list=free.to(DEV), free_count=_i32([len(left)]))
    s["positions"] = _i32([m - 1 for m in lens])
    if case["kind"] == "turnover":
        done, ask = _leaving(case)
        s["done"], s["ask"], s["granted"] = _i32(done), _i32(ask), torch.zeros(R, dtype=torch.int32, device=DEV)
    else:
        L, Hkv, d, dt = case["layers"], case["kv_heads"], case["head_dim"], TYPES[case["cache"]]
        s["parents"], s["children"] = _i32(now), _i32(list(range(R, R + len(now))))
        s["lengths"] = _i32(take) if case["prefix"] else None
        s["forked"] = torch.zeros(len(now), dtype=torch.int32, device=DEV)
        if case["cache"] == "q8":
            s["pool"] = torch.randint(0, 120, (L, 2, pool, Hkv, PAGE, d), generator=gen, device=DEV, dtype=torch.uint8)
            s["scales"] = torch.rand(L, 2, pool, Hkv, generator=gen, device=DEV)
        else:
            s["pool"] = torch.randn(L, 2, pool, Hkv, PAGE, d, generator=gen, device=DEV, dtype=dt)
            s["scales"] = None
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps between calls: the layers and the page state as the library takes them, rotary frequencies,
    workspaces."""
    import paper_2609_03494_amd as gp
    case = s["case"]
    s["state"] = gp.PageState(**vars(s["ps"]))
    if case["kind"] == "fork":
        pool, scales = s["pool"], s["scales"]
        s["layers"] = gp.Layers(gp.KV8Layer(pool[i, 0], pool[i, 1], scales[i, 0], scales[i, 1]) if scales is not None else
                                gp.KVLayer(pool[i, 0], pool[i, 1]) for i in range(case["layers"]))
    if case["kind"] in ("prompt", "rotary"):
        s["layer"] = (gp.KV8Layer if case["cache"] == "q8" else gp.KVLayer)(**vars(s["kv"]))
    if case["kind"] == "prompt":
        s["ws"] = gp.workspace(gp.GP_OP_PROMPT, case["reqs"], s["q"].shape[0], case["q_heads"], case["kv_heads"],
                               case["head_dim"], s["ps"].page_table.shape[1], TYPES[case["cache"]])
    if case["kind"] == "rotary":
        pairs = gp.GP_ROPE_INTERLEAVED if case["pairs"] == "interleaved" else gp.GP_ROPE_HALF
        s["rope"] = gp.Rope(pairs, gp.gp_rope_frequencies(case["rotary_dim"], THETA, case["factor"], case["low"],
                                                          case["high"], case["context"]), _magnitude(case))


# --------------------------------------------------------------------- run --

def run(s):
    if own:
        return _own(s, s["case"])
    return {"prompt": _plain_prompt, "rotary": _plain_rotary, "fork": _plain_fork, "turnover": _plain_turnover}[s["case"]["kind"]](s)


def _own(s, case):
    import paper_2609_03494_amd as gp
    ps, q8 = s["state"], case["cache"] == "q8"
    if case["kind"] == "prompt":
        # as every layer of a model but the last calls it: the lengths advance with the last layer
        (gp.gp_prompt_attention_q8 if q8 else gp.gp_prompt_attention)(s["layer"], ps, s["q"], s["scale"], s["out"], s["ws"],
                                                                      tok_start=s["tok_start"], advanced=False)
        return s["out"]
    if case["kind"] == "rotary":
        Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        q, k, v = s["rows"].view(-1, Hq + 2 * Hkv, d).split([Hq, Hkv, Hkv], 1)
        (gp.gp_append_rotary_q8 if q8 else gp.gp_append_rotary)(s["layer"], ps, s["positions"], k, v, s["rope"], q=q,
                                                                q_out=s["q_out"], tok_start=s["tok_start"], advance=False)
        return _cache(s)
    if case["kind"] == "fork":
        gp.gp_pages_release(ps, s["children"])
        (gp.gp_pages_fork_q8 if q8 else gp.gp_pages_fork)(s["layers"], ps, s["parents"], s["children"], s["forked"],
                                                          lengths=s["lengths"], positions=s["positions"])
        return _pages(s)
    gp.gp_pages_release(ps, s["done"])
    gp.gp_pages_reserve(ps, s["ask"], s["granted"])
    return _pages(s)


def _cache(s):
    kv, more = s["kv"], {}
    if s["case"]["cache"] == "q8":
        more = {"k_scale": kv.k_scale, "v_scale": kv.v_scale}
    return {"k": kv.k, "v": kv.v, "q": s["q_out"], **more}


def _pages(s):
    out = dict(vars(s["ps"]))
    if s["case"]["kind"] == "turnover":
        return {**out, "granted": s["granted"]}
    pool = s["pool"]
    out.update(forked=s["forked"], positions=s["positions"], pool=pool)
    return out if s["scales"] is None else {**out, "pool": pool.view(torch.float8_e4m3fn), "scales": s["scales"]}


def _groups(case):
    """Requests to pad together: of like numbers of new tokens, as many as 8 GB of scores hold."""
    held, new = _lengths(case)
    groups, cell = [], 4 * case["q_heads"]
    for r in sorted(range(len(new)), key=lambda r: (new[r], held[r])):
        if groups:
            g = groups[-1]
            n, m = max(new[x] for x in g + [r]), max(held[x] + new[x] for x in g + [r])
            if n <= 2 * new[g[0]] + 8 and (len(g) + 1) * n * m * cell <= 8e9:
                g.append(r)
                continue
        groups.append([r])
    return [(g, max(new[r] for r in g), max(held[r] + new[r] for r in g)) for g in groups]


def _plain_prompt(s):
    case, kv, ps = s["case"], s["kv"], s["ps"]
    Hq, Hkv, d, q8 = case["q_heads"], case["kv_heads"], case["head_dim"], case["cache"] == "q8"
    G, T = Hq // Hkv, s["q"].shape[0]
    new = _lengths(case)[1]
    for reqs, n, m in _groups(case):
        r = torch.tensor(reqs, device=DEV)
        P = -(-m // PAGE)
        page = ps.page_table[r, :P].long().clamp_min(0)                               # [R][P]
        K, V = ((x.view(torch.uint8)[page].view(x.dtype) if q8 else x[page]).float() for x in (kv.k, kv.v))
        if q8:
            K *= kv.k_scale[page][..., None, None]
            V *= kv.v_scale[page][..., None, None]
        K, V = (x.transpose(1, 2).flatten(2, 3) for x in (K, V))                      # [R][Hkv][16 P][d]
        first, held, counts = s["tok_start"][r], ps.seq_lens[r], [new[x] for x in reqs]
        count = s["tok_start"][r + 1] - first
        j = torch.arange(n, device=DEV)
        at = (first[:, None] + j).clamp_max(T - 1)                                    # [R][n]
        q = s["q"][at].float().view(len(reqs), n, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(len(reqs), Hkv, G * n, d)
        z = (q @ K.transpose(-1, -2)).view(len(reqs), Hkv, G, n, -1).mul_(s["scale"])
        see = torch.arange(P * PAGE, device=DEV) <= (held[:, None] + j)[..., None]    # [R][n][16 P]
        z.masked_fill_(~see[:, None, None], -math.inf)
        w = z.sub_(z.amax(-1, keepdim=True)).exp_()
        total = w.sum(-1, keepdim=True)
        V = torch.where(torch.arange(P * PAGE, device=DEV)[:, None] < (held + count)[:, None, None, None], V, 0.0)
        o = (w.flatten(2, 3) @ V).view(len(reqs), Hkv, G, n, d) / total
        gr, gj = _flat(counts)
        s["out"][first[gr] + gj] = o.permute(0, 3, 1, 2, 4).reshape(len(reqs), n, Hq, d)[gr, gj].to(s["out"].dtype)
    return s["out"]


def _flat(counts):
    """(request, place within it) of each of sum(counts) things in a row, counts known on the host."""
    n = torch.tensor(counts, device=DEV)
    r = torch.repeat_interleave(torch.arange(len(counts), device=DEV), n, output_size=sum(counts))
    return r, torch.arange(sum(counts), device=DEV) - (n.cumsum(0) - n)[r]


def _turn(x, c, si, case):
    """x [tokens][heads][d]: its first rotary_dim dims rotated pair by pair, the others as they are."""
    n = case["rotary_dim"]
    x, rest = x[..., :n].float(), x[..., n:].float()
    if case["pairs"] == "interleaved":
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.cat([torch.stack([a * c - b * si, b * c + a * si], -1).flatten(-2), rest], -1)
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * si, b * c + a * si, rest], -1)


def _plain_rotary(s):
    case, kv, ps = s["case"], s["kv"], s["ps"]
    Hq, Hkv, d, dt = case["q_heads"], case["kv_heads"], case["head_dim"], TYPES[case["cache"]]
    held, new = _lengths(case)
    r, j = _flat(new)
    m = ps.seq_lens[r] + j
    # angles of far positions need 64 bits
    ang = (s["positions"][r] + 1 + j).double()[:, None] * torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
    mag = _magnitude(case)
    c, si = (mag * ang.cos()).float().unsqueeze(1), (mag * ang.sin()).float().unsqueeze(1)
    q, k, v = s["rows"].view(-1, Hq + 2 * Hkv, d).split([Hq, Hkv, Hkv], 1)
    s["q_out"].copy_(_turn(q, c, si, case))
    k = _turn(k, c, si, case)
    if case["cache"] != "q8":
        page, slot = ps.page_table[r, m // PAGE].long(), m % PAGE
        kv.k[page, :, slot] = k.to(dt)
        kv.v[page, :, slot] = v
        return _cache(s)
    # 8 bits: the pages that get rows, whole, with their old rows under the old scale
    span = _touched(case)
    pr, pj = _flat([n for _, n in span])
    first = ps.seq_lens // PAGE
    page = ps.page_table[pr, first[pr] + pj].long()
    start = torch.tensor([0] + [n for _, n in span[:-1]], device=DEV).cumsum(0)
    at, slot = start[r] + m // PAGE - first[r], m % PAGE
    token = (first[pr] + pj)[:, None] * PAGE + torch.arange(PAGE, device=DEV)
    before = (token < ps.seq_lens[pr][:, None])[:, None, :, None]
    total = ps.seq_lens + torch.tensor(new, device=DEV)
    inside = (token < total[pr][:, None])[:, None, :, None]
    for pool, scales, x in ((kv.k, kv.k_scale, k), (kv.v, kv.v_scale, v.float())):
        old = pool[page].float()
        rows = torch.zeros_like(old)
        rows[at, :, slot] = x
        scale = _scale_for(rows.abs().amax((-1, -2)))
        had = before.any(2).squeeze(-1)
        scale = torch.where(had, torch.maximum(scale, scales[page]), scale)
        rows = torch.where(before, old * scales[page][..., None, None], rows) / scale[..., None, None]
        pool[page] = torch.where(inside, rows, old).to(torch.float8_e4m3fn)
        scales[page] = scale
    return _cache(s)


def _plain_release(ps, reqs):
    """Every page of the requests loses one reference; pages without any go onto the stack, the lowest id first."""
    pool, width = ps.refcount.numel(), ps.page_table.shape[1]
    reqs = reqs.long()
    held = torch.arange(width, device=DEV) < ps.num_pages[reqs][:, None]
    ids = torch.where(held, ps.page_table[reqs], pool).flatten().long()
    drops = torch.zeros(pool + 1, dtype=torch.int32, device=DEV).index_add_(0, ids, torch.ones_like(ids, dtype=torch.int32))[:pool]
    ps.refcount.sub_(drops)
    freed = (drops > 0) & (ps.refcount == 0)
    to = torch.where(freed, ps.free_count + freed.cumsum(0) - 1, pool)
    stack = torch.cat([ps.free_list, ps.free_list[:1]])
    stack[to] = torch.arange(pool, dtype=torch.int32, device=DEV)
    ps.free_list.copy_(stack[:pool])
    ps.free_count.add_(freed.sum())
    ps.num_pages[reqs] = 0
    ps.seq_lens[reqs] = 0


def _plain_fork(s):
    case, ps = s["case"], s["ps"]
    par, chi = s["parents"].long(), s["children"].long()
    _plain_release(ps, s["children"])
    m = ps.seq_lens[par]
    L = m if s["lengths"] is None else torch.minimum(m, s["lengths"])
    full, rem = L // PAGE, L % PAGE
    need = rem > 0
    rank = need.cumsum(0) - 1
    fits = ~need | (rank < ps.free_count)
    fresh = ps.free_list[(ps.free_count - 1 - rank).clamp_min(0)]
    width, pool = ps.page_table.shape[1], ps.refcount.numel()
    col = torch.arange(width, device=DEV)
    mine = fits[:, None]
    shared = mine & (col < full[:, None])
    row = torch.where(shared, ps.page_table[par], ps.page_table[chi])
    got = fits & need
    row = torch.where(got[:, None] & (col == full[:, None]), fresh[:, None], row)
    ids = torch.where(shared, row, pool).flatten().long()
    more = torch.cat([ps.refcount, ps.refcount[:1]]).index_add_(0, ids, torch.ones_like(ids, dtype=torch.int32))
    more[torch.where(got, fresh, pool).long()] = 1
    ps.refcount.copy_(more[:pool])
    # the rows of the last page that is not full, on every layer
    src = ps.page_table[par, full.clamp_max(width - 1)].long().clamp_min(0)
    dst = torch.where(got, fresh, src).long()
    rows = (torch.arange(PAGE, device=DEV) < rem[:, None])[None, None, :, None, :, None]
    p = s["pool"]
    p[:, :, dst] = torch.where(rows, p[:, :, src], p[:, :, dst])
    if s["scales"] is not None:
        s["scales"][:, :, dst] = s["scales"][:, :, src]
    ps.page_table[chi] = row
    ps.num_pages[chi] = torch.where(fits, full + need.int(), ps.num_pages[chi])
    ps.seq_lens[chi] = torch.where(fits, L, ps.seq_lens[chi])
    s["positions"][chi] = torch.where(fits, s["positions"][par] - (m - L), s["positions"][chi])
    ps.free_count.sub_(got.sum())
    s["forked"].copy_(fits)
    return _pages(s)


def _plain_turnover(s):
    ps = s["ps"]
    _plain_release(ps, s["done"])
    width, pool = ps.page_table.shape[1], ps.refcount.numel()
    want = (ps.seq_lens + s["ask"] + PAGE - 1) // PAGE
    fits = want <= width
    need = torch.where(fits, (want - ps.num_pages).clamp_min(0), 0)
    upto = need.cumsum(0)
    granted = fits & ((need == 0) | (upto <= ps.free_count))
    need = torch.where(granted, need, 0)
    col = torch.arange(width, device=DEV)
    fresh = (col >= ps.num_pages[:, None]) & (col < (ps.num_pages + need)[:, None])
    # pages leave the stack from its top, in the order of the requests
    at = (ps.free_count - 1)[:, None] - (upto - need)[:, None] - (col - ps.num_pages[:, None])
    row = torch.where(fresh, ps.free_list[at.clamp(0, pool - 1)], ps.page_table)
    refs = torch.cat([ps.refcount, ps.refcount[:1]])
    refs[torch.where(fresh, row, pool).flatten().long()] = 1
    ps.refcount.copy_(refs[:pool])
    ps.page_table.copy_(row)
    ps.num_pages.add_(need)
    ps.free_count.sub_(need.sum())
    s["granted"].copy_(granted)
    return _pages(s)


# -------------------------------------------------------------------- work --

def work(case):
    held, new = _lengths(case)
    R, Hq, Hkv, d, kind = case["reqs"], case["q_heads"], case["kv_heads"], case["head_dim"], case["kind"]
    e = 4 if case["cache"] == "f32" else 2
    c = 1 if case["cache"] == "q8" else e
    scales = 8 * Hkv if case["cache"] == "q8" else 0            # of one page
    if kind == "prompt":
        pages = sum(-(-(m + n) // PAGE) for m, n in zip(held, new))
        pairs = sum(n * m + n * (n + 1) // 2 for m, n in zip(held, new))
        return dict(bytes=2 * sum(new) * Hq * d * e + sum(m + n for m, n in zip(held, new)) * Hkv * d * 2 * c + pages * (scales + 4),
                    flops=4 * pairs * Hq * d)
    if kind == "rotary":
        T = sum(new)
        touched = sum(n for _, n in _touched(case))
        old = sum(m % PAGE for m in held) * 2 * Hkv * d if case["cache"] == "q8" else 0
        return dict(bytes=T * d * (2 * Hq * e + 2 * Hkv * (e + c)) + touched * (4 + 2 * scales) + old,
                    flops=3 * T * (Hq + Hkv) * case["rotary_dim"])
    if kind == "fork":
        # references are dropped and taken (read and written), table entries read and written, rows read and written
        _, _, taken, take = _forks(case)
        pages = sum(-(-x // PAGE) for x in taken + take)
        rows = sum(x % PAGE for x in take)
        copies = sum(x % PAGE > 0 for x in take)
        return dict(bytes=pages * 16 + case["layers"] * (rows * Hkv * d * c * 4 + copies * scales * 2), flops=pages)
    done, ask = _leaving(case)
    pages = sum(-(-held[r] // PAGE) + -(-ask[r] // PAGE) for r in done)
    return dict(bytes=pages * 16 + R * 16, flops=pages)


# ------------------------------------------------------------------- exact --

def _e4m3(x):
    """The nearest e4m3 value of |x| <= 448, ties to even: 3 bits below the leading one, from 2^-6 on."""
    step = _power(torch.frexp(x)[1].clamp_min(-5) - 4).double()
    return (x / step).round() * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "prompt":
        return _exact_prompt(s, case)
    if case["kind"] == "rotary":
        return _exact_rotary(s, case)
    return _exact_pages(s, case)


def _exact_prompt(s, case):
    kv, ps = s["kv"], s["ps"]
    held, new = _lengths(case)
    Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    G, t = Hq // Hkv, 0
    scale = float(torch.tensor(s["scale"], dtype=torch.float32))
    out = torch.zeros(sum(new), Hq, d, dtype=torch.float64, device=DEV)
    for r, (m, n) in enumerate(zip(held, new)):
        ids = ps.page_table[r, :-(-(m + n) // PAGE)].long()
        for h in range(Hkv):
            K, V = kv.k[ids, h].double(), kv.v[ids, h].double()
            if case["cache"] == "q8":
                K, V = K * kv.k_scale[ids, h].double()[:, None, None], V * kv.v_scale[ids, h].double()[:, None, None]
            K, V = K.reshape(-1, d)[:m + n], V.reshape(-1, d)[:m + n]
            step = max(1, int(2e8 / (m + n) / G))
            for a in range(0, n, step):
                b = min(n, a + step)
                q = s["q"][t + a:t + b, h * G:(h + 1) * G].double()                   # [tokens][G][d]
                z = scale * (q.flatten(0, 1) @ K[:m + b].T).view(b - a, G, m + b)
                late = torch.arange(m + b, device=DEV)[None, :] > m + torch.arange(a, b, device=DEV)[:, None]
                z[late[:, None].expand(-1, G, -1)] = -math.inf
                out[t + a:t + b, h * G:(h + 1) * G] = (torch.softmax(z, -1).flatten(0, 1) @ V[:m + b]).view(b - a, G, d)
        t += n
    return out


def _exact_rotary(s, case):
    kv, ps, q8 = s["kv"], s["ps"], case["cache"] == "q8"
    held, new = _lengths(case)
    Hq, Hkv, d, n2 = case["q_heads"], case["kv_heads"], case["head_dim"], case["rotary_dim"] // 2
    i = torch.arange(n2, dtype=torch.float64, device=DEV)
    freq = torch.exp(-math.log(THETA) * i / n2)
    if case["high"] > 0:
        turns = case["context"] * freq / (2 * math.pi)
        keep = ((turns - case["low"]) / (case["high"] - case["low"])).clamp(0, 1)
        freq = freq * keep + freq / case["factor"] * (1 - keep)
    else:
        freq = freq / case["factor"]
    mag = 1.0 + 0.1 * math.log(case["factor"]) if case["high"] > 0 else 1.0
    first, second = (2 * i.long(), 2 * i.long() + 1) if case["pairs"] == "interleaved" else (i.long(), i.long() + n2)
    k, v = kv.k.double(), kv.v.double()
    out = {"q": torch.zeros(sum(new), Hq, d, dtype=torch.float64, device=DEV)}
    ks, vs = (kv.k_scale.double(), kv.v_scale.double()) if q8 else (None, None)
    t = 0
    for r, (m, n) in enumerate(zip(held, new)):
        x = s["rows"][t:t + n].double().view(n, Hq + 2 * Hkv, d)
        ang = (torch.arange(n, dtype=torch.float64, device=DEV) + m)[:, None, None] * freq
        turned, a, b = x.clone(), x[..., first], x[..., second]
        turned[..., first] = mag * (a * ang.cos() - b * ang.sin())
        turned[..., second] = mag * (b * ang.cos() + a * ang.sin())
        out["q"][t:t + n] = turned[:, :Hq]
        kn, vn = turned[:, Hq:Hq + Hkv].transpose(0, 1), x[:, Hq + Hkv:].transpose(0, 1)       # [Hkv][n][d]
        t += n
        f = m // PAGE
        ids = ps.page_table[r, f:(m + n - 1) // PAGE + 1].long()
        for pool, scales, y in ((k, ks, kn), (v, vs, vn)):
            tile = pool[ids].transpose(0, 1).flatten(1, 2)                         # [Hkv][16 pages][d]
            at, end = m - f * PAGE, m - f * PAGE + n
            if q8:
                old = scales[ids].T                                                # [Hkv][pages]
                tile = tile * old.repeat_interleave(PAGE, 1).unsqueeze(-1)
                fresh = torch.zeros_like(tile)
                fresh[:, at:end] = y
                need = fresh.abs().view(Hkv, -1, PAGE * d).amax(-1)
                e = torch.ceil(torch.log2(need / TOP)).clamp_min(LEAST)
                e = torch.where(need > TOP * torch.exp2(e), e + 1, torch.where(need <= TOP * torch.exp2(e - 1), e - 1, e))
                sc = _power(e.clamp_min(LEAST).int()).double()
                if at:
                    sc[:, 0] = torch.maximum(sc[:, 0], old[:, 0])
                per = sc.repeat_interleave(PAGE, 1).unsqueeze(-1)
                rest = (tile / old.repeat_interleave(PAGE, 1).unsqueeze(-1))[:, end:].clone()
                tile[:, at:end] = y
                tile = _e4m3(tile / per)
                tile[:, end:] = rest
                scales[ids] = sc.T
            else:
                tile[:, at:end] = y
            pool[ids] = tile.view(Hkv, -1, PAGE, d).transpose(0, 1)
    out.update(k=k, v=v)
    if q8:
        out.update(k_scale=ks, v_scale=vs)
    return out


def _exact_pages(s, case):
    """The state after the pass, kept in lists; of the copied rows the whole pools (in the type that holds them exactly)."""
    ps = s["ps"]
    table, P, m = ps.page_table.tolist(), ps.num_pages.tolist(), ps.seq_lens.tolist()
    refs, stack, pos = ps.refcount.tolist(), ps.free_list.tolist(), s["positions"].tolist()
    height = int(ps.free_count[0])
    leave = s["children" if case["kind"] == "fork" else "done"].tolist()
    freed = []
    for r in leave:
        for p in table[r][:P[r]]:
            refs[p] -= 1
            if refs[p] == 0:
                freed.append(p)
        P[r] = m[r] = 0
    for p in sorted(freed):
        stack[height] = p
        height += 1
    out, ok = {}, []
    if case["kind"] == "turnover":
        spent = False
        for r, t in enumerate(s["ask"].tolist()):
            want = -(-(m[r] + t) // PAGE) - P[r]
            if want <= 0 or (not spent and want <= height and P[r] + want <= len(table[r])):
                for _ in range(max(0, want)):
                    height -= 1
                    table[r][P[r]] = stack[height]
                    refs[stack[height]] = 1
                    P[r] += 1
                ok.append(1)
            else:
                spent = spent or P[r] + want <= len(table[r])
                ok.append(0)
        out["granted"] = ok
    else:
        pool = s["pool"]
        lengths = s["lengths"].tolist() if s["lengths"] is not None else m
        for k, (p, c) in enumerate(zip(s["parents"].tolist(), s["children"].tolist())):
            L = min(m[p], lengths[k] if s["lengths"] is not None else m[p])
            if L % PAGE and height == 0:
                ok.append(0)
                continue
            for j in range(L // PAGE):
                table[c][j] = table[p][j]
                refs[table[p][j]] += 1
            P[c] = -(-L // PAGE)
            if L % PAGE:
                height -= 1
                to = table[c][P[c] - 1] = stack[height]
                refs[to] = 1
                pool[:, :, to, :, :L % PAGE] = pool[:, :, table[p][P[c] - 1], :, :L % PAGE]
                if s["scales"] is not None:
                    s["scales"][:, :, to] = s["scales"][:, :, table[p][P[c] - 1]]
            m[c], pos[c] = L, pos[p] - (m[p] - L)
            ok.append(1)
        out.update(forked=ok, positions=pos, pool=pool if s["scales"] is None else pool.view(torch.float8_e4m3fn))
        if s["scales"] is not None:
            out["scales"] = s["scales"]
    out.update(page_table=table, num_pages=P, seq_lens=m, refcount=refs, free_list=stack, free_count=[height])
    return {k: _i32(x) if isinstance(x, list) else x for k, x in out.items()}
