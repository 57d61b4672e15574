"""Rotary positions in either pairing, over a part of the head, with scaled frequencies
and a magnitude: appends and boundary scoring against float64."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_03494_amd as gp
import test_cache_ops_gpu as base
import workloads as W
from _harness import DeviceCase, library_params, to_numpy
from test_cache_ops_gpu import BF16, DEV, F32, RAGGED, SINGLE, _append_case, _check_append, _i32

pytestmark = pytest.mark.gpu


def _turned(x, pos, rope):
    """x [tokens][heads][d] float64, positions [tokens] as `rope` turns them, and the magnitude times |a| + |b| of each
    element's pair (zero behind the rotated part, which has to come out as it went in, rounded once)."""
    n = len(rope.freq)
    first, second = ((2 * torch.arange(n), 2 * torch.arange(n) + 1) if rope.layout == gp.GP_ROPE_INTERLEAVED else
                     (torch.arange(n), torch.arange(n) + n))
    mag = float(np.float32(rope.magnitude))
    ang = pos.double()[:, None, None] * torch.tensor(rope.freq, dtype=torch.float64)
    out, size = x.clone(), torch.zeros_like(x)
    a, b = x[..., first], x[..., second]
    out[..., first] = mag * (a * ang.cos() - b * ang.sin())
    out[..., second] = mag * (b * ang.cos() + a * ang.sin())
    size[..., first] = size[..., second] = mag * (a.abs() + b.abs())
    return out, size


def _rope(layout, n, d, scaled):
    if scaled:
        return gp.Rope(layout, gp.gp_rope_frequencies(n, 1.0e4, 8.0, 1.0, 4.0, 8192), 0.1 * math.log(8.0) + 1.0)
    return gp.Rope(layout, gp.gp_rope_frequencies(n, 1.0e6))


HALF, SIDE = gp.GP_ROPE_HALF, gp.GP_ROPE_INTERLEAVED
FORMS = [(HALF, 128, True), (HALF, 64, False), (HALF, 48, True), (HALF, 16, False), (SIDE, 128, False), (SIDE, 64, True),
         (SIDE, 32, True), (SIDE, 112, False)]


@pytest.mark.parametrize("cache,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 3, 3, 64), ("f32", 8, 1, 64), ("f32", 4, 2, 128),
                                            ("q8", 32, 8, 128), ("q8", 5, 5, 64), ("q8", 16, 2, 64), ("q8", 4, 2, 128)])
@pytest.mark.parametrize("layout,n,scaled", FORMS)
@pytest.mark.parametrize("form", ["ragged", "single", "fused"])
def test_append_rotary(monkeypatch, cache, hq, hkv, d, layout, n, scaled, form):
    if n > d:
        n = d
    rope = _rope(layout, n, d, scaled)
    reqs = SINGLE if form == "single" else RAGGED
    s = _append_case(cache, reqs, hq, hkv, d, 11 + hq, form == "fused", 0 if form == "ragged" else 3, form == "single")
    q_out = torch.full((s["q"].shape[0], hq, d), 7.0, dtype=s["dt"], device=DEV)
    s["position_tensor"] = _i32(s["pos"])
    fn = gp.gp_append_rotary_q8 if cache == "q8" else gp.gp_append_rotary
    advance = form != "fused"
    fn(s["kv"], s["ps"], s["position_tensor"], s["k"], s["v"], rope, q=s["q"], q_out=q_out, tok_start=s["start"], advance=advance)
    torch.cuda.synchronize()
    monkeypatch.setattr(base, "_rotated", _turned)
    _check_append(s, cache, reqs, hq, hkv, d, rope, q_out, advance)


@pytest.mark.parametrize("cache", ["bf16", "f32", "q8"])
def test_whole_head_at_theta_is_append_rope(cache):
    """Half-split pairs of the whole head at theta^(-2 i / d), magnitude 1: what gp_append_rope writes, to the rounding
    of its angles (bytes but for a few)."""
    d, out = 128, []
    for own in (False, True):
        s = _append_case(cache, RAGGED, 8, 2, d, 3, False, 0, False)
        q_out = torch.zeros((s["q"].shape[0], 8, d), dtype=s["dt"], device=DEV)
        args = (s["kv"], s["ps"], _i32([m - 1 for m, _, _ in RAGGED]), s["k"], s["v"])
        if own:
            fn, by = (gp.gp_append_rotary_q8 if cache == "q8" else gp.gp_append_rotary), gp.Rope(HALF, gp.gp_rope_frequencies(d, 1e6))
        else:
            fn, by = (gp.gp_append_rope_q8 if cache == "q8" else gp.gp_append_rope), 1e6
        fn(*args, by, q=s["q"], q_out=q_out, tok_start=s["start"])
        torch.cuda.synchronize()
        out.append([q_out, *vars(s["kv"]).values()])
    for x, y in zip(*out):
        assert (x.view(torch.uint8) != y.view(torch.uint8)).float().mean() < 1e-3


def test_append_rotary_in_place_and_captured():
    """q_out may be q; replays with eager calls between give the same bytes."""
    rope = _rope(SIDE, 64, 128, True)
    s = _append_case("bf16", RAGGED, 8, 2, 128, 3, False, 0, False)
    pos = _i32(s["pos"])
    want = torch.zeros_like(s["q"])
    args = (s["kv"], s["ps"], pos, s["k"], s["v"], rope)
    gp.gp_append_rotary(*args, q=s["q"], q_out=want, tok_start=s["start"], advance=False)
    k = s["kv"].k.clone()
    q = s["q"].clone()
    gp.gp_append_rotary(*args, q=q, q_out=q, tok_start=s["start"], advance=False)
    torch.cuda.synchronize()
    live = torch.cat([torch.full((n,), m >= 0) for m, _, n in RAGGED])
    assert torch.equal(q[live], want[live])
    out, graph, stream = torch.zeros_like(q), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        gp.gp_append_rotary(*args, q=s["q"], q_out=out, tok_start=s["start"], advance=False)
    for _ in range(3):
        out.zero_()
        s["kv"].k.copy_(s["before"][0])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(s["kv"].k.view(torch.int16), k.view(torch.int16))
        gp.gp_append_rotary(*args, q=s["q"], q_out=torch.empty_like(out), tok_start=s["start"], advance=False)
        torch.cuda.synchronize()


@pytest.mark.parametrize("layout,n,scaled", FORMS)
@pytest.mark.parametrize("workload", ["tiny", "high"])
def test_boundary_score_rotary(monkeypatch, workload, layout, n, scaled):
    """Counts and scores of the boundary requests against the oracle with its rotation replaced."""
    w = W.tiny() if workload == "tiny" else W.high_concurrency()
    n = min(n, w.head_dim)
    rope = _rope(layout, n, w.head_dim, scaled)

    def turn(x, pos, theta):
        out, _ = _turned(torch.from_numpy(np.asarray(x, np.float64)).reshape(1, 1, -1), torch.tensor([pos]), rope)
        return out.reshape(-1).numpy()

    monkeypatch.setattr(O.growpage_oracle, "rope", turn)
    dc = DeviceCase(w)
    bnd = np.asarray(w.boundary[:4], np.int32)
    params = O.Params()
    p32, max_cand, hkv = params.as_f32(w.head_dim), (w.max_pages - 1) * w.page_size, w.num_kv_heads
    counts = torch.full((len(bnd), hkv, 2), -7, dtype=torch.int32, device=DEV)
    scores = torch.full((len(bnd), hkv, max_cand), -1.0, device=DEV)
    ws = gp.workspace(gp.GP_OP_SCORE, w.num_reqs, len(bnd), w.num_q_heads, hkv, w.head_dim, w.max_pages, dc.q_pre.dtype)
    gp.gp_boundary_score_rotary(dc.layers[0], dc.ps, dc.q_pre, dc.qstate, dc.slot_ids, dc.positions, _i32(bnd),
                                library_params(params, w.head_dim), rope, counts, scores, ws)
    torch.cuda.synchronize()
    counts, scores = counts.cpu().numpy(), scores.cpu().numpy()
    for i, r in enumerate(bnd):
        P, b = int(w.num_pages[r]), w.page_size
        toks = dc.gather(w.page_table[r], (P - 1) * b, "k")
        c, sc, a32 = O.score_request(toks, w.dtype, P, b, w.q_pre[r], w.qstate[w.slot_ids[r]], int(w.positions[r]), p32, p32.scale)
        for h in range(hkv):
            np.testing.assert_allclose(scores[i, h, :(P - 1) * b], sc[h], rtol=1e-5, atol=0)
            for x in range(2):
                assert counts[i, h, x] == c[h, x] or O.top_p_fragile(a32[x, h], p32.p), (i, h, x)
