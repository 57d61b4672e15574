"""A serving step in which some requests get no pages: nothing of theirs goes into the cache or comes out of it in any layer,
and they go on when there is room."""
from __future__ import annotations

import pytest
import torch

import paper_2609_03494_amd as gp
from test_cache_ops_gpu import DEV, _i32
from test_prompt_run_gpu import HALF, Server

pytestmark = pytest.mark.gpu


def _step(s, ns, want):
    """ns[r] new tokens of each request, of which those with want[r] get their pages: lengths move once, behind the last layer."""
    tokens, granted = _i32(ns), _i32([-1] * s.R)
    gp.gp_pages_reserve(s.ps, tokens, granted)
    starts = [0]
    for n in ns:
        starts.append(starts[-1] + n)
    T, q8, start = starts[-1], s.kind == "q8", _i32(starts)
    made = []
    for kv in s.layers:
        rows = torch.randn(T, s.hq + 2 * s.hkv, s.d, generator=s.gen).to(s.dt).to(DEV)
        q, k, v = rows[:, :s.hq], rows[:, s.hq:s.hq + s.hkv], rows[:, s.hq + s.hkv:]
        q_out, out = (torch.full((T, s.hq, s.d), x, dtype=s.dt, device=DEV) for x in (5.0, 7.0))
        (gp.gp_append_rotary_q8 if q8 else gp.gp_append_rotary)(kv, s.ps, s.positions, k, v, s.rope, q=q, q_out=q_out, tok_start=start,
                                                                advance=False)
        (gp.gp_prompt_attention_q8 if q8 else gp.gp_prompt_attention)(kv, s.ps, q_out, s.scale, out, s.ws, tok_start=start)
        made.append((q, q_out, k, v, out))
    taken = tokens * granted
    s.ps.seq_lens += taken
    s.positions += taken
    torch.cuda.synchronize()
    assert granted.tolist() == want
    for l, (q, q_out, k, v, out) in enumerate(made):
        for r in range(s.R):
            if want[r]:
                s.took(l, r, slice(starts[r], starts[r + 1]), q, q_out, k, v, out)
            else:
                assert bool((out[starts[r]:starts[r + 1]] == 0).all()), (l, r)
    for r in range(s.R):
        s.pos[r] += ns[r] * want[r]
    assert s.positions.tolist() == s.pos
    s.check_pages()


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8"])
def test_requests_that_wait(kind):
    print(f"[waiting] {kind}", flush=True)
    s = Server(kind, gp.Rope(HALF, gp.gp_rope_frequencies(32, 1.0e6)), R=5, pool=12)
    _step(s, [37, 16, 5, 0, 16], [1, 1, 1, 1, 1])
    _step(s, [80, 40, 3, 20, 0], [1, 0, 1, 0, 1])             # the second has no pages, the fourth may not overtake it
    _step(s, [1, 40, 1, 20, 0], [1, 0, 1, 0, 1])
    s.release([0])
    _step(s, [0, 40, 1, 20, 1], [1, 1, 1, 1, 1])
