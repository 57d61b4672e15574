"""The operators on a prompt's way into the decode step refuse what they do not take,
before any launch; rotary frequencies, which are made on the host."""
import ctypes
import math

import pytest
import torch

import paper_2609_03494_amd as gp
from paper_2609_03494_amd import _lib
from test_cache_ops import _NoLaunch, FAKE, INVALID, ROPE, UNSUPPORTED, WORKSPACE, _kv, _kv8, _ps, lib  # noqa: F401


def _rope(layout=0, n=128, mag=1.0, freq=None):
    r = _lib._Rope(layout, n, mag)
    for i in range(64):
        r.freq[i] = 1.0 / (i + 1)
    if freq is not None:
        r.freq[freq[0]] = freq[1]
    return ctypes.byref(r)


def _rotary(fn, kv, ps, rope, **kw):
    a = dict(ROPE, **kw)
    return fn(kv, ps, a["positions"], rope, a["start"], a["tokens"], a["q"], a["q_stride"], a["q_out"], a["k"], a["k_stride"],
              a["v"], a["v_stride"], a["hq"], a["advance"], None)


@pytest.mark.parametrize("q8", [False, True])
def test_append_rotary_refusals(lib, q8):  # noqa: F811
    fn, kv = (lib.gp_append_rotary_q8, _kv8) if q8 else (lib.gp_append_rotary, _kv)
    nan, inf = float("nan"), float("inf")
    for bad in (None, _rope(layout=2), _rope(layout=-1), _rope(n=0), _rope(n=-16), _rope(n=144), _rope(mag=0.0), _rope(mag=-1.0),
                _rope(mag=nan), _rope(mag=inf), _rope(freq=(0, inf)), _rope(freq=(63, nan))):
        assert _rotary(fn, kv(), _ps(), bad) == INVALID
    assert _rotary(fn, kv(d=64), _ps(), _rope(n=128), k_stride=512, v_stride=512, q_stride=2048) == INVALID
    for n in (2, 8, 24, 120):
        assert _rotary(fn, kv(), _ps(), _rope(n=n)) == UNSUPPORTED
    good = _rope(n=64)
    for bad in (dict(tokens=3), dict(k_stride=1023), dict(q_stride=4095), dict(positions=None), dict(k=None), dict(q_out=None),
                dict(q_out=0x100000 + 256), dict(q_out=0x300000 - 4)):
        assert _rotary(fn, kv(), _ps(), good, **bad) == INVALID, bad
    assert _rotary(fn, None, _ps(), good) == _rotary(fn, kv(), None, good) == INVALID
    assert _rotary(fn, kv(d=96), _ps(), good) == _rotary(fn, kv(), _ps(), good, hq=24) == UNSUPPORTED
    assert _rotary(fn, kv(), _ps(), _rope(n=64, freq=(32, nan)), tokens=0, start=FAKE) == 0     # (behind the pairs: not looked at)


def test_boundary_score_rotary_refusals(lib):  # noqa: F811
    p = _lib._Params(0.9, 0.999, 0.99, 0.0, 0.088, 0.0, 4, 0)          # rope_theta is not looked at

    def call(rope, stages=3, n=1 << 40, params=p, cand=144):
        return lib.gp_boundary_score_rotary(_kv(), _ps(), FAKE, FAKE, 512, FAKE, FAKE, FAKE, 2, 32, ctypes.byref(params), rope,
                                            FAKE, FAKE, cand, FAKE, n, None, stages)
    assert call(None) == call(_rope(layout=5)) == call(_rope(mag=0.0)) == call(_rope(), stages=0) == call(_rope(), stages=4) == INVALID
    assert call(_rope(), cand=16) == INVALID
    assert call(_rope(n=40)) == UNSUPPORTED
    assert call(_rope(), n=16) == WORKSPACE


def test_rope_frequencies(lib):  # noqa: F811
    for n in (2, 16, 96, 128):
        f = gp.gp_rope_frequencies(n, 1.0e6)
        assert len(f) == n // 2 and f[0] == 1.0
        for i, x in enumerate(f):
            assert abs(x - 1.0e6 ** (-2.0 * i / n)) <= 1e-15 * x
        for i, (x, y) in enumerate(zip(f, gp.gp_rope_frequencies(n, 1.0e6, 4.0))):
            assert y == x / 4
        g = gp.gp_rope_frequencies(n, 1.0e6, 8.0, 1.0, 4.0, 8192)
        for i, (x, y) in enumerate(zip(f, g)):
            u = 8192 * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (u - 1.0) / 3.0))
            assert abs(y - x * (keep + (1 - keep) / 8)) <= 1e-14 * x
    freq = (ctypes.c_double * 64)()
    call = lambda n=64, theta=1e6, factor=2.0, low=1.0, high=4.0, ctx=8192.0, to=freq: lib.gp_rope_frequencies(  # noqa: E731
        to, n, theta, factor, low, high, ctx)
    nan, inf = float("nan"), float("inf")
    assert call() == 0
    for bad in (dict(to=None), dict(n=0), dict(n=63), dict(n=130), dict(theta=0.0), dict(theta=nan), dict(theta=inf),
                dict(factor=0.5), dict(factor=nan), dict(factor=inf), dict(low=-1.0), dict(low=nan), dict(low=4.0),
                dict(high=0.5), dict(high=-1.0), dict(high=nan), dict(high=inf), dict(ctx=0.0), dict(ctx=nan), dict(ctx=inf)):
        assert call(**bad) == INVALID, bad
    with pytest.raises(gp.GrowPageError):
        gp.gp_rope_frequencies(64, -1.0)
    with pytest.raises(ValueError):
        gp.gp_rope_frequencies(256, 1.0e6)
    with pytest.raises(ValueError):
        gp.Rope(0, [])


PROMPT = dict(start=FAKE, tokens=40, advanced=0, q=0x100000, q_stride=4096, hq=32, scale=0.088, out=0x900000, ws=FAKE, ws_bytes=1 << 40)


@pytest.mark.parametrize("q8", [False, True])
def test_prompt_attention_refusals(lib, q8):  # noqa: F811
    fn, kv = (lib.gp_prompt_attention_q8, _kv8) if q8 else (lib.gp_prompt_attention, _kv)

    def call(kv_=None, ps=None, **kw):
        a = dict(PROMPT, **kw)
        return fn(kv_ or kv(), ps or _ps(), a["start"], a["tokens"], a["advanced"], a["q"], a["q_stride"], a["hq"], a["scale"], a["out"],
                  a["ws"], a["ws_bytes"], None)
    nan, inf = float("nan"), float("inf")
    assert fn(None, _ps(), FAKE, 40, 0, FAKE, 4096, 32, 0.1, FAKE, FAKE, 1 << 40, None) == INVALID
    assert fn(kv(), None, FAKE, 40, 0, FAKE, 4096, 32, 0.1, FAKE, FAKE, 1 << 40, None) == INVALID
    for bad in (dict(scale=0.0), dict(scale=-0.1), dict(scale=nan), dict(scale=inf), dict(scale=2.0 ** 127), dict(tokens=-1), dict(start=None),
                dict(q_stride=4095), dict(q_stride=(1 << 30) + 1), dict(q=None), dict(out=None), dict(ws=None), dict(out=0x100000),
                dict(out=0x100000 + 8), dict(out=0x100000 + 39 * 8192 + 8190), dict(out=0x100000 - 40 * 8192 + 2)):
        assert call(**bad) == INVALID, bad
    if q8:
        assert call(scale=2.0 ** 111) == INVALID
    for bad in (kv(k=FAKE + 8), kv(v=FAKE + 4), kv(pool=99)):
        assert call(bad) == INVALID
    for bad in (kv(d=96), kv(page=32)):
        assert call(bad) == UNSUPPORTED
    for hq in (24, 4, 0, 128):
        assert call(hq=hq) == UNSUPPORTED
    assert call(ps=_ps(R=65536)) == call(ps=_ps(width=8193)) == UNSUPPORTED
    assert call(tokens=1 << 25) == UNSUPPORTED                         # 2^25 * 4 / 128 pieces of 8 heads
    assert call(tokens=2 ** 31 - 1, q_stride=1 << 30) == UNSUPPORTED
    size = gp.gp_workspace_bytes(gp.GP_OP_PROMPT, 4, 40, 32, 8, 128, 10, torch.bfloat16)
    assert call(ws_bytes=size - 1) == call(ws_bytes=256) == call(ws_bytes=0) == WORKSPACE
    assert call(tokens=0, q=None, out=None, ws=None) == call(ps=_ps(R=0), q=None) == 0


def test_prompt_workspace(lib):  # noqa: F811
    """A workspace of more tokens, or more requests, is no smaller; none of what is no shape."""
    size = lambda R=4, T=40, hq=32, hkv=8, d=128, dt=torch.bfloat16: gp.gp_workspace_bytes(gp.GP_OP_PROMPT, R, T, hq, hkv, d, 10, dt)  # noqa: E731
    for hq, hkv, d in ((32, 8, 128), (64, 8, 64), (5, 5, 64), (8, 1, 128), (64, 64, 64)):
        for dt in (torch.bfloat16, torch.float32):
            steps = [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1000, 30000]
            sizes = [size(R=R, T=T, hq=hq, hkv=hkv, d=d, dt=dt) for R in (1, 3, 64, 65, 700) for T in steps]
            for i, x in enumerate(sizes):
                assert 0 < x < 1 << 31
                if i % len(steps):
                    assert x >= sizes[i - 1]
                if i >= len(steps):
                    assert x >= sizes[i - len(steps)]
    for bad in (dict(hq=24), dict(d=96), dict(R=-1), dict(T=-1)):
        with pytest.raises(gp.GrowPageError):
            size(**bad)


def _state(R=4, width=10, pool=100, **none):
    a = dict(table=FAKE, pages=FAKE, lens=FAKE, refs=FAKE, stack=FAKE, height=FAKE)
    a.update(none)
    return ctypes.byref(_lib._PageState(a["table"], a["pages"], a["lens"], a["refs"], a["stack"], a["height"], R, width, pool))


BAD_STATES = [dict(table=None), dict(pages=None), dict(lens=None), dict(refs=None), dict(stack=None), dict(height=None),
              dict(pool=0), dict(R=-1), dict(width=0)]


def test_pages_refusals(lib):  # noqa: F811
    reserve = lambda ps=None, tokens=FAKE, keep=0, granted=FAKE: lib.gp_pages_reserve(ps or _state(), tokens, keep, granted, None)  # noqa: E731
    release = lambda ps=None, reqs=FAKE, n=3: lib.gp_pages_release(ps or _state(), reqs, n, None)  # noqa: E731
    for bad in BAD_STATES:
        assert reserve(_state(**bad)) == release(_state(**bad)) == INVALID, bad
    assert lib.gp_pages_reserve(None, FAKE, 0, FAKE, None) == lib.gp_pages_release(None, FAKE, 1, None) == INVALID
    assert reserve(tokens=None) == reserve(granted=None) == reserve(keep=-1) == release(reqs=None) == release(n=-1) == INVALID
    for call in (reserve, release):
        assert call(_state(R=65536)) == call(_state(width=8193)) == UNSUPPORTED
        assert call(_state(R=0)) == 0
    assert release(n=65536) == UNSUPPORTED
    assert release(n=0, reqs=None) == 0


@pytest.mark.parametrize("q8", [False, True])
def test_fork_refusals(lib, q8):  # noqa: F811
    fn = lib.gp_pages_fork_q8 if q8 else lib.gp_pages_fork

    def layers(*kw):
        kind = _lib._KV8Layer if q8 else _lib._KVLayer
        made = []
        for k in kw:
            a = dict(k=FAKE, v=FAKE, pool=100, hkv=8, page=16, d=128)
            a.update(k)
            made.append(kind(a["k"], a["v"], *((FAKE, FAKE) if q8 else ()), a["pool"], a["hkv"], a["page"], a["d"],
                             *(() if q8 else (a.get("dtype", 1),))))
        return (kind * len(made))(*made)

    def call(ls=None, n=None, ps=None, parents=FAKE, children=FAKE, forks=2, forked=FAKE):
        ls = layers({}, {}) if ls is None else ls
        return fn(ls, len(ls) if n is None else n, ps or _state(), parents, children, None, forks, None, forked, None)
    assert fn(None, 1, _state(), FAKE, FAKE, None, 2, None, FAKE, None) == call(n=0) == call(n=-3) == INVALID
    assert call(parents=None) == call(children=None) == call(forked=None) == call(forks=-1) == INVALID
    for bad in (dict(k=None), dict(v=None), dict(pool=99), dict(hkv=4), dict(d=64), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(hkv=0)):
        assert call(layers({}, bad)) == INVALID, bad
    assert call(layers(dict(pool=99), dict(pool=99))) == INVALID                  # another pool than the state's
    if not q8:
        assert call(layers({}, dict(dtype=0))) == call(layers({}, dict(dtype=7))) == INVALID
    for bad in BAD_STATES:
        assert call(ps=_state(**bad)) == INVALID, bad
    assert call(layers(dict(d=96))) == call(layers(dict(page=32))) == call(forks=2049) == UNSUPPORTED
    assert call(layers(*([{}] * 257))) == call(layers(dict(hkv=8193))) == call(ps=_state(R=65536)) == UNSUPPORTED
    assert call(forks=0, parents=None) == call(ps=_state(R=0)) == 0


def test_binding_refusals():
    """What the Python calls check themselves, on tensors that no GPU has to hold."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    ps = gp.PageState(i32(4, 10), i32(4), i32(4), i32(100), i32(100), i32(1))
    k = torch.zeros(100, 2, 16, 64, dtype=torch.bfloat16)
    layer = gp.KVLayer(k, k)
    with pytest.raises(ValueError):
        gp.gp_pages_release(ps, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        gp.gp_pages_reserve(ps, i32(4), torch.zeros(4))
    for v in (k[:99], k.float(), k[:, :1]):                             # pools of two shapes or types
        with pytest.raises(ValueError, match="one shape"):
            gp.KVLayer(k, v).c()
        with pytest.raises(ValueError, match="one shape"):
            gp.Layers([layer, gp.KVLayer(k, v)])
    with pytest.raises(ValueError):                                     # not on a GPU
        gp.gp_pages_reserve(ps, i32(4), i32(4))
    with pytest.raises(ValueError):
        gp.Layers([])
    with pytest.raises(ValueError):
        gp.Layers([layer, gp.KV8Layer(k.view(torch.uint8)[..., :64].contiguous(), k.view(torch.uint8)[..., :64].contiguous(),
                                      torch.zeros(100, 2), torch.zeros(100, 2))])


def _device_calls():
    """Each call of the binding on a prompt's way, with every tensor that its kernels reach, by name."""
    pool, hkv, d, R = 6, 2, 64, 3
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    state = lambda: gp.PageState(i32(R, 4), i32(R), i32(R), i32(pool), i32(pool), i32(1))  # noqa: E731
    layers = {"": lambda: gp.KVLayer(bf(pool, hkv, 16, d), bf(pool, hkv, 16, d)),
              "_q8": lambda: gp.KV8Layer(u8(pool, hkv, 16, d), u8(pool, hkv, 16, d), torch.ones(pool, hkv), torch.ones(pool, hkv))}
    of_state = lambda ps: dict(page_table=ps.page_table, num_pages=ps.num_pages, seq_lens=ps.seq_lens)  # noqa: E731
    rope = gp.Rope(gp.GP_ROPE_HALF, [1.0] * 16)
    for q8, layer in layers.items():
        kv, ps, t = layer(), state(), dict(positions=i32(R), k_new=bf(R, hkv, d), v_new=bf(R, hkv, d), q=bf(R, hkv, d),
                                           q_out=bf(R, hkv, d), tok_start=i32(R + 1))
        yield f"gp_append_rotary{q8}", {**vars(kv), **of_state(ps), **t}, lambda fn, kv=kv, ps=ps, t=t: fn(
            kv, ps, t["positions"], t["k_new"], t["v_new"], rope, q=t["q"], q_out=t["q_out"], tok_start=t["tok_start"])
        kv, ps, t = layer(), state(), dict(q=bf(R, hkv, d), out=bf(R, hkv, d), ws=u8(64), tok_start=i32(R + 1))
        yield f"gp_prompt_attention{q8}", {**vars(kv), **of_state(ps), **t}, lambda fn, kv=kv, ps=ps, t=t: fn(
            kv, ps, t["q"], 0.1, t["out"], t["ws"], tok_start=t["tok_start"])
        kv, ps, t = layer(), state(), dict(parents=i32(2), children=i32(2), forked=i32(2), lengths=i32(2), positions=i32(R))
        yield f"gp_pages_fork{q8}", {**vars(kv), **vars(ps), **t}, lambda fn, kv=kv, ps=ps, t=t: fn(
            [kv], ps, t["parents"], t["children"], t["forked"], lengths=t["lengths"], positions=t["positions"])
    kv, ps, t = layers[""](), state(), dict(q_pre=bf(R, hkv, d), qstate=torch.zeros(R, 2, hkv, d), slot_ids=i32(R), positions=i32(R),
                                            bnd=i32(1), k_counts=i32(1, hkv, 2), scores=torch.zeros(1, hkv, 48), ws=u8(64))
    yield "gp_boundary_score_rotary", {**vars(kv), **of_state(ps), **t}, lambda fn: fn(
        kv, ps, t["q_pre"], t["qstate"], t["slot_ids"], t["positions"], t["bnd"], gp.Params(), rope, t["k_counts"], t["scores"], t["ws"])
    ps1, t1 = state(), dict(tokens=i32(R), granted=i32(R))
    yield "gp_pages_reserve", {**vars(ps1), **t1}, lambda fn: fn(ps1, t1["tokens"], t1["granted"])
    ps2, t2 = state(), dict(reqs=i32(2))
    yield "gp_pages_release", {**vars(ps2), **t2}, lambda fn: fn(ps2, t2["reqs"])


def test_every_tensor_lies_on_the_current_device(monkeypatch):
    """Host tensors that say they lie on device 0: the call goes through.  One of them at a time on the host or on
    another device, whichever it is: the call is refused and the library not reached."""
    fake = _NoLaunch()
    monkeypatch.setattr(_lib, "load", lambda: fake)
    monkeypatch.setattr(_lib, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    names = set()
    for name, tensors, call in _device_calls():
        fn = getattr(gp, name)
        for t in tensors.values():
            t.get_device = lambda: 0
        fake.calls = 0
        call(fn)
        assert fake.calls == 1, name
        for what, t in tensors.items():
            for dev in (-1, 1):
                t.get_device = lambda dev=dev: dev
                with pytest.raises(ValueError, match="device"):
                    call(fn)
                assert fake.calls == 1, (name, what)
            t.get_device = lambda: 0
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)      # all on a device that is not the current one
        with pytest.raises(ValueError, match="current device"):
            call(fn)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
        names.add(name)
    assert len(names) == 9
