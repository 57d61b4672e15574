"""The operators around the paged cache refuse what they do not take, before any
launch: rotated appends, the 8-bit cache, page bounds, selection and attention
over listed pages."""
import ctypes
import os

import pytest
import torch

import paper_2609_03494_amd as gp
from paper_2609_03494_amd import _lib

FAKE = 0x1000
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_03494_amd import build
        build.build()
    return gp.load()


def _kv(k=FAKE, v=FAKE, pool=100, hkv=8, page=16, d=128, dtype=1):
    return ctypes.byref(_lib._KVLayer(k, v, pool, hkv, page, d, dtype))


def _kv8(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, pool=100, hkv=8, page=16, d=128):
    return ctypes.byref(_lib._KV8Layer(k, v, ks, vs, pool, hkv, page, d))


def _ps(R=4, width=10, pool=100, table=FAKE):
    return ctypes.byref(_lib._PageState(table, FAKE, FAKE, FAKE, FAKE, FAKE, R, width, pool))


ROPE = dict(positions=FAKE, start=None, tokens=4, q=0x100000, q_stride=4096, q_out=0x200000, k=0x300000, k_stride=1024,
            v=0x400000, v_stride=1024, hq=32, theta=1e6, advance=1)


def _rope(fn, kv, ps, **kw):
    a = dict(ROPE, **kw)
    return fn(kv, ps, a["positions"], a["start"], a["tokens"], a["q"], a["q_stride"], a["q_out"], a["k"], a["k_stride"],
              a["v"], a["v_stride"], a["hq"], a["theta"], a["advance"], None)


@pytest.mark.parametrize("q8", [False, True])
def test_append_rope_refusals(lib, q8):
    fn = lib.gp_append_rope_q8 if q8 else lib.gp_append_rope
    kv = _kv8 if q8 else _kv
    for bad in (dict(tokens=3), dict(tokens=-1, start=FAKE), dict(theta=0.0), dict(theta=float("nan")),
                dict(theta=float("inf")), dict(k_stride=1023), dict(v_stride=0), dict(q_stride=4095),
                dict(k_stride=(1 << 30) + 1), dict(positions=None), dict(k=None), dict(v=None), dict(q_out=None),
                # outputs over inputs: other than in place
                dict(q_out=0x100000 + 256), dict(q_out=0x100000, q_stride=8192), dict(q_out=0x300000 - 4),
                dict(q_out=0x400000)):
        assert _rope(fn, kv(), _ps(), **bad) == INVALID, bad
    assert _rope(fn, None, _ps()) == INVALID
    assert _rope(fn, kv(), None) == INVALID
    assert _rope(fn, kv(), _ps(pool=99)) == INVALID
    assert _rope(fn, kv(d=96), _ps()) == UNSUPPORTED
    assert _rope(fn, kv(page=32), _ps()) == UNSUPPORTED
    assert _rope(fn, kv(), _ps(), hq=24) == UNSUPPORTED
    assert _rope(fn, kv(), _ps(width=8193)) == UNSUPPORTED
    assert _rope(fn, kv(), _ps(R=65536), tokens=65536) == UNSUPPORTED
    assert _rope(fn, kv(), _ps(), tokens=(1 << 27) + 1, start=FAKE, q=None) == UNSUPPORTED
    assert _rope(fn, kv(hkv=8193), _ps(), q=None, k_stride=1 << 21, v_stride=1 << 21) == UNSUPPORTED
    # nothing to do
    assert _rope(fn, kv(), _ps(R=0), tokens=0) == 0
    assert _rope(fn, kv(), _ps(), tokens=0, start=FAKE) == 0


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(pool=0), dict(hkv=0),
                                 dict(k=FAKE + 8), dict(v=FAKE + 4)])
def test_8bit_layer_refusals(lib, bad):
    """A null pool or scale, and pools off 16 bytes, in every call that takes such a layer."""
    ps = _ps(pool=bad.get("pool", 100))
    assert _rope(lib.gp_append_rope_q8, _kv8(**bad), ps) == INVALID
    assert lib.gp_decode_attention_q8(_kv8(**bad), ps, FAKE, 32, 0.1, FAKE, FAKE, 1 << 30, None) == INVALID
    assert lib.gp_page_bounds_q8(_kv8(**bad), ps, None, 0, FAKE, None) == INVALID
    assert lib.gp_decode_attention_pages_q8(_kv8(**bad), ps, FAKE, 8, FAKE, 32, 0.1, FAKE, FAKE, 1 << 30, None) == INVALID


def test_decode_q8_refusals(lib):
    call = lambda kv=None, ps=None, q=FAKE, hq=32, scale=0.1, out=FAKE, ws=FAKE, n=1 << 30: lib.gp_decode_attention_q8(  # noqa: E731
        kv or _kv8(), ps or _ps(), q, hq, scale, out, ws, n, None)
    assert call(q=None) == call(out=None) == call(ws=None) == call(scale=0.0) == call(scale=float("inf")) == INVALID
    assert call(ps=_ps(pool=7)) == call(ps=_ps(table=None)) == INVALID
    assert call(hq=24) == call(kv=_kv8(d=96)) == call(ps=_ps(width=8193)) == UNSUPPORTED
    need = gp.gp_workspace_bytes(gp.GP_OP_DECODE, 4, 0, 32, 8, 128, 10, torch.bfloat16)
    assert call(n=need - 1) == WORKSPACE
    assert call(ps=_ps(R=0), ws=None, n=0) == 0


def test_page_bounds_refusals(lib):
    for fn, kv in ((lib.gp_page_bounds, _kv), (lib.gp_page_bounds_q8, _kv8)):
        assert fn(kv(), _ps(), None, -1, FAKE, None) == fn(kv(), _ps(), None, 0, None, None) == INVALID
        assert fn(None, _ps(), None, 0, FAKE, None) == fn(kv(), None, None, 0, FAKE, None) == INVALID
        assert fn(kv(), _ps(pool=99), None, 0, FAKE, None) == INVALID
        assert fn(kv(d=256), _ps(), None, 0, FAKE, None) == fn(kv(), _ps(width=8193), None, 0, FAKE, None) == UNSUPPORTED
        assert fn(kv(), _ps(R=0), None, 0, None, None) == 0


def test_select_refusals(lib):
    base = dict(bounds=FAKE, dtype=1, ps=None, q=FAKE, hq=32, hkv=8, d=128, budget=8, first=1, last=2, sel=FAKE, ws=FAKE,
                n=1 << 30)

    def call(**kw):
        a = dict(base, **kw)
        return lib.gp_select_pages(a["bounds"], a["dtype"], a["ps"] or _ps(), a["q"], a["hq"], a["hkv"], a["d"], a["budget"],
                                   a["first"], a["last"], a["sel"], a["ws"], a["n"], None)
    for bad in (dict(bounds=None), dict(q=None), dict(sel=None), dict(ws=None), dict(dtype=2), dict(budget=0),
                dict(budget=8193), dict(first=-1), dict(last=-1), dict(first=7), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
                dict(ps=_ps(pool=0)), dict(ps=_ps(R=-1))):
        assert call(**bad) == INVALID, bad
    assert call(hq=24) == call(d=96) == call(ps=_ps(width=8193)) == UNSUPPORTED
    need = gp.gp_workspace_bytes(gp.GP_OP_SELECT, 4, 0, 32, 8, 128, 10, torch.bfloat16)
    assert need >= 4 * 8 * 10 * 4
    assert call(n=need - 1) == WORKSPACE
    assert call(ps=_ps(R=0), bounds=None, q=None, sel=None, ws=None, n=0) == 0


def test_decode_pages_refusals(lib):
    for fn, kv in ((lib.gp_decode_attention_pages, _kv), (lib.gp_decode_attention_pages_q8, _kv8)):
        call = lambda sel=FAKE, budget=8, ps=None, n=1 << 30, hq=32: fn(kv(), ps or _ps(), sel, budget, FAKE, hq, 0.1, FAKE,  # noqa: E731
                                                                        FAKE, n, None)
        assert call(sel=None) == call(budget=0) == call(budget=-1) == call(budget=8193) == INVALID
        assert call(hq=24) == call(ps=_ps(width=8193)) == UNSUPPORTED
        need = gp.gp_workspace_bytes(gp.GP_OP_DECODE, 4, 0, 32, 8, 128, 8, torch.bfloat16)
        assert call(n=need - 1) == WORKSPACE
        assert call(ps=_ps(R=0), n=0) == 0


def test_binding_refusals():
    """The binding names the argument whose type or shape does not fit, without a device."""
    pool, hkv, d, R = 6, 2, 64, 3
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    ps = gp.PageState(i32(R, 4), i32(R), i32(R), i32(pool), i32(pool), i32(1))
    codes, scale = torch.zeros(pool, hkv, 16, d, dtype=torch.uint8), torch.ones(pool, hkv)
    kv8 = gp.KV8Layer(codes, codes.clone(), scale, scale.clone())
    kv = gp.KVLayer(torch.zeros(pool, hkv, 16, d), torch.zeros(pool, hkv, 16, d))
    new = torch.zeros(R, hkv, d, dtype=torch.bfloat16)
    q = torch.zeros(R, 2 * hkv, d, dtype=torch.bfloat16)
    pos = i32(R)
    for layer in (gp.KV8Layer(codes.float(), codes, scale, scale), gp.KV8Layer(codes, codes[:5], scale, scale),
                  gp.KV8Layer(codes, codes, scale.double(), scale), gp.KV8Layer(codes, codes, scale, scale[:5])):
        with pytest.raises(ValueError):
            layer.c()
    for k, v, more in ((new.float(), new, {}), (new, new[:2], {}), (new, new[:, :1], {}), (new[..., :32], new, {}),
                       (new, new, dict(q=q)), (new, new, dict(q=q, q_out=q.float())),
                       (new, new, dict(q=q[:2], q_out=q[:2])), (new, new, dict(tok_start=i32(R))),
                       (new, new, dict(tok_start=torch.zeros(R + 1, dtype=torch.int64))),
                       (new.transpose(1, 2).contiguous().transpose(1, 2), new, {})):
        with pytest.raises(ValueError):
            gp.gp_append_rope_q8(kv8, ps, pos, k, v, 1e4, **more)
    with pytest.raises(ValueError):
        gp.gp_append_rope(kv, ps, pos, new, new, 1e4)                      # bfloat16 rows, float32 pools
    with pytest.raises(ValueError):
        gp.gp_decode_attention_q8(kv8, ps, q.float(), 0.1, q, codes)
    with pytest.raises(ValueError):
        gp.gp_page_bounds(kv, ps, torch.zeros(pool, hkv, 2, d, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        gp.gp_page_bounds_q8(kv8, ps, torch.zeros(pool, hkv, 2, d, dtype=torch.bfloat16), from_tokens=i32(R + 1))
    bounds = torch.zeros(pool, hkv, 2, d, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        gp.gp_select_pages(bounds, ps, q.float(), 1, 1, i32(R, hkv, 4), codes)
    with pytest.raises(ValueError):
        gp.gp_select_pages(bounds, ps, q, 1, 1, i32(R, hkv + 1, 4), codes)
    with pytest.raises(ValueError):
        gp.gp_select_pages(bounds[:5], ps, q, 1, 1, i32(R, hkv, 4), codes)
    with pytest.raises(ValueError):
        gp.gp_decode_attention_pages_q8(kv8, ps, i32(R, hkv, 4).long(), q, 0.1, q, codes)
    # what fits otherwise, but lies in host memory
    for call in (lambda: gp.gp_append_rope_q8(kv8, ps, pos, new, new, 1e4), lambda: gp.gp_page_bounds_q8(kv8, ps, bounds),
                 lambda: gp.gp_decode_attention_q8(kv8, ps, q, 0.1, q, codes),
                 lambda: gp.gp_select_pages(bounds, ps, q, 1, 1, i32(R, hkv, 4), codes),
                 lambda: gp.gp_decode_attention_pages_q8(kv8, ps, i32(R, hkv, 4), q, 0.1, q, codes)):
        with pytest.raises(ValueError, match="device"):
            call()


def test_binding_refuses_short_queries_and_positions():
    """Arguments with fewer rows than the page state has requests, which a kernel would read past."""
    pool, hkv, d, R = 6, 2, 64, 3
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    ps = gp.PageState(i32(R, 4), i32(R), i32(R), i32(pool), i32(pool), i32(1))
    codes, scale = torch.zeros(pool, hkv, 16, d, dtype=torch.uint8), torch.ones(pool, hkv)
    kv8 = gp.KV8Layer(codes, codes.clone(), scale, scale.clone())
    kv = gp.KVLayer(torch.zeros(pool, hkv, 16, d), torch.zeros(pool, hkv, 16, d))
    new = torch.zeros(R, hkv, d, dtype=torch.bfloat16)
    for positions in (i32(R - 1), torch.zeros(R, dtype=torch.int64)):
        with pytest.raises(ValueError, match="positions"):
            gp.gp_append_rope_q8(kv8, ps, positions, new, new, 1e4)
        with pytest.raises(ValueError, match="positions"):
            gp.gp_append_rope(kv, ps, positions, new.float(), new.float(), 1e4)
    q, lists = torch.zeros(R, 2 * hkv, d, dtype=torch.bfloat16), i32(R, hkv, 4)
    for x, out in ((q[:2], q), (q, q[:2]), (q[:2], q[:2]), (q[..., :32], q[..., :32]), (q, q[:, :2]), (q[0], q[0])):
        with pytest.raises(ValueError, match="q_post and out"):
            gp.gp_decode_attention_q8(kv8, ps, x, 0.1, out, codes)
        with pytest.raises(ValueError, match="q_post and out"):
            gp.gp_decode_attention_pages_q8(kv8, ps, lists, x, 0.1, out, codes)
        with pytest.raises(ValueError, match="q_post and out"):
            gp.gp_decode_attention_pages(kv, ps, lists, x.float(), 0.1, out.float(), codes)


def test_q8_scale_limit(lib):
    """The 8-bit calls take softmax scales below 2^111 only; the others any."""
    for scale, want in ((2.0 ** 111, INVALID), (3.0e38, INVALID), (2.0 ** 110, WORKSPACE)):
        assert lib.gp_decode_attention_q8(_kv8(), _ps(), FAKE, 32, scale, FAKE, FAKE, 0, None) == want
        assert lib.gp_decode_attention_pages_q8(_kv8(), _ps(), FAKE, 8, FAKE, 32, scale, FAKE, FAKE, 0, None) == want
        assert lib.gp_decode_attention_pages(_kv(), _ps(), FAKE, 8, FAKE, 32, scale, FAKE, FAKE, 0, None) == WORKSPACE


class _NoLaunch:
    """The library's place: counts calls, launches nothing."""
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


def _device_calls():
    """Each call of the binding around the cache, with every tensor that its kernels reach, by name."""
    pool, hkv, d, R = 6, 2, 64, 3
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    state = lambda: gp.PageState(i32(R, 4), i32(R), i32(R), i32(pool), i32(pool), i32(1))  # noqa: E731
    layers = {"": lambda: gp.KVLayer(bf(pool, hkv, 16, d), bf(pool, hkv, 16, d)),
              "_q8": lambda: gp.KV8Layer(u8(pool, hkv, 16, d), u8(pool, hkv, 16, d), torch.ones(pool, hkv), torch.ones(pool, hkv))}
    of_state = lambda ps: dict(page_table=ps.page_table, num_pages=ps.num_pages, seq_lens=ps.seq_lens)  # noqa: E731
    for q8, layer in layers.items():
        kv, ps, t = layer(), state(), dict(positions=i32(R), k_new=bf(R, hkv, d), v_new=bf(R, hkv, d), q=bf(R, hkv, d),
                                           q_out=bf(R, hkv, d), tok_start=i32(R + 1))
        yield f"gp_append_rope{q8}", {**vars(kv), **of_state(ps), **t}, lambda fn, kv=kv, ps=ps, t=t: fn(
            kv, ps, t["positions"], t["k_new"], t["v_new"], 1e4, q=t["q"], q_out=t["q_out"], tok_start=t["tok_start"])
        kv, ps, t = layer(), state(), dict(bounds=bf(pool, hkv, 2, d), from_tokens=i32(R))
        yield f"gp_page_bounds{q8}", {**vars(kv), **of_state(ps), **t}, lambda fn, kv=kv, ps=ps, t=t: fn(
            kv, ps, t["bounds"], from_tokens=t["from_tokens"])
        kv, ps, t = layer(), state(), dict(selected=i32(R, hkv, 4), q=bf(R, hkv, d), out=bf(R, hkv, d), ws=u8(64))
        yield f"gp_decode_attention_pages{q8}", {**vars(kv), **of_state(ps), **t}, lambda fn, kv=kv, ps=ps, t=t: fn(
            kv, ps, t["selected"], t["q"], 0.1, t["out"], t["ws"])
    kv, ps, t = layers["_q8"](), state(), dict(q=bf(R, hkv, d), out=bf(R, hkv, d), ws=u8(64))
    yield "gp_decode_attention_q8", {**vars(kv), **of_state(ps), **t}, lambda fn, kv=kv, ps=ps, t=t: fn(
        kv, ps, t["q"], 0.1, t["out"], t["ws"])
    ps, t = state(), dict(bounds=bf(pool, hkv, 2, d), q=bf(R, hkv, d), selected=i32(R, hkv, 4), ws=u8(64))
    yield "gp_select_pages", {**of_state(ps), **t}, lambda fn, ps=ps, t=t: fn(
        t["bounds"], ps, t["q"], 1, 1, t["selected"], t["ws"])


def test_binding_checks_the_device_of_every_tensor(monkeypatch):
    """Host tensors that say they lie on device 0: the call goes through.  One of them at a time on the host or on
    another device, whichever it is: the call is refused and the library not reached."""
    lib = _NoLaunch()
    monkeypatch.setattr(_lib, "load", lambda: lib)
    monkeypatch.setattr(_lib, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    seen = 0
    for name, tensors, call in _device_calls():
        fn = getattr(gp, name)
        for t in tensors.values():
            t.get_device = lambda: 0
        lib.calls = 0
        call(fn)
        assert lib.calls == 1, name
        for what, t in tensors.items():
            for dev in (-1, 1):
                t.get_device = lambda dev=dev: dev
                with pytest.raises(ValueError, match="device"):
                    call(fn)
                assert lib.calls == 1, (name, what)
                seen += 1
            t.get_device = lambda: 0
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)      # all on a device that is not the current one
        with pytest.raises(ValueError, match="current device"):
            call(fn)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert seen == 2 * 77                                 # tensors of the eight calls


def test_decode_pages_refuses_pools_off_16_bytes(lib):
    """bfloat16 pools; float32 ones may lie at any multiple of 4."""
    call = lambda kv: lib.gp_decode_attention_pages(kv, _ps(), FAKE, 8, FAKE, 32, 0.1, FAKE, FAKE, 0, None)  # noqa: E731
    assert call(_kv(k=FAKE + 2)) == call(_kv(v=FAKE + 8)) == INVALID
    assert call(_kv()) == call(_kv(k=FAKE + 4, v=FAKE + 8, dtype=0)) == WORKSPACE
