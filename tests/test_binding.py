"""What the binding hands to the library: page states without the parts that a call does not need."""
import ctypes
import gc
import weakref
import gc
import weakref

import pytest
import torch

import paper_2609_03494_amd as gp
from paper_2609_03494_amd import _lib
from test_cache_ops import _NoLaunch, lib  # noqa: F401


def _i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def _state(**none):
    a = dict(page_table=_i32(4, 10), num_pages=_i32(4), seq_lens=_i32(4), refcount=_i32(100), free_list=_i32(100), free_count=_i32(1))
    return gp.PageState(**{**a, **none})


def test_page_state_without_a_stack(monkeypatch):
    """The attention and append calls do not look at the free stack, so a state may come without one."""
    for none in (("free_list",), ("free_count",), ("free_list", "free_count")):
        ps = _state(**{k: None for k in none})
        c = ps.c()
        for key in ("page_table", "num_pages", "seq_lens", "refcount", "free_list", "free_count"):
            assert getattr(c, key) == (None if key in none else getattr(ps, key).data_ptr()), (none, key)
        assert (c.num_reqs, c.max_pages, c.pool_pages) == (4, 10, 100)
    with pytest.raises(ValueError, match="contiguous"):
        _state(free_list=_i32(200)[::2]).c()
    with pytest.raises(ValueError, match="contiguous"):
        _state(seq_lens=_i32(8)[::2]).c()
    # a call that needs none of it reaches the library, the calls on pages say what is missing
    fake, ps = _NoLaunch(), _state(free_list=None, free_count=None)
    monkeypatch.setattr(_lib, "load", lambda: fake)
    monkeypatch.setattr(_lib, "_stream", lambda stream: 0)
    kv = gp.KVLayer(torch.zeros(100, 2, 16, 64), torch.zeros(100, 2, 16, 64))
    gp.gp_decode_attention(kv, ps, torch.zeros(4, 4, 64), 0.1, torch.zeros(4, 4, 64), torch.zeros(64, dtype=torch.uint8))
    assert fake.calls == 1
    for call in (lambda: gp.gp_pages_release(ps, _i32(2)), lambda: gp.gp_pages_reserve(ps, _i32(4), _i32(4)),
                 lambda: gp.gp_pages_fork([kv], ps, _i32(2), _i32(2), _i32(2))):
        with pytest.raises(ValueError, match="free_list"):
            call()
    assert fake.calls == 1


def test_state_without_lengths_is_the_library_s_to_refuse(lib):  # noqa: F811
    for key in ("num_pages", "seq_lens"):
        c = _state(**{key: None}).c()
        assert getattr(c, key) is None
        assert lib.gp_pages_release(ctypes.byref(c), 0x1000, 1, None) == 1


def test_layers_hold_the_tensors_that_they_point_to():
    """A layer whose pool is replaced later: the handle keeps the one that it was made of."""
    pool = lambda dt=torch.float32: torch.zeros(6, 2, 16, 64).to(dt)  # noqa: E731
    layer, layer8 = gp.KVLayer(pool(), pool()), gp.KV8Layer(pool(torch.uint8), pool(torch.uint8), torch.ones(6, 2), torch.ones(6, 2))
    for x in (layer, layer8):
        handle = gp.Layers([x])
        old = {name: weakref.ref(t) for name, t in vars(x).items()}
        at = {name: t.data_ptr() for name, t in vars(x).items()}
        for name, t in list(vars(x).items()):
            setattr(x, name, torch.ones_like(t))
        gc.collect()
        for name, t in old.items():
            assert t() is not None and t().data_ptr() == getattr(handle._c[0], name) == at[name], name
