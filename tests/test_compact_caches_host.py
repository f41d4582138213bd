"""Refusals and sizes of compact caches that need no GPU: bad arguments come back as error codes before anything is launched."""
import ctypes as C

import pytest

from paper_2405_10637_b200 import binding as lk

A = 0x100000          # a plausible, aligned address


def test_null_caches_and_arrays_are_refused():
    L = lk.lib()
    assert L.lckv_cache_read_kv(None, 0, A, A, 0, 4, 1, None) == lk.EINVAL
    assert L.lckv_attention_weights(None, 0, 0, A, A, None, A, 0, 1, None) == lk.EINVAL
    assert L.lckv_evict_kv(None, 0, None, 0, None, 0, None, 0, A, 0, 0, 4, 1, 0, None) == lk.EINVAL


@pytest.mark.parametrize("kw", [dict(kv_bits=8), dict(kv_bits=-4), dict(kv_bits=2), dict(kv_bits=4, kernel_kind=1)])
def test_configurations_that_do_not_exist(kw):
    cfg = lk.make_config(1, 0, 4, 4, 64, 2, 16, **kw)
    out = C.c_void_p()
    assert lk.lib().lckv_cache_bytes(C.byref(cfg)) == 0
    assert lk.lib().lckv_cache_alloc(C.byref(out), C.byref(cfg), A, 1 << 40) == lk.EINVAL


def test_a_caller_without_the_new_field_is_understood():
    """A configuration of the size that it had before kv_bits: the rest is not read."""
    cfg = lk.make_config(4, 1, 4, 4, 64, 2, 16, kv_bits=77)       # odd w: refused whatever else it says
    out = C.c_void_p()
    old = lk.Config.kv_bits.offset
    assert old == C.sizeof(lk.Config) - 4
    for size, w in ((old, 1), (old - 4, 2), (C.sizeof(lk.Config) + 4, 2), (0, 2)):
        cfg.struct_size, cfg.n_warmup = size, w
        assert lk.lib().lckv_cache_alloc(C.byref(out), C.byref(cfg), A, 1 << 40) == lk.EINVAL
    cfg.struct_size, cfg.n_warmup = old, 2                        # kv_bits = 77 lies behind its end: the buffer is the next to be refused
    assert lk.lib().lckv_cache_alloc(C.byref(out), C.byref(cfg), A + 1, 1 << 40) == lk.ENOMEM
