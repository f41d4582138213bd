"""Refusals of the operators around the attention (rotary positions, rotated append, residual norm, 4-bit products):
every bad argument comes back as an error code before anything is launched, so these run without a GPU.  The
pointers are never dereferenced."""
import ctypes as C

import pytest

from paper_2405_10637_b200 import binding as lk

A = 0x100000          # a plausible, aligned address
FAR = 0x40000000      # and one far from it


def rope(cos=A, sin=FAR, rot_dim=128, interleaved=0, positions=64, size=None):
    return lk.Rope(C.sizeof(lk.Rope) if size is None else size, rot_dim, interleaved, positions, cos, sin)


def scaling(**kw):
    s = lk.make_rope_scaling()
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def tables(cos=A, sin=FAR, positions=64, rot_dim=128, s=None):
    s = s or scaling()
    return lk.lib().lckv_rope_tables(cos, sin, positions, rot_dim, C.addressof(s), None)


def test_rope_tables_refuses():
    bad = [dict(cos=None), dict(sin=None), dict(positions=0), dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=130),
           dict(cos=A + 2), dict(sin=A), dict(sin=A + 64 * 64 * 4 - 4),
           dict(s=scaling(kind=4)), dict(s=scaling(kind=-1)), dict(s=scaling(base=1.0)), dict(s=scaling(base=float("nan"))),
           dict(s=scaling(base=float("inf"))), dict(s=scaling(kind=1, factor=0.0)), dict(s=scaling(kind=2, factor=-1.0)),
           dict(s=scaling(kind=3, factor=2.0, original=0.0)), dict(s=scaling(kind=3, factor=2.0, original=8.0, low=4.0, high=4.0)),
           dict(s=scaling(kind=3, factor=2.0, original=8.0, low=-1.0)), dict(s=scaling(amplitude=float("inf"))),
           dict(s=scaling(struct_size=8))]
    for kw in bad:
        assert tables(**kw) == lk.EINVAL, kw
    assert lk.lib().lckv_rope_tables(A, FAR, 64, 128, None, None) == lk.EINVAL


def apply(r=None, pos=A, x=A, xt=4096, xh=128, y=FAR, yt=4096, yh=128, tokens=4, heads=32, d=128, dtype=0, tr=0):
    r = r or rope()
    return lk.lib().lckv_rope_apply(C.addressof(r), pos, x, xt, xh, y, yt, yh, tokens, heads, d, dtype, tr, None)


def test_rope_apply_refuses():
    bad = [dict(r=rope(size=4)), dict(r=rope(cos=None)), dict(r=rope(sin=None)), dict(r=rope(rot_dim=0)), dict(r=rope(rot_dim=5)),
           dict(r=rope(rot_dim=130)), dict(r=rope(positions=0)), dict(r=rope(interleaved=2)), dict(r=rope(cos=A + 2)),
           dict(pos=None), dict(x=None), dict(y=None), dict(tokens=0), dict(heads=0), dict(heads=65537), dict(d=96), dict(dtype=2),
           dict(tr=2), dict(x=A + 1), dict(y=FAR + 1), dict(pos=A + 2), dict(x=A + 2, dtype=1),
           dict(xt=-1), dict(xh=-1), dict(yt=0), dict(yh=0), dict(yh=64), dict(yt=4000),        # y would overlap itself
           dict(y=A + 2), dict(y=A, yt=8192), dict(y=A + 64 * 2), dict(y=A + 4096 * 2)]          # x and y share memory
    for kw in bad:
        assert apply(**kw) == lk.EINVAL, kw
    assert apply(r=rope(rot_dim=128), d=64) == lk.EINVAL
    assert lk.lib().lckv_rope_apply(None, A, A, 4096, 128, FAR, 4096, 128, 4, 32, 128, 0, 0, None) == lk.EINVAL


def test_rotated_append_refuses_a_null_cache():
    r = rope()
    f, g = lk.lib().lckv_rope_append_kv, lk.lib().lckv_rope_prefill_write_kv
    assert f(None, 0, C.addressof(r), A, 0, FAR, A, A, 0, 1, 1, 0, None) == lk.EINVAL
    assert g(None, 0, C.addressof(r), A, 0, FAR, A, A, 0, 1, 1, None) == lk.EINVAL


def norm(x=A, xs=0, xd=0, r=None, ro=None, rd=0, w=FAR, wd=0, y=4 * FAR, kind=0, scale=None, group=0, rows=4, width=64,
         eps=1e-6):
    return lk.lib().lckv_rms_norm(x, xs, xd, r, ro, rd, w, wd, y, kind, scale, group, rows, width, eps, None)


def test_rms_norm_refuses():
    R = 2 * FAR
    bad = [dict(x=None), dict(w=None), dict(y=None), dict(rows=0), dict(width=0), dict(width=32769), dict(xd=2), dict(rd=2),
           dict(wd=-1), dict(kind=3), dict(kind=-1), dict(kind=2), dict(scale=R), dict(kind=2, scale=R, group=64), dict(group=128),
           dict(ro=R), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(xs=63), dict(xs=-64),
           dict(x=A + 1), dict(x=A + 2, xd=1), dict(r=R + 1), dict(r=R, ro=R + 1), dict(w=FAR + 1), dict(y=4 * FAR + 1),
           dict(kind=2, scale=R + 2), dict(y=A + 2), dict(y=A, xs=128), dict(y=A, kind=1), dict(y=FAR), dict(r=R, ro=R + 2),
           dict(r=R, ro=A, rd=1), dict(r=R, ro=4 * FAR), dict(kind=2, scale=4 * FAR + 16)]
    for kw in bad:
        assert norm(**kw) == lk.EINVAL, kw


def linear(w=A, n=64, k=128, group=128, zeros=0, x=FAR, xs=0, xk=0, sc=None, sg=0, y=2 * FAR, ys=0, yd=0, rows=4, st=None):
    return lk.lib().lckv_quant_linear(w, n, k, group, zeros, x, xs, xk, sc, sg, y, ys, yd, rows, st, None)


def test_quant_refuses():
    S = 4 * FAR
    bad = [dict(w=None), dict(x=None), dict(y=None), dict(n=0), dict(k=0), dict(n=(1 << 24) + 1), dict(k=100), dict(group=16),
           dict(k=192), dict(group=256), dict(zeros=2), dict(rows=0), dict(rows=(1 << 19) + 1), dict(xk=2), dict(yd=2),
           dict(xk=1), dict(sc=S), dict(sg=128), dict(xk=1, sc=S, sg=64), dict(xs=120), dict(xs=132), dict(ys=63),
           dict(w=A + 128), dict(x=FAR + 8), dict(y=2 * FAR + 1), dict(y=2 * FAR + 2, yd=1), dict(xk=1, sc=S + 2),
           dict(y=FAR), dict(y=A + 64), dict(xk=1, sc=S, xs=136), dict(st=S + 2)]
    for kw in bad:
        assert linear(**kw) == lk.EINVAL, kw
    size = lk.lib().lckv_quant_bytes
    assert size(64, 128, 128, 0) == 128 * 128 // 2 + 128 * 2
    assert size(1, 32, 32, 1) == 128 * 128 // 2 + 128 * 4 * 3          # padded to 128 features and 128 columns
    for n, k, g, z in [(0, 128, 128, 0), (64, 0, 128, 0), (64, 96, 64, 0), (64, 128, 16, 0), (64, 128, 128, 2)]:
        assert size(n, k, g, z) == 0
    pack = lk.lib().lckv_quant_pack
    assert pack(None, FAR, None, 64, 128, 128, A, 1 << 20, None) == lk.EINVAL
    assert pack(FAR, None, None, 64, 128, 128, A, 1 << 20, None) == lk.EINVAL
    assert pack(FAR, 2 * FAR, None, 64, 128, 128, None, 1 << 20, None) == lk.EINVAL
    assert pack(FAR, 2 * FAR + 1, None, 64, 128, 128, A, 1 << 20, None) == lk.EINVAL
    assert pack(FAR, 2 * FAR, None, 64, 130, 128, A, 1 << 20, None) == lk.EINVAL
    assert pack(FAR, 2 * FAR, None, 64, 128, 128, A + 16, 1 << 20, None) == lk.ENOMEM
    assert pack(FAR, 2 * FAR, None, 64, 128, 128, A, 4096, None) == lk.ENOMEM
    assert pack(A, 2 * FAR, None, 64, 128, 128, A, 1 << 20, None) == lk.EINVAL


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    t = torch.zeros(4, 64)
    with pytest.raises(lk.LckvError) as e:
        lk.make_rope(t, t)
    assert e.value.status == lk.EINVAL
    with pytest.raises(lk.LckvError):
        lk.lckv_rms_norm(t, torch.ones(64), torch.zeros(4, 64))
    with pytest.raises(lk.LckvError):
        lk.lckv_quant_pack(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.bfloat16))


def test_rope_tables_refuses_frequencies_outside_fp64():
    assert tables(rot_dim=4, s=scaling(kind=2, factor=1e-300)) == lk.EINVAL         # the base becomes 0, a frequency infinite
    assert tables(s=scaling(kind=1, factor=1e-310)) == lk.EINVAL
    assert tables(s=scaling(amplitude=1e300)) == lk.EINVAL                          # infinite in fp32


def test_outputs_apart_from_what_is_read():
    cos, sin, pos, y = 16 * FAR, 20 * FAR, 24 * FAR, 2 * FAR
    r = rope(cos=cos, sin=sin)
    size = 64 * 64 * 4
    for bad in (cos, cos + size - 256, sin - 128, pos):
        assert apply(r=r, pos=pos, y=bad) == lk.EINVAL
    S = 4 * FAR
    assert linear(xk=1, sc=y + 64 * 2, y=y) == lk.EINVAL
    assert linear(xk=1, sc=S, st=y + 8, y=y) == lk.EINVAL
