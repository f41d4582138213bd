"""The operators around the attention against plain forms in 64 bits: rotary tables, rotation, rotated append, residual
norm, products with 4-bit weights, and a run of them with the decode attention.

Tolerances, from the number formats: a rounding to bf16 is off by at most 2^-8 of the value, to e4m3 by 2^-4 (2^-10 of the
scale below the normal range), an fp32 operation by 2^-24 of its result; each check says how many it counts."""
import math

import numpy as np
import pytest
import torch

from paper_2405_10637_b200 import binding as lk

from helpers import Case, NAN_BITS, compare
from paper_2405_10637_b200 import inputs as syn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def within(got, want, tol, what=""):
    """Finite, and |got - want| <= tol, in 64 bits."""
    got = got.double()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = ((got - want).abs() - tol).max().item() if got.numel() else 0.0
    assert over <= 0, f"{what}: {over:.3e} over the tolerance"


# ---- rotary positions ---------------------------------------------------------------------------------------------------


def thetas(rot, kind, base, factor, original, low, high):
    out = []
    for j in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if kind == 2 and rot > 2 else base
        th = b ** (-2.0 * j / rot)
        if kind == 1:
            th /= factor
        if kind == 3:
            g = min(1.0, max(0.0, (original * th / (2 * math.pi) - low) / (high - low)))
            th = th * g + th / factor * (1 - g)
        out.append(th)
    return torch.tensor(out, dtype=torch.float64)


def tables64(rot, positions):
    ang = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * thetas(rot, 0, 1e4, 1, 1, 1, 2).to(DEV)
    return torch.cos(ang), torch.sin(ang)


def rotate64(x, cos, sin, rot, interleaved, sign=1.0):
    """x [..., heads, d], cos / sin [..., rot / 2] -> rotated, and the bound's magnitude |x0 c| + |x1 s|, in 64 bits."""
    x = x.double()
    c, s = cos.double()[..., None, :], sign * sin.double()[..., None, :]
    y, mag = x.clone(), torch.zeros_like(x)
    i0 = torch.arange(rot // 2, device=x.device)
    i0, i1 = (2 * i0, 2 * i0 + 1) if interleaved else (i0, i0 + rot // 2)
    a, b = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = a * c - b * s, b * c + a * s
    mag[..., i0], mag[..., i1] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, mag


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
@pytest.mark.parametrize("positions,rot", [(1, 2), (7, 6), (1000, 64), (131072, 128), (333, 128)])
def test_rope_tables(positions, rot, kind):
    base, factor, original, low, high, amp = 500000.0, 8.0, 8192.0, 1.0, 4.0, 1.2079
    cos, sin = (torch.full((positions, rot // 2), float("nan"), device=DEV) for _ in range(2))
    lk.lckv_rope_tables(cos, sin, lk.make_rope_scaling(kind, base, factor, original, low, high, amp))
    ang = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * thetas(rot, kind, base, factor, original, low, high).to(DEV)
    # the reduced angle in half turns, at most 1, is rounded once (2^-24 half turns = pi 2^-24 off), the function (2 ulp of
    # at most 1: 2^-22) and the product (2^-24) follow; the 64-bit angles of both sides differ by 1e5 * 2^-51
    tol = amp * (math.pi * E + 4 * E + E) + 2e-10
    within(cos, amp * torch.cos(ang), tol)
    within(sin, amp * torch.sin(ang), tol)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (128, 16), (128, 50), (64, 64), (64, 32), (64, 2), (64, 62)])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (1, 32), (3, 5), (130, 8), (2100, 33)])
def test_rope_apply(tokens, heads, d, rot, interleaved, dtype):
    g = gen(tokens * 131 + heads + rot)
    positions = 77
    cos, sin = (t.float() for t in tables64(rot, positions))
    rope = lk.make_rope(cos, sin, interleaved)
    x = randn(g, tokens, heads, d, dtype=dtype)
    pos = torch.randint(0, positions, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    pos[0], pos[-1] = 0, positions - 1
    for transpose in (False, True):
        y = lk.lckv_rope_apply(rope, pos, x, torch.full_like(x, float("nan")), transpose=transpose)
        want, mag = rotate64(x, cos[pos.long()], sin[pos.long()], rot, interleaved, -1.0 if transpose else 1.0)
        # two products and a sum in fp32, then the output's rounding (which sees a value off by those)
        within(y, want, 3 * E * mag * (1 + HALF[dtype]) + HALF[dtype] * want.abs())
        assert torch.equal(y[..., rot:], x[..., rot:])
    z = x.clone()
    assert lk.lckv_rope_apply(rope, pos, z, z) is z
    assert torch.equal(z, lk.lckv_rope_apply(rope, pos, x)), "in place differs"


@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_apply_strides(shift, interleaved):
    """Views of a fused projection, heads outside tokens, odd offsets; what lies between stays as it was."""
    g = gen(5)
    T, H, d = 19, 6, 64
    cos, sin = (t.float() for t in tables64(d, 40))
    rope = lk.make_rope(cos, sin, interleaved)
    pos = torch.randint(0, 40, (T,), generator=g, device=DEV, dtype=torch.int32)
    flat = randn(g, T * 3 * H * d + 64)
    x = flat[shift:shift + T * 3 * H * d].view(T, 3 * H, d)[:, H:2 * H]
    want = lk.lckv_rope_apply(rope, pos, x.contiguous())
    buf = torch.full((T * 2 * H * d + 64,), 7.0, dtype=torch.bfloat16, device=DEV)
    out = buf[shift:shift + T * 2 * H * d].view(T, 2 * H, d)[:, :H]
    lk.lckv_rope_apply(rope, pos, x, out)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((buf == 7.0).all()), "wrote outside the output"
    across = torch.empty(H, T, d, dtype=torch.bfloat16, device=DEV).transpose(0, 1)      # heads outside tokens
    assert torch.equal(lk.lckv_rope_apply(rope, pos, x, across), want)
    one = randn(g, 1, H, d).expand(T, H, d)                                               # one token, rotated T ways
    assert torch.equal(lk.lckv_rope_apply(rope, pos, one), lk.lckv_rope_apply(rope, pos, one.contiguous()))
    both = randn(g, T, 2 * H, d)                                                          # other heads of the same tokens
    want = lk.lckv_rope_apply(rope, pos, both[:, :H].contiguous())
    lk.lckv_rope_apply(rope, pos, both[:, :H], both[:, H:])
    assert torch.equal(both[:, H:], want)


def test_rope_transpose_is_the_gradient():
    """Against differences of the scalar sum(rotation(x) * u) in fp32, whose rotation is linear in x."""
    g = gen(9)
    cos, sin = (t.float() for t in tables64(64, 9))
    rope = lk.make_rope(cos, sin)
    pos = torch.tensor([3, 8], dtype=torch.int32, device=DEV)
    x, u = randn(g, 2, 3, 64, dtype=torch.float32), randn(g, 2, 3, 64, dtype=torch.float32)
    grad = lk.lckv_rope_apply(rope, pos, u, transpose=True)
    for idx in [(0, 0, 0), (1, 2, 5), (0, 1, 40), (1, 0, 63)]:
        up, down = x.clone(), x.clone()
        up[idx] += 1.0
        down[idx] -= 1.0
        diff = ((lk.lckv_rope_apply(rope, pos, up).double() - lk.lckv_rope_apply(rope, pos, down).double()) * u.double()).sum() / 2
        # 2 values of size <= 8 change, each with 3 fp32 operations a side, times |u| <= 5; the gradient itself has 3
        assert abs(diff.item() - grad[idx].item()) <= 2 * 2 * 4 * 8 * E * 5 + 3 * E * 10
    back = lk.lckv_rope_apply(rope, pos, lk.lckv_rope_apply(rope, pos, x), transpose=True)
    within(back, x.double(), 16 * E * 8)       # c^2 + s^2 = 1 up to the tables' rounding; |x| <= 5 and its partner


# ---- rotated append -----------------------------------------------------------------------------------------------------


def fused(g, B, n, hq, hkv, d):
    t = randn(g, B, n, hq + 2 * hkv, d)
    return t[:, :, :hq], t[:, :, hq:hq + hkv], t[:, :, hq + hkv:]


def expect_rows(c, slot, k64, mag, v, lens, n, prompt):
    """Writes the new rows into the host caches (rounded like the kernel within a unit: taken from the GPU after the check)
    and compares every byte of the slot."""
    kt, vt = c.cache.slot_tensors(slot)
    torch.cuda.synchronize()
    before_k, before_v = c.hK[slot].copy(), c.hV[slot].copy()
    for b in range(c.B):
        gk, gv = ((c._gather(kt, b), c._gather(vt, b)) if c.page_rows else (syn.bits(kt[b]), syn.bits(vt[b])))
        count = int(lens[b]) if prompt else n
        new = []
        for i in range(count):
            p = i if prompt else int(lens[b]) + i
            row = p
            if c.stream_sink and p >= c.T_cap:
                row = c.stream_sink + (p - c.stream_sink) % (c.T_cap - c.stream_sink)
            new.append(row)
            got = syn.from_bits(gk[:, row]).double()
            w, m = k64[b, i].cpu(), mag[b, i].cpu()
            within(got, w, 3 * E * m * (1 + 2.0 ** -8) + 2.0 ** -8 * w.abs(), f"key seq {b} token {i}")
            assert np.array_equal(gv[:, row], syn.bits(v[b, i])), f"value seq {b} token {i}"
            c.hK[slot][b][:, row], c.hV[slot][b][:, row] = gk[:, row], gv[:, row]
        n_rows = min(gk.shape[1], c.T_cap)
        keep = np.ones(n_rows, bool)
        keep[[r for r in new if r < n_rows]] = False
        if c.page_rows:
            keep[max([int(lens[b])] + [r + 1 for r in new]):] = False       # rows of owned pages that were never defined
        assert np.array_equal(gk[:, :n_rows][:, keep], before_k[b][:, :n_rows][:, keep]), f"seq {b}: other keys changed"
        assert np.array_equal(gv[:, :n_rows][:, keep], before_v[b][:, :n_rows][:, keep]), f"seq {b}: other values changed"


LAYOUTS = {"contiguous": {}, "paged": dict(page_rows=64, n_pages=40), "ring": dict(stream_sink=4)}


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("n,is_fused,interleaved,rot", [(1, True, False, None), (1, False, True, 32), (3, True, True, None), (9, False, False, 24), (70, True, False, None)])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (8, 2, 128)])
def test_rotated_append(Hq, Hkv, d, n, is_fused, interleaved, rot, layout):
    lens = [0, 61, 64, 5, 127]
    T_cap = 200
    if layout == "ring":
        T_cap, lens = 90, [0, 61, 89, 90, 500]
    c = Case(L=2, w=0, Hq=Hq, Hkv=Hkv, d=d, lens=lens, T_cap=T_cap, seed=3, B_max=6, **LAYOUTS[layout])
    rot = rot or d
    g = gen(n + d)
    cos, sin = (t.float() for t in tables64(rot, 600))
    rope = lk.make_rope(cos, sin, interleaved)
    B = c.B
    q, k, v = fused(g, B, n, Hq, Hkv, d) if is_fused else (randn(g, B, n, h, d) for h in (Hq, Hkv, Hkv))
    pos = torch.tensor(lens, device=DEV)[:, None] + torch.arange(n, device=DEV)
    want_q, mag_q = rotate64(q, cos[pos], sin[pos], rot, interleaved)
    want_k, mag_k = rotate64(k, cos[pos], sin[pos], rot, interleaved)
    out = c.cache.lckv_rope_append_kv(0, rope, q, k, v, advance_len=1)
    assert c.cache.lckv_cache_status() == 0
    within(out, want_q, 3 * E * mag_q * (1 + 2.0 ** -8) + 2.0 ** -8 * want_q.abs(), "q")
    expect_rows(c, 0, want_k, mag_k, v, lens, n, False)
    c.lens += n
    assert c.cache.lckv_cache_lengths(B) == c.lens.tolist()
    # a condensed layer has a query only: the same rotation, at the lengths as they are now, and no row is touched
    pos = torch.tensor(c.lens.tolist(), device=DEV)[:, None] + torch.arange(n, device=DEV)
    if int(pos.max()) < 600 and (layout == "ring" or int(pos.max()) < T_cap):
        kt = c.cache.slot_tensors(0)[0].clone()
        want_q, mag_q = rotate64(q, cos[pos], sin[pos], rot, interleaved)
        out = c.cache.lckv_rope_append_kv(0, rope, q, None, None)
        within(out, want_q, 3 * E * mag_q * (1 + 2.0 ** -8) + 2.0 ** -8 * want_q.abs(), "q alone")
        assert torch.equal(c.cache.slot_tensors(0)[0].view(torch.int16), kt.view(torch.int16))
    # and the attention reads what was stored
    qq = syn.randn_bf16((B, Hq, d), 5)
    got = c.cache.lckv_decode_attention(0, lk.MODE_CONDENSED, qq.to(DEV))
    from oracle import lckv_oracle as orc
    want, _ = orc.decode_attention(syn.bits(qq), c.hK[0], c.hV[0], c.lens, 0, c.scale, n_sink=c.stream_sink)
    compare(got, want, "attention over appended rows")
    c.close()


@pytest.mark.parametrize("page_rows", [0, 64])
@pytest.mark.parametrize("is_fused,interleaved,rot", [(True, False, 128), (False, True, 64), (False, False, 6)])
def test_rotated_prompt(is_fused, interleaved, rot, page_rows):
    lens, n_max, Hq, Hkv, d = [0, 1, 64, 130, 37], 133, 6, 3, 128
    c = Case(L=2, w=0, Hq=Hq, Hkv=Hkv, d=d, lens=lens, T_cap=140, seed=8, poison=False, page_rows=page_rows,
             n_pages=20 if page_rows else 0)
    g = gen(1)
    cos, sin = (t.float() for t in tables64(rot, 130))
    rope = lk.make_rope(cos, sin, interleaved)
    q, k, v = fused(g, c.B, n_max, Hq, Hkv, d) if is_fused else (randn(g, c.B, n_max, h, d) for h in (Hq, Hkv, Hkv))
    pos = torch.arange(n_max, device=DEV).clamp(max=129).expand(c.B, n_max)
    want_q, mag_q = rotate64(q, cos[pos], sin[pos], rot, interleaved)
    want_k, mag_k = rotate64(k, cos[pos], sin[pos], rot, interleaved)
    out = torch.full((c.B, n_max, Hq, d), 3.0, dtype=torch.bfloat16, device=DEV)
    c.cache.lckv_rope_prefill_write_kv(0, rope, q, k, v, out)
    for b, n in enumerate(lens):
        within(out[b, :n], want_q[b, :n], 3 * E * mag_q[b, :n] * (1 + 2.0 ** -8) + 2.0 ** -8 * want_q[b, :n].abs(), "q")
        assert bool((out[b, n:] == 3.0).all()), "rows behind a prompt were written"
    expect_rows(c, 0, want_k, mag_k, v, lens, n_max, True)
    assert c.cache.lckv_cache_lengths(c.B) == lens
    c.close()


def refused(status, f, *a, **kw):
    with pytest.raises(lk.LckvError) as e:
        f(*a, **kw)
    assert e.value.status == status, e.value


def test_rotated_append_refuses():
    c = Case(L=2, w=0, Hq=4, Hkv=2, d=64, lens=[3, 60], T_cap=64, seed=2, page_rows=64, n_pages=2)
    f = c.cache.lckv_rope_append_kv
    g = gen(3)
    rope = lk.make_rope(*(t.float() for t in tables64(64, 128)))
    q, k, v = (randn(g, 2, 1, h, 64) for h in (4, 2, 2))
    before = [t.clone() for t in c.cache.slot_tensors(0)]
    refused(lk.EINVAL, f, 2, rope, q, k, v)                                   # no such slot
    refused(lk.EINVAL, f, 0, rope, None, k, None)                             # a key without its value
    refused(lk.EINVAL, f, 0, rope, q, None, None, advance_len=1)
    refused(lk.EINVAL, f, 0, rope, q.float(), k, v)
    refused(lk.EINVAL, f, 0, rope, q[:, :, :3], k, v)
    refused(lk.EINVAL, f, 0, rope, q.cpu(), k, v)
    refused(lk.EINVAL, f, 0, rope, q, k[:1].expand(2, 1, 2, 64), v)           # tokens that share memory
    refused(lk.EINVAL, f, 0, lk.make_rope(*(t.float() for t in tables64(64, 60))), q, k, v)    # position 60 is not there
    refused(lk.EINVAL, f, 0, lk.make_rope(*(t.float() for t in tables64(128, 128))), q, k, v)  # wider than a head
    five = [randn(g, 2, 5, h, 64) for h in (4, 2, 2)]
    refused(lk.ECAPACITY, f, 0, rope, *five)                                  # 60 + 5 > 64
    t = randn(g, 2, 1, 8, 64)
    refused(lk.EINVAL, f, 0, rope, t[:, :, :4], t[:, :, 4:6], t[:, :, 6:], q_out=t.view(-1)[:2 * 4 * 64].view(2, 1, 4, 64))
    refused(lk.EINVAL, f, 0, rope, q, k, v, stream=None, q_out=torch.empty(2, 1, 4, 64, device=DEV))
    p = c.cache.lckv_rope_prefill_write_kv
    refused(lk.EINVAL, p, 0, rope, *(randn(g, 2, 59, h, 64) for h in (4, 2, 2)))     # a prompt of 60 in 59 tokens
    assert c.cache.lckv_cache_lengths(2) == [3, 60]
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, c.cache.slot_tensors(0)))
    c.close()
    c = Case(L=2, w=0, Hq=2, Hkv=2, d=64, lens=[3, 5], T_cap=16, seed=2, stream_sink=4)
    rope = lk.make_rope(*(t.float() for t in tables64(64, 64)))
    refused(lk.EINVAL, c.cache.lckv_rope_append_kv, 0, rope, *(randn(g, 2, 13, 2, 64) for _ in range(3)))
    refused(lk.EINVAL, c.cache.lckv_rope_prefill_write_kv, 0, rope, *(randn(g, 2, 8, 2, 64) for _ in range(3)))
    c.close()


def test_rotated_append_captured():
    """A captured call replays at the lengths on the device; growth and advance inside a capture are refused; a replay that
    finds no room writes nothing and says so."""
    c = Case(L=2, w=0, Hq=2, Hkv=2, d=64, lens=[3, 62], T_cap=130, seed=2, page_rows=64, n_pages=5)
    rope = lk.make_rope(*(t.float() for t in tables64(64, 256)))
    g = gen(4)
    q, k, v = (randn(g, 2, 2, 64) for _ in range(3))
    out = torch.empty_like(q)
    f = c.cache.lckv_rope_append_kv
    f(0, rope, q, k, v, out)                     # pages for the next row are there
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        f(0, rope, q, k, v, out)
        refused(lk.EINVAL, f, 0, rope, q, k, v, out, advance_len=1)
        refused(lk.EINVAL, f, 0, rope, *(randn_like_n(t, 3) for t in (q, k, v)))      # 62 + 3 needs a page
    for step in range(4):                        # lengths 62 .. 65: the last two need the second page
        q.copy_(randn(g, 2, 2, 64)); k.copy_(randn(g, 2, 2, 64)); v.copy_(randn(g, 2, 2, 64))
        out.zero_()
        if step == 2:
            # an eager call makes the page (and would be followed by replays for the other slots)
            f(0, rope, q, k, v, torch.empty_like(q))
        graph.replay()
        got = out.clone()
        want = f(0, rope, q, k, v)               # eager, the same token again
        assert torch.equal(got, want)
        kt, _ = c.cache.slot_tensors(0)
        row = torch.stack([syn.from_bits(c._gather(kt, b)[:, int(c.lens[b])]) for b in range(2)]).to(DEV)
        kk, mag = rotate64(k, rope.tables[0][torch.tensor(c.lens.tolist(), device=DEV)], rope.tables[1][torch.tensor(c.lens.tolist(), device=DEV)], 64, False)
        within(row, kk, 3 * E * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * kk.abs())
        f(0, rope, q, k, v, out, advance_len=1)
        c.lens += 1
        assert c.cache.lckv_cache_status() == 0
    assert c.cache.lckv_cache_lengths(2) == c.lens.tolist()
    # no eager call makes room: sequence 1 grows to the end of its pages on the host's side only
    c.cache.lckv_cache_reset([3, 64])
    graph.replay()                               # row 64 of sequence 1 has no page
    assert c.cache.lckv_cache_status() == lk.ECAPACITY
    c.cache.lckv_cache_reset([3, 62])
    assert c.cache.lckv_cache_status() == 0
    c.close()


def randn_like_n(t, n):
    return torch.zeros(t.shape[0], n, *t.shape[1:], dtype=t.dtype, device=t.device)


# ---- residual and norm --------------------------------------------------------------------------------------------------


def norm64(x, r, w, eps):
    h = x.double() + (r.double() if r is not None else 0.0)
    return h, h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.double()


# fp32 errors of the norm relative to y: at most 128 additions on a path of the sum (32768 columns over 256 threads) and 10
# in the reductions, each 2^-24 of a sum of squares whose root halves it; the square, division, root and two products
NORM = (138 / 2 + 8) * E


def check_norm(y, scale, y64, group):
    """An output of lckv_rms_norm against y64."""
    if scale is None:
        within(y, y64, y64.abs() * (NORM * 1.01 + HALF[y.dtype]) + 1e-38)
        return
    rows, width = y64.shape
    step = group or width
    s = scale.double().view(rows, -1)
    for b in range(s.shape[1]):
        blk = y64[:, b * step:(b + 1) * step]
        top = blk.abs().max(1).values / 448.0
        within(s[:, b], top, top * (NORM + 2 * E) + 1e-45)
        got = y[:, b * step:(b + 1) * step].float().double() * s[:, b:b + 1]
        # one rounding to e4m3 of a quotient that carries the errors above; below 2^-6 the steps are 2^-9 of the scale
        within(got, blk, blk.abs() * (2.0 ** -4 + 2 * NORM) * (1 + 2.0 ** -10) + 2.0 ** -10 * top[:, None] * 1.001)


WIDTHS = [1, 7, 8, 64, 100, 128, 250, 256, 1000, 1024, 2048, 2056, 4095, 4096, 8192, 9000, 16384, 20000, 32768]


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3row", "e4m3block"])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm(width, out):
    g = gen(width)
    for rows, x32, r32, w32, res in [(1, False, False, False, True), (5, True, True, True, True), (33, False, True, False, True), (4, False, False, True, False)]:
        x = randn(g, rows, width, dtype=torch.float32 if x32 else torch.bfloat16)
        r = randn(g, rows, width, dtype=torch.float32 if r32 else torch.bfloat16, std=3.0) if res else None
        w = 1 + randn(g, width, dtype=torch.float32, std=0.2)
        w = w if w32 else w.to(torch.bfloat16)
        eps = 1e-5
        group = 128 if out == "e4m3block" else 0
        dt = {"bf16": torch.bfloat16, "fp32": torch.float32}.get(out, torch.float8_e4m3fn)
        y = torch.empty(rows, width, dtype=dt, device=DEV)
        scale = torch.full((rows, -(-width // 128) if group else 1), float("nan"), device=DEV) if dt == torch.float8_e4m3fn else None
        h = torch.empty_like(r) if res else None
        lk.lckv_rms_norm(x, w, y, residual=r, residual_out=h, out_scale=scale, scale_group=group, eps=eps)
        h64, y64 = norm64(x, r, w, eps)
        check_norm(y, scale, y64, group)
        if res:
            within(h, h64, h64.abs() * (HALF[h.dtype] + E) * (1 + E))      # the sum in fp32, then its type
            # in place gives the same bits
            r2, y2 = r.clone(), torch.empty_like(y)
            lk.lckv_rms_norm(x, w, y2, residual=r2, residual_out=r2, out_scale=scale, scale_group=group, eps=eps)
            assert torch.equal(r2, h) and torch.equal(y2.view(torch.uint8), y.view(torch.uint8))
        if dt == x.dtype and not res:
            x2 = x.clone()
            lk.lckv_rms_norm(x2, w, x2, eps=eps)
            assert torch.equal(x2, y)


@pytest.mark.parametrize("width,pad,shift", [(256, 8, 0), (256, 3, 1), (77, 5, 1), (4096, 4096, 8)])
def test_norm_strides(width, pad, shift):
    g = gen(2)
    flat = randn(g, 9 * (width + pad) + 16)
    x = flat[shift:shift + 9 * (width + pad)].view(9, width + pad)[:, :width]
    w = torch.ones(width, dtype=torch.bfloat16, device=DEV)
    y = lk.lckv_rms_norm(x, w, torch.empty(9, width, dtype=torch.bfloat16, device=DEV))
    assert torch.equal(y, lk.lckv_rms_norm(x.contiguous(), w, torch.empty_like(y))) or width % 8
    check_norm(y, None, norm64(x, None, w, 1e-6)[1], 0)


@pytest.mark.parametrize("width", [96, 1024, 1030])
def test_norm_special_values(width):
    """Rows of zeros, of the largest and smallest values, an infinity and a NaN among others; eps 0."""
    g = gen(6)
    x = randn(g, 8, width, dtype=torch.float32)
    x[1] = 0
    x[2] *= 1e18                      # squares up to 1e37 and sums up to 1e38 stay finite
    x[3] *= 1e-30                     # eps dominates: y is x / sqrt(eps)
    x[4, 5] = float("inf")
    x[5, 7] = float("nan")
    x[6, 128 % width:] = 0            # blocks of zeros beside others
    w = torch.ones(width, device=DEV)
    for group in (0, 128):
        y = torch.empty(8, width, dtype=torch.float8_e4m3fn, device=DEV)
        s = torch.empty(8, -(-width // 128) if group else 1, device=DEV)
        lk.lckv_rms_norm(x, w, y, out_scale=s, scale_group=group, eps=1e-6)
        ok = [0, 1, 2, 3, 6, 7]
        y64 = norm64(x, None, w, 1e-6)[1]
        check_norm(y[ok], s[ok], y64[ok], group)
        assert bool((y[1].float() == 0).all()) and bool((s[1] == 0).all())
        assert bool(torch.isnan(y[5].float()).all()) and bool(torch.isnan(s[5]).all())
        assert bool(torch.isnan(s[4, 0])) and bool(torch.isnan(y[4, 5].float()))
    y = lk.lckv_rms_norm(x, w, torch.empty_like(x), eps=1e-6)
    check_norm(y[ok], None, norm64(x, None, w, 1e-6)[1][ok], 0)
    assert bool(torch.isnan(y[4, 5])) and bool((y[4, :5] == 0).all()) and bool(torch.isnan(y[5]).all())
    y = lk.lckv_rms_norm(x[:1], w, torch.empty_like(x[:1]), eps=0.0)
    check_norm(y, None, norm64(x[:1], None, w, 0.0)[1], 0)
    # outputs so small that the scale's inverse is out of range
    tiny = torch.full((1, width), 2.0 ** -140, device=DEV)
    y, s = torch.empty(1, width, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(1, device=DEV)
    lk.lckv_rms_norm(tiny, w, y, out_scale=s, eps=1.0)
    assert s.item() > 0 and bool(((y.float() - 448.0).abs() <= 32).all())        # s is a subnormal: 2^-149 of 2^-148.8 off


def test_norm_refuses():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV), torch.ones(64, device=DEV)
    y = torch.empty_like(x)
    f = lk.lckv_rms_norm
    refused(lk.EINVAL, f, x.half(), w, y)
    refused(lk.EINVAL, f, x, w[:63], y)
    refused(lk.EINVAL, f, x, w, y[:3])
    refused(lk.EINVAL, f, x, w, y.cpu())
    refused(lk.EINVAL, f, x[:1].expand(4, 64), w, y)
    refused(lk.EINVAL, f, x, w, y, residual_out=torch.empty_like(x))
    refused(lk.EINVAL, f, x, w, y, residual=x.t().contiguous().t())
    refused(lk.EINVAL, f, x, w, y.to(torch.float8_e4m3fn))
    refused(lk.EINVAL, f, x, w, y.to(torch.float8_e4m3fn), out_scale=torch.empty(5, device=DEV))
    refused(lk.EINVAL, f, x, w, y, out_scale=torch.empty(4, device=DEV))
    refused(lk.EINVAL, f, torch.zeros(1, 32769, device=DEV), torch.ones(32769, device=DEV), torch.empty(1, 32769, device=DEV))


# ---- products with 4-bit weights ----------------------------------------------------------------------------------------


def make_weight(g, n, k, group, has_zeros):
    codes = torch.randint(0, 16, (n, k), generator=g, device=DEV, dtype=torch.uint8)
    packed = codes[:, 0::2] | (codes[:, 1::2] << 4)
    scales = ((torch.rand((n, k // group), generator=g, device=DEV) + 0.1) * 0.02).to(torch.bfloat16)
    zeros = torch.randint(0, 16, (n, k // group), generator=g, device=DEV, dtype=torch.uint8) if has_zeros else None
    z = zeros.double().repeat_interleave(group, 1) if has_zeros else 8.0
    w64 = (codes.double() - z) * scales.double().repeat_interleave(group, 1)
    return lk.lckv_quant_pack(packed, scales, zeros), w64


def make_x(g, rows, k, kind):
    """-> x, x_scale, x in 64 bits."""
    if kind == "bf16":
        x = randn(g, rows, k)
        return x, None, x.double()
    x = (torch.randn((rows, k), generator=g, device=DEV) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    blocks = 1 if kind == "row" else -(-k // 128)
    s = torch.rand((rows, blocks), generator=g, device=DEV) * 0.01 + 1e-3
    wide = s.double() if kind == "row" else s.double().repeat_interleave(128, 1)[:, :k]
    return x, s, x.float().double() * wide


def check_linear(y, x64, w64, k):
    want = x64 @ w64.t()
    mag = x64.abs() @ w64.abs().t()
    # products of a code and x are exact; an accumulation on the tensor cores is off by at most 2^-23 (it may truncate) of the
    # partial sums' magnitude: k / 16 of them and 16 inside each, then the scalings and the additions of partial sums
    tol = mag * 2.0 ** -23 * (k / 16 + 16 + 4 + 64)
    within(y, want, tol * (1 + HALF[y.dtype]) + HALF[y.dtype] * want.abs())


SHAPES = [(1, 32, 32), (16, 64, 32), (64, 128, 128), (63, 96, 32), (65, 160, 32), (100, 192, 64), (300, 1024, 128), (520, 2048, 64),
          (129, 4096, 32), (1000, 1152, 128), (64, 8192, 128)]


@pytest.mark.parametrize("kind", ["bf16", "row", "block"])
@pytest.mark.parametrize("has_zeros", [False, True])
@pytest.mark.parametrize("n,k,group", SHAPES)
def test_quant_linear(n, k, group, has_zeros, kind):
    g = gen(n + k + group)
    w, w64 = make_weight(g, n, k, group, has_zeros)
    for rows, dt in [(1, torch.bfloat16), (2, torch.float32), (8, torch.bfloat16), (9, torch.float32), (16, torch.float32), (17, torch.bfloat16),
                     (33, torch.float32), (64, torch.float32), (100, torch.bfloat16), (129, torch.float32), (300, torch.float32)]:
        x, s, x64 = make_x(g, rows, k, kind)
        y = lk.lckv_quant_linear(w, x, torch.full((rows, n), float("nan"), dtype=dt, device=DEV), x_scale=s)
        check_linear(y, x64, w64, k)
        again = lk.lckv_quant_linear(w, x, torch.empty_like(y), x_scale=s)
        assert torch.equal(y, again), "not repeatable"


@pytest.mark.parametrize("rows", [1, 8, 13, 40, 200])
def test_quant_linear_strides(rows):
    """Rows of x inside wider rows, y as a part of a fused output; what lies beside y stays as it was."""
    g = gen(11)
    n, k = 70, 256
    w, w64 = make_weight(g, n, k, 64, True)
    x = randn(g, rows, 2 * k + 8)[:, k:2 * k]
    buf = torch.full((rows, 3 * n + 1), 7.0, device=DEV)
    y = buf[:, n:2 * n]
    lk.lckv_quant_linear(w, x, y)
    check_linear(y, x.double(), w64, k)
    assert torch.equal(y, lk.lckv_quant_linear(w, x.contiguous(), torch.empty(rows, n, device=DEV)))
    y.fill_(7.0)
    assert bool((buf == 7.0).all()), "wrote outside the output"


@pytest.mark.parametrize("rows", [3, 16, 50, 140])
@pytest.mark.parametrize("kind", ["bf16", "block"])
def test_quant_linear_keeps_rows_apart(kind, rows):
    """A row with an infinity or a NaN changes no other row."""
    g = gen(12)
    n, k = 130, 384
    w, w64 = make_weight(g, n, k, 128, False)
    x, s, x64 = make_x(g, rows, k, kind)
    clean = lk.lckv_quant_linear(w, x, torch.empty(rows, n, device=DEV), x_scale=s)
    x2 = x.clone()
    x2[1, 200] = float("nan")
    if kind == "bf16":
        x2[2, 3] = float("inf")
    y = lk.lckv_quant_linear(w, x2, torch.empty(rows, n, device=DEV), x_scale=s)
    assert bool(torch.isnan(y[1]).all())
    if kind == "bf16":
        assert not bool(torch.isfinite(y[2]).any())
    rest = [0] + list(range(3, rows))
    assert torch.equal(y[rest], clean[rest])


def test_quant_refuses():
    g = gen(1)
    w, _ = make_weight(g, 64, 128, 128, False)
    f = lk.lckv_quant_linear
    x = randn(g, 4, 128)
    refused(lk.EINVAL, f, w, x.float())
    refused(lk.EINVAL, f, w, x[:, :64])
    refused(lk.EINVAL, f, w, x.cpu())
    refused(lk.EINVAL, f, w, x, torch.empty(4, 63, device=DEV))
    refused(lk.EINVAL, f, w, x, torch.empty(4, 64, device=DEV, dtype=torch.float16))
    refused(lk.EINVAL, f, w, x[:1].expand(4, 128))
    refused(lk.EINVAL, f, w, x, x_scale=torch.ones(4, device=DEV))
    refused(lk.EINVAL, f, w, x.to(torch.float8_e4m3fn))
    refused(lk.EINVAL, f, w, x.to(torch.float8_e4m3fn), x_scale=torch.ones(3, device=DEV))
    refused(lk.EINVAL, f, w, torch.zeros(4 * 128 + 8, dtype=torch.bfloat16, device=DEV)[4:4 + 512].view(4, 128))     # rows off the 16-byte grid
    codes = torch.zeros(64, 64, dtype=torch.uint8, device=DEV)
    refused(lk.EINVAL, lk.lckv_quant_pack, codes, torch.ones(64, 8, dtype=torch.bfloat16, device=DEV))               # groups of 16
    refused(lk.EINVAL, lk.lckv_quant_pack, codes, torch.ones(64, 1, device=DEV))
    refused(lk.EINVAL, lk.lckv_quant_pack, codes, torch.ones(64, 1, dtype=torch.bfloat16, device=DEV), torch.zeros(64, 2, dtype=torch.uint8, device=DEV))


# ---- all of them, as a decode step uses them ------------------------------------------------------------------------------


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("streams", [False, True])
def test_layer_step(eight_bit, streams):
    """norm -> fused q|k|v projection -> rotation and append -> attention -> output projection -> residual and norm, for three
    tokens, against the same steps in 64 bits (each step from the GPU's own rounded inputs, so that tolerances do not pile up);
    eager, and on a side stream."""
    B, Hq, Hkv, d, width = 5, 8, 4, 64, 512
    c = Case(L=2, w=0, Hq=Hq, Hkv=Hkv, d=d, lens=[0, 9, 63, 64, 100], T_cap=192, seed=21, page_rows=64, n_pages=15)
    g = gen(33)
    rope = lk.make_rope(*lk.lckv_rope_tables(torch.empty(192, d // 2, device=DEV), torch.empty(192, d // 2, device=DEV),
                                             lk.make_rope_scaling(3, 1e4, 4.0, 64.0)))
    n_qkv = (Hq + 2 * Hkv) * d
    w_qkv, w64_qkv = make_weight(g, n_qkv, width, 128, True)
    w_o, w64_o = make_weight(g, width, Hq * d, 64, False)
    norm_w = (1 + randn(g, width, std=0.1)).to(torch.bfloat16)
    res = randn(g, B, width, dtype=torch.float32)
    delta = randn(g, B, width)
    stream = torch.cuda.Stream() if streams else torch.cuda.current_stream()
    stream.wait_stream(torch.cuda.current_stream())
    from oracle import lckv_oracle as orc
    for token in range(3):
        with torch.cuda.stream(stream):
            old = res.clone()
            y = torch.empty(B, width, dtype=torch.float8_e4m3fn if eight_bit else torch.bfloat16, device=DEV)
            s = torch.empty(B, 4, device=DEV) if eight_bit else None
            lk.lckv_rms_norm(delta, norm_w, y, residual=res, residual_out=res, out_scale=s, scale_group=128 if eight_bit else 0)
            qkv = lk.lckv_quant_linear(w_qkv, y, x_scale=s).view(B, Hq + 2 * Hkv, d)
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            q_rot = c.cache.lckv_rope_append_kv(0, rope, q, k, v)
            o = c.cache.lckv_decode_attention(0, lk.MODE_STANDARD, q_rot)
            new_delta = lk.lckv_quant_linear(w_o, o.view(B, Hq * d))
            c.cache.lckv_rope_append_kv(0, rope, None, k, v, advance_len=1)      # the same row again, then the next token
        torch.cuda.synchronize()
        assert c.cache.lckv_cache_status() == 0
        h64, y64 = norm64(delta, old, norm_w, 1e-6)
        within(res, h64, h64.abs() * 2 * E)
        check_norm(y, s, y64, 128 if eight_bit else 0)
        y_in = y.float().double() * s.double().repeat_interleave(128, 1) if eight_bit else y.double()
        check_linear(qkv.view(B, -1), y_in, w64_qkv, width)
        pos = torch.tensor(c.lens.tolist(), device=DEV)
        want_q, mag = rotate64(q, rope.tables[0][pos], rope.tables[1][pos], d, False)
        within(q_rot, want_q, 3 * E * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * want_q.abs())
        want_k, mag_k = rotate64(k, rope.tables[0][pos], rope.tables[1][pos], d, False)
        expect_rows(c, 0, want_k[:, None], mag_k[:, None], v[:, None], c.lens, 1, False)
        want, _ = orc.decode_attention(syn.bits(q_rot), c.hK[0], c.hV[0], c.lens, 1, c.scale)
        # The grouped-head kernel rounds probabilities to bf16: p' = p (1 + e), |e| <= 2^-8, normalised by their own sum, so
        # |sum p' v / sum p' - sum p v| <= 2^-8 (1 + 2^-7) sum p |v - o| <= 2^-8 (1 + 2^-7) 2 max|v|.  Scores are sums of 64 fp32
        # products, each at most max|q| max|k|, scaled by 1/8: off by at most 64 * 64 * max|q| max|k| / 8 * 2^-24, which moves a
        # probability by that share of itself.  Then the output's rounding.  (Values here are larger than the unit values
        # that compare()'s absolute bound is made for.)
        rows = [[syn.from_bits(t[0][b][:, :int(c.lens[b]) + 1]).double().abs().numpy() for b in range(B)] for t in (c.hK, c.hV)]
        off = 64 * 64 / 8 * E * q_rot.abs().max().item() * max(r.max() for r in rows[0])
        top = np.repeat(np.stack([r.max(1) for r in rows[1]]), Hq // Hkv, axis=1)
        tol = (2.0 ** -8 * (1 + 2.0 ** -7) + off) * 2 * top + 2.0 ** -8 * np.abs(want)
        within(o.cpu(), torch.from_numpy(want), torch.from_numpy(tol), "attention")
        assert np.linalg.norm(o.double().cpu().numpy() - want) <= 5e-3 * np.linalg.norm(want)
        check_linear(new_delta, o.view(B, -1).double(), w64_o, Hq * d)
        c.lens += 1
        assert c.cache.lckv_cache_lengths(B) == c.lens.tolist()
        delta = new_delta
    c.close()


def test_step_in_a_graph():
    """The operators without host-side growth, captured once and replayed with other inputs, equal eager calls bit for bit;
    two graphs share no workspace."""
    g = gen(44)
    B, width = 7, 512
    w, _ = make_weight(g, 768, width, 64, False)
    norm_w = torch.ones(width, dtype=torch.bfloat16, device=DEV)
    rope = lk.make_rope(*(t.float() for t in tables64(128, 64)))
    pos = torch.arange(B, dtype=torch.int32, device=DEV)

    def step(x, y, h, z):
        lk.lckv_rms_norm(x, norm_w, y)
        lk.lckv_quant_linear(w, y, h)
        lk.lckv_rope_apply(rope, pos, h.view(B, 6, 128), z)

    sets = [(randn(g, B, width), torch.empty(B, width, dtype=torch.bfloat16, device=DEV), torch.empty(B, 768, dtype=torch.bfloat16, device=DEV),
             torch.empty(B, 6, 128, dtype=torch.bfloat16, device=DEV)) for _ in range(2)]
    step(*sets[0])
    torch.cuda.synchronize()
    graphs = []
    for s in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(*s)
    for trial in range(3):
        for s in sets:
            s[0].copy_(randn(g, B, width))
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in sets]
        for st, gr in zip(streams, graphs):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for s in sets:
            got = [t.clone() for t in s[1:]]
            fresh = [torch.empty_like(t) for t in s[1:]]
            step(s[0], *fresh)
            assert all(torch.equal(a, b) for a, b in zip(got, fresh))
