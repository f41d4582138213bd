"""The operators around the attention at the kernels that only many rows, tokens or features reach, at offsets beyond 32
bits, on streams other than the current one and in two streams at once.  Tolerances: see test_gpu_operators.py."""
import pytest
import torch

from paper_2405_10637_b200 import binding as lk

from helpers import Case
from test_gpu_operators import (DEV, E, HALF, check_linear, check_norm, fused, gen, make_weight, make_x, norm64, randn,
                                refused, rotate64, tables64, within)

pytestmark = pytest.mark.gpu


# ---- many rows, tokens, features -----------------------------------------------------------------------------------------


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3row", "e4m3block"])
@pytest.mark.parametrize("width", [1, 40, 64, 100, 128, 256, 1000, 1030, 2056, 4095, 4096, 6152, 8192, 9000, 16384, 20001])
def test_norm_many_rows(width, out):
    """More rows than the GPU runs thread blocks at once, and a last thread block of rows that is not full."""
    g = gen(width + 1)
    eps = 1e-5
    group = 128 if out == "e4m3block" else 0
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}.get(out, torch.float8_e4m3fn)
    for rows, x32, r32, w32, res in [(150, False, False, False, True), (1501, False, False, True, False), (700, False, True, False, True),
                                     (700, True, False, False, True), (301, True, True, True, True), (1203, True, False, False, False)]:
        if width <= 64:
            rows *= 16
        x = randn(g, rows, width, dtype=torch.float32 if x32 else torch.bfloat16)
        r = randn(g, rows, width, dtype=torch.float32 if r32 else torch.bfloat16, std=3.0) if res else None
        w = 1 + randn(g, width, dtype=torch.float32, std=0.2)
        w = w if w32 else w.to(torch.bfloat16)
        y = torch.empty(rows, width, dtype=dt, device=DEV)
        scale = torch.full((rows, -(-width // 128) if group else 1), float("nan"), device=DEV) if dt == torch.float8_e4m3fn else None
        h = torch.empty_like(r) if res else None
        lk.lckv_rms_norm(x, w, y, residual=r, residual_out=h, out_scale=scale, scale_group=group, eps=eps)
        h64, y64 = norm64(x, r, w, eps)
        check_norm(y, scale, y64, group)
        if res:
            within(h, h64, h64.abs() * (HALF[h.dtype] + E) * (1 + E))
            r2, y2 = r.clone(), torch.empty_like(y)
            lk.lckv_rms_norm(x, w, y2, residual=r2, residual_out=r2, out_scale=scale, scale_group=group, eps=eps)
            assert torch.equal(r2, h) and torch.equal(y2.view(torch.uint8), y.view(torch.uint8))
        if dt == x.dtype and not res:
            x2 = x.clone()
            lk.lckv_rms_norm(x2, w, x2, eps=eps)
            assert torch.equal(x2, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [64, 1030, 4096])
def test_norm_many_rows_apart(width, dtype):
    """Rows whose squares overflow or vanish in fp32, zeros, an infinity and a NaN change no other row."""
    g = gen(9)
    rows, eps = 1000, 2.0 ** -133
    x = randn(g, rows, width, dtype=dtype)
    w = torch.ones(width, device=DEV)
    clean = lk.lckv_rms_norm(x, w, torch.empty_like(x), eps=eps)
    x2 = x.clone()
    x2[::7] = 0
    x2[1::7] *= 1e25
    x2[2::7] *= 1e-25
    x2[3::7, 5] = float("inf")
    x2[4::7, width - 1] = float("nan")
    y = lk.lckv_rms_norm(x2, w, torch.empty_like(x), eps=eps)
    for i in (5, 6):
        assert torch.equal(y[i::7], clean[i::7])
    assert bool((y[::7] == 0).all()) and bool(torch.isnan(y[4::7]).all()) and bool(torch.isnan(y[3::7, 5]).all())
    for i in (1, 2):
        check_norm(y[i::7], None, norm64(x2[i::7], None, w, eps)[1], 0)


@pytest.mark.parametrize("page_rows", [0, 64])
@pytest.mark.parametrize("interleaved,rot,prompt", [(False, 128, False), (True, 64, False), (False, 24, False), (True, 50, True), (False, 96, True)])
def test_rotated_append_many_tokens(interleaved, rot, prompt, page_rows):
    """Several heads per thread, and tokens that end inside a thread block."""
    B, n, Hq, Hkv, d = 41, 67, 21, 7, 128
    lens = [(b * 13) % (n + 1) for b in range(B)] if prompt else [(b * 5) % 60 for b in range(B)]
    c = Case(L=2, w=0, Hq=Hq, Hkv=Hkv, d=d, lens=lens, T_cap=140, seed=8, poison=False, page_rows=page_rows, n_pages=3 * B if page_rows else 0)
    g = gen(1)
    cos, sin = (t.float() for t in tables64(rot, 140))
    rope = lk.make_rope(cos, sin, interleaved)
    q, k, v = fused(g, B, n, Hq, Hkv, d)
    pos = torch.arange(n, device=DEV)[None] + (0 if prompt else torch.tensor(lens, device=DEV)[:, None])
    pos = pos.expand(B, n)
    want_q, mag_q = rotate64(q, cos[pos], sin[pos], rot, interleaved)
    want_k, mag_k = rotate64(k, cos[pos], sin[pos], rot, interleaved)
    out = torch.full((B, n, Hq, d), 3.0, dtype=torch.bfloat16, device=DEV)
    (c.cache.lckv_rope_prefill_write_kv if prompt else c.cache.lckv_rope_append_kv)(0, rope, q, k, v, out)
    for b in range(B):
        m = lens[b] if prompt else n
        within(out[b, :m], want_q[b, :m], 3 * E * mag_q[b, :m] * (1 + 2.0 ** -8) + 2.0 ** -8 * want_q[b, :m].abs(), "q")
        assert bool((out[b, m:] == 3.0).all())
    kt, vt = c.cache.slot_tensors(0)
    table = c.cache.lckv_cache_page_table() if page_rows else None
    for b in range(B):
        m, first = (lens[b], 0) if prompt else (n, lens[b])
        for i in range(m):
            row = first + i
            at = (b, slice(None), row) if not page_rows else (int(table[b, row // page_rows]), slice(None), row % page_rows)
            if i in (0, m // 2, m - 1):
                within(kt[at], want_k[b, i], 3 * E * mag_k[b, i] * (1 + 2.0 ** -8) + 2.0 ** -8 * want_k[b, i].abs(), "k")
                assert torch.equal(vt[at], v[b, i])
    c.close()


@pytest.mark.parametrize("Hq,Hkv,d", [(64, 16, 64), (32, 32, 128), (7, 7, 64)])
def test_long_ragged_prompts(Hq, Hkv, d):
    """Thread blocks that hold several tokens, of different prompts and behind their ends."""
    lens, n = [3301, 0, 1, 1650, 3300], 3301
    cfg = lk.make_config(2, 0, Hq, Hkv, d, len(lens), 3328, page_rows=64, n_pages=52 * len(lens))
    c = lk.Cache(cfg)
    c.lckv_cache_reset(lens)
    g = gen(12)
    cos, sin = (t.float() for t in tables64(d, n))
    rope = lk.make_rope(cos, sin)
    q, k, v = fused(g, len(lens), n, Hq, Hkv, d)
    out = torch.full((len(lens), n, Hq, d), 3.0, dtype=torch.bfloat16, device=DEV)
    c.lckv_rope_prefill_write_kv(0, rope, q, k, v, out)
    kt, vt = c.slot_tensors(0)
    table = c.lckv_cache_page_table().to(DEV)
    for b, m in enumerate(lens):
        assert bool((out[b, m:] == 3.0).all())
        if m == 0:
            continue
        want, mag = rotate64(q[b, :m], cos[:m], sin[:m], d, False)
        within(out[b, :m], want, 3 * E * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs(), "q")
        row = torch.arange(m, device=DEV)
        page, at = table[b, row // 64], row % 64
        want, mag = rotate64(k[b, :m], cos[:m], sin[:m], d, False)
        within(kt[page, :, at], want, 3 * E * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs(), "k")
        assert torch.equal(vt[page, :, at], v[b, :m])
    assert c.lckv_cache_status() == 0
    c.close()


@pytest.mark.parametrize("heads,d", [(96, 64), (44, 128), (11, 128)])
def test_rotation_many_tokens(heads, d):
    g = gen(13)
    tokens = 16500
    cos, sin = (t.float() for t in tables64(d, 999))
    x = randn(g, tokens, heads, d)
    pos = torch.randint(0, 999, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    y = lk.lckv_rope_apply(lk.make_rope(cos, sin), pos, x)
    want, mag = rotate64(x, cos[pos.long()], sin[pos.long()], d, False)
    within(y, want, 3 * E * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs())


@pytest.mark.parametrize("kind", ["bf16", "row", "block"])
@pytest.mark.parametrize("n,k,group,has_zeros", [(9001, 288, 32, True), (20000, 640, 128, False), (2561, 4096, 64, True)])
def test_quant_linear_many_features(n, k, group, has_zeros, kind):
    g = gen(n)
    w, w64 = make_weight(g, n, k, group, has_zeros)
    for rows in (1, 7, 16, 31, 65, 257):
        x, s, x64 = make_x(g, rows, k, kind)
        check_linear(lk.lckv_quant_linear(w, x, torch.full((rows, n), float("nan"), device=DEV), x_scale=s), x64, w64, k)


# ---- offsets beyond 32 bits ----------------------------------------------------------------------------------------------


def test_largest_tables():
    """2^31 - 1 positions of one pair: the last ones, by their angle modulo a turn (theta = 1)."""
    n = 2 ** 31 - 1
    cos, sin = (torch.empty(n, 1, device=DEV) for _ in range(2))
    lk.lckv_rope_tables(cos, sin, lk.make_rope_scaling())
    for at in (0, 2 ** 30 - 3, n - 5):
        p = torch.arange(at, at + 5, dtype=torch.float64, device=DEV)
        # the turns of a position are a product of p and a number off by 2^-53; the argument here is as far off in fp64
        tol = 2.0 ** -22 + n * 2.0 ** -50
        within(cos[at:at + 5, 0], torch.cos(p), tol)
        within(sin[at:at + 5, 0], torch.sin(p), tol)


def test_rotation_far_offsets():
    tokens, heads, d = 2 ** 18 + 3, 64, 128                       # 2^31 + 24576 elements
    g = gen(2)
    cos, sin = (t.float() for t in tables64(128, 512))
    rope = lk.make_rope(cos, sin)
    x = randn(g, tokens, 1, d).expand(tokens, heads, d)           # one head, read for all
    pos = torch.randint(0, 512, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    y = lk.lckv_rope_apply(rope, pos, x)
    t = slice(tokens - 6, tokens)
    want, mag = rotate64(x[t], cos[pos[t].long()], sin[pos[t].long()], 128, False)
    within(y[t], want, 3 * E * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs())


@pytest.mark.parametrize("page_rows", [0, 64])
def test_append_far_offsets(page_rows):
    T, d = 2 ** 24 + 128, 128                                     # a slot of 2^31 + 16384 elements
    cfg = lk.make_config(2, 0, 1, 1, d, 1, T, page_rows=page_rows, n_pages=T // 64 if page_rows else 0)
    c = lk.Cache(cfg)
    g = gen(3)
    cos, sin = (torch.rand(T, 1, generator=g, device=DEV) for _ in range(2))
    rope = lk.make_rope(cos, sin)
    first = T - 64 - 3
    c.lckv_cache_reset([first])
    q, k, v = (randn(g, 1, 5, 1, d) for _ in range(3))
    out = c.lckv_rope_append_kv(0, rope, q, k, v, advance_len=1)
    at = slice(first, first + 5)
    kt, vt = c.slot_tensors(0)
    if page_rows:
        table = c.lckv_cache_page_table()[0]
        rows = torch.arange(first, first + 5)
        ids = table[rows // 64]
        assert int(ids.min()) >= 0
        got_k, got_v = (torch.stack([t[int(i), 0, int(r) % 64] for i, r in zip(ids, rows)]) for t in (kt, vt))
    else:
        got_k, got_v = kt[0, 0, at], vt[0, 0, at]
    for got, src in ((out[0, :, 0], q[0, :, 0]), (got_k, k[0, :, 0])):
        want, mag = rotate64(src[:, None], cos[at], sin[at], 2, False)
        within(got, want[:, 0], 3 * E * mag[:, 0] * (1 + 2.0 ** -8) + 2.0 ** -8 * want[:, 0].abs())
    assert torch.equal(got_v, v[0, :, 0])
    assert c.lckv_cache_lengths(1) == [first + 5] and c.lckv_cache_status() == 0
    c.close()


@pytest.mark.parametrize("width,step", [(4096, 4096), (4095, 4095), (4093, 4096)])
def test_norm_far_offsets(width, step):
    rows = 2 ** 31 // width + 200
    x = torch.randn(rows, step, device=DEV, generator=gen(4), dtype=torch.bfloat16)[:, :width]
    w = torch.ones(width, device=DEV)
    y = lk.lckv_rms_norm(x, w, torch.empty(rows, width, dtype=torch.bfloat16, device=DEV))
    for t in (slice(0, 3), slice(rows - 205, rows)):
        check_norm(y[t], None, norm64(x[t], None, w, 1e-6)[1], 0)


@pytest.mark.parametrize("rows", [2, 33])
def test_quant_far_offsets(rows):
    n, k, group = 2 ** 20 + 70, 8192, 128                         # 4.4 GB packed
    g = gen(5)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.rand((n, k // group), generator=g, device=DEV).to(torch.bfloat16)
    w = lk.lckv_quant_pack(codes, scales)
    x = randn(g, rows, k)
    y = lk.lckv_quant_linear(w, x, torch.empty(rows, n, device=DEV))
    for t in (slice(0, 40), slice(n - 200, n)):
        c = torch.stack([codes[t] & 15, codes[t] >> 4], -1).view(-1, k)
        w64 = (c.double() - 8) * scales[t].double().repeat_interleave(group, 1)
        check_linear(y[:, t], x.double(), w64, k)


# ---- streams -------------------------------------------------------------------------------------------------------------


def test_made_outputs_belong_to_the_stream():
    """An output that a call on another stream makes is neither filled nor still in use on the current one."""
    lens, n, H, d = [3, 9], 9, 2, 64
    c = Case(L=2, w=0, Hq=H, Hkv=H, d=d, lens=lens, T_cap=16, seed=2, poison=False)
    g = gen(6)
    rope = lk.make_rope(*(t.float() for t in tables64(64, 64)))
    q, k, v = (randn(g, 2, n, H, d) for _ in range(3))
    want = c.cache.lckv_rope_prefill_write_kv(0, rope, q, k, v)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                    # the current stream is busy for a tenth of a second
    got = c.cache.lckv_rope_prefill_write_kv(0, rope, q, k, v, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    c.close()


def test_two_streams_at_once():
    """Calls that run side by side share nothing: each gives the bits that it gives alone."""
    g = gen(7)
    w, _ = make_weight(g, 4096, 2048, 64, True)
    jobs = []
    for rows in (1, 16, 24, 200):
        x, s, _ = make_x(g, rows, 2048, "block")
        jobs.append((x, s, lk.lckv_quant_linear(w, x, x_scale=s)))
    h = randn(g, 2000, 2048)
    ones = torch.ones(2048, device=DEV)
    normed = lk.lckv_rms_norm(h, ones, torch.empty_like(h))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    out = [[] for _ in streams]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                for x, s, _ in jobs[i:] + jobs[:i]:
                    out[i].append(lk.lckv_quant_linear(w, x, x_scale=s))
                out[i].append(lk.lckv_rms_norm(h, ones, torch.empty_like(h)))
    torch.cuda.synchronize()
    for i in range(len(streams)):
        order = [y for _, _, y in jobs[i:] + jobs[:i]] + [normed]
        for j, y in enumerate(out[i]):
            assert torch.equal(y, order[j % len(order)])


def test_numbers_that_do_not_fit_are_refused():
    x = torch.zeros(2, 256, dtype=torch.bfloat16, device=DEV)
    y, s = torch.empty(2, 256, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(2, 2, device=DEV)
    refused(lk.EINVAL, lk.lckv_rms_norm, x, torch.ones(256, device=DEV), y, out_scale=s, scale_group=2 ** 32 + 128)
    c = Case(L=2, w=0, Hq=2, Hkv=2, d=64, lens=[1], T_cap=8, seed=2)
    rope = lk.make_rope(*(t.float() for t in tables64(64, 64)))
    refused(lk.EINVAL, c.cache.lckv_rope_append_kv, 2 ** 32, rope, *(torch.zeros(1, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(3)))
    c.close()
