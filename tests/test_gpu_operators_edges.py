"""The operators around the attention at the ends of what their documentation allows.  Tolerances: see
test_gpu_operators.py."""
import pytest
import torch

from paper_2405_10637_b200 import binding as lk

from test_gpu_operators import DEV, E, HALF, check_linear, check_norm, gen, make_weight, make_x, norm64, randn, refused, rotate64, tables64, within

pytestmark = pytest.mark.gpu


# ---- the widest rows -----------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3row", "e4m3block"])
@pytest.mark.parametrize("width,shift", [(32761, 0), (32762, 0), (32767, 0), (32768, 1)])
def test_norm_widest_rows(width, shift, out):
    """Rows that touch 4096 and 4097 vectors of 8; width 32768 with a weight off the 16-byte grid."""
    g = gen(width)
    group = 128 if out == "e4m3block" else 0
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}.get(out, torch.float8_e4m3fn)
    for rows, x32, r32, w32, res in [(1, False, False, False, True), (3, True, True, True, True), (301, False, True, True, True),
                                     (301, False, False, False, False)]:
        x = randn(g, rows, width, dtype=torch.float32 if x32 else torch.bfloat16)
        r = randn(g, rows, width, dtype=torch.float32 if r32 else torch.bfloat16, std=3.0) if res else None
        w = (1 + randn(g, width + 8, dtype=torch.float32, std=0.2)).to(torch.float32 if w32 else torch.bfloat16)[shift:shift + width]
        y = torch.full((rows, width), float("nan"), device=DEV).to(dt)
        scale = torch.full((rows, -(-width // 128) if group else 1), float("nan"), device=DEV) if dt == torch.float8_e4m3fn else None
        h = torch.full_like(r, float("nan")) if res else None
        lk.lckv_rms_norm(x, w, y, residual=r, residual_out=h, out_scale=scale, scale_group=group, eps=1e-5)
        h64, y64 = norm64(x, r, w, 1e-5)
        check_norm(y, scale, y64, group)
        if res:
            within(h, h64, h64.abs() * (HALF[h.dtype] + E) * (1 + E))


# ---- replays of a rotated append -------------------------------------------------------------------------------------------


SHORT = 8                              # positions of the tables


def replayed(c, g, lens, n, rot, interleaved, with_kv, prompt, aligned):
    """Captures a call with tables of SHORT positions at lengths that fit, replays it at `lens`, and compares with an eager call
    that has longer tables: tokens with a position are the same, of the others nothing is written."""
    B, (Hq, Hkv, d) = len(lens), c.heads
    cos, sin = (t.float() for t in tables64(rot, 64))
    rope, short = lk.make_rope(cos, sin, interleaved), lk.make_rope(cos[:SHORT].contiguous(), sin[:SHORT].contiguous(), interleaved)
    flat = randn(g, B * n * (Hq + 2 * Hkv) * d + 8)[0 if aligned else 1:][:B * n * (Hq + 2 * Hkv) * d]
    flat = flat.view(B, n, Hq + 2 * Hkv, d)
    q, k, v = flat[:, :, :Hq], flat[:, :, Hq:Hq + Hkv], flat[:, :, Hq + Hkv:]
    if not with_kv:
        k = v = None

    def call(r, out):
        if prompt:
            c.lckv_rope_prefill_write_kv(0, r, q, k, v, out)
        else:
            c.lckv_rope_append_kv(0, r, q, k, v, out)

    pools = c.slot_tensors(0)
    c.lckv_cache_reset(lens)
    for t in pools:
        t.fill_(5.0)
    want = torch.full((B, n, Hq, d), 9.0, dtype=torch.bfloat16, device=DEV)
    call(rope, want)
    want_pools = [t.clone() for t in pools]
    assert c.lckv_cache_status() == 0

    c.lckv_cache_reset([0] * B)
    for t in pools:
        t.fill_(5.0)
    out = torch.full_like(want, 9.0)
    if prompt:
        c.lckv_cache_reset([1] * B)
    call(short, out)                                  # pages for the captured call
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(short, out)
    c.lckv_cache_reset(lens)
    for t in (*pools, out):
        t.fill_(5.0 if t is not out else 9.0)
    graph.replay()
    status = c.lckv_cache_status()
    lost = False
    for b in range(B):
        for i in range(n):
            if prompt and i >= lens[b]:
                assert bool((out[b, i] == 9.0).all())
                continue
            at = i if prompt else lens[b] + i
            if at < SHORT:
                assert torch.equal(out[b, i], want[b, i]), (b, i)
            else:
                lost = True
                assert bool((out[b, i] == 9.0).all()), (b, i)
                # the rows that the eager call wrote for this token stay as they were
                if with_kv:
                    row = at
                    if c.cfg.stream_sink and row >= c.cfg.max_seq:
                        row = c.cfg.stream_sink + (row - c.cfg.stream_sink) % (c.cfg.max_seq - c.cfg.stream_sink)
                    for t, w in zip(pools, want_pools):
                        place = (b, slice(None), row) if not c.cfg.page_rows else (int(c.lckv_cache_page_table()[b, row // c.cfg.page_rows]), slice(None), row % c.cfg.page_rows)
                        w[place] = 5.0
    if not c.cfg.page_rows:
        for t, w in zip(pools, want_pools):
            assert torch.equal(t, w)
    else:
        # (pages may have changed hands between the two)
        assert with_kv or bool((pools[0] == 5.0).all())
        for b in range(B):
            for i in range(n):
                at = i if prompt else lens[b] + i
                if (prompt and i >= lens[b]) or not with_kv:
                    continue
                page = int(c.lckv_cache_page_table()[b, at // c.cfg.page_rows])
                got = pools[1][page, :, at % c.cfg.page_rows]
                assert torch.equal(got, v[b, i]) if at < SHORT else bool((got == 5.0).all())
    assert lost and status == lk.ECAPACITY
    c.lckv_cache_reset([0] * B)
    assert c.lckv_cache_status() == 0


REPLAY_LAYOUTS = {"contiguous": dict(), "paged": dict(page_rows=64, n_pages=6), "ring": dict(stream_sink=4)}


@pytest.mark.parametrize("layout", list(REPLAY_LAYOUTS))
@pytest.mark.parametrize("rot,interleaved,aligned", [(64, False, True), (50, False, True), (22, True, True), (64, True, False)])
def test_replay_behind_the_tables(rot, interleaved, aligned, layout):
    g = gen(rot)
    T = 12 if layout == "ring" else 40
    c = lk.Cache(lk.make_config(2, 0, 4, 2, 64, 3, T, **REPLAY_LAYOUTS[layout]))
    for with_kv in (True, False):
        replayed(c, g, [3, 20, 8], 1, rot, interleaved, with_kv, False, aligned)
        replayed(c, g, [7, 2, 30], 3, rot, interleaved, with_kv, False, aligned)
        if layout != "ring":
            replayed(c, g, [11, 3, 0], 12, rot, interleaved, with_kv, True, aligned)
    c.close()


# ---- products whose device-side waits run out --------------------------------------------------------------------------------


@pytest.fixture
def copy_limits():
    yield lk.lckv_quant_set_copy_limits
    lk.lckv_quant_set_copy_limits()


@pytest.mark.parametrize("weights,x_blocks", [(-1, 0), (1, -1), (-1, 3), (2, 2)])
@pytest.mark.parametrize("rows,n,k,group,has_zeros,kind", [(17, 130, 512, 128, False, "bf16"), (32, 1000, 4096, 64, True, "block"),
                                                           (200, 600, 2048, 32, False, "row"), (129, 300, 11008, 128, True, "bf16")])
def test_quant_waits_that_run_out(rows, n, k, group, has_zeros, kind, weights, x_blocks, copy_limits):
    """Copies that are not requested: the outputs are NaN and that is reported, nothing else is written, and calls queued
    behind are right (what the call that gave up still had under way does not reach their memory)."""
    g = gen(rows)
    w, w64 = make_weight(g, n, k, group, has_zeros)
    x, s, x64 = make_x(g, rows, k, kind)
    clean = lk.lckv_quant_linear(w, x, torch.empty(rows, n, device=DEV), x_scale=s)
    check_linear(clean, x64, w64, k)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    buf = torch.full((rows, n + 8), 7.0, device=DEV)
    after = [torch.full((rows, n), 3.0, device=DEV) for _ in range(2)]
    copy_limits(weights, x_blocks)
    lk.lckv_quant_linear(w, x, buf[:, 4:4 + n], x_scale=s, dev_status=status)
    copy_limits()
    for y in after:
        lk.lckv_quant_linear(w, x, y, x_scale=s)
    torch.cuda.synchronize()
    assert status.item() == lk.ETIMEOUT
    assert bool(torch.isnan(buf[:, 4:4 + n]).all())
    assert bool((buf[:, :4] == 7.0).all()) and bool((buf[:, 4 + n:] == 7.0).all())
    assert all(torch.equal(y, clean) for y in after)


# ---- products: weights at and beside their zero point, one large activation --------------------------------------------------


@pytest.mark.parametrize("kind", ["bf16", "row", "block"])
@pytest.mark.parametrize("rows", [1, 8, 16, 17, 40])
@pytest.mark.parametrize("k,group,has_zeros", [(128, 128, False), (1024, 64, True), (2080, 32, True), (4096, 128, True)])
def test_quant_small_weights_large_activation(k, group, has_zeros, rows, kind):
    """c - z is exact before it meets x: a feature whose codes are its zero points gives 0 whatever x is, and an x of some
    thousands leaves no trace in a feature that has a zero weight there."""
    g = gen(k + rows)
    n = 72
    zeros = torch.randint(1, 15, (n, k // group), generator=g, device=DEV, dtype=torch.uint8) if has_zeros else None
    z = zeros.repeat_interleave(group, 1) if has_zeros else torch.full((n, k), 8, dtype=torch.uint8, device=DEV)
    w = torch.randint(-1, 2, (n, k), generator=g, device=DEV, dtype=torch.int32)
    w[:16] = 0
    big = 37
    w[16:48, big] = 0
    codes = (z.int() + w).to(torch.uint8)
    scales = (torch.rand((n, k // group), generator=g, device=DEV) + 0.5).to(torch.bfloat16)
    packed = lk.lckv_quant_pack(codes[:, 0::2] | (codes[:, 1::2] << 4), scales, zeros)
    w64 = w.double() * scales.double().repeat_interleave(group, 1)
    x, s, _ = make_x(g, rows, k, kind)
    if kind == "bf16":
        x[:, big] = 3333.0
        x64 = x.double()
    else:
        x = (x.float() / 64).to(torch.float8_e4m3fn)
        x[:, big] = 448.0
        x64 = x.float().double() * (s.double() if kind == "row" else s.double().repeat_interleave(128, 1)[:, :k])
    y = lk.lckv_quant_linear(packed, x, torch.empty(rows, n, device=DEV), x_scale=s)
    assert bool((y[:, :16] == 0).all())
    check_linear(y, x64, w64, k)


def test_quant_sums_of_large_activations():
    """x whose products with 16 + c would leave fp32 while those with c - z do not."""
    g = gen(8)
    n, k = 64, 256
    codes = torch.full((n, k // 2), 0x88, dtype=torch.uint8, device=DEV)
    codes[:, 5] = 0x89                                       # one weight of 1, the others 0
    w = lk.lckv_quant_pack(codes, torch.ones(n, 2, dtype=torch.bfloat16, device=DEV))
    for rows in (1, 16, 17):
        x = torch.full((rows, k), 1e38, device=DEV).to(torch.bfloat16)
        y = lk.lckv_quant_linear(w, x, torch.empty(rows, n, device=DEV))
        assert torch.equal(y, x[:, :1].float().expand(rows, n))


# ---- rows of the smallest and the largest numbers -----------------------------------------------------------------------------


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3row", "e4m3block"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [8, 64, 1000, 1030, 4096, 20001, 32767, 32768])
def test_norm_of_extreme_rows(width, dtype, out):
    """Rows near the smallest and the largest numbers of their type beside ordinary ones, with an eps of zero and one that is as
    small as the squares; the factor of such a row lies outside fp32."""
    g = gen(width)
    group = 128 if out == "e4m3block" else 0
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}.get(out, torch.float8_e4m3fn)
    tiny = 2.0 ** -126 if dtype == torch.bfloat16 else 2.0 ** -140
    unit = torch.tensor([1.0, tiny, 1e38, tiny * 2 ** 60, 3e19], dtype=torch.float64, device=DEV)
    for rows in (5, 305):
        x = torch.randn((rows, width), generator=g, device=DEV).double() * unit[torch.arange(rows, device=DEV) % 5, None]
        x = x.clamp(-3e38, 3e38).to(dtype)
        x[:, 0] = torch.where(x[:, 0] == 0, unit[torch.arange(rows, device=DEV) % 5].to(dtype), x[:, 0])       # no row of zeros
        x[2] = 3e38                                        # the sum of these squares, at the first scale that suffices for most
        w = 1 + randn(g, width, dtype=torch.float32, std=0.2)
        for eps in (0.0, 2.0 ** -149, 1e-30):
            y = torch.empty(rows, width, device=DEV, dtype=dt)
            scale = torch.empty(rows, -(-width // 128) if group else 1, device=DEV) if dt == torch.float8_e4m3fn else None
            lk.lckv_rms_norm(x, w, y, out_scale=scale, scale_group=group, eps=eps)
            check_norm(y, scale, norm64(x, None, w, torch.tensor(eps, dtype=torch.float32).double().item())[1], group)


# ---- zero points above 15 --------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("n,k,group", [(1, 32, 32), (70, 256, 64), (3000, 4096, 128)])
def test_zero_points_above_15_are_refused(n, k, group):
    g = gen(n)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.ones(n, k // group, dtype=torch.bfloat16, device=DEV)
    zeros = torch.randint(0, 16, (n, k // group), generator=g, device=DEV, dtype=torch.uint8)
    zeros.view(-1)[0] = zeros.view(-1)[-1] = 15
    x = randn(g, 3, k)
    w = lk.lckv_quant_pack(codes, scales, zeros)
    c = torch.stack([codes & 15, codes >> 4], -1).view(n, k)
    check_linear(lk.lckv_quant_linear(w, x, torch.empty(3, n, device=DEV)), x.double(), c.double() - zeros.double().repeat_interleave(group, 1), k)
    for at, value in [(0, 16), (-1, 16), (zeros.numel() // 2, 255)]:
        bad = zeros.clone()
        bad.view(-1)[at] = value
        refused(lk.EINVAL, lk.lckv_quant_pack, codes, scales, bad)


# ---- a query alone behind the last row ----------------------------------------------------------------------------------------


@pytest.mark.parametrize("layout", [dict(), dict(page_rows=64, n_pages=4)])
@pytest.mark.parametrize("rot", [64, 24])
def test_query_alone_needs_no_row(rot, layout):
    """A condensed layer's query at the end of a full cache: it has a position, and no row is written for it."""
    g = gen(rot)
    c = lk.Cache(lk.make_config(2, 0, 4, 2, 64, 2, 128, **layout))
    c.lckv_cache_reset([128, 126])
    pools = [t.fill_(5.0) for t in c.slot_tensors(0)]
    cos, sin = (t.float() for t in tables64(rot, 131))
    rope = lk.make_rope(cos, sin)
    q, k, v = (randn(g, 2, 3, h, 64) for h in (4, 2, 2))
    out = c.lckv_rope_append_kv(0, rope, q, None, None)
    pos = torch.tensor([128, 126], device=DEV)[:, None] + torch.arange(3, device=DEV)
    want, mag = rotate64(q, cos[pos], sin[pos], rot, False)
    within(out, want, 3 * E * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs())
    assert c.lckv_cache_status() == 0 and all(bool((t == 5.0).all()) for t in pools)
    refused(lk.ECAPACITY, c.lckv_rope_append_kv, 0, rope, q, k, v)
    refused(lk.EINVAL, c.lckv_rope_append_kv, 0, rope, *(randn(g, 2, 4, 4, 64), None, None))       # position 131 is not there
    c.close()


# ---- operands that the kernel in front has written ----------------------------------------------------------------------------


def test_operands_of_the_kernel_in_front():
    """A launch may begin before the one in front has ended: tables, positions' products, weights, scales and x that the calls
    in front wrote into the same memory, queued without a pause, give the bits that they give with a pause after each call."""
    g = gen(77)
    T, H, d, width = 64, 16, 128, 2048
    w, _ = make_weight(g, width, width, 64, True)
    pos = torch.randint(0, 200, (T,), generator=g, device=DEV, dtype=torch.int32)
    xs = [randn(g, T, H, d, dtype=torch.float32) for _ in range(3)]
    scalings = [lk.make_rope_scaling(0, base) for base in (1e4, 5e5, 1e3)]
    cache = lk.Cache(lk.make_config(2, 0, H, H, d, T, 256))
    cache.lckv_cache_reset(list(range(T)))

    def chain(pause):
        cos, sin = (torch.empty(256, d // 2, device=DEV) for _ in range(2))
        rope = lk.make_rope(cos, sin)
        turned = torch.empty_like(xs[0])
        normed, scale = torch.empty(T, width, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(T, width // 128, device=DEV)
        few = torch.empty(8, width, device=DEV)
        y, q = torch.empty(T, width, dtype=torch.bfloat16, device=DEV), torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV)
        outs = []
        torch.cuda.synchronize()
        for step in range(12):
            for call in (lambda: lk.lckv_rope_tables(cos, sin, scalings[step % 3]),
                         lambda: lk.lckv_rope_apply(rope, pos, xs[step % 3], turned),
                         # the norm's weight is a row that the rotation has just written
                         lambda: lk.lckv_rms_norm(turned.view(T, width), turned.view(T, width)[step], normed, out_scale=scale, scale_group=128),
                         lambda: lk.lckv_quant_linear(w, normed, y, x_scale=scale),
                         lambda: lk.lckv_quant_linear(w, normed[:8], few, x_scale=scale[:8]),
                         lambda: lk.lckv_rope_tables(cos, sin, scalings[(step + 1) % 3]),
                         lambda: cache.lckv_rope_append_kv(0, rope, y.view(T, H, d), y.view(T, H, d), y.view(T, H, d), q)):
                call()
                if pause:
                    torch.cuda.synchronize()
            outs.append([t.clone() for t in (turned, normed.view(torch.uint8), scale, y, few, q)])
        torch.cuda.synchronize()
        return outs

    want = chain(True)
    for _ in range(5):
        for got, ref in zip(chain(False), want):
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
    cache.close()


@pytest.mark.parametrize("layout", [dict(), dict(page_rows=64, n_pages=4)])
def test_prompts_captured_while_they_are_empty(layout):
    """A call captured at lengths of zero writes the prompts that a replay finds."""
    g = gen(5)
    c = lk.Cache(lk.make_config(2, 0, 4, 2, 64, 2, 128, **layout))
    rope = lk.make_rope(*(t.float() for t in tables64(64, 64)))
    q, k, v = (randn(g, 2, 9, h, 64) for h in (4, 2, 2))
    out = torch.full((2, 9, 4, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    c.lckv_cache_reset([0, 0])
    c.lckv_rope_prefill_write_kv(0, rope, q, k, v, out)
    assert bool((out == 9.0).all()) and c.lckv_cache_status() == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.lckv_rope_prefill_write_kv(0, rope, q, k, v, out)
    c.lckv_cache_reset([9, 4])
    graph.replay()
    got, pools = out.clone(), [t.clone() for t in c.slot_tensors(0)]
    want = torch.full_like(out, 9.0)
    for t in c.slot_tensors(0):
        t.fill_(0)
    c.lckv_rope_prefill_write_kv(0, rope, q, k, v, want)
    assert torch.equal(got, want) and bool((got[1, 4:] == 9.0).all()) and c.lckv_cache_status() == 0
    table = c.lckv_cache_page_table() if c.cfg.page_rows else None
    for b, m in ((0, 9), (1, 4)):
        page = b if table is None else int(table[b, 0])
        for a, w in zip(pools, c.slot_tensors(0)):
            assert torch.equal(a[page, :, :m], w[page, :, :m])
    c.close()
