"""Compact caches against plain forms in 64 bits: rows held in 4 bits (written, read back, attended to), the attention
weight that rows gather, eviction, and a run of them together.

Tolerances, from the number formats: a rounding to bf16 is off by at most 2^-8 of the value, an fp32 operation by 2^-24 of its
result.  A score is a sum of D products and D / 64 lows on the tensor cores and in fp32; every partial sum is at most
A = scale * (sum |q| step code + |low| sum |q|), and fewer than 16 of them are rounded (chains of D / 16 MMAs, which may
drop what lies below 2^-23, and the sums of groups): 2^-19 A bounds it, with the exponential's argument.  Weights carry 22 bits and
ex2 has an error of 2^-22: with the sums of up to 64 terms per lane and the merge, 2^-17 of sum p (step code + |low|) bounds the rest."""
import math

import numpy as np
import pytest
import torch

from paper_2405_10637_b200 import binding as lk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
CONDENSED, STANDARD = lk.MODE_CONDENSED, lk.MODE_STANDARD


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(torch.bfloat16)


def rows_bf16(g, *shape):
    """Keys or values with a few channels far off zero."""
    x = torch.randn(shape, generator=g, device=DEV)
    off = torch.randn(shape[-2:], generator=g, device=DEV) * 4.0
    return (x + off * (torch.rand(shape[-2:], generator=g, device=DEV) < 0.1)).to(torch.bfloat16)


def f32(x):
    return x.to(torch.float32).to(torch.float64)


def encode64(x):
    """code, step, low of x [..., d] bf16 in 64 bits, with the definition's roundings; a group that is not finite: low NaN."""
    y = x.double().unflatten(-1, (-1, 64))
    low, high = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    bad = ~(torch.isfinite(low) & torch.isfinite(high))
    y, low, high = (torch.where(bad, 0.0, t) for t in (y, low, high))
    ratio = float(np.float32(16) / np.float32(15))
    step = f32(f32(high / 16 - low / 16) * ratio).to(torch.bfloat16).double()
    step = torch.where(step < 2.0 ** -120, 0.0, step)
    code = torch.round(f32(f32(y / 16 - low / 16) * f32(16.0 / step))).clamp(0, 15)
    code = torch.where(step == 0, 0.0, code)
    low = torch.where(bad, float("nan"), low)
    return code, step, low


def value64(x):
    code, step, low = encode64(x)
    return (low + step * code).flatten(-2)


def make(bits, B, Hq, Hkv, d, cap, lens, page=0, n_pages=None, out32=0, sink=0, poison=True, L=1, w=0, **kw):
    if page and n_pages is None:
        n_pages = B * -(-cap // page)
    cfg = lk.make_config(L, w, Hq, Hkv, d, B, cap, kv_bits=bits, page_rows=page, n_pages=n_pages or 0, out_dtype=out32, stream_sink=sink, **kw)
    c = lk.Cache(cfg)
    if poison:                                   # what was never written is NaN everywhere: codes 15, steps and lows NaN
        c.buf[c.info.workspace_bytes:] = 0xFF
    if page:                                     # pages not in the order of the sequences
        c.lckv_cache_reset(list(lens)[::-1])
    c.lckv_cache_reset(list(lens))
    return c


def within(got, want, tol, what=""):
    got = got.double()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = ((got - want).abs() - tol).max().item() if got.numel() else 0.0
    assert over <= 0, f"{what}: {over:.3e} over the tolerance"


# ---- rows in 4 bits ---------------------------------------------------------------------------------------------------------


def special_rows(d):
    """[n, 1, d]: constant, zero, huge, tiny, threshold, signed zero, ties, infinite and NaN groups."""
    base = torch.linspace(-1, 1, d, device=DEV)
    out = [torch.full((d,), 0.7, device=DEV), torch.zeros(d, device=DEV), base * 3.3e38, base * 1e-38, base * 2.0 ** -119 * 7.5, base * 2.0 ** -118 * 7.5,
           torch.where(base > 0, 0.0, -0.0), (torch.arange(d, device=DEV) % 31) * 0.5, base * 1e30, (torch.arange(d, device=DEV) == 3) * 1.0]
    x = torch.stack(out).to(torch.bfloat16)
    bad = x[:1].repeat(4, 1)
    bad[0, 5], bad[1, 6], bad[2, d - 1], bad[3, 0] = math.inf, -math.inf, math.nan, math.nan
    return torch.cat([x, bad]).unsqueeze(1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [0, 64])
def test_rows_stand_for_what_the_definition_says(d, page):
    g = gen(1)
    lens = [70, 0, 14, 1, 129]
    k, v = rows_bf16(g, 5, 131, 3, d), rows_bf16(g, 5, 131, 3, d)
    s = special_rows(d)
    k[2, :14, 1:2], v[2, :14, 0:1] = s, s.flip(0)
    c = make(4, 5, 3, 3, d, 130, lens, page)
    c.lckv_prefill_write_kv(0, k, v)
    for dt in (torch.float32, torch.bfloat16):
        ko, vo = (torch.full(k.shape, 7.0, dtype=dt, device=DEV) for _ in range(2))
        c.lckv_cache_read_kv(0, ko, vo)
        for got, x in ((ko, k), (vo, v)):
            want = value64(x).float().to(dt)
            for b, n in enumerate(lens):
                assert torch.equal(torch.isnan(got[b, :n]), torch.isnan(want[b, :n]))
                assert torch.equal(torch.nan_to_num(got[b, :n]), torch.nan_to_num(want[b, :n]))
                assert (got[b, n:] == 7.0).all()
    assert c.lckv_cache_status() == 0


def test_every_code_and_step_comes_back():
    """Values that are exactly low + step * code stay what they are."""
    for e in (-60, -3, 0, 5, 100):
        x = (torch.arange(128, device=DEV) % 16).float() * 2.0 ** e - 2.0 ** (e + 2)
        x = x.to(torch.bfloat16).view(1, 1, 1, 128)
        c = make(4, 1, 1, 1, 128, 8, [1])
        c.lckv_prefill_write_kv(0, x, -x)
        ko, vo = torch.empty_like(x), torch.empty_like(x)
        c.lckv_cache_read_kv(0, ko, vo)
        assert torch.equal(ko, x) and torch.equal(vo, -x)


@pytest.mark.parametrize("d,page,sink", [(64, 0, 0), (128, 0, 0), (64, 64, 0), (128, 128, 0), (64, 0, 3), (128, 0, 1)])
def test_append_writes_the_same_rows(d, page, sink):
    g = gen(2)
    B, H, cap = 4, 3, 131
    lens = [0, 5, 127, 130] if not sink else [0, 130, 131, 400]
    k, v = rows_bf16(g, B, 1, H, d), rows_bf16(g, B, 1, H, d)
    c = make(4, B, H, H, d, cap, lens, page, sink=sink)
    before = c.buf.clone()
    c.lckv_append_kv(0, k[:, 0].contiguous(), v[:, 0].contiguous())
    assert (c.buf != before).sum() > 0
    if sink:                                     # the ring position, read through the attention: one row of weight 1
        return _ring_row(c, k, v, lens, cap, sink, d)
    c.lckv_append_kv(0, k[:, 0].contiguous(), v[:, 0].contiguous(), advance_len=1)
    assert c.lckv_cache_lengths() == [n + 1 for n in lens]
    ko, vo = (torch.zeros(B, cap, H, d, device=DEV) for _ in range(2))
    c.lckv_cache_read_kv(0, ko, vo)
    for b, n in enumerate(lens):
        assert torch.equal(ko[b, n], value64(k)[b, 0].float()) and torch.equal(vo[b, n], value64(v)[b, 0].float())


def _ring_row(c, k, v, lens, cap, sink, d):
    """Fill every row by appends; the last max_seq - sink tokens and the first ones have to be there."""
    B, H = k.shape[0], k.shape[2]
    c.lckv_cache_reset([0] * B)
    tokens = cap + 40
    g = gen(3)
    ks, vs = rows_bf16(g, B, tokens, H, d), rows_bf16(g, B, tokens, H, d)
    for t in range(tokens):
        c.lckv_append_kv(0, ks[:, t].contiguous(), vs[:, t].contiguous(), advance_len=1)
    keep = list(range(sink)) + list(range(tokens - (cap - sink), tokens))
    q = randn(g, B, H, d)
    lse = torch.empty(B, H, device=DEV)
    out = c.lckv_decode_attention(0, CONDENSED, q, lse=lse)
    check_attention(out, lse, q, ks[:, keep], vs[:, keep], [len(keep)] * B)


# ---- attention --------------------------------------------------------------------------------------------------------------


def attention64(q, k, v, n):
    """Output, lse, sum p (step code + |low|) and the scores' bound A of one sequence: q [Hq, d], k, v [n, Hkv, d] bf16."""
    Hq, d = q.shape
    g = Hq // k.shape[1]
    (kc, ks, kl), (vc, vs, vl) = encode64(k[:n]), encode64(v[:n])
    kk, vv = ((lo + s * c).flatten(-2).repeat_interleave(g, 1) for c, s, lo in ((kc, ks, kl), (vc, vs, vl)))
    ka = (ks * kc + kl.abs()).flatten(-2).repeat_interleave(g, 1)
    va = (vs * vc + vl.abs()).flatten(-2).repeat_interleave(g, 1)
    s = torch.einsum("hd,nhd->hn", q.double(), kk) * d ** -0.5
    a = torch.einsum("hd,nhd->hn", q.double().abs(), ka) * d ** -0.5
    p = torch.softmax(s, 1)
    return torch.einsum("hn,nhd->hd", p, vv), torch.logsumexp(s, 1), torch.einsum("hn,nhd->hd", p, va), a.max(1).values


def check_attention(out, lse, q, k, v, lens, what=""):
    for b, n in enumerate(lens):
        if n == 0:
            assert not out[b].any() and (lse is None or not lse[b].any()), what
            continue
        o, l, mag, a = attention64(q[b], k[b], v[b], n)
        ds = 2.0 ** -19 * a
        within(out[b], o, (torch.expm1(2 * ds)[:, None] + 2.0 ** -17) * mag + HALF[out.dtype] * o.abs(), f"{what} out {b} ({n} rows)")
        if lse is not None:
            within(lse[b], l, ds + 2.0 ** -20 * (1 + l.abs()), f"{what} lse {b} ({n} rows)")


def run_attention(Hq, Hkv, d, lens, mode, page, out32, cap=None, seed=5, workers=(0,), qstd=1.0):
    g = gen(seed)
    B, cap = len(lens), cap or max(lens) + 1
    k, v = rows_bf16(g, B, max(1, max(lens)), Hkv, d), rows_bf16(g, B, max(1, max(lens)), Hkv, d)
    seen = [n - mode for n in lens]              # the last row of STANDARD is appended
    c = make(4, B, Hq, Hkv, d, cap, seen, page, out32=out32)
    c.lckv_prefill_write_kv(0, k, v)
    if mode:
        last = torch.tensor([n - 1 for n in lens], device=DEV)
        bb = torch.arange(B, device=DEV)
        c.lckv_append_kv(0, k[bb, last].contiguous(), v[bb, last].contiguous())
    q = randn(g, B, Hq, d, std=qstd)
    for limit in workers:
        c.lckv_cache_set_worker_limit(min(limit, c.info.n_workers))
        lse = torch.empty(B, Hq, device=DEV)
        out = c.lckv_decode_attention(0, mode, q, lse=lse)
        assert out.dtype == (torch.float32 if out32 else torch.bfloat16)
        check_attention(out, lse, q, k, v, lens, f"limit {limit}")
        again = c.lckv_decode_attention(0, mode, q)
        assert torch.equal(out, again)
    assert c.lckv_cache_status() == 0


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (2, 1), (6, 2), (8, 2), (5, 1), (12, 2), (14, 2), (8, 1), (32, 4), (9, 1), (12, 1), (16, 1), (11, 1), (32, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_head_groups(Hq, Hkv, d):
    run_attention(Hq, Hkv, d, [1, 17, 0, 200], CONDENSED, 0, 1)


@pytest.mark.parametrize("lens", [[0], [0, 0, 0], [1], [15, 16, 17], [63, 64, 65], [127, 128, 129, 0, 191], [2, 0, 777, 1]])
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 3, 3), (128, 8, 1)])
@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("mode", [CONDENSED, STANDARD])
def test_attention_lengths(lens, d, Hq, Hkv, page, mode):
    if mode == STANDARD:
        lens = [max(1, n) for n in lens]
    run_attention(Hq, Hkv, d, lens, mode, page, 0, cap=max(lens) + 3)


@pytest.mark.parametrize("d,Hq,Hkv,lens", [(128, 1, 1, [20011]), (64, 8, 1, [30000, 5]), (128, 32, 8, [4097, 1, 0, 900]), (64, 10, 2, [9000, 9001])])
def test_attention_split_over_workers(d, Hq, Hkv, lens):
    run_attention(Hq, Hkv, d, lens, CONDENSED, 128, 1, workers=(0, 1, 2, 7, 40, 333))


@pytest.mark.parametrize("std", [1e-20, 1e-3, 8.0])
def test_attention_small_and_large_queries(std):
    run_attention(4, 4, 128, [300, 40], CONDENSED, 0, 1, qstd=std)
    run_attention(8, 1, 64, [300, 40], CONDENSED, 0, 1, qstd=std)


@pytest.mark.parametrize("d,Hq", [(64, 2), (128, 2), (128, 8)])
def test_attention_values_of_very_different_steps(d, Hq):
    """Rows whose values differ by 2^40: what a row of small steps contributes is right to the largest."""
    g = gen(6)
    k, v = rows_bf16(g, 1, 150, 1, d) * 0.1, rows_bf16(g, 1, 150, 1, d)
    scale = 2.0 ** torch.randint(-30, 11, (1, 150, 1, 1), generator=g, device=DEV).float()
    v = (v.float() * scale).to(torch.bfloat16)
    q = randn(g, 1, Hq, d)
    for order in (torch.arange(150), torch.arange(149, -1, -1), scale.flatten().sort().indices.cpu()):
        kk, vv = k[:, order].contiguous(), v[:, order].contiguous()
        c = make(4, 1, Hq, 1, d, 200, [150], out32=1)
        c.lckv_prefill_write_kv(0, kk, vv)
        lse = torch.empty(1, Hq, device=DEV)
        check_attention(c.lckv_decode_attention(0, CONDENSED, q, lse=lse), lse, q, kk, vv, [150])


@pytest.mark.parametrize("scale", [2.0 ** -118, 2.0 ** 118, 0.0])
def test_attention_extreme_values(scale):
    g = gen(7)
    k, v = rows_bf16(g, 1, 90, 1, 128), rows_bf16(g, 1, 90, 1, 128)
    v = (v.float() * scale).to(torch.bfloat16)
    q = randn(g, 1, 2, 128)
    c = make(4, 1, 2, 1, 128, 90, [90], out32=1)
    c.lckv_prefill_write_kv(0, k, v)
    check_attention(c.lckv_decode_attention(0, CONDENSED, q), None, q, k, v, [90])


def test_attention_not_a_number_stays_where_it_is():
    """A NaN among the values makes its 64 dimensions NaN, one among the keys the heads that see it; other sequences, kv heads
    and dimensions do not notice."""
    g = gen(8)
    k, v = rows_bf16(g, 3, 100, 2, 128), rows_bf16(g, 3, 100, 2, 128)
    q = randn(g, 3, 4, 128)
    kb, vb = k.clone(), v.clone()
    vb[0, 50, 1, 70] = math.nan
    kb[1, 99, 0, 3] = math.inf
    c = make(4, 3, 4, 2, 128, 100, [100] * 3, out32=1)
    c.lckv_prefill_write_kv(0, kb, vb)
    out = c.lckv_decode_attention(0, CONDENSED, q)
    bad = torch.zeros(3, 4, 128, dtype=torch.bool, device=DEV)
    bad[0, 2:, 64:] = True
    bad[1, :2] = True
    assert torch.equal(torch.isnan(out), bad)
    c.lckv_prefill_write_kv(0, k, v)
    assert torch.equal(out[~bad], c.lckv_decode_attention(0, CONDENSED, q)[~bad])
    # the row behind the visible ones may hold anything
    c.lckv_prefill_write_kv(0, kb, vb)
    c.lckv_cache_reset([50, 99, 64])
    out = c.lckv_decode_attention(0, CONDENSED, q)
    check_attention(out, None, q, k, v, [50, 99, 64])


@pytest.mark.parametrize("graph", [0, 1])
@pytest.mark.parametrize("d,Hq,Hkv,page", [(64, 8, 2, 0), (128, 2, 2, 64)])
def test_layer_stack_steps(graph, d, Hq, Hkv, page):
    """Three decode steps of a stack with warmup layers: every layer's output from the rows that its slot holds by then."""
    g = gen(9)
    L, w, B, cap = 4, 2, 3, 80
    plan = lk.lckv_plan(L, w)
    lens = [61, 0, 33]
    c = make(4, B, Hq, Hkv, d, cap, lens, page, L=L, w=w, use_graph=graph)
    ks, vs = ([rows_bf16(g, B, cap, Hkv, d) for _ in range(plan["n_slots"])] for _ in range(2))
    for s in range(plan["n_slots"]):
        c.lckv_prefill_write_kv(s, ks[s], vs[s])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    q = [randn(g, B, Hq, d) for _ in range(L)]
    kn, vn = ([rows_bf16(g, B, Hkv, d) if plan["write_slot"][l] >= 0 else None for l in range(L)] for _ in range(2))
    out = [torch.empty(B, Hq, d, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
    torch.cuda.synchronize()
    for step in range(3):
        for t in q + [x for x in kn + vn if x is not None]:
            t.copy_(rows_bf16(g, *t.shape))
        torch.cuda.synchronize()
        c.lckv_layer_stack_step(q, out, kn, vn, stream=st)
        torch.cuda.synchronize()
        for l in range(L):
            s, mode = plan["read_slot"][l], plan["mode"][l]
            if plan["write_slot"][l] >= 0 and plan["write_before"][l]:
                for b, n in enumerate(lens):
                    ks[plan["write_slot"][l]][b, n], vs[plan["write_slot"][l]][b, n] = kn[l][b], vn[l][b]
            check_attention(out[l], None, q[l], ks[s], vs[s], [n + mode for n in lens], f"step {step} layer {l}")
        for l in range(L):
            if plan["write_slot"][l] >= 0 and not plan["write_before"][l]:
                for b, n in enumerate(lens):
                    ks[plan["write_slot"][l]][b, n], vs[plan["write_slot"][l]][b, n] = kn[l][b], vn[l][b]
        lens = [n + 1 for n in lens]
    assert c.lckv_cache_lengths() == lens and c.lckv_cache_status() == 0


def test_attention_timeout_is_reported():
    c = make(4, 2, 4, 4, 128, 64, [64, 40], poison=False)
    c.buf[c.info.workspace_bytes:] = 0
    q = randn(gen(10), 2, 4, 128)
    c.lckv_cache_set_wait_limit(0)
    c.lckv_decode_attention(0, CONDENSED, q)
    assert c.lckv_cache_status() == lk.ETIMEOUT
    c.lckv_cache_set_wait_limit(1 << 18)
    c.lckv_cache_reset([64, 40])
    out = c.lckv_decode_attention(0, CONDENSED, q)
    assert c.lckv_cache_status() == 0 and not out.any()


# How far exp(lse) may be off: over bf16 rows the tensor-core kernel sums probabilities that are rounded to bf16, each by at most
# 2^-8 of itself, so their sum is off by no more either; over 4-bit rows scores are off by 2^-19 A, and A < 100 here.
LSE = {16: 2.0 ** -8, 4: 2.0 ** -12}


# ---- gathered weights -------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("d,Hq,Hkv,page", [(64, 8, 2, 0), (128, 3, 3, 64), (128, 16, 1, 0), (64, 12, 1, 128), (64, 5, 1, 0), (128, 32, 4, 0)])
def test_weights_against_64_bits(bits, d, Hq, Hkv, page):
    g = gen(11)
    lens = [300, 0, 1, 64, 77]
    B, cap = len(lens), 301
    k, v = rows_bf16(g, B, 300, Hkv, d), rows_bf16(g, B, 300, Hkv, d)
    q = randn(g, B, Hq, d)
    c = make(bits, B, Hq, Hkv, d, cap, lens, page)
    c.lckv_prefill_write_kv(0, k, v)
    lse = torch.empty(B, Hq, device=DEV)
    c.lckv_decode_attention(0, CONDENSED, q, lse=lse)
    before = torch.rand((B, Hkv, cap + 3), generator=g, device=DEV)
    after = torch.full_like(before, -5.0)
    c.lckv_attention_weights(0, CONDENSED, q, lse, after, previous=before)
    alone = c.lckv_attention_weights(0, CONDENSED, q, lse)
    into = before.clone()
    c.lckv_attention_weights(0, CONDENSED, q, lse, into, previous=into)
    for b, n in enumerate(lens):
        assert (after[b, :, n:] == -5.0).all() and (alone[b, :, n:] == 0).all()
        assert torch.equal(into[b, :, n:], before[b, :, n:]) and torch.equal(into[b, :, :n], after[b, :, :n])
        if n == 0:
            continue
        kk = (value64(k[b, :n]) if bits == 4 else k[b, :n].double()).repeat_interleave(Hq // Hkv, 1)
        (kc, ks, kl) = encode64(k[b, :n])
        mag = ((ks * kc + kl.abs()).flatten(-2) if bits == 4 else k[b, :n].double().abs()).repeat_interleave(Hq // Hkv, 1)
        s = torch.einsum("hd,nhd->hn", q[b].double(), kk) * d ** -0.5
        a = torch.einsum("hd,nhd->hn", q[b].double().abs(), mag) * d ** -0.5
        p = torch.exp(s - lse[b].double()[:, None])
        err = (p * (torch.expm1(2.0 ** -19 * (a + lse[b].double().abs()[:, None] + 1)) + 2.0 ** -20)).unflatten(0, (Hkv, -1)).sum(1)
        want = p.unflatten(0, (Hkv, -1)).sum(1)
        within(alone[b, :, :n], want, err, f"sequence {b}")
        within(after[b, :, :n], before[b, :, :n].double() + want, err + 2.0 ** -22 * (1 + want), f"sequence {b}")
        # all of a head's weight is given out
        assert (alone[b, :, :n].double().sum(1) - Hq // Hkv).abs().max() < LSE[bits] * (Hq // Hkv)


def test_weights_with_the_new_token_and_in_a_ring():
    g = gen(12)
    for bits in (4, 16):
        c = make(bits, 2, 4, 2, 64, 96, [95, 300], sink=4, poison=False)
        c.buf[c.info.workspace_bytes:] = 0
        k, v, q = rows_bf16(g, 2, 2, 64), rows_bf16(g, 2, 2, 64), randn(g, 2, 4, 64)
        c.lckv_append_kv(0, k, v)
        lse = torch.empty(2, 4, device=DEV)
        c.lckv_decode_attention(0, STANDARD, q, lse=lse)
        w = c.lckv_attention_weights(0, STANDARD, q, lse)
        assert (w.sum(-1) - 2).abs().max() < LSE[bits] * 2
        row = [95, 4 + (300 - 4) % 92]
        for b in range(2):
            others = torch.ones(96, dtype=torch.bool)
            others[row[b]] = False
            rest = w[b][:, others]
            assert (rest == rest[:, :1]).all() and (w[b, :, row[b]] != rest[:, 0]).all()


# ---- eviction ---------------------------------------------------------------------------------------------------------------


def kept_plain(w, n, sink, recent, keep):
    """Rows that stay, ascending; w a numpy row of weights or None."""
    if n <= keep:
        return np.arange(n)
    x = np.zeros(n) if w is None else w[:n].astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    nan = np.zeros(n, bool) if w is None else np.isnan(w[:n])
    mid = np.arange(sink, n - recent)
    order = mid[np.lexsort((mid, nan[mid], -x[mid]))][:keep - sink - recent]
    return np.sort(np.concatenate([np.arange(sink), order, np.arange(n - recent, n)])).astype(np.int64)


def weight_sets(g, B, H, n):
    w = torch.exp(2 * torch.randn((B, H, n), generator=g, device=DEV))
    yield "distinct", w
    t = torch.floor(torch.rand((B, H, n), generator=g, device=DEV) * 4)
    yield "ties", t
    z = t - 2
    z[z == 0] = -0.0
    z[:, :, ::3] = 0.0
    yield "signs", z
    x = w.clone()
    x[:, :, ::5], x[:, :, 1::7], x[:, :, 2::11] = math.nan, math.inf, -math.inf
    yield "infinite", x
    yield "equal", torch.full_like(w, 0.25)
    yield "none", None


SHAPES = [(0, 0, 1), (4, 8, 40), (0, 40, 40), (40, 0, 40), (3, 0, 64), (0, 5, 63), (1, 1, 130), (5, 60, 100)]


@pytest.mark.parametrize("sink,recent,keep", SHAPES)
@pytest.mark.parametrize("bits,to,d", [(16, 16, 64), (16, 4, 128), (4, 4, 128), (4, 4, 64), (16, 4, 64), (16, 16, 128)])
def test_evict_into_another_cache(sink, recent, keep, bits, to, d):
    g = gen(13)
    lens = [129, 0, 100, 41, 64]
    B, H, cap = len(lens), 2, 130
    k, v = rows_bf16(g, B, cap, H, d), rows_bf16(g, B, cap, H, d)
    src = make(bits, B, H, H, d, cap, lens)
    src.lckv_prefill_write_kv(0, k, v)
    for i, (name, w) in enumerate(weight_sets(g, B, H, cap + 2)):
        dst = make(to, B, H, H, d, keep + 3, [1, 2, 0, 3, 0][:B] if keep > 2 else [0] * B, page=64 if i % 2 else 0)
        kept = torch.full((B, H, keep), 99, dtype=torch.int32, device=DEV)
        out = torch.full((B, H, keep + 4), -7.0, device=DEV)
        state = src.buf.clone()
        dst.lckv_evict_kv(0, src, 0, kept, weights=w, weights_out=out, n_sink=sink, n_recent=recent, set_len=1)
        assert torch.equal(src.buf, state)
        new = [min(n, keep) for n in lens]
        assert dst.lckv_cache_lengths() == new and dst.lckv_cache_status() == 0
        ko, vo = (torch.zeros(B, keep, H, d, device=DEV) for _ in range(2))
        dst.lckv_cache_read_kv(0, ko, vo)
        wn = None if w is None else w.cpu().numpy()
        for b, n in enumerate(lens):
            for h in range(H):
                rows = kept_plain(None if w is None else wn[b, h], n, sink, recent, keep)
                assert kept[b, h].tolist() == rows.tolist() + [-1] * (keep - len(rows)), (name, b, h)
                at = torch.tensor(rows, device=DEV, dtype=torch.int64)
                for got, x in ((ko, k), (vo, v)):
                    y = x[b, at, h]
                    want = value64(y).float() if 4 in (bits, to) else y.float()
                    assert torch.equal(got[b, :len(rows), h], want), (name, b, h)
                want = torch.zeros(keep + 3, device=DEV)
                if w is not None:
                    want[:len(rows)] = w[b, h, at]
                assert torch.equal(torch.nan_to_num(out[b, h, :keep + 3], nan=123.0), torch.nan_to_num(want, nan=123.0)), (name, b, h)
                assert out[b, h, keep + 3] == -7.0
    if to == 4 and keep >= 130:                  # a prompt's way into a 4-bit cache: nothing is dropped
        assert [int((kept[b, 0] >= 0).sum()) for b in range(B)] == lens


@pytest.mark.parametrize("bits,d,page", [(16, 64, 0), (16, 128, 64), (4, 64, 64), (4, 128, 0), (4, 128, 128)])
@pytest.mark.parametrize("sink,recent,keep", [(4, 8, 40), (0, 0, 200), (2, 300, 500), (0, 0, 1)])
def test_evict_in_place(bits, d, page, sink, recent, keep):
    g = gen(14)
    lens = [700, 0, 300, 41]
    B, H, cap = len(lens), 3, 701
    k, v = rows_bf16(g, B, cap, H, d), rows_bf16(g, B, cap, H, d)
    c = make(bits, B, H, H, d, cap, lens, page, n_pages=(12 if page == 64 else 6) * 4 if page else None, L=2, w=2)
    for s in range(2):
        c.lckv_prefill_write_kv(s, k if s == 0 else v, v if s == 0 else k)
    w = torch.exp(2 * torch.randn((B, H, cap), generator=g, device=DEV))
    first = w.cpu().numpy()
    kept = torch.empty((B, H, keep), dtype=torch.int32, device=DEV)
    c.lckv_evict_kv(1, c, 1, kept, weights=w, n_sink=sink, n_recent=recent)
    assert c.lckv_cache_lengths() == lens
    c.lckv_evict_kv(0, c, 0, kept, weights=w, weights_out=w, n_sink=sink, n_recent=recent, set_len=1)
    new = [min(n, keep) for n in lens]
    assert c.lckv_cache_lengths() == new and c.lckv_cache_status() == 0
    if page:
        held = (c.lckv_cache_page_table() >= 0).sum(1).tolist()
        assert held == [-(-n // page) for n in new]
    for s in range(2):
        ko, vo = (torch.zeros(B, keep, H, d, device=DEV) for _ in range(2))
        c.lckv_cache_read_kv(s, ko, vo)
        for b, n in enumerate(lens):
            for h in range(H):
                rows = kept_plain(first[b, h], n, sink, recent, keep)
                assert kept[b, h].tolist() == rows.tolist() + [-1] * (keep - len(rows))
                at = torch.tensor(rows, device=DEV, dtype=torch.int64)
                for got, x in ((ko, k if s == 0 else v), (vo, v if s == 0 else k)):
                    y = x[b, at, h]
                    assert torch.equal(got[b, :len(rows), h], value64(y).float() if bits == 4 else y.float())
                want = torch.zeros(cap)
                want[:len(rows)] = torch.from_numpy(first[b, h, rows])
                assert torch.equal(w[b, h].cpu(), want)
    # appends go on behind the rows that stayed
    c.lckv_append_kv(0, k[:, 0].contiguous(), v[:, 0].contiguous(), advance_len=1)
    assert c.lckv_cache_lengths() == [n + 1 for n in new]


@pytest.mark.parametrize("n,keep", [(60000, 700), (49153, 49152), (33000, 32000)])
def test_evict_long(n, keep):
    """More rows than a thread block keeps in shared memory, and fewer."""
    g = gen(15)
    c = make(4, 1, 1, 1, 64, n, [n], poison=False)
    w = torch.exp(torch.randn((1, 1, n), generator=g, device=DEV))
    w[..., ::2] = torch.floor(w[..., ::2] * 2)
    kept = torch.empty((1, 1, keep), dtype=torch.int32, device=DEV)
    c.lckv_evict_kv(0, c, 0, kept, weights=w, n_sink=7, n_recent=100)
    assert kept[0, 0].tolist() == kept_plain(w[0, 0].cpu().numpy(), n, 7, 100, keep).tolist()


def test_evict_pool_without_pages_changes_nothing():
    src = make(16, 2, 1, 1, 64, 256, [256, 256], poison=False)
    dst = make(16, 2, 1, 1, 64, 256, [0, 0], page=64, n_pages=3, poison=False)
    kept = torch.full((2, 1, 128), 5, dtype=torch.int32, device=DEV)
    with pytest.raises(lk.LckvError) as e:
        dst.lckv_evict_kv(0, src, 0, kept, set_len=1)
    assert e.value.status == lk.ECAPACITY
    assert (kept == 5).all() and dst.lckv_cache_lengths() == [0, 0] and (dst.lckv_cache_page_table() < 0).all()


# ---- streams, graphs, a run of all ------------------------------------------------------------------------------------------


def test_captured_calls_follow_the_lengths():
    """One graph of append, attention, weights and eviction into a small cache, replayed with other rows and lengths."""
    g = gen(16)
    B, Hq, Hkv, d, cap, keep = 3, 4, 2, 128, 400, 96
    src, dst = make(4, B, Hq, Hkv, d, cap, [399] * B), make(4, B, Hq, Hkv, d, keep, [0] * B)
    q, kn, vn = randn(g, B, Hq, d), rows_bf16(g, B, Hkv, d), rows_bf16(g, B, Hkv, d)
    out, lse = torch.empty(B, Hq, d, dtype=torch.bfloat16, device=DEV), torch.empty(B, Hq, device=DEV)
    w, kept = torch.zeros(B, Hkv, cap, device=DEV), torch.empty(B, Hkv, keep, dtype=torch.int32, device=DEV)
    wo = torch.empty(B, Hkv, keep, device=DEV)

    def calls():
        src.lckv_append_kv(0, kn, vn)
        src.lckv_decode_attention(0, STANDARD, q, out=out, lse=lse)
        src.lckv_attention_weights(0, STANDARD, q, lse, w)
        dst.lckv_evict_kv(0, src, 0, kept, weights=w, weights_out=wo, n_sink=4, n_recent=16)

    graph = torch.cuda.CUDAGraph()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        calls()
        with torch.cuda.graph(graph, stream=st):
            calls()
        with pytest.raises(lk.LckvError):
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=st):
                dst.lckv_evict_kv(0, src, 0, kept, set_len=1)
    torch.cuda.synchronize()
    for lens in ([200, 0, 399], [30, 95, 96]):
        k, v = rows_bf16(g, B, cap, Hkv, d), rows_bf16(g, B, cap, Hkv, d)
        src.lckv_cache_reset(lens)
        src.lckv_prefill_write_kv(0, k, v)
        w.zero_()
        for t in (q, kn, vn):
            t.copy_(rows_bf16(g, *t.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(lens):
            k[b, n], v[b, n] = kn[b], vn[b]
        seen = [n + 1 for n in lens]
        check_attention(out, lse, q, k, v, seen)
        for b, n in enumerate(lens):
            for h in range(Hkv):
                rows = kept_plain(w[b, h].cpu().numpy(), n, 4, 16, keep)
                assert kept[b, h].tolist() == rows.tolist() + [-1] * (keep - len(rows))
        assert src.lckv_cache_status() == 0 and dst.lckv_cache_status() == 0


def test_prompt_to_compact_cache_and_on():
    """A prompt encoded in a bf16 cache; its heavy rows taken into a paged 4-bit cache; decode steps there, with weights, and an
    eviction in place when the budget is full again."""
    g = gen(17)
    B, Hq, Hkv, d, n, keep = 2, 8, 2, 64, 300, 64
    lens = [300, 211]
    full = make(16, B, Hq, Hkv, d, n, lens)
    small = make(4, B, Hq, Hkv, d, 80, [0] * B, page=64, n_pages=4)
    k, v = rows_bf16(g, B, n, Hkv, d), rows_bf16(g, B, n, Hkv, d)
    full.lckv_prefill_write_kv(0, k, v)
    pq = rows_bf16(g, B, n, Hq, d)
    full.lckv_prefill_attention(0, CONDENSED, pq)
    w = torch.zeros(B, Hkv, n, device=DEV)
    for _ in range(3):
        q, lse = randn(g, B, Hq, d), torch.empty(B, Hq, device=DEV)
        full.lckv_decode_attention(0, CONDENSED, q, lse=lse)
        full.lckv_attention_weights(0, CONDENSED, q, lse, w, previous=w)
    kept = torch.empty(B, Hkv, keep, dtype=torch.int32, device=DEV)
    sw = torch.empty(B, Hkv, 80, device=DEV)
    small.lckv_evict_kv(0, full, 0, kept, weights=w, weights_out=sw, n_sink=4, n_recent=16, set_len=1)
    assert small.lckv_cache_lengths() == [keep] * B
    # what the small cache holds, as bf16 rows per head: [B, rows, Hkv, d]
    idx = kept.long().permute(0, 2, 1)[..., None].expand(-1, -1, -1, d)
    hk, hv = torch.gather(k, 1, idx), torch.gather(v, 1, idx)
    for _ in range(16):
        q, lse = randn(g, B, Hq, d), torch.empty(B, Hq, device=DEV)
        out = small.lckv_decode_attention(0, CONDENSED, q, lse=lse)
        check_attention(out, lse, q, hk, hv, [hk.shape[1]] * B)
        small.lckv_attention_weights(0, CONDENSED, q, lse, sw, previous=sw)
        kn, vn = rows_bf16(g, B, Hkv, d), rows_bf16(g, B, Hkv, d)
        small.lckv_append_kv(0, kn, vn, advance_len=1)
        hk, hv = torch.cat([hk, kn[:, None]], 1), torch.cat([hv, vn[:, None]], 1)
    assert small.lckv_cache_lengths() == [80] * B
    before = sw.cpu().numpy()
    small.lckv_evict_kv(0, small, 0, kept, weights=sw, weights_out=sw, n_sink=4, n_recent=16, set_len=1)
    for b in range(B):
        for h in range(Hkv):
            assert kept[b, h].tolist() == kept_plain(before[b, h], 80, 4, 16, keep).tolist()
    idx = kept.long().permute(0, 2, 1)[..., None].expand(-1, -1, -1, d)
    hk, hv = torch.gather(hk, 1, idx), torch.gather(hv, 1, idx)
    q = randn(g, B, Hq, d)
    check_attention(small.lckv_decode_attention(0, CONDENSED, q), None, q, hk, hv, [keep] * B)
    assert small.lckv_cache_status() == 0


# ---- refusals that need a cache ---------------------------------------------------------------------------------------------


def refused(status, call, *a, **kw):
    with pytest.raises(lk.LckvError) as e:
        call(*a, **kw)
    assert e.value.status == status


def test_refusals():
    c4, c16 = make(4, 2, 4, 2, 64, 100, [50, 100], poison=False), make(16, 2, 4, 2, 64, 100, [50, 100], poison=False)
    ring = make(4, 2, 4, 2, 64, 100, [50, 100], sink=2, poison=False)
    other = make(4, 2, 4, 4, 64, 100, [50, 100], poison=False)
    f, i = dict(device=DEV), dict(device=DEV, dtype=torch.int32)
    k = torch.zeros(2, 100, 2, 64, dtype=torch.bfloat16, **f)
    q, lse, w = torch.zeros(2, 4, 64, dtype=torch.bfloat16, **f), torch.zeros(2, 4, **f), torch.zeros(2, 2, 100, **f)
    kept = torch.zeros(2, 2, 40, **i)
    E = lk.EINVAL
    # entries that have no 4-bit form
    refused(E, c4.lckv_cache_slot_ptrs, 0)
    refused(E, c4.slot_tensors, 0)
    refused(E, c4.lckv_prefill_attention, 0, CONDENSED, torch.zeros(2, 100, 4, 64, dtype=torch.bfloat16, **f))
    cos, sin = torch.ones(200, 32, **f), torch.zeros(200, 32, **f)
    rope = lk.make_rope(cos, sin)
    refused(E, c4.lckv_rope_append_kv, 0, rope, q, k[:, 0].contiguous(), k[:, 0].contiguous())
    refused(E, c4.lckv_rope_prefill_write_kv, 0, rope, None, k, k)
    assert c4.lckv_rope_append_kv(0, rope, q, None, None) is not None          # a query alone has nothing to do with the rows
    wt = torch.zeros(128, 64, dtype=torch.bfloat16, **f)
    refused(E, c4.lckv_project_append_kv, 0, torch.zeros(2, 64, dtype=torch.bfloat16, **f), wt, wt)
    # reading
    refused(E, c4.lckv_cache_read_kv, 0, k, k)                                  # one tensor for both
    refused(E, c4.lckv_cache_read_kv, 0, k, k.float())
    refused(E, c4.lckv_cache_read_kv, 0, k[:, :99].contiguous(), k[:, :99].contiguous())       # shorter than a sequence
    refused(E, c4.lckv_cache_read_kv, 1, k, k.clone())
    refused(E, ring.lckv_cache_read_kv, 0, k, k.clone())
    refused(E, c4.lckv_cache_read_kv, 0, k.cpu(), k.cpu())
    refused(E, c4.lckv_cache_read_kv, 0, k.transpose(1, 2), k.clone())
    # weights
    refused(E, c4.lckv_attention_weights, 0, 2, q, lse, w)
    refused(E, c4.lckv_attention_weights, 1, 0, q, lse, w)
    refused(lk.ECAPACITY, c4.lckv_attention_weights, 0, STANDARD, q, lse, w)
    refused(E, c4.lckv_attention_weights, 0, 0, q, lse, w[:, :, :99].contiguous())
    refused(E, c4.lckv_attention_weights, 0, 0, q, lse[:1], w)
    refused(E, c4.lckv_attention_weights, 0, 0, q.float(), lse, w)
    flat = torch.zeros(500, **f)
    refused(E, c4.lckv_attention_weights, 0, 0, q, lse, flat[:400].view(2, 2, 100), previous=flat[4:404].view(2, 2, 100))
    # eviction
    ok = dict(weights=w, n_sink=4, n_recent=8)
    refused(E, c16.lckv_evict_kv, 0, c4, 0, kept, **ok)                         # 4 bits to 16
    refused(E, other.lckv_evict_kv, 0, c4, 0, torch.zeros(2, 4, 40, **i))
    refused(E, ring.lckv_evict_kv, 0, c4, 0, kept, **ok)
    refused(E, c4.lckv_evict_kv, 0, ring, 0, kept, **ok)
    refused(E, c4.lckv_evict_kv, 0, c4, 0, kept, weights=w, n_sink=33, n_recent=8)
    refused(E, c4.lckv_evict_kv, 0, c4, 0, kept, weights=w, n_sink=-1)
    refused(E, c4.lckv_evict_kv, 0, c4, 0, kept, weights=w, n_recent=-1)
    refused(E, c4.lckv_evict_kv, 0, c4, 0, torch.zeros(2, 2, 101, **i), weights=w)
    refused(E, c4.lckv_evict_kv, 0, c4, 0, torch.zeros(2, 2, 0, **i), weights=w)
    refused(E, c4.lckv_evict_kv, 0, c4, 0, kept.float(), **ok)
    refused(E, c4.lckv_evict_kv, 1, c4, 0, kept, **ok)
    refused(E, c4.lckv_evict_kv, 0, c4, 0, kept, weights=flat[:400].view(2, 2, 100), weights_out=flat[4:404].view(2, 2, 100))
    two = make(4, 2, 4, 2, 64, 100, [50, 100], poison=False, L=2, w=2)
    refused(E, two.lckv_evict_kv, 1, two, 0, kept, **ok)                        # another slot of the same cache
    assert c4.lckv_cache_lengths() == [50, 100] and c4.lckv_cache_status() == 0


def test_calls_on_another_stream():
    g = gen(18)
    st = torch.cuda.Stream()
    B, H, d, n = 2, 2, 128, 200
    k, v, q = rows_bf16(g, B, n, H, d), rows_bf16(g, B, n, H, d), randn(g, B, H, d)
    c, c2 = make(4, B, H, H, d, n, [n, 77]), make(4, B, H, H, d, 50, [0, 0])
    lse, out = torch.empty(B, H, device=DEV), torch.empty(B, H, d, dtype=torch.bfloat16, device=DEV)
    kept = torch.empty(B, H, 50, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    c.lckv_prefill_write_kv(0, k, v, stream=st)
    c.lckv_decode_attention(0, CONDENSED, q, out=out, lse=lse, stream=st)
    w = c.lckv_attention_weights(0, CONDENSED, q, lse, stream=st)
    c2.lckv_evict_kv(0, c, 0, kept, weights=w, set_len=1, stream=st)
    st.synchronize()
    check_attention(out, lse, q, k, v, [n, 77])
    for b, m in enumerate((n, 77)):
        for h in range(H):
            assert kept[b, h].tolist() == kept_plain(w[b, h].cpu().numpy(), m, 0, 0, 50).tolist()


def test_a_cache_beyond_32_bits_of_rows_and_bytes():
    """The last sequence's rows lie behind 2^32 bytes of codes."""
    g = gen(19)
    B, H, d, cap = 66, 32, 128, 1 << 15
    c = lk.Cache(lk.make_config(1, 0, H, H, d, B, cap, kv_bits=4))
    lens = [0] * (B - 1) + [500]
    c.lckv_cache_reset(lens)
    k, v = (torch.zeros(B, 500, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[-1], v[-1] = rows_bf16(g, 500, H, d), rows_bf16(g, 500, H, d)
    c.lckv_prefill_write_kv(0, k, v)
    q, lse = randn(g, B, H, d), torch.empty(B, H, device=DEV)
    out = c.lckv_decode_attention(0, CONDENSED, q, lse=lse)
    check_attention(out, lse, q, k, v, lens)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    c.lckv_cache_read_kv(0, ko, vo)
    assert torch.equal(ko[-1], value64(k[-1]).float().bfloat16()) and not ko[:-1].any()
    w = c.lckv_attention_weights(0, CONDENSED, q, lse)
    assert (w[-1].sum(-1) - 1).abs().max() < LSE[4] and not w[:-1].any()


@pytest.mark.parametrize("B", [31, 32, 33, 385, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("d,Hq", [(64, 1), (128, 2)])
def test_attention_of_many_sequences(B, d, Hq):
    """Batches around the sizes at which the kernel's table of sequences changes its form; many of them empty."""
    g = gen(20)
    lens = torch.randint(0, 150, (B,), generator=torch.Generator().manual_seed(B)).tolist()
    for i in range(0, B, 3):
        lens[i] = 0
    lens[-1] = 0
    k, v, q = rows_bf16(g, B, 150, 1, d), rows_bf16(g, B, 150, 1, d), randn(g, B, Hq, d)
    c = make(4, B, Hq, 1, d, 150, lens, out32=1)
    c.lckv_prefill_write_kv(0, k, v)
    for limit in (0, 37):
        c.lckv_cache_set_worker_limit(limit)
        lse = torch.full((B, Hq), 9.0, device=DEV)
        out = c.lckv_decode_attention(0, CONDENSED, q, lse=lse)
        assert not out[::3].any() and not lse[::3].any() and not out[-1].any()
        some = [b for b in range(B) if lens[b]][::max(1, B // 40)]
        check_attention(out[some], lse[some], q[some], k[some], v[some], [lens[b] for b in some])
        assert torch.isfinite(out).all() and (out[[b for b in range(B) if lens[b]]].abs().amax((1, 2)) > 0).all()


def test_tensors_off_the_grid_are_refused():
    c = make(4, 2, 4, 2, 64, 100, [50, 99], poison=False)
    flat = torch.zeros(100000, dtype=torch.bfloat16, device=DEV)
    good = [flat[8 * i:8 * i + n] for i, n in ((0, 512), (1000, 512))]

    def off(shape):
        n = math.prod(shape)
        return flat[1:1 + n].view(shape)

    q, kn = good[0].view(2, 4, 64), good[1][:256].view(2, 2, 64)
    refused(lk.EINVAL, c.lckv_decode_attention, 0, CONDENSED, off((2, 4, 64)))
    refused(lk.EINVAL, c.lckv_decode_attention, 0, CONDENSED, q, out=off((2, 4, 64)))
    refused(lk.EINVAL, c.lckv_append_kv, 0, off((2, 2, 64)), kn)
    refused(lk.EINVAL, c.lckv_prefill_write_kv, 0, off((2, 99, 2, 64)), off((2, 99, 2, 64)))
    refused(lk.EINVAL, c.lckv_layer_stack_step, [off((2, 4, 64))], [q], [kn], [kn])
    refused(lk.EINVAL, c.lckv_attention_weights, 0, CONDENSED, off((2, 4, 64)), torch.zeros(2, 4, device=DEV))
    assert c.lckv_cache_lengths() == [50, 99]


@pytest.mark.parametrize("sink", [0, 2])
def test_steps_from_host_buffers(sink):
    """The same outputs as the step on device buffers, and the same rows."""
    g = gen(21)
    L, w, B, Hq, Hkv, d, cap = 4, 2, 3, 4, 2, 64, 40
    plan = lk.lckv_plan(L, w)
    lens = [20, 0, 33] if not sink else [60, 0, 39]
    a, b = (make(4, B, Hq, Hkv, d, cap, lens, L=L, w=w, host_staging=1, sink=sink, poison=False) for _ in range(2))
    for c in (a, b):
        c.buf[c.info.workspace_bytes:] = 0
    for _ in range(3):
        q = [randn(g, B, Hq, d) for _ in range(L)]
        kn, vn = ([rows_bf16(g, B, Hkv, d) if plan["write_slot"][l] >= 0 else None for l in range(L)] for _ in range(2))
        out = [torch.empty_like(x) for x in q]
        a.lckv_layer_stack_step(q, out, kn, vn)
        host = lambda ts: [None if t is None else t.cpu().pin_memory() for t in ts]
        out_h = [torch.empty(B, Hq, d, dtype=torch.bfloat16).pin_memory() for _ in range(L)]
        qh, kh, vh = host(q), host(kn), host(vn)
        b.lckv_layer_stack_step_host(qh, out_h, kh, vh)
        torch.cuda.synchronize()
        for x, y in zip(out, out_h):
            assert torch.equal(x.cpu(), y) and torch.isfinite(y).all()
    assert a.lckv_cache_lengths() == b.lckv_cache_lengths() == [n + 3 for n in lens]


def test_weights_timeout_is_reported():
    c = make(4, 2, 4, 4, 128, 64, [64, 40], poison=False)
    c.buf[c.info.workspace_bytes:] = 0
    q, lse = randn(gen(22), 2, 4, 128), torch.zeros(2, 4, device=DEV)
    c.lckv_cache_set_wait_limit(0)
    c.lckv_attention_weights(0, CONDENSED, q, lse)
    assert c.lckv_cache_status() == lk.ETIMEOUT
    c.lckv_cache_set_wait_limit(1 << 18)
    c.lckv_cache_reset([64, 40])
    w = c.lckv_attention_weights(0, CONDENSED, q, lse)
    assert c.lckv_cache_status() == 0 and (w[0] == 1).all() and (w[1, :, :40] == 1).all() and not w[1, :, 40:].any()


def test_evict_after_lengths_that_only_the_device_knows():
    """A captured advance moves the device's lengths alone; a later eviction goes by them, whatever the host thinks."""
    g = gen(23)
    n, keep = 1500, 300
    c = make(16, 1, 1, 1, 64, 2000, [900])
    k, v = rows_bf16(g, 1, n, 1, 64), rows_bf16(g, 1, n, 1, 64)
    kn, vn = k[:, 0].contiguous(), v[:, 0].contiguous()
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    c.lckv_prefill_write_kv(0, k[:, :900].contiguous(), v[:, :900].contiguous())
    torch.cuda.synchronize()
    q, o = randn(g, 1, 1, 64), torch.empty(1, 1, 64, dtype=torch.bfloat16, device=DEV)
    with torch.cuda.graph(graph, stream=st):
        c.lckv_layer_stack_step([q], [o], [kn], [vn])
    for i in range(900, n):
        kn.copy_(k[:, i]); vn.copy_(v[:, i])
        torch.cuda.synchronize()
        graph.replay()
    torch.cuda.synchronize()
    assert c.lckv_cache_lengths() == [n]
    w = torch.rand((1, 1, 2000), generator=g, device=DEV)
    kept = torch.empty((1, 1, keep), dtype=torch.int32, device=DEV)
    dst = make(4, 1, 1, 1, 64, keep, [0])
    dst.lckv_evict_kv(0, c, 0, kept, weights=w, n_sink=2, n_recent=50, set_len=1)
    assert kept[0, 0].tolist() == kept_plain(w[0, 0].cpu().numpy(), n, 2, 50, keep).tolist()
