"""The forms that sizes choose among: selection at the limits of its thread blocks, rows read back one and four a thread, gathered weights
of two tiles a warp and of sequences that outgrew a captured launch."""
import math

import pytest
import torch

from test_gpu_compact_caches import CONDENSED, DEV, gen, kept_plain, make, randn, rows_bf16, value64, within

pytestmark = pytest.mark.gpu


def weights_of(kind, g, shape):
    w = torch.exp(2 * torch.randn(shape, generator=g, device=DEV))
    if kind == "ties":
        w = torch.floor(torch.rand(shape, generator=g, device=DEV) * 5) - 2.0
        w[w == 0] = -0.0
    if kind == "infinite":
        w[..., ::5], w[..., 1::7], w[..., 2::11] = math.nan, math.inf, -math.inf
    return w


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2500, 4096, 4097, 6001, 8192, 8193, 16384, 16385, 20000, 32767, 32768, 32769])
@pytest.mark.parametrize("kind", ["distinct", "ties", "infinite"])
def test_selection_of_any_number_of_rows(n, kind):
    """Both sides of every size at which the thread block changes, weights of the rows that stay in place of all."""
    g = gen(61)
    B = 3
    c = make(4, B, 1, 1, 64, n + 5, [n, n - 1, n // 2])
    k = rows_bf16(g, B, n, 1, 64)
    c.lckv_prefill_write_kv(0, k, -k)
    for sink, recent, keep in ((7, 100, n // 2), (0, 0, n - 1), (3, 0, 10), (0, 64, n - 2)):
        w = weights_of(kind, g, (B, 1, n + 5))
        held = w.clone()
        kept = torch.empty((B, 1, keep), dtype=torch.int32, device=DEV)
        dst = make(4, B, 1, 1, 64, keep, [0] * B)
        dst.lckv_evict_kv(0, c, 0, kept, weights=w, n_sink=sink, n_recent=recent, set_len=1)
        assert torch.equal(w.view(torch.int32), held.view(torch.int32))
        again = torch.empty_like(kept)
        if keep == n - 2:                                    # the last: in place, rows and weights
            c.lckv_evict_kv(0, c, 0, again, weights=w, weights_out=w, n_sink=sink, n_recent=recent, set_len=1)
            assert torch.equal(again, kept)
        for b, m in enumerate((n, n - 1, n // 2)):
            rows = kept_plain(held[b, 0].cpu().numpy(), m, sink, recent, keep)
            assert kept[b, 0].tolist() == rows.tolist() + [-1] * (keep - len(rows))
            if keep == n - 2:
                want = torch.zeros(n + 5, device=DEV)
                want[:len(rows)] = held[b, 0, torch.tensor(rows, device=DEV)]
                assert torch.equal(torch.nan_to_num(w[b, 0], nan=123.0), torch.nan_to_num(want, nan=123.0))
    ko, vo = (torch.zeros((B, n, 1, 64), device=DEV) for _ in range(2))
    c.lckv_cache_read_kv(0, ko, vo)
    for b, m in enumerate((n, n - 1, n // 2)):
        rows = torch.tensor(kept_plain(held[b, 0].cpu().numpy(), m, 0, 64, n - 2), device=DEV)
        assert torch.equal(ko[b, :len(rows)], value64(k)[b, rows].float()) and torch.equal(vo[b, :len(rows)], value64(-k)[b, rows].float())
    assert c.lckv_cache_status() == 0


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("H,lens", [(3, [70, 0, 2, 67]), (8, [2001, 1998, 3, 0, 1995, 1, 2000])])
def test_rows_read_back(bits, d, page, H, lens):
    """Small calls take one token a thread, large ones four: lengths of every remainder, both row types, both outputs."""
    g = gen(62)
    B, n = len(lens), max(lens)
    many = n * B * H * (d // 8) >= 148 * 16 * 256            # (four blocks of 256 threads, four tokens each, for every SM)
    assert many == (n > 1000)
    k, v = rows_bf16(g, B, n, H, d), rows_bf16(g, B, n, H, d)
    c = make(bits, B, H, H, d, n, lens, page)
    c.lckv_prefill_write_kv(0, k, v)
    for dt in (torch.bfloat16, torch.float32):
        ko, vo = (torch.full(k.shape, 7.0, dtype=dt, device=DEV) for _ in range(2))
        c.lckv_cache_read_kv(0, ko, vo)
        for got, x in ((ko, k), (vo, v)):
            want = (value64(x).float() if bits == 4 else x).to(dt)
            for b, m in enumerate(lens):
                assert torch.equal(got[b, :m], want[b, :m]) and (got[b, m:] == 7.0).all()
    assert c.lckv_cache_status() == 0


def check_weights(w, before, q, k, lse, lens, bits):
    """Scores: chains of d / 16 MMAs that may each drop 2^-23 of a partial sum, at most 2^-20 of the magnitudes' sum, and as much again for
    scaling, lse and their difference: 2^-19 of both; exponentials 2^-22 each, at most 2^-20 with the sums over heads."""
    B, Hkv = w.shape[:2]
    d = q.shape[-1]
    for b, n in enumerate(lens):
        assert torch.equal(w[b, :, n:], before[b, :, n:])
        if n == 0:
            continue
        kk = (value64(k[b, :n]) if bits == 4 else k[b, :n].double()).permute(1, 2, 0)                 # [Hkv, d, n]
        qq = q[b].double().view(Hkv, -1, d)
        s, a = qq @ kk * d ** -0.5, qq.abs() @ kk.abs() * d ** -0.5
        l = lse[b].double().view(Hkv, -1, 1)
        p = torch.exp(s - l)
        err = (p * (torch.expm1(2.0 ** -19 * (a + l.abs() + 1)) + 2.0 ** -20)).sum(1)
        want = before[b, :, :n].double() + p.sum(1)
        within(w[b, :, :n], want, err + 2.0 ** -22 * want.abs(), f"sequence {b}")


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 32, 32), (128, 64, 32), (64, 384, 32)])
def test_weights_of_many_tiles(bits, d, Hq, Hkv):
    """More than 64 tiles an SM: a warp over bf16 keys takes two of them, the last one alone."""
    g = gen(63)
    lens = [2350, 2304, 2305, 0, 1, 65, 128, 2350]
    B, n = len(lens), max(lens)
    assert -(-n // 64) * B * Hkv >= 64 * 148 and -(-n // 64) % 2 == 1
    k, q = rows_bf16(g, B, n, Hkv, d), randn(g, B, Hq, d)
    c = make(bits, B, Hq, Hkv, d, n, lens)
    c.lckv_prefill_write_kv(0, k, k)
    lse = torch.zeros(B, Hq, device=DEV)
    c.lckv_decode_attention(0, CONDENSED, q, lse=lse)
    before = torch.rand((B, Hkv, n), generator=g, device=DEV)
    w = before.clone()
    c.lckv_attention_weights(0, CONDENSED, q, lse, w, previous=before)
    check_weights(w, before, q, k, lse, lens, bits)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 2, 2), (128, 12, 1)])
def test_weights_of_sequences_that_outgrew_the_launch(bits, d, Hq, Hkv):
    """Captured with short sequences, replayed with long ones (and the other way round)."""
    g = gen(64)
    B, n = 3, 777
    k, q = rows_bf16(g, B, n, Hkv, d), randn(g, B, Hq, d)
    c = make(bits, B, Hq, Hkv, d, n, [10, 0, 64])
    lse, before = torch.zeros(B, Hq, device=DEV), torch.rand((B, Hkv, n), generator=g, device=DEV)
    w = before.clone()
    torch.cuda.synchronize()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=st):
        c.lckv_attention_weights(0, CONDENSED, q, lse, w, previous=before)
    for lens in ([777, 0, 641], [1, 130, 3], [10, 0, 64]):
        c.lckv_cache_reset(lens)
        c.lckv_prefill_write_kv(0, k, k)
        c.lckv_decode_attention(0, CONDENSED, q, lse=lse)
        w.copy_(before)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_weights(w, before, q, k, lse, lens, bits)
    assert c.lckv_cache_status() == 0
