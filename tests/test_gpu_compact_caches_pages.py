"""Compact caches in pages: what may follow an eviction that gave pages back, and captured calls next to it."""
import pytest
import torch

from paper_2405_10637_b200 import binding as lk
from test_gpu_compact_caches import CONDENSED, DEV, check_attention, gen, kept_plain, make, randn, refused, rows_bf16, value64

pytestmark = pytest.mark.gpu


def after_eviction(bits, d=64, Hq=4, H=2, seed=41):
    """A paged cache that was evicted in place, giving pages back, and its rows per head [B][rows, H, d]."""
    g = gen(seed)
    lens, keep, cap = [300, 0, 130, 64], 70, 301
    B = len(lens)
    k, v = rows_bf16(g, B, cap, H, d), rows_bf16(g, B, cap, H, d)
    c = make(bits, B, Hq, H, d, cap, lens, 64)
    c.lckv_prefill_write_kv(0, k, v)
    w = torch.rand((B, H, cap), generator=g, device=DEV)
    kept = torch.empty((B, H, keep), dtype=torch.int32, device=DEV)
    c.lckv_evict_kv(0, c, 0, kept, weights=w, n_sink=2, n_recent=9, set_len=1)
    rows = [[kept_plain(w[b, h].cpu().numpy(), lens[b], 2, 9, keep) for h in range(H)] for b in range(B)]
    stay = [[torch.stack([x[b, torch.tensor(rows[b][h], device=DEV), h] for h in range(H)], 1) for b in range(B)] for x in (k, v)]
    return g, c, [min(n, keep) for n in lens], stay


def same_rows(c, lens, stay, four):
    B, H, d = len(lens), c.cfg.n_kv_heads, c.cfg.head_dim
    out = [torch.zeros((B, max(lens), H, d), device=DEV) for _ in range(2)]
    c.lckv_cache_read_kv(0, *out)
    for got, x in zip(out, stay):
        for b, n in enumerate(lens):
            assert torch.equal(got[b, :n], value64(x[b][:n]).float() if four else x[b][:n].float())


@pytest.mark.parametrize("bits", [4, 16])
def test_out_of_a_cache_that_gave_pages_back(bits):
    g, c, lens, stay = after_eviction(bits)
    to = make(4, 4, 4, 2, 64, 80, [80] * 4, 64)             # two pages a sequence: it gives some back as well
    kept = torch.empty((4, 2, 50), dtype=torch.int32, device=DEV)
    to.lckv_evict_kv(0, c, 0, kept, set_len=1)               # equal weights: the lowest rows
    assert to.lckv_cache_lengths() == [min(n, 50) for n in lens]
    same_rows(to, [min(n, 50) for n in lens], stay, True)
    last = make(4, 4, 4, 2, 64, 50, [0] * 4)
    last.lckv_evict_kv(0, to, 0, kept[:, :, :40].contiguous(), set_len=1)
    same_rows(last, [min(n, 40) for n in lens], stay, True)
    same_rows(c, lens, stay, bits == 4)
    assert c.lckv_cache_status() == to.lckv_cache_status() == last.lckv_cache_status() == 0


@pytest.mark.parametrize("bits", [4, 16])
def test_captures_right_after_pages_were_given_back(bits):
    """Attention, weights, reading and another eviction in one graph; then the pages change places, and a replay goes by the new ones."""
    g, c, lens, stay = after_eviction(bits)
    B, Hq, H, d, cap = 4, 4, 2, 64, 301
    q, lse = randn(g, B, Hq, d), torch.empty(B, Hq, device=DEV)
    out = torch.empty(B, Hq, d, dtype=torch.bfloat16, device=DEV)
    w = torch.zeros(B, H, cap, device=DEV)
    read = [torch.zeros(B, 70, H, d, device=DEV) for _ in range(2)]
    small, kept = make(4, B, Hq, H, d, 50, [0] * B), torch.empty((B, H, 50), dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=st):
        c.lckv_attention_weights(0, CONDENSED, q, lse, w)
        c.lckv_decode_attention(0, CONDENSED, q, out=out, lse=lse)
        c.lckv_attention_weights(0, CONDENSED, q, lse, w)
        c.lckv_cache_read_kv(0, *read)
        small.lckv_evict_kv(0, c, 0, kept, weights=w, n_sink=3, n_recent=5)

    def check():
        graph.replay()
        torch.cuda.synchronize()
        assert c.lckv_cache_status() == small.lckv_cache_status() == 0
        for got, x in zip(read, stay):
            for b, n in enumerate(lens):
                assert torch.equal(got[b, :n], value64(x[b]).float() if bits == 4 else x[b].float())
        if bits == 4:
            pad = [torch.cat([torch.cat([x, x.new_zeros(70 - x.shape[0], H, d)])[None] for x in s]) for s in stay]
            check_attention(out, lse, q, *pad, lens)
        wn = w.cpu().numpy()
        for b, n in enumerate(lens):
            assert abs(w[b].sum().item() - Hq) < 0.05 if n else not w[b].any()
            for h in range(H):
                rows = kept_plain(wn[b, h], n, 3, 5, 50).tolist()
                assert kept[b, h].tolist() == rows + [-1] * (50 - len(rows))

    check()
    before = c.lckv_cache_page_table()
    c.lckv_cache_reset([129] * 4)
    c.lckv_cache_reset(lens)
    assert not torch.equal(before, c.lckv_cache_page_table())
    k, v = (torch.zeros(B, 70, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for b, n in enumerate(lens):
        k[b, :n], v[b, :n] = stay[0][b], stay[1][b]
    c.lckv_prefill_write_kv(0, k, v)
    for t in (*read, w):
        t.zero_()
    check()


def test_reading_is_captured_only_with_the_table_on_the_device():
    """A cache whose table no call has brought to the device yet: the upload does not belong into the caller's graph."""
    c = lk.Cache(lk.make_config(1, 0, 4, 2, 64, 2, 100, page_rows=64, n_pages=4, kv_bits=4))
    out = [torch.full((2, 100, 2, 64), 3.0, device=DEV) for _ in range(2)]
    other = torch.zeros(4, device=DEV)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=st):
        refused(lk.EINVAL, c.lckv_cache_read_kv, 0, *out)
        other.add_(1.0)                                      # (so that the graph is not empty)
    assert (out[0] == 3.0).all()
    c.lckv_cache_read_kv(0, *out)                            # eager: uploads; no rows yet
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        c.lckv_cache_read_kv(0, *out)
    c.lckv_cache_reset([70, 1])
    k = rows_bf16(gen(43), 2, 100, 2, 64)
    c.lckv_prefill_write_kv(0, k, -k)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    for got, x in zip(out, (k, -k)):
        for b, n in enumerate((70, 1)):
            assert torch.equal(got[b, :n], value64(x)[b, :n].float()) and (got[b, n:] == 3.0).all()
