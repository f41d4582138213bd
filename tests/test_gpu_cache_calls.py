"""What a user of the Python binding may rely on around a cache's calls: views of its memory, and the checks of tensors."""
import pytest
import torch

from paper_2405_10637_b200 import binding as lk
from test_gpu_compact_caches import CONDENSED, DEV, gen, make, randn, refused, rows_bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [0, 64])
def test_views_of_a_slot_are_the_callers_own(page):
    """What one caller does to a view's shape or gradient flag is not seen by the next; the memory is the same."""
    c = make(16, 2, 4, 2, 64, 100, [100, 3], page)
    k = rows_bf16(gen(51), 2, 100, 2, 64)
    c.lckv_prefill_write_kv(0, k, k)
    first = c.slot_tensors(0)
    shape, held = first[0].shape, first[0].clone()
    first[0].unsqueeze_(0)
    first[1].t_() if first[1].dim() == 2 else first[1].transpose_(0, 1)
    first[0].requires_grad_()
    again = c.slot_tensors(0)
    for t in again:
        assert t.shape == shape and t.is_contiguous() and not t.requires_grad
    assert again[0].data_ptr() == first[0].data_ptr() and again[1].data_ptr() == first[1].data_ptr()
    assert torch.equal(again[0].view(torch.int16), held.view(torch.int16))
    again[0].zero_()
    assert not c.slot_tensors(0)[0].any() and not first[0].any()


@pytest.mark.parametrize("bits,out32", [(16, 0), (16, 1), (4, 0), (4, 1)])
def test_tensors_that_do_not_fit_are_refused(bits, out32):
    B, Hq, H, d, n = 3, 4, 2, 64, 50
    g = gen(52)
    c = make(bits, B, Hq, H, d, n + 1, [n, 7, 0], out32=out32)
    k, v = rows_bf16(g, B, n, H, d), rows_bf16(g, B, n, H, d)
    q, kn = randn(g, B, Hq, d), rows_bf16(g, B, H, d)
    out = torch.empty(B, Hq, d, dtype=torch.float32 if out32 else torch.bfloat16, device=DEV)
    other = torch.empty_like(out, dtype=torch.bfloat16 if out32 else torch.float32)
    state = c.buf.clone()
    E = lk.EINVAL
    bad = lambda t: (t.cpu(), t.float(), t.half(), t.transpose(0, 1), t[..., ::2], t[:1], None)
    for t in bad(q):
        refused(E, c.lckv_decode_attention, 0, CONDENSED, t, out=out, batch=B)
    for t in (other, out.cpu(), out.transpose(0, 1), out[:2], out.half()):
        refused(E, c.lckv_decode_attention, 0, CONDENSED, q, out=t)
    for t in (torch.empty(B, Hq, device=DEV, dtype=torch.float64), torch.empty(B, Hq), torch.empty(B, Hq - 1, device=DEV), torch.empty(Hq, B, device=DEV).t()):
        refused(E, c.lckv_decode_attention, 0, CONDENSED, q, out=out, lse=t)
    for t in bad(kn):
        refused(E, c.lckv_append_kv, 0, t, kn, batch=B)
        refused(E, c.lckv_append_kv, 0, kn, t, batch=B)
    for t in bad(k)[:-1]:
        refused(E, c.lckv_prefill_write_kv, 0, k, t)
    for t in bad(k)[:3]:
        refused(E, c.lckv_prefill_write_kv, 0, t, v)
    refused(E, c.lckv_prefill_write_kv, 0, k.transpose(1, 2), v)
    torch.cuda.synchronize()
    assert torch.equal(c.buf, state)
    # what fits: raw 16-bit patterns, room to spare, other shapes of the same elements, fewer sequences
    c.lckv_prefill_write_kv(0, k.view(torch.int16), v.flatten(2))
    want = c.lckv_decode_attention(0, CONDENSED, q)
    lse = torch.full((B + 1, Hq), 5.0, device=DEV)
    got = c.lckv_decode_attention(0, CONDENSED, q.view(torch.uint16).flatten(1), out=out, lse=lse)
    assert got is out and torch.equal(want, got) and (lse[B] == 5.0).all()
    two = c.lckv_decode_attention(0, CONDENSED, q, out=torch.zeros_like(out), batch=2)
    assert not two[2].any() and (two[:2].float() - want[:2].float()).abs().max() < 0.05
    c.lckv_append_kv(0, kn.view(torch.int16), kn[:, None], advance_len=1)
    assert c.lckv_cache_lengths() == [n + 1, 8, 1] and c.lckv_cache_status() == 0


def test_calls_use_the_caches_device_and_a_stream_of_it():
    c = make(4, 1, 2, 2, 64, 10, [3], poison=False)
    c.buf[c.info.workspace_bytes:] = 0
    q = randn(gen(53), 1, 2, 64)

    class Elsewhere:
        device, cuda_stream = torch.device("cuda", 7), 0

    refused(lk.EINVAL, c.lckv_decode_attention, 0, CONDENSED, q, stream=Elsewhere())
    refused(lk.EINVAL, c.lckv_append_kv, 0, q, q, stream=Elsewhere())
    refused(lk.EINVAL, c.lckv_prefill_write_kv, 0, torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16, device=DEV),
            torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16, device=DEV), stream=Elsewhere())
    st = torch.cuda.Stream()
    out = torch.ones(1, 2, 64, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    c.lckv_decode_attention(0, CONDENSED, q, out=out, stream=st)
    st.synchronize()
    assert not out.any()
    c.close()
    refused(lk.EINVAL, c.lckv_decode_attention, 0, CONDENSED, q, out=out)
    refused(lk.EINVAL, c.lckv_append_kv, 0, q, q)


def test_outputs_made_by_a_call_belong_to_its_stream():
    """An output that a call makes on a given stream is made, and for prompts zeroed, there: not behind what the current stream still does."""
    n = 200
    g = gen(54)
    c = make(16, 1, 2, 2, 64, n, [n])
    k, q, pq = rows_bf16(g, 1, n, 2, 64), randn(g, 1, 2, 64), randn(g, 1, n, 2, 64)
    c.lckv_prefill_write_kv(0, k, k)
    want, want_p = c.lckv_decode_attention(0, CONDENSED, q), c.lckv_prefill_attention(0, CONDENSED, pq)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)                            # some 10 ms of the current stream
    got, got_p = c.lckv_decode_attention(0, CONDENSED, q, stream=st), c.lckv_prefill_attention(0, CONDENSED, pq, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_p, want_p)
