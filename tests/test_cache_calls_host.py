"""Tensors that a cache's calls cannot take are refused before the library is entered; no GPU."""
import pytest
import torch

from paper_2405_10637_b200 import binding as lk

B, HQ, HKV, D = 2, 4, 2, 64
Q, K = torch.zeros(B, HQ, D, dtype=torch.bfloat16), torch.zeros(B, HKV, D, dtype=torch.bfloat16)
P = torch.zeros(B, 9, HKV, D, dtype=torch.bfloat16)


def closed(handle):
    """A cache without memory; its handle is not looked at where a tensor is refused."""
    c = lk.Cache.__new__(lk.Cache)
    c.cfg = lk.make_config(1, 0, HQ, HKV, D, B, 16)
    c.h, c.call, c.heads, c.out_torch_dtype = None, (handle, 0), (HQ, HKV, D), torch.bfloat16
    return c


CALLS = [
    ("lckv_decode_attention", lambda c, q: c.lckv_decode_attention(0, 0, q, out=Q.clone())),
    ("lckv_decode_attention", lambda c, q: c.lckv_decode_attention(0, 0, q, out=Q.clone(), batch=10 ** 9)),
    ("lckv_decode_attention", lambda c, q: c.lckv_decode_attention(0, 0, q, out=Q.clone(), lse=torch.zeros(B, HQ))),
    ("lckv_append_kv", lambda c, q: c.lckv_append_kv(0, K, K)),
    ("lckv_append_kv", lambda c, q: c.lckv_append_kv(0, K, None)),
    ("lckv_append_kv", lambda c, q: c.lckv_append_kv(0, K, K, batch=-1)),
    ("lckv_prefill_write_kv", lambda c, q: c.lckv_prefill_write_kv(0, P, P)),
    ("lckv_prefill_write_kv", lambda c, q: c.lckv_prefill_write_kv(0, P, None)),
]


@pytest.mark.parametrize("handle", [None, 0, 1 << 20])
@pytest.mark.parametrize("i", range(len(CALLS)))
def test_tensors_of_the_host_are_refused(handle, i):
    name, call = CALLS[i]
    with pytest.raises(lk.LckvError) as e:
        call(closed(handle), Q)
    assert e.value.status == lk.EINVAL
    assert name in str(e.value) and "on the cache's device" in str(e.value)


def test_what_is_no_tensor_is_refused():
    c = closed(1 << 20)
    for bad in (3, "q", [Q]):
        with pytest.raises(lk.LckvError) as e:
            c.lckv_decode_attention(0, 0, bad, out=Q, batch=B)
        assert e.value.status == lk.EINVAL
