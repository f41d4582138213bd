"""What a user of the Python binding may rely on around a cache's calls: views of its memory, and the checks of tensors."""
import pytest
import torch

from test_gpu_compact_caches import DEV, gen, make, rows_bf16

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
