"""The operators around the attention at the ends of what their documentation allows.  Tolerances: see
test_gpu_operators.py."""
import pytest
import torch

from paper_2405_10637_b200 import binding as lk

from test_gpu_operators import DEV, E, HALF, check_norm, gen, norm64, randn, within

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
