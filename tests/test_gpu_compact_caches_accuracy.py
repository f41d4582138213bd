"""How exact the operators over 4-bit rows are over many rows: root mean squares of the errors against 64 bits, with bounds from the
statistics of the roundings (the largest errors that could add up are far above them)."""
import pytest
import torch

from test_gpu_compact_caches import CONDENSED, DEV, attention64, encode64, gen, make, randn

pytestmark = pytest.mark.gpu


def rms(x):
    return x.double().pow(2).mean().sqrt().item()


@pytest.mark.parametrize("d,Hq", [(128, 1), (128, 4), (128, 8), (64, 2), (64, 3), (64, 8)])
@pytest.mark.parametrize("workers", [1, 5, 0])
def test_bf16_outputs_of_many_rows_in_one_warp(d, Hq, workers):
    """32768 rows whose values cancel: sums of step * code and of lows are hundreds of times the output.

    Bound of the rms error: the output's rounding (at most 2^-8 of it, evenly spread: / sqrt 3); every weight times step in 11 bits
    (2^-11 of it, / sqrt 3, independent); and fp32 sums: a chain of four MMAs, which may drop what lies below 2^-23 of the partial sum
    (2^-21), and the roundings (2^-24 / sqrt 3 each) of up to 512 sums over tiles and 8192 lows of a lane, together 2^-19 of
    sum p (step code + |low|)."""
    g = gen(31)
    n = 32768
    k, v = randn(g, 1, n, 1, d), randn(g, 1, n, 1, d)
    q = randn(g, 1, Hq, d)
    c = make(4, 1, Hq, 1, d, n, [n])
    c.lckv_prefill_write_kv(0, k, v)
    c.lckv_cache_set_worker_limit(workers)
    out = c.lckv_decode_attention(0, CONDENSED, q)[0].double()
    want, lse, mag, _ = attention64(q[0], k[0], v[0], n)
    code, step, low = encode64(k[0])
    s = torch.einsum("hd,nd->hn", q[0].double(), (low + step * code).flatten(-2)[:, 0]) * d ** -0.5
    code, step, low = encode64(v[0])
    term = (step * code).flatten(-2)[:, 0]
    weights = torch.einsum("hn,nd->hd", torch.exp(s - lse[:, None]) ** 2, term ** 2)
    tol = ((2.0 ** -8 * want) ** 2 / 3 + 2.0 ** -22 / 3 * weights).mean().sqrt().item() * 1.1 + 2.0 ** -19 * mag.mean().item()
    err = rms(out - want)
    print(f"d {d} heads {Hq} workers {workers}: rms error {err / rms(want):.3e} of the output's, bound {tol / rms(want):.3e}")
    assert err <= tol
