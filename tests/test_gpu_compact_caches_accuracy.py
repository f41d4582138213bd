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


def exact_rows(q, k, n):
    """Scores [Hq, n] of one kv head in 64 bits."""
    code, step, low = encode64(k[:n, 0])
    return q.double() @ (low + step * code).flatten(-2).T * q.shape[-1] ** -0.5


# Queries off zero: with mean 0, 1 and 8 scores reach 16, 16 and 64 (base 2) and the partial sums of a group's codes less 8 about 1, 4 and 8 in
# a score's units (of codes as they are, about 6, 20 and 110).  Scores, lse and their difference are rounded at 2^-24 of what they reach, a few
# times; a score's MMAs, four a group, may each drop 2^-23 of a partial sum, always with one sign.
BOUND = {0.0: 2.0 ** -19, 1.0: 2.0 ** -18, 8.0: 2.0 ** -17}
SHAPES = [(128, 1, 4096, 0), (128, 4, 32768, 0), (128, 8, 32768, 1), (128, 8, 700, 0), (64, 2, 4096, 0), (64, 4, 9000, 3), (64, 8, 32768, 0), (64, 8, 32768, 1)]


@pytest.mark.parametrize("d,Hq,n,workers", SHAPES)
@pytest.mark.parametrize("mean", list(BOUND))
def test_fp32_outputs_and_lse(d, Hq, n, workers, mean):
    """fp32 outputs keep what 11 bits of a weight, codes that are all positive and truncated sums over rows would lose.

    Rms of the outputs' errors over that of the outputs: BOUND for the scores.  Then a warp's N blocks of 16 rows are added one by one
    in fp32: codes are 7.5 in the mean, so with codes less 8 the sum grows to S = |sum p step (code - 8)|, half a step or so whatever
    the output is, and the sum of the lows to about the same; the i-th of N roundings is at most 2^-24 of S i / N, evenly spread:
    sqrt(N / 3) 2^-24 / sqrt 3 of S, for both.  lse: BOUND."""
    g = gen(32)
    k, v = randn(g, 1, n, 1, d), randn(g, 1, n, 1, d)
    q = (torch.randn((1, Hq, d), generator=g, device=DEV) + mean).to(torch.bfloat16)
    c = make(4, 1, Hq, 1, d, n, [n], out32=1)
    c.lckv_prefill_write_kv(0, k, v)
    c.lckv_cache_set_worker_limit(workers)
    lse = torch.empty(1, Hq, device=DEV)
    out = c.lckv_decode_attention(0, CONDENSED, q, lse=lse)[0].double()
    want, l, _, _ = attention64(q[0], k[0], v[0], n)
    err, err_l = rms(out - want) / rms(want), (lse[0].double() - l).abs().max().item()
    code, step, _ = encode64(v[0])
    grown = torch.softmax(exact_rows(q[0], k[0], n), 1) @ (step * (code - 8)).flatten(-2)[:, 0]
    blocks = -(-n // 16 // (workers or c.info.n_workers))
    tol = BOUND[mean] + 2.0 ** -24 * (2 * blocks) ** 0.5 / 3 * rms(grown) / rms(want)
    print(f"d {d} heads {Hq} rows {n} workers {workers} mean {mean}: out {err:.2e} ({tol:.2e}) lse {err_l:.2e}")
    assert err <= tol
    assert err_l <= BOUND[mean]


@pytest.mark.parametrize("d,Hq,n", [(128, 1, 4096), (128, 8, 2000), (64, 2, 500), (64, 8, 9000)])
@pytest.mark.parametrize("mean", list(BOUND))
def test_lse_next_to_bf16_outputs(d, Hq, n, mean):
    """Codes enter as they are: a group's four MMAs (two over 64 dimensions a side) may each drop 2^-23 of partial sums of up to half of A, the
    largest row's scale * sum (|q| step code + |q low|); fp32 steps behind them 2^-24 each: 2^-21 A, and BOUND."""
    g = gen(33)
    k, v = randn(g, 1, n, 1, d), randn(g, 1, n, 1, d)
    q = (torch.randn((1, Hq, d), generator=g, device=DEV) + mean).to(torch.bfloat16)
    c = make(4, 1, Hq, 1, d, n, [n])
    c.lckv_prefill_write_kv(0, k, v)
    lse = torch.empty(1, Hq, device=DEV)
    c.lckv_decode_attention(0, CONDENSED, q, lse=lse)
    _, l, _, a = attention64(q[0], k[0], v[0], n)
    err = (lse[0].double() - l).abs()
    print(f"d {d} heads {Hq} rows {n} mean {mean}: lse {err.max().item():.2e}, A {a.max().item():.1f}")
    assert (err <= 2.0 ** -21 * a + BOUND[mean]).all()


@pytest.mark.parametrize("d,Hq,n", [(128, 1, 4096), (128, 8, 2000), (64, 2, 500), (64, 8, 9000), (64, 12, 300)])
@pytest.mark.parametrize("mean", list(BOUND))
def test_gathered_weights(d, Hq, n, mean):
    """Rms of a weight's error over the weight, given lse."""
    g = gen(34)
    k = randn(g, 1, n, 1, d)
    q = (torch.randn((1, Hq, d), generator=g, device=DEV) + mean).to(torch.bfloat16)
    c = make(4, 1, Hq, 1, d, n, [n])
    c.lckv_prefill_write_kv(0, k, k)
    s = exact_rows(q[0], k[0], n)
    lse = torch.logsumexp(s, 1).float()
    w = c.lckv_attention_weights(0, CONDENSED, q, lse[None])[0, 0, :n].double()
    want = torch.exp(s - lse.double()[:, None]).sum(0)
    err = rms(w / want - 1)
    print(f"d {d} heads {Hq} rows {n} mean {mean}: {err:.2e}")
    assert err <= BOUND[mean]
