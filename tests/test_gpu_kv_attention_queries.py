"""What the tensor core's terms leave of the queries: attention over the 8-bit cache where a query's features differ much in size.

A row is scaled so that its largest feature lies in [128, 256).  bf16 results: two terms, exact for the features from 2^-13 of the
largest on.  FP32 results: three terms, exact from 2^-16 of the largest on; smaller features are off by 2^-24 of the largest at most."""
import pytest
import torch

import kv_ref as R
from paper_2307_09782_b200 import binding

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("lens,new,Hq,H,D,page", [([700, 40], [1, 1], 4, 2, 128, 64), ([700, 40], [7, 3], 8, 2, 64, 16),
                                                  ([500, 300], [400, 120], 4, 2, 128, 32)])
@pytest.mark.parametrize("out,exponent", [(BF16, -3), (BF16, -6), (F32, -3), (F32, -6), (F32, -9)])
def test_small_features_beside_a_large_one(lens, new, Hq, H, D, page, out, exponent):
    """One feature of 200 that all keys answer with zero, the others 2^exponent 183 / 128, a number of 8 bits, against
    positive keys: whatever is lost of one is lost of all, and shows in the logarithm of the sum.  That is FP32 for both
    types: off by 2^-18 of sum |q| |k| and 2^-17 at most, as in test_gpu_kv_attention.py."""
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
    codes[:, 0] &= 0x7F
    codes[:, 0, :, :, 5] = 0
    q = torch.full((cu[-1], Hq, D), 2.0 ** exponent * 183 / 128, device="cuda").to(BF16)
    q[..., 5] = 200.0
    sm = 2.0 ** -exponent / D  # scores of a few units
    _, lse = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), sm_scale=sm, out_dtype=out,
                                  lse=True)
    _, ref, (_, qk, _) = R.attention(codes, scale, q, table, lens, cu, sm, True, 0)
    err, tol = (lse.to(R.F64) - ref).abs(), 2.0 ** -17 + 2.0 ** -18 * qk + 2.0 ** -22 * ref.abs()
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("case", [([4096], [130], 4, 4, 128, 32, True, 0), ([4000] * 3, [1] * 3, 16, 8, 128, 64, True, 0),
                                  ([2000, 90], [9, 60], 8, 2, 64, 64, True, 0)])
@pytest.mark.parametrize("factor", [20.0, 100.0])
def test_fp32_results_beside_a_large_feature(case, factor):
    """In the 2-norm, one feature of each query `factor` times as large as the others.  What the three terms leave is nothing beside the
    rest; a score of the size s = factor D^-1/2 is summed up in 3 D / 32 <= 12 steps, each off by 2^-23 of a partial sum at most
    and half of it on average: 6 2^-23 s < 2^-17.2 for factor 100 (s = 8.9; D = 64: 3 2^-23 12.5), which counts in the numerator and in the
    sum, and two roundings of scores and factors (2^-24 s each): < 2^-15.9."""
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page, spread=0.0)
    q = torch.randn((cu[-1], Hq, D), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    q[..., 17] *= factor
    q = q.to(BF16)
    got = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), out_dtype=F32)
    ref, _, _ = R.attention(codes, scale, q, table, lens, cu, D ** -0.5, causal, window)
    err = float((got.to(R.F64) - ref).norm() / ref.norm())
    print(f"factor {factor}: {err:.2e}")
    assert err <= 2.0 ** -15.5


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("L,n,Hq,H,D,window", [(8192, 513, 64, 64, 128, 0), (8192, 257, 128, 128, 64, 0), (5000, 4100, 32, 8, 128, 0),
                                               (4500, 700, 64, 32, 64, 3000), (40000, 256, 160, 160, 64, 0)])
def test_long_sums(L, n, Hq, H, D, window, out):
    """Values around 1 and scores near zero: what the sums over many tokens lose shows as a part of every result.  The tensor core cuts off
    2^-23 of a sum at most with each product of 16 tokens.  FP32 results: sums of 8 steps of 64 tokens with two terms each, 64 2^-23 = 2^-17
    at most, and less than that for all else.  bf16 results: L / 16 2^-23 = L 2^-27 at most; they are rounded by 2^-9 of themselves at
    most, all in one direction if they are nearly equal, as here."""
    page = 128
    per = -(-L // page)
    cache = binding.make_kv_cache(per, H, D, page)
    g = torch.Generator(device="cuda").manual_seed(3)
    table = torch.arange(per, dtype=torch.int32, device="cuda").view(1, per)
    for i in range(0, L, 4096):  # in parts: the inputs in 32 bits are large
        m = min(4096, L - i)
        k = torch.randn((m, H, D), generator=g, device="cuda").to(BF16)
        v = (1 + 0.1 * torch.randn((m, H, D), generator=g, device="cuda")).to(BF16)
        binding.kv_cache_write(cache, k, v, table, R.ints([i + m]), cu=R.ints([0, m]))
    q = (0.2 * torch.randn((n, Hq, D), generator=g, device="cuda")).to(BF16)
    got = binding.kv_attention(cache, q, table, R.ints([L]), cu=R.ints([0, n]), window=window, out_dtype=out)
    heads = 2
    codes, scale = cache.codes[:, :, :heads].contiguous(), cache.scale[:, :, :heads].contiguous()
    G = Hq // H
    ref, _, _ = R.attention(codes, scale, q[:, :heads * G].contiguous(), table, [L], [0, n], D ** -0.5, True, window)
    got = got[:, :heads * G].to(R.F64)
    shrunk = float(1 - got.sum() / ref.sum())
    print(f"{out} {L}: {shrunk:.2e}, 2-norm {float((got - ref).norm() / ref.norm()):.2e}")
    assert abs(shrunk) <= (2.0 ** -16 if out == F32 else L * 2.0 ** -27 + 2.0 ** -9)
    if out == F32:
        assert (got - ref).norm() <= 2.0 ** -16 * ref.norm()
