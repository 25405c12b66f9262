"""Attention over the 8-bit cache, in every form for both result types: which kernel takes a sequence goes by the type as well as by
its rows, so what holds for one is looked at for the other.  And the cache's writes where a CTA has several rounds of blocks.

Tolerances as in test_gpu_kv_attention.py; FP32 results come from probabilities of two FP16 numbers, which are off by 2^-22 of
themselves, or by 2^-25 where the row's largest is 2^8 at least: 2^-33 (largest p scale) (sum of |codes|)."""
import math

import pytest
import torch

import kv_ref as R
from paper_2307_09782_b200 import binding
from test_gpu_kv_attention import ATTN_CASES, attn_tolerance, check_attention, half_step, same_scales

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("out", [BF16, F32])


def tolerance(ref, bound, out):
    if out == BF16:
        return attn_tolerance(ref, bound, out)
    pv, qk, low = bound
    return half_step(out) * ref.abs() + pv * (2.0 ** -22 + 2 * 2.0 ** -18 * qk[..., None] + 2.0 ** -17) + 2.0 ** -33 * low + 1e-30


def compare(case, out, codes, scale, table, lens, cu, q, sm=None):
    _, _, Hq, H, D, page, causal, window = case
    got = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), causal=causal, window=window,
                               sm_scale=sm, out_dtype=out)
    ref, _, bound = R.attention(codes, scale, q, table, lens, cu, D ** -0.5 if sm is None else sm, causal, window)
    err, tol = (got.to(R.F64) - ref).abs(), tolerance(ref, bound, out)
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))
    return got


def plain(case, out, seed=0, sm=None):
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page, seed)
    return compare(case, out, codes, scale, table, lens, cu, R.heads(cu[-1], Hq, D, seed + 7), sm)


@pytest.mark.parametrize("case", ATTN_CASES)
def test_fp32_results_keep_both_terms(case):
    plain(case, F32)


@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (5, 1), (8, 1), (3, 3), (16, 1), (17, 1), (8, 4), (11, 3), (1, 64), (1, 65), (64, 1), (65, 1), (16, 4),
                                 (13, 5), (5, 13), (1, 128), (1, 129), (1, 256), (1, 257), (3, 86)])
@TYPES
def test_rows_at_the_borders(G, n, out):
    """Of the instances for 4, 8, 16, 32 and 64 rows, of the two kernels, of row tiles and items."""
    plain(([700, 129], [n, 1], 2 * G, 2, 128, 64, True, 0), out)
    plain(([700, n + 60], [n, n], 2 * G, 2, 64, 32, True, 50), out)


@pytest.mark.parametrize("case", [
    ([2500, 2500, 40, 1900], [700, 1, 40, 650], 12, 12, 64, 32, True, 0),
    ([900] * 9, [200] * 9, 32, 8, 128, 64, True, 0),
    ([1500] * 3, [150] * 3, 40, 8, 128, 64, True, 200),
    ([70] * 90, [70] * 90, 2, 1, 64, 16, True, 0),
    ([6000], [100], 4, 1, 128, 128, False, 0),
    ([40, 0, 900] * 40, [40, 0, 33] * 40, 4, 2, 64, 64, True, 0),
    ([300, 2000, 17, 900], [1, 500, 1, 16], 8, 2, 128, 64, True, 0),  # decoding beside chunks
])
@TYPES
def test_blocks_over_ctas(case, out):
    plain(case, out)


@pytest.mark.parametrize("sm", [1.0, 0.01])
@pytest.mark.parametrize("case", [ATTN_CASES[2], ATTN_CASES[8], ATTN_CASES[10]])
def test_scales_of_scores(case, sm):
    check_attention(case, BF16, 3, sm_scale=sm)


@pytest.mark.parametrize("case", [ATTN_CASES[2], ATTN_CASES[8], ATTN_CASES[11]])
@TYPES
def test_zero_and_extreme_blocks(case, out):
    """Blocks of zero values, of the smallest scale and of scales 2^40 apart."""
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
    owned = table[table >= 0].long()
    scale[owned[::3], 1] = 2.0 ** -20
    scale[owned[1::3], 1] = 2.0 ** 20
    codes[owned[0], 1] = 0
    scale[owned[0], 1] = 2.0 ** -39
    scale[owned[0], 0] = 2.0 ** -64
    compare(case, out, codes, scale, table, lens, cu, R.heads(cu[-1], Hq, D, 7))


@pytest.mark.parametrize("L,n,Hq,H,D,page", [(700, 1, 8, 2, 128, 64), (700, 5, 4, 2, 64, 16), (500, 300, 4, 2, 128, 32)])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 30, 2.0 ** 48])
@TYPES
def test_written_zeros_beside_values(L, n, Hq, H, D, page, size, out):
    """Padding: tokens whose values are zeros fill blocks (their scale is the smallest, 2^-64), the others' values are as large as `size`."""
    per = -(-L // page)
    cache = binding.make_kv_cache(per + 1, H, D, page)
    k, v = R.heads(L, H, D, 1), R.heads(L, H, D, 2) * size
    v[page:3 * page] = 0
    k[2 * page:4 * page] = 0
    table = torch.randperm(per, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(1, per).cuda()
    binding.kv_cache_write(cache, k, v, table, R.ints([L]), cu=R.ints([0, L]))
    assert (cache.scale[table[0, 1].long(), 1] == 2.0 ** -64).all()
    case = ([L], [n], Hq, H, D, page, True, 0)
    compare(case, out, cache.codes, cache.scale, table, [L], [0, n], R.heads(n, Hq, D, 7))


@pytest.mark.parametrize("case", [([300, 200], [1, 1], 8, 2, 128, 64, True, 0), ([300, 200], [1, 1], 2, 2, 64, 16, True, 0),
                                  ([300, 200], [6, 3], 8, 2, 128, 64, True, 0), ([300, 200], [8, 2], 4, 2, 64, 16, True, 40),
                                  ([300, 200], [24, 3], 4, 2, 128, 16, True, 0), ([2000, 40], [1, 1], 64, 2, 128, 128, True, 0),
                                  ([300, 200], [250, 200], 4, 2, 64, 32, True, 0), ([300, 200], [250, 90], 4, 2, 128, 16, True, 40)])
@pytest.mark.parametrize("what", ["key", "value", "page"])
@TYPES
def test_nan_blocks(case, what, out):
    """A block that stands for NaN reaches the rows that see it and no others; so does a page the table names wrongly."""
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
    i = 2 if page >= 64 else 17 if page == 16 and (new[0] == 24 or window) else 5
    p = int(table[0, i])
    if what == "page":
        table[0, i] = -3
    else:
        scale[p, 0 if what == "key" else 1, 1] = math.nan
        codes[p, 0 if what == "key" else 1, 1] = 0
    q = R.heads(cu[-1], Hq, D, 7)
    got = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), causal=causal, window=window,
                               out_dtype=out)
    ref, _, bound = R.attention(codes, scale, q, table, lens, cu, D ** -0.5, causal, window)
    L, n = lens[0], cu[1]
    hit = torch.zeros((cu[-1], Hq), dtype=torch.bool, device="cuda")
    for r in range(n):
        pos = L - n + r
        lo = max(0, pos + 1 - window) if window else 0
        if lo < (i + 1) * page and pos >= i * page:
            hit[r, slice(None) if what == "page" else slice(Hq // H, 2 * Hq // H)] = True
    assert hit.any()
    assert got[hit].isnan().all()
    assert ((got.to(R.F64) - ref).abs() <= tolerance(ref, bound, out))[~hit].all()


@pytest.mark.parametrize("case", [([300, 200], [5, 1], 8, 2, 128, 64, True, 0), ([300, 200], [90, 70], 8, 2, 128, 64, True, 0),
                                  ([3000, 200], [40, 33], 10, 2, 64, 32, True, 0), ([1500, 300], [1200, 300], 4, 4, 64, 16, True, 0)])
@TYPES
def test_not_finite_queries(case, out):
    """A query that is not finite gives NaN in its own row and head only."""
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
    q = R.heads(cu[-1], Hq, D, 7)
    args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
    good, sums = binding.kv_attention(*args, cu=R.ints(cu), out_dtype=out, lse=True)
    bad = [(2, 3, 9, math.nan), (cu[-1] - 1, 0, 0, math.inf), (0, 1, D - 1, -math.inf)]
    hit = torch.zeros((cu[-1], Hq), dtype=torch.bool, device="cuda")
    for t, h, d, value in bad:
        q[t, h, d] = value
        hit[t, h] = True
    got, lse = binding.kv_attention(*args, cu=R.ints(cu), out_dtype=out, lse=True)
    assert got[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(got[~hit], good[~hit]) and torch.equal(lse[~hit], sums[~hit])


@pytest.mark.parametrize("case", [ATTN_CASES[0], ATTN_CASES[2], ATTN_CASES[8], ATTN_CASES[11], ATTN_CASES[12],
                                  ([5000], [1], 8, 2, 128, 64, True, 0), ([3000], [40], 8, 2, 128, 64, True, 0)])
def test_results_in_the_place_of_queries(case):
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
    q = R.heads(cu[-1], Hq, D, 7, 2)
    args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
    want = binding.kv_attention(*args, cu=R.ints(cu), causal=causal, window=window)
    got = binding.kv_attention(*args, cu=R.ints(cu), causal=causal, window=window, out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want)


def test_one_token_each_with_and_without_offsets():
    """64 sequences of one new token, said by offsets or left unsaid."""
    lens = [37 * i % 900 + 1 for i in range(64)]
    codes, scale, table, lens, cu = R.batch(lens, [1] * 64, 2, 128, 64)
    q = R.heads(64, 8, 128, 7)
    args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
    ref, _, bound = R.attention(codes, scale, q, table, lens, cu, 128 ** -0.5, True, 0)
    for cu_ in (None, R.ints(cu)):
        got = binding.kv_attention(*args, cu=cu_)
        assert ((got.to(R.F64) - ref).abs() <= attn_tolerance(ref, bound, BF16)).all()


# ---- writing, many blocks ---------------------------------------------------------------------------------------------
def write(codes, scale, k, v, table, lens, cu, mode):
    """As kv_ref.write, the keys' and values' heads of a page at once."""
    codes, scale = codes.clone(), scale.clone()
    page = codes.shape[3]
    x = torch.stack([k, v]).float()  # [2, T, H, D]
    tab = table.tolist()
    for b in range(len(lens)):
        r, n = cu[b], cu[b + 1] - cu[b]
        pos, end = lens[b] - n, lens[b]
        while pos < end:
            stop = min(end, (pos // page + 1) * page)
            p, lo, m = tab[b][pos // page], pos % page, stop - pos
            new = x[:, r:r + m].transpose(1, 2)  # [2, H, m, D]
            s, old = R.scale_of(new.abs().amax((2, 3)), mode), scale[p].clone()
            if lo > 0:
                s = torch.where(torch.isnan(old) | (s <= old), old, s)
                again = R.codes_of(codes[p, :, :, :lo].view(torch.float8_e4m3fn).float() * old[..., None, None], s[..., None, None])
                keep = (s == old) | torch.isnan(old)
                codes[p, :, :, :lo] = torch.where(keep[..., None, None], codes[p, :, :, :lo], again)
            codes[p, :, :, lo:lo + m] = R.codes_of(new, s[..., None, None])
            scale[p] = s
            r, pos = r + m, stop
    return codes, scale


@pytest.mark.parametrize("B,H,D,page,mode", [(3, 2, 64, 16, "none"), (75, 64, 64, 16, "M1"), (75, 64, 64, 16, "none"), (80, 9, 128, 128, "none"),
                                             (90, 40, 64, 32, "M1"), (90, 33, 128, 32, "none"), (60, 20, 128, 64, "M1")])
def test_several_rounds_of_blocks_per_cta(B, H, D, page, mode):
    """Up to 75 sequences of some 20 new tokens and 128 blocks each: more than find room at once.  Teams of 32 to 512 threads."""
    g = torch.Generator().manual_seed(B)
    new = torch.randint(1, 40, (B,), generator=g).tolist()
    lens = [n + int(torch.randint(0, 50, (1,), generator=g)) for n in new]
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page, mode=mode)
    k, v = R.heads(cu[-1], H, D, 3, 2), R.heads(cu[-1], H, D, 4)
    k[::3] *= 30
    expect = write(codes, scale, k, v, table, lens, cu, mode)
    if B == 3:
        simple = R.write(codes, scale, k, v, table, lens, cu, mode)
        assert torch.equal(simple[0], expect[0]) and same_scales(simple[1], expect[1])
    binding.kv_cache_write(binding.Fp8KvCache(codes, scale), k, v, table, R.ints(lens), cu=R.ints(cu), mode=mode)
    assert torch.equal(codes, expect[0]) and same_scales(scale, expect[1])


# ---- the layer ----------------------------------------------------------------------------------------------------------
def test_padding_of_a_batch_reaches_nobody():
    """Rows behind the last sequence, whatever they hold: the others' results and the cache are the same."""
    from test_gpu_kv_attention_calls import block, inputs

    b, new = block(), [40, 1, 70]
    pages = torch.arange(30, dtype=torch.int32, device="cuda").view(3, 10)
    results = []
    for fill in (0.0, math.nan, 1e30):
        cache = b.new_cache(30, 16)
        x = inputs(128)
        x[111:] = fill
        positions = torch.cat([torch.arange(n) for n in new] + [torch.full((17,), -1 if fill else 0)]).to(torch.int32).cuda()
        y = b.forward(x, cache, pages, R.ints(new), positions, cu=R.ints([0, 40, 41, 111]))
        results.append((y[:111].clone(), cache.codes, cache.scale))
    for other in results[1:]:
        assert all(torch.equal(a, o) for a, o in zip(results[0], other))
    assert not results[0][0].isnan().any()
