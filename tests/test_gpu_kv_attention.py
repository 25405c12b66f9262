"""The attention half of a decoder layer against plain 64-bit forms: norms with the position rotation, the 8-bit cache,
attention over it.

Tolerances.  A result of type t is off by at most finfo(t).eps / 2 of its value for its own rounding.  Before it:
norms: FP32 sums of D squares and a few products, 2^-20 of the larger feature of a pair.
attention: a probability is rounded to 11 bits (2^-11); FP32 scores are off by 2^-18 of sum |q| |k| at most (two tensor-core
sums of 128 products that round towards zero, and the parts of q below 2^-17 of its row's largest), which counts twice, in the
numerator and in the sum; the power of two and the sums of a few thousand terms add 2^-18.  Small ones end: a
probability times its value's scale, with the row's largest at 2^8 or more, is held in steps of 2^-24 (FP16) where there are many
rows, and as three E4M3 numbers, the third in steps of 2^-9 / 2^8, where there are few: it is off by 2^-18 / 2^8 = 2^-26 of the largest at
most, which multiplies its code: 2^-26 (largest p scale) (sum of |codes|).  (That shows where the tokens with the large
probabilities have a code of zero: with sm_scale = 1 one result in 150000 is 3e-11 beside others of 1.)
"""
import math

import pytest
import torch

import kv_ref as R
from paper_2307_09782_b200 import binding

pytestmark = pytest.mark.gpu
EPS = 1e-6


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- norms and rotation ---------------------------------------------------------------------------------------------
NORM_CASES = [
    # T, Hq, H, D, rot, pairs, norm, extra heads in a row
    (1, 12, 12, 64, 64, "halves", True, 0),
    (33, 32, 8, 128, 128, "halves", True, 8),
    (7, 5, 1, 128, 64, "neighbours", True, 3),
    (130, 9, 3, 64, 16, "neighbours", True, 0),
    (65, 17, 2, 64, 32, "halves", True, 1),
    (19, 8, 8, 128, 16, "halves", False, 0),
    (1000, 3, 3, 128, 128, "neighbours", True, 0),
]


def norm_inputs(case, seed=0):
    T, Hq, H, D, rot, pairs, norm, extra = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k = R.heads(T, Hq, D, seed + 1, extra), R.heads(T, H, D, seed + 2, extra)
    w = (1 + 0.3 * torch.randn((2, D), generator=g, device="cuda")) if norm else (None, None)
    table = binding.rotary_table(4099, rot)
    positions = torch.randint(0, 4099, (T,), generator=g, device="cuda", dtype=torch.int32)
    return q, k, w[0], w[1], table, positions


@pytest.mark.parametrize("case", NORM_CASES)
def test_norm_rope(case):
    q, k, wq, wk, table, positions = norm_inputs(case)
    yq, yk = binding.qk_norm_rope(q, k, table, positions, wq=wq, wk=wk, eps=EPS, pairs=case[5])
    for x, w, y in ((q, wq, yq), (k, wk, yk)):
        ref = R.norm_rope(x.to(R.F64), None if w is None else w.to(R.F64), table, positions, EPS, case[5])
        big = ref.abs().amax(-1, keepdim=True)
        assert ((y.to(R.F64) - ref).abs() <= half_step(torch.bfloat16) * ref.abs() + 2.0 ** -20 * big).all()


def test_norm_rope_in_place_and_zero_rows():
    case = NORM_CASES[1]
    q, k, wq, wk, table, positions = norm_inputs(case)
    q[3] = 0
    expect = binding.qk_norm_rope(q, k, table, positions, wq=wq, wk=wk)
    assert not expect[0][3].any()
    got = binding.qk_norm_rope(q, k, table, positions, wq=wq, wk=wk, out=(q, k))
    assert got[0].data_ptr() == q.data_ptr() and torch.equal(q, expect[0]) and torch.equal(k, expect[1])


def test_norm_rope_unknown_positions():
    """Outside the table: NaN in the rotated features, the others as usual; neighbours in the batch are not touched."""
    q, k, wq, wk, table, positions = norm_inputs((8, 4, 2, 128, 64, "halves", True, 0))
    good = binding.qk_norm_rope(q, k, table, positions, wq=wq, wk=wk)
    bad = positions.clone()
    bad[1], bad[5], bad[6] = -1, 4099, 2 ** 31 - 1
    got = binding.qk_norm_rope(q, k, table, bad, wq=wq, wk=wk)
    rows = torch.tensor([t not in (1, 5, 6) for t in range(8)], device="cuda")
    for y, ref in zip(got, good):
        assert torch.equal(y[rows], ref[rows]) and torch.equal(y[..., 64:], ref[..., 64:])
        assert y[~rows][..., :64].isnan().all()


@pytest.mark.parametrize("case", NORM_CASES)
def test_norm_rope_backward(case):
    q, k, wq, wk, table, positions = norm_inputs(case)
    T, Hq, H, D = case[:4]
    dq, dk = R.heads(T, Hq, D, 11, 2), R.heads(T, H, D, 12)
    got = binding.qk_norm_rope_backward(dq, dk, q, k, table, positions, wq=wq, wk=wk, eps=EPS, pairs=case[5])
    for x, w, dy, dx, dw in ((q, wq, dq, got[0], got[2]), (k, wk, dk, got[1], got[3])):
        x64 = x.to(R.F64).requires_grad_()
        w64 = None if w is None else w.to(R.F64).requires_grad_()
        R.norm_rope(x64, w64, table, positions, EPS, case[5]).backward(dy.to(R.F64))
        ref = x64.grad
        # a difference of two terms of the size of the rotated gradient / the row's norm
        size = (dy.to(R.F64).abs().amax(-1, keepdim=True) if w is None else
                dy.to(R.F64).norm(dim=-1, keepdim=True) * 2 * w.abs().max() / (x.to(R.F64).square().mean(-1, keepdim=True) + EPS).sqrt())
        assert ((dx.to(R.F64) - ref).abs() <= half_step(torch.bfloat16) * ref.abs() + 2.0 ** -19 * size).all()
        if w is None:
            assert dw is None
        else:
            n = (x.to(R.F64) / (x.to(R.F64).square().mean(-1, keepdim=True) + EPS).sqrt()).abs()
            terms = (dy.to(R.F64).norm(dim=-1, keepdim=True) * n).sum((0, 1))  # |g| is at most the norm of dy
            assert ((dw.to(R.F64) - w64.grad).abs() <= 2.0 ** -20 * terms).all()


def test_norm_rope_backward_against_differences():
    """Along random directions, from the forward pass in 64 bits: the operator's gradient against what the loss does."""
    case = (5, 2, 1, 64, 32, "halves", True, 0)
    q, k, wq, wk, table, positions = norm_inputs(case)
    dq, dk = R.heads(5, 2, 64, 11), R.heads(5, 1, 64, 12)
    gq, gk, gwq, gwk = binding.qk_norm_rope_backward(dq, dk, q, k, table, positions, wq=wq, wk=wk, eps=EPS)

    def loss(x, w, dy):
        return (R.norm_rope(x, w, table, positions, EPS, "halves") * dy.to(R.F64)).sum()
    for x, w, dy, gx, gw in ((q, wq, dq, gq, gwq), (k, wk, dk, gk, gwk)):
        g = torch.Generator(device="cuda").manual_seed(5)
        vx, vw = torch.randn(x.shape, generator=g, device="cuda").to(R.F64), torch.randn(w.shape, generator=g, device="cuda").to(R.F64)
        h = 1e-5
        x64, w64 = x.to(R.F64), w.to(R.F64)
        diff = (loss(x64 + h * vx, w64 + h * vw, dy) - loss(x64 - h * vx, w64 - h * vw, dy)) / (2 * h)
        ours = (gx.to(R.F64) * vx).sum() + (gw.to(R.F64) * vw).sum()
        # each gradient is rounded to bf16 (half a step), the differences are good to about h^2
        tol = half_step(torch.bfloat16) * (gx.to(R.F64) * vx).abs().sum() + 1e-6 * abs(diff) + 1e-6
        assert abs(diff - ours) <= tol


def test_norm_rope_no_tokens():
    q, k, wq, wk, table, positions = norm_inputs((4, 2, 2, 64, 64, "halves", True, 0))
    yq, _ = binding.qk_norm_rope(q[:0], k[:0], table, positions[:0], wq=wq, wk=wk)
    assert yq.shape == (0, 2, 64)
    got = binding.qk_norm_rope_backward(q[:0], k[:0], q[:0], k[:0], table, positions[:0], wq=wq, wk=wk)
    assert not got[2].any() and not got[3].any()


# ---- the cache ------------------------------------------------------------------------------------------------------
WRITE_CASES = [
    # lens, new, H, D, page, mode
    ([1], [1], 1, 64, 16, "none"),
    ([17, 64, 65], [1, 1, 1], 3, 128, 64, "none"),
    ([40, 1, 100, 33], [39, 1, 0, 33], 2, 64, 32, "M1"),
    ([300, 7], [129, 7], 2, 128, 128, "none"),
    ([50, 50], [17, 50], 5, 64, 16, "M1"),
    ([257], [200], 1, 128, 16, "none"),
    ([130, 128], [2, 128], 2, 64, 128, "M1"),
]


def same_scales(a, b):
    return torch.equal(a.nan_to_num(nan=-1.0), b.nan_to_num(nan=-1.0))


@pytest.mark.parametrize("case", WRITE_CASES)
def test_cache_write(case):
    lens, new, H, D, page, mode = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page, mode=mode)
    T = cu[-1]
    k, v = R.heads(T + 2, H, D, 3, 2), R.heads(T + 2, H, D, 4)  # two rows behind the last sequence
    k[T:] = math.nan
    k[:T // 2] *= 30  # scales that grow, and some that do not
    expect = R.write(codes, scale, k, v, table, lens, cu, mode)
    cache = binding.Fp8KvCache(codes, scale)
    binding.kv_cache_write(cache, k, v, table, R.ints(lens), cu=R.ints(cu), mode=mode)
    assert torch.equal(codes, expect[0]) and same_scales(scale, expect[1])
    if all(n == 1 for n in new):
        codes2, scale2, table, lens, cu = R.batch(lens, new, H, D, page, mode=mode)
        binding.kv_cache_write(binding.Fp8KvCache(codes2, scale2), k[:T], v[:T], table, R.ints(lens), mode=mode)
        assert torch.equal(codes2, expect[0]) and same_scales(scale2, expect[1])


def test_cache_write_token_by_token():
    """A page grows from zeros over small to large values and one that is not finite; another head stays as it is."""
    cache = binding.make_kv_cache(2, 2, 64, 16)
    codes, scale = cache.codes.clone(), cache.scale.clone()
    table = R.ints([[1, 0]])
    for i, f in enumerate([0.0, 1e-20, 1e-3, 1.0, 0.5, 1e4, math.inf, 1.0] + [1.0] * 10):
        k, v = R.heads(1, 2, 64, i), R.heads(1, 2, 64, 100 + i)
        if math.isinf(f):
            k[0, 0, 5] = f
        else:
            k[:, 0] *= f
        binding.kv_cache_write(cache, k, v, table, R.ints([i + 1]))
        codes, scale = R.write(codes, scale, k, v, table, [i + 1], [0, 1], "none")
        assert torch.equal(cache.codes, codes) and same_scales(cache.scale, scale), i
    assert scale[1, 0, 0].isnan() and not codes[1, 0, 0].any()  # the poisoned block: NaN, and no code that is one
    assert not scale[0].isnan().any() and not scale[1, :, 1].isnan().any()


def test_cache_write_wrong_names():
    """Pages outside the cache or the table, offsets that do not fit: nothing is written there, the others are."""
    codes, scale, table, lens, cu = R.batch([40, 40, 40, 40], [20, 20, 20, 20], 2, 64, 16)
    k, v = R.heads(80, 2, 64, 3), R.heads(80, 2, 64, 4)
    table[0, 2], table[1, 1] = -1, codes.shape[0]
    lens = [40, 40, 60, 19]  # the third runs out of the table, the fourth has fewer tokens than new ones
    expect = R.write(codes, scale, k, v, table, lens, cu, "none")
    binding.kv_cache_write(binding.Fp8KvCache(codes, scale), k, v, table, R.ints(lens), cu=R.ints(cu))
    assert torch.equal(codes, expect[0]) and same_scales(scale, expect[1])
    before = codes.clone(), scale.clone()
    for wrong in ([0, 0, 0, 0, 81], [-5, -5, -5, -5, -5], [9, 8, 7, 6, 5]):
        binding.kv_cache_write(binding.Fp8KvCache(codes, scale), k, v, table, R.ints([40, 40, 40, 40]), cu=R.ints(wrong))
    assert torch.equal(codes, before[0]) and same_scales(scale, before[1])


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,H,D,page", [([1], 1, 64, 16), ([130, 0, 64, 7], 3, 128, 64), ([33, 95], 2, 64, 32), ([200], 5, 128, 128)])
def test_cache_read(lens, H, D, page, out):
    codes, scale, table, lens, cu = R.batch(lens, lens, H, D, page)
    k, v = binding.kv_cache_read(binding.Fp8KvCache(codes, scale), table, R.ints(cu), cu[-1], out_dtype=out)
    for b in range(len(lens)):
        ref = R.gather(codes, scale, table[b].tolist(), lens[b])
        for i, x in enumerate((k, v)):
            r = ref[i].transpose(0, 1)
            # one product rounded to FP32 and then to the result's type
            assert ((x[cu[b]:cu[b + 1]].to(R.F64) - r).abs() <= (half_step(out) + 2.0 ** -24) * 1.01 * r.abs()).all()


def test_cache_read_missing_pages():
    codes, scale, table, lens, cu = R.batch([40], [40], 1, 64, 16)
    table[0, 1] = codes.shape[0] + 5
    k, _ = binding.kv_cache_read(binding.Fp8KvCache(codes, scale), table, R.ints([0, 60]), 60)
    assert k[16:32].isnan().all() and k[48:].isnan().all() and not k[:16].isnan().any()


# ---- attention ------------------------------------------------------------------------------------------------------
ATTN_CASES = [
    # lens, new, Hq, H, D, page, causal, window
    ([1], [1], 1, 1, 64, 16, True, 0),
    ([17], [1], 12, 12, 64, 16, True, 0),
    ([128, 129, 127, 1, 64], [1] * 5, 32, 8, 128, 64, True, 0),
    ([1000, 3, 0, 513], [1] * 4, 8, 1, 128, 32, True, 0),
    ([3000, 40], [1, 1], 7, 1, 64, 128, True, 0),
    ([1500, 700], [1, 1], 10, 2, 128, 16, True, 100),
    ([600, 30], [1, 1], 64, 1, 128, 64, True, 0),
    ([600, 30], [1, 1], 71, 1, 64, 64, True, 0),
    ([257, 40, 700], [4, 1, 9], 12, 4, 128, 64, True, 0),
    ([257, 40, 700], [4, 40, 9], 6, 6, 64, 32, True, 33),
    ([300], [300], 4, 2, 128, 128, True, 0),
    ([513, 1, 77, 400], [513, 1, 70, 0], 6, 2, 128, 16, True, 0),
    ([1030, 333], [130, 333], 5, 5, 64, 64, True, 0),
    ([1030, 333], [130, 333], 5, 5, 64, 64, True, 64),
    ([700, 129], [129, 1], 8, 4, 128, 64, False, 0),
    ([260, 5], [300, 9], 4, 2, 64, 16, True, 0),      # more new tokens than tokens: the first rows see nothing
    ([2049], [257], 16, 2, 128, 64, True, 1),
    ([5000], [3], 9, 3, 128, 128, True, 1300),
]


def attn_tolerance(ref, bound, out):
    pv, qk, low = bound
    return half_step(out) * ref.abs() + pv * (2.0 ** -11 + 2 * 2.0 ** -18 * qk[..., None] + 2.0 ** -17) + 2.0 ** -26 * low + 1e-30


def check_attention(case, out, seed=0, lens_override=None, **kw):
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page, seed)
    T = cu[-1]
    q = R.heads(T + 3, Hq, D, seed + 7, 2)
    single = all(n == 1 for n in new)
    res = torch.full((T + 3, Hq, D), 7.0, dtype=out, device="cuda")
    q_, res_ = (q[:T], res[:T]) if single else (q, res)
    sm = kw.pop("sm_scale", None)
    _, lse = binding.kv_attention(binding.Fp8KvCache(codes, scale), q_, table, R.ints(lens), cu=None if single else R.ints(cu),
                                  causal=causal, window=window, out=res_, lse=True, sm_scale=sm, **kw)
    assert (res[T:] == 7.0).all()  # rows behind the last sequence
    ref, ref_lse, bound = R.attention(codes, scale, q[:T], table, lens, cu, D ** -0.5 if sm is None else sm, causal, window)
    err, tol = (res[:T].to(R.F64) - ref).abs(), attn_tolerance(ref, bound, out)
    assert not res[:T].isnan().any()
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))
    lse = lse[:T].to(R.F64)
    none = ref_lse.isinf()
    assert torch.equal(lse[none], ref_lse[none])
    lerr, ltol = (lse - ref_lse)[~none].abs(), (2.0 ** -17 + 2.0 ** -18 * bound[1] + 2.0 ** -22 * ref_lse.abs())[~none]
    assert (lerr <= ltol).all(), float((lerr / ltol).max())


@pytest.mark.parametrize("case", ATTN_CASES)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_attention(case, out):
    check_attention(case, out)


@pytest.mark.parametrize("case", [
    ([2500, 2500, 40, 1900], [700, 1, 40, 650], 12, 12, 64, 32, True, 0),  # fewer row blocks than CTAs: several for each
    ([900] * 9, [200] * 9, 32, 8, 128, 64, True, 0),                       # more of them: CTAs that end inside one
    ([1500] * 3, [150] * 3, 40, 8, 128, 64, True, 200),                    # tokens' heads that do not fill a tile
    ([70] * 90, [70] * 90, 2, 1, 64, 16, True, 0),
    ([6000], [100], 4, 1, 128, 128, False, 0),                             # two blocks for all CTAs
    ([40, 0, 900] * 40, [40, 0, 33] * 40, 4, 2, 64, 64, True, 0),          # most sequences have none
])
def test_attention_blocks_over_ctas(case):
    check_attention(case, torch.float32)


@pytest.mark.parametrize("case", [([6001], [200], 4, 4, 128, 32, True, 0), ([9000] * 5, [1] * 5, 16, 8, 128, 64, True, 0),
                                  ([700, 30], [5, 30], 8, 2, 64, 64, True, 0)])
def test_attention_fp32_results_keep_more_than_probabilities_of_12_bits(case):
    """In the 2-norm.  The queries' two terms leave at most 2^-18 of a row's largest feature (about 4 sigma) per feature; over D independent
    ones times D^-1/2 a score is off by 4 / sqrt(3) 2^-18 < 2^-16.  Powers, FP32 sums and products (1e-8 each) are below that."""
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
    q = R.heads(cu[-1], Hq, D, 7)
    got = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), out_dtype=torch.float32)
    ref, _, _ = R.attention(codes, scale, q, table, lens, cu, D ** -0.5, causal, window)
    assert (got.to(R.F64) - ref).norm() <= 2.0 ** -16 * ref.norm()


@pytest.mark.parametrize("pad", [8, 64, 128])
def test_attention_rows_of_other_strides(pad):
    """Queries and results inside wider rows, whole heads wide or not."""
    for lens, new, Hq, H, D, page, causal, window in (ATTN_CASES[10], ATTN_CASES[11], ATTN_CASES[12]):
        codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
        q = R.heads(cu[-1], Hq, D, 7)
        args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
        want = binding.kv_attention(*args, cu=R.ints(cu), causal=causal, window=window)
        wide = torch.full((cu[-1], Hq * D + pad), float("nan"), device="cuda", dtype=torch.bfloat16)
        rows = wide[:, :Hq * D].view(cu[-1], Hq, D)
        rows.copy_(q)
        out = torch.zeros((cu[-1], Hq * D + pad), device="cuda", dtype=torch.bfloat16)
        binding.kv_attention(args[0], rows, *args[2:], cu=R.ints(cu), causal=causal, window=window, out=out[:, :Hq * D].view(cu[-1], Hq, D))
        assert torch.equal(out[:, :Hq * D].reshape(want.shape), want)
        assert not out[:, Hq * D:].any()


@pytest.mark.parametrize("sm_scale", [1.0, 0.01])
def test_attention_scale(sm_scale):
    check_attention(ATTN_CASES[2], torch.float32, 3, sm_scale=sm_scale)
    check_attention(ATTN_CASES[10], torch.float32, 3, sm_scale=sm_scale)


@pytest.mark.parametrize("case", [ATTN_CASES[2], ATTN_CASES[8], ATTN_CASES[11]])
def test_attention_zero_and_extreme_blocks(case):
    """Blocks of zero values, of the smallest scale and of scales 2^40 apart."""
    lens, new, Hq, H, D, page, causal, window = case
    codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
    owned = table[table >= 0].long()
    scale[owned[::3], 1] = 2.0 ** -20
    scale[owned[1::3], 1] = 2.0 ** 20
    codes[owned[0], 1] = 0
    scale[owned[0], 1] = 2.0 ** -39
    scale[owned[0], 0] = 2.0 ** -64
    q = R.heads(cu[-1], Hq, D, 7)
    got = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), causal=causal, window=window,
                               out_dtype=torch.float32)
    ref, _, bound = R.attention(codes, scale, q, table, lens, cu, D ** -0.5, causal, window)
    assert ((got.to(R.F64) - ref).abs() <= attn_tolerance(ref, bound, torch.float32)).all()


@pytest.mark.parametrize("case", [([300, 200], [1, 1], 8, 2, 128, 64, True, 0), ([300, 200], [6, 3], 8, 2, 128, 64, True, 0),
                                  ([300, 200], [24, 3], 4, 2, 128, 16, True, 0), ([300, 200], [250, 200], 4, 2, 64, 32, True, 0), ([300, 200], [250, 90], 4, 2, 128, 16, True, 40)])
def test_attention_nan_blocks(case):
    """A block that stands for NaN reaches the rows that see it and no others; so does a page the table names wrongly."""
    lens, new, Hq, H, D, page, causal, window = case
    for what in ("key", "value", "page"):
        codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
        i = 2 if page >= 64 else 17 if page == 16 and new[0] == 24 else 5  # (17: some of the first sequence's rows end before it)
        p = int(table[0, i])
        if what == "page":
            table[0, i] = -3
        else:
            scale[p, 0 if what == "key" else 1, 1] = math.nan
            codes[p, 0 if what == "key" else 1, 1] = 0
        q = R.heads(cu[-1], Hq, D, 7)
        got = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), causal=causal, window=window,
                                   out_dtype=torch.float32)
        ref, _, bound = R.attention(codes, scale, q, table, lens, cu, D ** -0.5, causal, window)
        # which rows see tokens of that page
        L, n = lens[0], cu[1]
        hit = torch.zeros((cu[-1], Hq), dtype=torch.bool, device="cuda")
        for r in range(n):
            pos = L - n + r
            lo = max(0, pos + 1 - window) if window else 0
            if lo < (i + 1) * page and pos >= i * page:
                hit[r, slice(None) if what == "page" else slice(Hq // H, 2 * Hq // H)] = True
        assert hit.any()
        assert got[hit].isnan().all()
        tol = attn_tolerance(ref, bound, torch.float32)
        assert ((got.to(R.F64) - ref).abs() <= tol)[~hit].all()


def test_attention_not_finite_queries():
    """A query that is not finite gives NaN in its own row and head only."""
    case = ([300, 200], [5, 1], 8, 2, 128, 64, True, 0)
    codes, scale, table, lens, cu = R.batch(*case[:2], *case[3:6])
    q = R.heads(6, 8, 128, 7)
    cache = binding.Fp8KvCache(codes, scale)
    good = binding.kv_attention(cache, q, table, R.ints(lens), cu=R.ints(cu))
    q[2, 3, 9], q[5, 0, 0] = math.nan, math.inf
    got = binding.kv_attention(cache, q, table, R.ints(lens), cu=R.ints(cu))
    hit = torch.zeros((6, 8), dtype=torch.bool, device="cuda")
    hit[2, 3] = hit[5, 0] = True
    assert got[hit].isnan().all() and torch.equal(got[~hit], good[~hit])


def test_attention_wrong_names():
    """Offsets that do not fit leave their rows alone; negative lengths are none."""
    codes, scale, table, lens, cu = R.batch([100, 100], [2, 2], 2, 64, 16)
    q = R.heads(4, 4, 64, 7)
    cache = binding.Fp8KvCache(codes, scale)
    for wrong in ([0, 5, 5], [-2, 0, 0], [3, 2, 1]):
        out = torch.full((4, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        binding.kv_attention(cache, q, table, R.ints(lens), cu=R.ints(wrong), out=out)
        assert (out == 7).all()
    out = binding.kv_attention(cache, q, table, R.ints([-5, 100]), cu=R.ints(cu))
    ref, _, bound = R.attention(codes, scale, q, table, [0, 100], cu, 0.125, True, 0)
    assert not out[:2].any()
    assert ((out.to(R.F64) - ref).abs() <= attn_tolerance(ref, bound, torch.bfloat16)).all()


def test_attention_repeats_its_bits():
    for case in (ATTN_CASES[3], ATTN_CASES[12]):
        lens, new, Hq, H, D, page, causal, window = case
        codes, scale, table, lens, cu = R.batch(lens, new, H, D, page)
        q = R.heads(cu[-1], Hq, D, 7)
        args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
        first = binding.kv_attention(*args, cu=R.ints(cu))
        for _ in range(5):
            assert torch.equal(binding.kv_attention(*args, cu=R.ints(cu)), first)
