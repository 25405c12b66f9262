"""FP8 products whose scales are all powers of two, many tokens: the tensor core applies the scales.

Integer codes and small powers of two make every sum exact in FP32, in any order, so those results are compared bit for bit.
Elsewhere the running sum stays in the tensor core over all K: each of its 4 KB additions of 32 products loses less than
33 x 2^-23 of the largest term or of the sum so far, hence |err| <= (132 KB + 2) 2^-23 S with S the sum of the absolute
products.
"""
import numpy as np
import pytest
import torch

import fp8_ref as R
from gpu_util import dev, host
from paper_2307_09782_b200 import binding
from test_gpu_fp8_block import acts, bf16_tensor, check_values, code_tol, ok, quantized_values, weight

pytestmark = pytest.mark.gpu


def ints(rng, shape):
    return rng.integers(-3, 4, shape).astype(np.float32)


def operand(codes_of, scales):
    return torch.from_numpy(R.e4m3_round(codes_of)).to(dev()), torch.from_numpy(np.ascontiguousarray(scales, np.float32)).to(dev())


def blocks(n):
    return (n + 127) // 128


# one tile pair and less, ragged everything, K of one block, more tile pairs than the device has, rings that wrap often
EXACT = [(100, 144, 300), (129, 16, 1), (200, 128, 256), (255, 272, 513), (384, 528, 257), (640, 3600, 384), (1100, 400, 8208),
         (300, 8208, 130)]


@pytest.mark.parametrize("M,K,N", EXACT)
@pytest.mark.parametrize("parts", [1, 2])
def test_linear_exact(M, K, N, parts):
    rng = np.random.default_rng(M + K + N)
    a, b = ints(rng, (parts, M, K)), ints(rng, (parts, N, K))
    sa = 2.0 ** rng.integers(0, 3, (parts, blocks(K), M))
    sb = 2.0 ** rng.integers(-1, 2, (parts, blocks(N), blocks(K)))
    row = 2.0 ** rng.integers(-20, 21, M)      # the same factor over a whole row: the sums stay exact
    ref = np.zeros((M, N))
    for i in range(parts):
        sa[i] *= row
        ref += (a[i] * np.repeat(sa[i].T, 128, 1)[:, :K]) @ (b[i] * np.repeat(np.repeat(sb[i], 128, 0)[:N], 128, 1)[:, :K]).T
    ca, ta = operand(a, sa)
    cb, tb = operand(b, sb)
    if parts == 1:
        q, w = binding.Fp8Block(ca[0], ta[0], pow2=True), binding.Fp8Weight(cb[0], tb[0], N, K)
    else:
        q, w = binding.Fp8Block(ca, ta, pow2=True), binding.Fp8Weight(cb, tb, N, K, parts=2)
    assert w.pow2
    ws = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(M, N, K))
    y = binding.fp8_block_linear(w, q=q, out_dtype=torch.bfloat16, workspace=ws)
    ok(ws)
    assert np.array_equal(host(y.float()), R.bf16(ref.astype(np.float32)))
    # and without the promise
    q.pow2 = False
    assert torch.equal(y, binding.fp8_block_linear(w, q=q, out_dtype=torch.bfloat16, workspace=ws))


@pytest.mark.parametrize("M,K,N", [(200, 272, 300), (700, 1040, 400)])
def test_linear_extreme_scales(M, K, N):
    """From the smallest scale there is to large ones; the other side makes up for it."""
    rng = np.random.default_rng(M)
    a, b = ints(rng, (M, K)), ints(rng, (N, K))
    e = rng.integers(-126, 101, blocks(K))                # per block of K: a's exponent, b's is the opposite, within its range
    sa = np.repeat(2.0 ** e[:, None], M, 1)
    sb = np.repeat(2.0 ** -np.clip(e, -120, 100)[None, :], blocks(N), 0)
    ref = (a * np.repeat(sa.T, 128, 1)[:, :K]) @ (b * np.repeat(np.repeat(sb, 128, 0)[:N], 128, 1)[:, :K]).T
    ca, ta = operand(a, sa)
    cb, tb = operand(b, sb)
    y = binding.fp8_block_linear(binding.Fp8Weight(cb, tb, N, K), q=binding.Fp8Block(ca, ta, pow2=True), out_dtype=torch.bfloat16)
    S = np.abs(a) @ np.abs(b).T
    check_values(y, ref, (132 * blocks(K) + 2) * 2.0 ** -23 * S, True)


def test_promise_is_not_made_for_other_scales():
    """A weight with other scales, or activations with the rule without powers of two, keep the FP32 scales."""
    M, K, N = 300, 400, 272
    x = acts(1, M, K)
    for wmode, mode in (("none", "M1"), ("M1", "none"), ("none", "none")):
        w, (wv,) = weight(9, N, K, wmode)
        assert w.pow2 == (wmode == "M1")
        xv = R.rows_values(*R.quantize_rows(x, mode))
        tol = (134 + 2 * blocks(K)) * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T)
        for args in (dict(x=bf16_tensor(x), mode=mode), dict(q=binding.quantize_fp8_block(bf16_tensor(x), mode))):
            check_values(binding.fp8_block_linear(w, out_dtype=torch.bfloat16, **args), xv @ wv.T, tol, True)
    w, _ = weight(9, N, K, "M1")
    assert binding.transpose_fp8_weight(binding.quantize_weight_fp8_block(torch.randn(256, 128, device=dev()), "M1")).pow2
    for other in (0.0, -0.5, float("inf"), 0.75, 2.0 ** -127):
        s = w.scale.clone()
        s[-1, -1] = other
        assert not binding.Fp8Weight(w.codes, s, N, K).pow2


@pytest.mark.parametrize("M", [140, 300, 513])
def test_not_finite(M):
    """A NaN or infinity reaches its own token's outputs and nobody else's."""
    K, N = 400, 272
    x = acts(3, M, K)
    x[M // 2, 140], x[M - 1, 399], x[0, 0] = np.nan, np.inf, -np.inf
    bad = [0, M // 2, M - 1]
    rest = np.delete(np.arange(M), bad)
    w, (wv,) = weight(4, N, K, "M1")
    y = host(binding.fp8_block_linear(w, x=bf16_tensor(x), mode="M1", out_dtype=torch.bfloat16).float())
    assert np.isnan(y[bad]).all() and np.isfinite(y[rest]).all()
    w, _ = weight(4, N, K, "M1", parts=2)
    h, hq, gu = binding.fp8_gated_linear(w, x=bf16_tensor(x), mode="M1", quantized=True, checkpoint=True)
    for v in (host(h.float()), quantized_values(hq), quantized_values(gu, 0), quantized_values(gu, 1)):
        assert np.isnan(v[bad]).all() and np.isfinite(v[rest]).all()


@pytest.mark.parametrize("M,K,F", [(100, 272, 144), (385, 8208, 272), (700, 400, 8208)])
@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "relu"])
def test_gated_and_backward(M, K, F, kind):
    x = acts(M + F, M, K)
    w, (wg, wu) = weight(F + 1, F, K, "M1", parts=2)
    xv = R.rows_values(*R.quantize_rows(x, "M1"))
    eps = (132 * blocks(K) + 2) * 2.0 ** -23
    g, u = xv @ wg.T, xv @ wu.T
    tg, tu = eps * (np.abs(xv) @ np.abs(wg).T), eps * (np.abs(xv) @ np.abs(wu).T)
    a, _ = R.act(g, kind)
    h = a * u
    th = 1.13 * tg * (np.abs(u) + tu) + (np.abs(a) + 1.13 * tg) * tu + 2.0 ** -18 * np.abs(h)
    ws = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(M, F, K))
    xq = binding.quantize_fp8_block(bf16_tensor(x), "M1")
    hb, hq, gu = binding.fp8_gated_linear(w, q=xq, act=kind, mode="M1", quantized=True, checkpoint=True, workspace=ws)
    ok(ws)
    check_values(hb, h, th, True)
    for b, i, v, t in ((hq, None, h, th), (gu, 0, g, tg), (gu, 1, u, tu)):
        assert (np.abs(quantized_values(b, i) - v) <= code_tol(v, "M1", t)).all()
    again = binding.fp8_gated_linear(w, x=bf16_tensor(x), act=kind, mode="M1", quantized=True, checkpoint=True, workspace=ws)
    assert torch.equal(again[0], hb) and torch.equal(again[1].codes, hq.codes) and torch.equal(again[2].codes, gu.codes)

    # the gradient's product from the same checkpoints: dy has K features, x's values serve
    wt, (wv,) = weight(F + 7, F, K, "M1")
    d, dq = binding.fp8_gated_linear_backward(wt, gu, q=xq, act=kind, mode="M1", workspace=ws)
    ok(ws)
    dh, t = xv @ wv.T, eps * (np.abs(xv) @ np.abs(wv).T)
    gv, uv = quantized_values(gu, 0), quantized_values(gu, 1)
    a, da = R.act(gv, kind)
    ea = 2.0 ** -18 * np.maximum(1.0, np.abs(gv))
    check_values(d[0], dh * uv * da, t * np.abs(uv * da) + (np.abs(dh) + t) * np.abs(uv) * ea, True)
    check_values(d[1], dh * a, t * np.abs(a) + (np.abs(dh) + t) * ea, True)
    for i in (0, 1):
        q = binding.quantize_fp8_block(d[i], "M1")
        assert torch.equal(q.codes, dq.codes[i]) and torch.equal(q.scale, dq.scale[i])


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("M,mode", [(5, "none"), (5, "M1"), (150, "M1")])
def test_gradient_far_out(M, mode, kind):
    """Far from zero the derivative is 0 or 1, also where the square of the argument overflows."""
    K, F = 144, 272
    rng = np.random.default_rng(M)
    dy = R.bf16(rng.standard_normal((M, K)) * 0.01)
    g, u = R.bf16(rng.standard_normal((M, F)) * 200), R.bf16(rng.standard_normal((M, F)))
    g[0], g[1], g[2, :128], g[2, 128:] = 1e20, -1e20, 90.0, -3e36
    wt, (wv,) = weight(F, F, K, mode)
    gq, uq = (binding.quantize_fp8_block(bf16_tensor(v), mode) for v in (g, u))
    gu = binding.Fp8Block(torch.stack([gq.codes, uq.codes]), torch.stack([gq.scale, uq.scale]))
    d, _ = binding.fp8_gated_linear_backward(wt, gu, dy=bf16_tensor(dy), act=kind, mode=mode)
    dyv = R.rows_values(*R.quantize_rows(dy, mode))
    dh, t = dyv @ wv.T, (134 + 2 * blocks(K)) * 2.0 ** -23 * (np.abs(dyv) @ np.abs(wv).T)
    gv, uv = quantized_values(gu, 0), quantized_values(gu, 1)
    a, da = R.act(gv, kind)
    ea = 2.0 ** -18 * np.maximum(1.0, np.abs(gv))
    check_values(d[0], dh * uv * da, t * np.abs(uv * da) + (np.abs(dh) + t) * np.abs(uv) * ea, True)
    check_values(d[1], dh * a, t * np.abs(a) + (np.abs(dh) + t) * ea, True)
