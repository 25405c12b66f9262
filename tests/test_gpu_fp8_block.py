"""The FP8 operators with block scales against plain 64-bit forms.

Tolerances.  The products of E4M3 values are exact in FP32.  The tensor core adds 32 of them at a time to a running
sum, aligned to the largest term, losing less than 2^-23 of it per term: at most 4 x 33 x 2^-23 of a block's
absolute sum.  The sum over KB blocks rounds twice per block (scale, FMA).  So |err| <= (132 + 2 KB + 2) 2^-23 S with S
the sum of the absolute products.  A bf16 result adds half a unit in its last place, 2^-8 of its value at most.
An E4M3 code is within 2^-4 of its value, or half a subnormal step (2^-10 of the scale), and the power-of-two scale of
a value at the edge can be the next one.
"""
import numpy as np
import pytest
import torch

import fp8_ref as R
from gpu_util import dev, host
from paper_2307_09782_b200 import binding, gated_ffn, synth

pytestmark = pytest.mark.gpu


def bf16_tensor(v):
    return torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(dev()).to(torch.bfloat16)


def acts(seed, M, K, zero_rows=True):
    x = synth.bf16_bits_to_f32(synth.make_x(seed, M, K, max(1, K // 100)))
    if zero_rows and M > 2:
        x[M // 2] = 0.0           # a token with nothing in it
        x[0, :min(K, 128)] = 0.0  # and a block
    return x


def sum_tol(S, K, parts=1):
    return (134 + 2 * parts * ((K + 127) // 128)) * 2.0 ** -23 * S


def check_values(y, ref, tol, bf16=False):
    y = host(y.float()).astype(np.float64)
    assert y.shape == ref.shape
    lim = tol + (2.0 ** -8 * (np.abs(ref) + tol) if bf16 else 0)
    bad = ~(np.abs(y - ref) <= lim)
    assert not bad.any(), f"{bad.sum()} of {bad.size}; worst {np.abs(y - ref).max():.3e}, first {np.argwhere(bad)[0]}"


def ok(ws):
    assert binding.device_status(ws) == (0, 0)


def weight(seed, N, K, mode, parts=1):
    W = np.stack([synth.make_w(seed + i, N, K) for i in range(parts)])
    if N > 128 and K > 128:
        W[:, :128, 128:256] = 0.0
    w = binding.quantize_weight_fp8_block(torch.from_numpy(W if parts > 1 else W[0]).to(dev()), mode)
    vals = []
    for i in range(parts):
        q, s = R.quantize_blocks(W[i], mode)
        assert np.array_equal(host(w.codes).reshape(parts, N, K)[i], q)
        assert np.array_equal(host(w.scale).reshape(parts, *s.shape)[i], s)
        vals.append(R.blocks_values(q, s))
    return w, vals


# ---- quantizers ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("mode", ["none", "M1"])
@pytest.mark.parametrize("M,K,pad", [(1, 16, 0), (1, 4096, 0), (3, 128, 8), (17, 144, 0), (33, 1040, 24), (300, 2048, 0),
                                     (2000, 528, 8)])
def test_quantize_rows(M, K, pad, mode):
    x = acts(M + K, M, K)
    xp = torch.zeros((M, K + pad), dtype=torch.bfloat16, device=dev())
    xp[:, :K] = bf16_tensor(x)
    q = binding.quantize_fp8_block(xp[:, :K], mode)
    qr, sr = R.quantize_rows(x, mode)
    assert np.array_equal(host(q.codes), qr)
    assert np.array_equal(host(q.scale), sr)
    assert np.array_equal(host(q.values()).astype(np.float64), R.rows_values(qr, sr).astype(np.float32))


@pytest.mark.parametrize("mode", ["none", "M1"])
def test_quantize_extremes(mode):
    """Largest and smallest numbers, exact powers of two at the edge of the rule, infinities and NaN in one block each."""
    x = np.zeros((10, 384), np.float32)
    x[0, 3] = 3.3895314e38
    x[1, 3] = 2.0 ** -126
    x[2, :] = 2.0 ** -133          # the smallest bf16 number
    x[3, 130] = 448.0
    x[4, 130] = 450.0
    x[5, 300] = 3.5
    x[6, 1], x[6, 200] = np.inf, 1.0
    x[7, 1], x[7, 200] = np.nan, 1.0
    x[8, 383] = -np.inf
    x[9, :] = -0.0
    q = binding.quantize_fp8_block(bf16_tensor(x), mode)
    qr, sr = R.quantize_rows(R.bf16(x), mode)
    np.testing.assert_array_equal(host(q.scale), sr)
    v, vr = host(q.values()).astype(np.float64), R.rows_values(qr, sr)
    np.testing.assert_array_equal(np.isnan(v), np.isnan(vr))
    fine = np.isfinite(vr)
    assert np.array_equal(host(q.codes)[fine], qr[fine])
    assert np.isnan(v[6, :128]).all() and np.isfinite(v[6, 128:]).all()


@pytest.mark.parametrize("mode", ["none", "M1"])
@pytest.mark.parametrize("N,K", [(1, 16), (128, 128), (144, 272), (1000, 528)])
def test_quantize_weight_and_transpose(N, K, mode):
    w, _ = weight(N + K, N, K, mode)
    if N % 16:
        with pytest.raises(binding.ZqError):
            binding.transpose_fp8_weight(w)
        return
    t = binding.transpose_fp8_weight(w)
    assert (t.N, t.K) == (K, N)
    assert torch.equal(t.codes, w.codes.t().contiguous()) and torch.equal(t.scale, w.scale.t().contiguous())


# ---- linear ------------------------------------------------------------------------------------------------------------
LINEAR = [(1, 16, 1), (1, 128, 128), (1, 4096, 300), (2, 528, 129), (7, 144, 1000), (16, 2048, 128), (17, 1040, 1001),
          (33, 272, 257), (64, 1536, 640), (65, 400, 2), (100, 1040, 1001), (129, 256, 384), (130, 2064, 513),
          (257, 144, 255), (500, 640, 900),
          (2, 8192, 130), (16, 8208, 128), (40, 8192, 130)]  # long rows: every ring of the kernels wraps around


@pytest.mark.parametrize("M,K,N", LINEAR)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", ["none", "M1"])
def test_linear(M, K, N, out, mode):
    x = acts(M * 3 + K, M, K)
    w, (wv,) = weight(N, N, K, mode)
    qr, sr = R.quantize_rows(x, mode)
    xv = R.rows_values(qr, sr)
    ref, S = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    ws = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(M, N, K))
    xt = bf16_tensor(x)
    y = binding.fp8_block_linear(w, x=xt, mode=mode, out_dtype=out, workspace=ws)
    ok(ws)
    check_values(y, ref, sum_tol(S, K), out == torch.bfloat16)
    # the quantized form of the same activations, and the same call again: the same bits
    y2 = binding.fp8_block_linear(w, q=binding.quantize_fp8_block(xt, mode), out_dtype=out, workspace=ws)
    assert torch.equal(y, y2)
    assert torch.equal(y, binding.fp8_block_linear(w, x=xt, mode=mode, out_dtype=out, workspace=ws))


@pytest.mark.parametrize("M,K,N", [(3, 144, 70), (33, 272, 257), (200, 528, 300)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_linear_strided(M, K, N, out):
    """Rows of x and y further apart than they are long, at an odd offset for y; nothing beside y's rows is written."""
    x = acts(5, M, K)
    w, (wv,) = weight(6, N, K, "none")
    xp = torch.full((M, K + 40), float("nan"), dtype=torch.bfloat16, device=dev())
    xp[:, :K] = bf16_tensor(x)
    for off, pad in ((1, 2), (0, 3), (8, 16)):
        big = torch.full((M, N + off + pad), 7.0, dtype=out, device=dev())
        y = big[:, off:off + N]
        binding.fp8_block_linear(w, x=xp[:, :K], y=y)
        xv = R.rows_values(*R.quantize_rows(x, "none"))
        check_values(y, xv @ wv.T, sum_tol(np.abs(xv) @ np.abs(wv).T, K), out == torch.bfloat16)
        assert (big[:, :off] == 7.0).all() and (big[:, off + N:] == 7.0).all()


@pytest.mark.parametrize("M,K,N", [(1, 256, 144), (40, 144, 300), (150, 528, 272)])
def test_linear_two_parts(M, K, N):
    w, (w0, w1) = weight(9, N, K, "none", parts=2)
    x0, x1 = acts(1, M, K), acts(2, M, K)
    q0, q1 = (binding.quantize_fp8_block(bf16_tensor(x)) for x in (x0, x1))
    q = binding.Fp8Block(torch.stack([q0.codes, q1.codes]), torch.stack([q0.scale, q1.scale]))
    y = binding.fp8_block_linear(w, q=q)
    v0, v1 = (R.rows_values(*R.quantize_rows(x, "none")) for x in (x0, x1))
    S = np.abs(v0) @ np.abs(w0).T + np.abs(v1) @ np.abs(w1).T
    check_values(y, v0 @ w0.T + v1 @ w1.T, sum_tol(S, K, 2))


@pytest.mark.parametrize("M", [1, 20, 70, 200])
def test_linear_not_finite(M):
    """A NaN reaches its own token's outputs and nobody else's."""
    K, N = 272, 200
    x = acts(3, M, K)
    x[M // 2, 140] = np.nan
    w, (wv,) = weight(4, N, K, "none")
    y = host(binding.fp8_block_linear(w, x=bf16_tensor(x)))
    assert np.isnan(y[M // 2]).all()
    rest = np.delete(np.arange(M), M // 2)
    assert np.isfinite(y[rest]).all()


def test_linear_empty():
    w, _ = weight(4, 200, 272, "none")
    y = binding.fp8_block_linear(w, x=torch.empty((0, 272), dtype=torch.bfloat16, device=dev()))
    assert y.shape == (0, 200)


def test_linear_side_stream():
    """On a stream of the caller's, behind work queued there."""
    x, (w, (wv,)) = acts(8, 50, 512), weight(8, 256, 512, "none")
    st = torch.cuda.Stream()
    xt = bf16_tensor(x * 0)
    src = bf16_tensor(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(2_000_000)
        xt.copy_(src)
        y = binding.fp8_block_linear(w, x=xt)
    st.synchronize()
    xv = R.rows_values(*R.quantize_rows(x, "none"))
    check_values(y, xv @ wv.T, sum_tol(np.abs(xv) @ np.abs(wv).T, 512))


# ---- gated layer -----------------------------------------------------------------------------------------------------
def code_tol(v, mode, extra):
    """How far a quantized value may be from a 64-bit one, itself known to `extra`."""
    M, N = v.shape
    p = R._pad(np.abs(v) + extra, [1]).reshape(M, -1, 128)
    s = np.maximum(p.max(2) / 448, 2.0 ** -126) * (2 if mode == "M1" else 1)
    step = np.repeat(s, 128, 1)[:, :N] * 2.0 ** -10 * (2 if mode == "M1" else 1)
    return 2.0 ** -4 * (1 + 2.0 ** -10) * (np.abs(v) + extra) + step + extra


def quantized_values(b, i=None):
    c, s = (b.codes, b.scale) if i is None else (b.codes[i], b.scale[i])
    return R.rows_values(host(c), host(s))


GATED = [(1, 16, 16), (1, 512, 400), (3, 144, 128), (16, 1040, 272), (30, 256, 144), (64, 272, 640), (70, 528, 720),
         (130, 400, 144), (300, 144, 272), (1, 8192, 144), (16, 8208, 128)]


@pytest.mark.parametrize("M,K,F", GATED)
@pytest.mark.parametrize("kind,mode", [("silu", "none"), ("gelu_tanh", "M1"), ("relu", "none"), ("silu", "M1")])
def test_gated(M, K, F, kind, mode):
    x = acts(M + F, M, K)
    w, (wg, wu) = weight(F + 1, F, K, mode, parts=2)
    xv = R.rows_values(*R.quantize_rows(x, mode))
    g, u = xv @ wg.T, xv @ wu.T
    tg, tu = sum_tol(np.abs(xv) @ np.abs(wg).T, K), sum_tol(np.abs(xv) @ np.abs(wu).T, K)
    a, _ = R.act(g, kind)
    h = a * u
    # |act'| <= 1.13; the fast exponential and division add 2^-18 of the value at most
    th = 1.13 * tg * (np.abs(u) + tu) + (np.abs(a) + 1.13 * tg) * tu + 2.0 ** -18 * np.abs(h)
    ws = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(M, F, K))
    hb, hq, gu = binding.fp8_gated_linear(w, x=bf16_tensor(x), act=kind, mode=mode, quantized=True, checkpoint=True,
                                          workspace=ws)
    ok(ws)
    check_values(hb, h, th, True)
    for b, i, v, t in ((hq, None, h, th), (gu, 0, g, tg), (gu, 1, u, tu)):
        err = np.abs(quantized_values(b, i) - v)
        assert (err <= code_tol(v, mode, t)).all(), (i, err.max())
    # each output alone is the same
    only, _, _ = binding.fp8_gated_linear(w, x=bf16_tensor(x), act=kind, mode=mode, workspace=ws)
    assert torch.equal(only, hb)
    q = binding.quantize_fp8_block(bf16_tensor(x), mode)
    none, only, _ = binding.fp8_gated_linear(w, q=q, act=kind, mode=mode, bf16=False, quantized=True, workspace=ws)
    assert none is None and torch.equal(only.codes, hq.codes) and torch.equal(only.scale, hq.scale)


@pytest.mark.parametrize("M", [2, 40, 140])
def test_gated_not_finite(M):
    x = acts(3, M, 144)
    x[1, 5] = np.inf
    w, _ = weight(4, 144, 144, "none", parts=2)
    h, hq, gu = binding.fp8_gated_linear(w, x=bf16_tensor(x), quantized=True, checkpoint=True)
    rest = np.delete(np.arange(M), 1)
    for v in (host(h.float()), quantized_values(hq), quantized_values(gu, 0), quantized_values(gu, 1)):
        assert np.isnan(v[1]).all() and np.isfinite(v[rest]).all()


# ---- backward --------------------------------------------------------------------------------------------------------
BACK = [(1, 16, 16), (5, 144, 272), (70, 528, 720), (130, 400, 144), (260, 272, 400)]


@pytest.mark.parametrize("M,K,F", BACK)
@pytest.mark.parametrize("kind,mode", [("silu", "M1"), ("gelu_tanh", "none"), ("relu", "M1")])
def test_gated_backward(M, K, F, kind, mode):
    rng = np.random.default_rng(M + F)
    dy = R.bf16(rng.standard_normal((M, K)) * 0.01)
    g, u = (R.bf16(rng.standard_normal((M, F)) * 2) for _ in range(2))
    if M > 1:
        dy[1] = 0.0
        g[0] = 0.0
    wt, (wv,) = weight(F, F, K, mode)    # the transposed down projection
    gq, uq = (binding.quantize_fp8_block(bf16_tensor(v), mode) for v in (g, u))
    gu = binding.Fp8Block(torch.stack([gq.codes, uq.codes]), torch.stack([gq.scale, uq.scale]))
    ws = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(M, F, K))
    d, dq = binding.fp8_gated_linear_backward(wt, gu, dy=bf16_tensor(dy), act=kind, mode=mode, workspace=ws)
    ok(ws)
    dyv = R.rows_values(*R.quantize_rows(dy, mode))
    dh, t = dyv @ wv.T, sum_tol(np.abs(dyv) @ np.abs(wv).T, K)
    gv, uv = quantized_values(gu, 0), quantized_values(gu, 1)
    a, da = R.act(gv, kind)
    # value and derivative by the fast exponential and division: 2^-18 of max(1, |g|)
    ea = 2.0 ** -18 * np.maximum(1.0, np.abs(gv))
    check_values(d[0], dh * uv * da, t * np.abs(uv * da) + (np.abs(dh) + t) * np.abs(uv) * ea, True)
    check_values(d[1], dh * a, t * np.abs(a) + (np.abs(dh) + t) * ea, True)
    # the quantized gradients are those of the bf16 ones, bit for bit
    for i in (0, 1):
        q = binding.quantize_fp8_block(d[i], mode)
        assert torch.equal(q.codes, dq.codes[i]) and torch.equal(q.scale, dq.scale[i])


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "relu"])
def test_backward_against_differences(kind):
    """dg and du against central differences of sum(dh * act(g) u) in 64 bits, at the checkpoint's g and u."""
    M, F, K = 20, 144, 144
    rng = np.random.default_rng(3)
    dy = R.bf16(rng.standard_normal((M, K)) * 0.1)
    g, u = (R.bf16(rng.standard_normal((M, F)) * 2) for _ in range(2))
    wt, (wv,) = weight(5, F, K, "M1")
    gq, uq = (binding.quantize_fp8_block(bf16_tensor(v), "M1") for v in (g, u))
    gu = binding.Fp8Block(torch.stack([gq.codes, uq.codes]), torch.stack([gq.scale, uq.scale]))
    d, _ = binding.fp8_gated_linear_backward(wt, gu, dy=bf16_tensor(dy), act=kind, mode="M1")
    dh = R.rows_values(*R.quantize_rows(dy, "M1")) @ wv.T
    gv, uv = quantized_values(gu, 0), quantized_values(gu, 1)
    e = 1e-5
    away = np.abs(gv) > 2 * e if kind == "relu" else np.ones_like(gv, bool)  # the kink has no difference quotient
    fd_g = dh * uv * (R.act(gv + e, kind)[0] - R.act(gv - e, kind)[0]) / (2 * e)
    fd_u = dh * (R.act(gv, kind)[0] * (uv + e) - R.act(gv, kind)[0] * (uv - e)) / (2 * e)
    # bf16 rounding, 2^-8; the rest (differences 1e-9, FP32 sums) is far below 2^-12 of the row's largest
    for i, fd in ((0, fd_g), (1, fd_u)):
        lim = 2.0 ** -8 * np.abs(fd) + 2.0 ** -12 * np.abs(fd).max(1, keepdims=True)
        assert (np.abs(host(d[i].float()) - fd) <= lim)[away].all()


# ---- weight gradient -------------------------------------------------------------------------------------------------
WGRAD = [(1, 16, 1, 1), (3, 128, 128, 1), (64, 144, 100, 1), (65, 272, 257, 1), (333, 768, 144, 1), (200, 400, 130, 2),
         (1000, 256, 512, 1), (129, 528, 8, 3),
         (2100, 144, 40, 1), (4500, 272, 300, 1), (8200, 128, 130, 1), (2100, 1552, 1500, 1)]  # few tiles, many tokens: clusters of 2, 4, 8


@pytest.mark.parametrize("M,K,N,parts", WGRAD)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", ["M1", "none"])
def test_weight_grad(M, K, N, parts, out, mode):
    rng = np.random.default_rng(M + N)
    x = acts(M + 1, M, K)
    ld = (N + 7) // 8 * 8 + 8
    G = R.bf16(rng.standard_normal((parts, M, N)) * 0.01)
    gt = torch.full((parts, M, ld), float("nan"), dtype=torch.bfloat16, device=dev())
    gt[:, :, :N] = bf16_tensor(G)
    gv = gt[:, :, :N] if parts > 1 else gt[0, :, :N]
    q = binding.quantize_fp8_block(bf16_tensor(x), mode)
    ws = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(0, 0, 16))
    dw = binding.fp8_weight_grad(gv, q, out_dtype=out, workspace=ws)
    ok(ws)
    xv = R.rows_values(*R.quantize_rows(x, mode))
    xb = R.bf16(xv.astype(np.float32)).astype(np.float64)
    if mode == "M1":
        assert np.array_equal(xb, xv)
    ref = np.stack([g.astype(np.float64).T @ xb for g in G])
    S = np.stack([np.abs(g.astype(np.float64)).T @ np.abs(xb) for g in G])
    # one running FP32 sum: tensor-core adds of 16 terms, each losing less than 2^-23 of the largest, and the sum of
    # the absolute products bounds every partial sum
    tol = (17 * ((M + 15) // 16) + 2) * 2.0 ** -23 * S
    check_values(dw, ref if parts > 1 else ref[0], tol if parts > 1 else tol[0], out == torch.bfloat16)
    assert torch.equal(dw, binding.fp8_weight_grad(gv, q, out_dtype=out, workspace=ws))


def test_weight_grad_empty():
    q = binding.quantize_fp8_block(torch.empty((0, 144), dtype=torch.bfloat16, device=dev()))
    dw = binding.fp8_weight_grad(torch.empty((0, 24), dtype=torch.bfloat16, device=dev()), q)
    assert dw.shape == (24, 144) and not dw.any()


def test_weight_grad_against_differences():
    """d/dW of sum(G * (x^ W^T)) by differences: the function is linear, so the difference quotient is the gradient."""
    rng = np.random.default_rng(0)
    M, N, K = 40, 24, 144
    G, x = R.bf16(rng.standard_normal((M, N))), acts(1, M, K)
    q = binding.quantize_fp8_block(bf16_tensor(x), "M1")
    dw = host(binding.fp8_weight_grad(bf16_tensor(G), q)).astype(np.float64)
    xv = R.rows_values(*R.quantize_rows(x, "M1"))
    loss = lambda W: (G.astype(np.float64) * (xv @ W.T)).sum()  # noqa: E731
    W = rng.standard_normal((N, K))
    S = np.abs(G).astype(np.float64).T @ np.abs(xv)
    for n, k in ((0, 0), (23, 143), (7, 100)):
        E = np.zeros((N, K))
        E[n, k] = 0.5
        fd = loss(W + E) - loss(W - E)
        assert abs(dw[n, k] - fd) <= (17 * 3 + 2) * 2.0 ** -23 * S[n, k] + 1e-9 * S.max()


# ---- the block ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("M", [1, 20, 150])
@pytest.mark.parametrize("mode", ["none", "M1"])
def test_block_step(M, mode):
    """Serving and training pass of the whole block against 64 bits.  The codes in between can fall on either side of a
    rounding boundary, so outputs are compared in the 2-norm: a flipped code moves its value by 2^-3 at most, and fewer
    than one in a thousand flips (FP32 sums are good to 2^-15 of a rounding step), which gives 2^-3 sqrt(1e-3) = 4e-3 on
    top of the bf16 rounding, 2^-9."""
    K, F = 528, 720
    rng = np.random.default_rng(M)
    x = acts(M, M, K)
    W = [synth.make_w(i, *s) for i, s in enumerate([(F, K), (F, K), (K, F)])]
    ffn = gated_ffn.GatedFfnFp8.from_weights(*[torch.from_numpy(w).to(dev()) for w in W], mode=mode, training=True)
    wg, wu, wd = [R.blocks_values(*R.quantize_blocks(w, mode)) for w in W]
    dy = R.bf16(rng.standard_normal((M, K)) * 0.01)
    xt, dyt = bf16_tensor(x), bf16_tensor(dy)
    y0 = ffn.forward(xt)
    y, saved = ffn.forward_train(xt)
    assert torch.equal(y, y0)
    dx, dwgu, dwd = ffn.backward(dyt, saved)
    ok(ffn.workspace(M))
    # the calls it strings together give the same bits
    xq = binding.quantize_fp8_block(xt, mode)
    h, hq, gu = binding.fp8_gated_linear(ffn.gate_up, q=xq, mode=mode, quantized=True, checkpoint=True)
    assert torch.equal(y, binding.fp8_block_linear(ffn.down, q=hq, out_dtype=torch.bfloat16))
    d, dq = binding.fp8_gated_linear_backward(ffn.down_t, gu, dy=dyt, mode=mode)
    assert torch.equal(dx, binding.fp8_block_linear(ffn.gate_up_t, q=dq, out_dtype=torch.bfloat16))
    assert torch.equal(dwgu, binding.fp8_weight_grad(d, xq, out_dtype=torch.bfloat16))
    assert torch.equal(dwd, binding.fp8_weight_grad(dyt, hq, out_dtype=torch.bfloat16))

    def fq(v):
        return R.rows_values(*R.quantize_rows(np.asarray(v, np.float32), mode))

    xv = fq(x)
    g, u = xv @ wg.T, xv @ wu.T
    hv = fq(R.act(g, "silu")[0] * u)
    gv, uv = fq(g), fq(u)
    dh = fq(dy) @ wd
    a, da = R.act(gv, "silu")
    dg, du = R.bf16(dh * uv * da), R.bf16(dh * a)
    xb, hb = R.bf16(xv).astype(np.float64), R.bf16(hv).astype(np.float64)
    ref = {"y": hv @ wd.T, "dx": fq(dg) @ wg + fq(du) @ wu,
           "dwg": dg.T.astype(np.float64) @ xb, "dwu": du.T.astype(np.float64) @ xb, "dwd": dy.T.astype(np.float64) @ hb}
    got = {"y": y, "dx": dx, "dwg": dwgu[0], "dwu": dwgu[1], "dwd": dwd}
    for k, r in ref.items():
        v = host(got[k].float()).astype(np.float64)
        rel = np.linalg.norm(v - r) / np.linalg.norm(r)
        assert rel <= 2.0 ** -9 + 4e-3, (k, rel)


def test_example_trains_and_serves():
    """The example's loop lowers its loss, and its single-token passes agree with the batch to bf16 rounding."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_ffn_fp8.py")
    spec = importlib.util.spec_from_file_location("gated_ffn_fp8_example", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses, ffn, x = ex.train(128, 256, 384, 25, log=None)
    assert losses[-1] < 0.7 * losses[0]
    whole = ffn.forward(x).float()
    one = torch.cat([ffn.forward(x[i:i + 1]) for i in range(4)]).float()
    # the sums differ in order only; a code of h in between can flip by one step (2^-3 of one of 384 terms)
    assert ((one - whole[:4]).norm() / whole[:4].norm()) < 2.0 ** -8 + 4e-3


def test_offsets_beyond_32_bits():
    """More than 2^31 codes and 2^32 bytes of activations: the last rows come out like a call on them alone."""
    M, K, N = 70_001, 32_768, 16
    x = torch.randn((1, K), device=dev()).to(torch.bfloat16).expand(M, K).contiguous()
    x[-3:] = torch.randn((3, K), device=dev()).to(torch.bfloat16)
    w, _ = weight(1, N, K, "none")
    q, ql = binding.quantize_fp8_block(x), binding.quantize_fp8_block(x[-3:])
    assert torch.equal(q.codes[-3:], ql.codes) and torch.equal(q.scale[:, -3:], ql.scale)
    y = binding.fp8_block_linear(w, q=q)
    yl = binding.fp8_block_linear(w, q=ql)
    assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[-4])
    S = ql.values().abs() @ w.values().abs().t()
    assert ((y[-3:] - yl).abs() <= 2 * sum_tol(S, K)).all()
    g = torch.zeros((M, 8), dtype=torch.bfloat16, device=dev())
    g[-3:] = 1.0
    dw = binding.fp8_weight_grad(g, q)
    dl = binding.fp8_weight_grad(g[-3:].contiguous(), ql)
    assert ((dw - dl).abs() <= 2.0 ** -20 * ql.values().abs().sum(0)).all()
