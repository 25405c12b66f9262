"""The FP8 operators with block scales without a GPU: what the C entry points refuse before anything is launched, what the
binding refuses, size queries, and the plain forms the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
import fp8_ref as R
from paper_2307_09782_b200 import binding, gated_ffn

NULL, P, ODD = None, 0x10000, 0x10004  # P: aligned to 256 bytes, never dereferenced
NONE, M1, M2 = 0, 1, 2
ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_MODE, ERR_WS = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def L():
    entry.build()
    return binding.lib()


def test_quantizer_refusals(L):
    f = L.zq_quantize_fp8_block

    def call(x=P, M=4, K=64, ldx=64, mode=NONE, q=P, s=P):
        return f(x, M, K, ldx, mode, q, s, None)

    assert call(mode=M2) == ERR_MODE and call(mode=7) == ERR_MODE
    assert call(K=60) == ERR_SHAPE and call(K=0) == ERR_SHAPE and call(ldx=56) == ERR_SHAPE and call(M=-1) == ERR_SHAPE
    assert call(x=NULL) == ERR_NULL and call(q=NULL) == ERR_NULL and call(s=NULL) == ERR_NULL
    assert call(x=ODD) == ERR_ALIGN and call(q=ODD) == ERR_ALIGN and call(ldx=68) == ERR_ALIGN
    assert call(M=0, x=NULL, q=NULL, s=NULL) == 0

    g = L.zq_quantize_weight_fp8_block
    assert g(P, 4, 64, M2, P, P, None) == ERR_MODE
    assert g(P, 4, 60, NONE, P, P, None) == ERR_SHAPE
    assert g(NULL, 4, 64, NONE, P, P, None) == ERR_NULL
    assert g(ODD, 4, 64, NONE, P, P, None) == ERR_ALIGN
    assert g(NULL, 0, 64, NONE, NULL, NULL, None) == 0

    t = L.zq_transpose_weight_fp8_block
    assert t(P, P, 24, 64, P, P, None) == ERR_SHAPE  # the transposed rows would not be multiples of 16
    assert t(P, P, 32, 60, P, P, None) == ERR_SHAPE
    assert t(P, NULL, 32, 64, P, P, None) == ERR_NULL
    assert t(ODD, P, 32, 64, P, P, None) == ERR_ALIGN


def test_linear_refusals(L):
    ws = binding.fp8_block_linear_workspace_bytes(4, 0, 64)

    def call(q=P, s=P, x=NULL, ldx=0, mode=NONE, parts=1, M=4, N=8, K=64, w=P, wsc=P, y=P, ydt=0, ldy=8, work=P, nws=ws):
        return L.zq_fp8_block_linear(q, s, x, ldx, mode, parts, M, N, K, w, wsc, y, ydt, ldy, work, nws, None)

    assert call(mode=M2) == ERR_MODE and call(ydt=2) == ERR_MODE
    for kw in (dict(K=72), dict(K=8), dict(N=-1), dict(M=-2), dict(ldy=7), dict(parts=0), dict(parts=3),
               dict(q=NULL, s=NULL, x=P, ldx=64, parts=2), dict(q=NULL, s=NULL, x=P, ldx=56)):
        assert call(**kw) == ERR_SHAPE, kw
    for kw in (dict(q=NULL), dict(s=NULL), dict(w=NULL), dict(wsc=NULL), dict(y=NULL), dict(x=P, ldx=64)):
        assert call(**kw) == ERR_NULL, kw  # the last: raw and quantized at once
    for kw in (dict(q=ODD), dict(w=ODD), dict(y=P + 2), dict(work=P + 16), dict(q=NULL, s=NULL, x=ODD, ldx=64),
               dict(q=NULL, s=NULL, x=P, ldx=68)):
        assert call(**kw) == ERR_ALIGN, kw
    assert call(work=NULL) == ERR_WS and call(nws=100) == ERR_WS
    assert call(q=NULL, s=NULL, x=P, ldx=64, nws=ws - 1) == ERR_WS
    assert call(M=0) == 0 and call(N=0, ldy=0) == 0


def test_gated_refusals(L):
    ws = binding.fp8_block_linear_workspace_bytes(4, 0, 64)

    def call(q=P, s=P, mode=NONE, M=4, F=32, K=64, w=P, wsc=P, act=0, h=P, ldh=32, hq=NULL, hs=NULL, gu=NULL, gus=NULL,
             work=P, nws=ws):
        return L.zq_fp8_gated_linear(q, s, NULL, 0, mode, M, F, K, w, wsc, act, h, ldh, hq, hs, gu, gus, work, nws, None)

    assert call(mode=M2) == ERR_MODE and call(act=3) == ERR_MODE
    assert call(F=24) == ERR_SHAPE and call(ldh=31) == ERR_SHAPE and call(K=24) == ERR_SHAPE
    assert call(h=NULL) == ERR_NULL and call(hq=P) == ERR_NULL and call(gu=P) == ERR_NULL and call(w=NULL) == ERR_NULL
    assert call(hq=ODD, hs=P) == ERR_ALIGN and call(gu=ODD, gus=P) == ERR_ALIGN and call(h=P + 1) == ERR_ALIGN
    assert call(nws=0) == ERR_WS and call(M=0) == 0

    def back(q=P, s=P, mode=NONE, F=32, K=64, act=0, wt=P, gu=P, d=P, dq=P, ds=P, work=P, nws=ws, M=4):
        return L.zq_fp8_gated_linear_backward(q, s, NULL, 0, mode, M, F, K, wt, P, act, gu, P, d, dq, ds, work, nws, None)

    assert back(mode=M2) == ERR_MODE and back(act=-1) == ERR_MODE
    assert back(F=20) == ERR_SHAPE
    assert back(gu=NULL) == ERR_NULL and back(d=NULL) == ERR_NULL and back(dq=NULL) == ERR_NULL and back(ds=NULL) == ERR_NULL
    assert back(d=ODD) == ERR_ALIGN and back(wt=ODD) == ERR_ALIGN
    assert back(work=NULL) == ERR_WS and back(M=0) == 0


def test_weight_grad_refusals(L):
    ws = binding.fp8_block_linear_workspace_bytes(0, 0, 16)

    def call(g=P, ldg=8, stride=0, parts=1, q=P, s=P, M=4, N=8, K=64, dw=P, dt=0, work=P, nws=ws):
        return L.zq_fp8_weight_grad(g, ldg, stride, parts, q, s, M, N, K, dw, dt, work, nws, None)

    assert call(dt=2) == ERR_MODE
    assert call(parts=2, stride=0) == ERR_SHAPE  # several parts in one place
    assert call(ldg=7) == ERR_SHAPE and call(parts=0) == ERR_SHAPE and call(parts=65) == ERR_SHAPE and call(K=40) == ERR_SHAPE
    assert call(g=NULL) == ERR_NULL and call(q=NULL) == ERR_NULL and call(dw=NULL) == ERR_NULL
    assert call(N=4, ldg=12) == ERR_ALIGN and call(stride=4, parts=2) == ERR_ALIGN and call(dw=ODD) == ERR_ALIGN
    assert call(nws=16) == ERR_WS and call(N=0, ldg=0) == 0


def test_ffn_refusals(L):
    M, K, F, N = 4, 64, 32, 48
    ws = binding.fp8_gated_ffn_workspace_bytes(M, K, F, N, True)

    def call(x=P, ldx=K, mode=NONE, M=M, K=K, F=F, N=N, gu=P, dn=P, act=0, y=P, ydt=1, ldy=N, saved=NULL, work=P, nws=ws):
        return L.zq_fp8_gated_ffn(x, ldx, mode, M, K, F, N, gu, P, dn, P, act, y, ydt, ldy, saved, work, nws, None)

    assert call(mode=M2) == ERR_MODE and call(act=9) == ERR_MODE and call(ydt=5) == ERR_MODE
    assert call(F=40) == ERR_SHAPE and call(ldx=32) == ERR_SHAPE and call(ldy=47) == ERR_SHAPE
    assert call(x=NULL) == ERR_NULL and call(dn=NULL) == ERR_NULL and call(y=NULL) == ERR_NULL
    assert call(saved=P + 16) == ERR_ALIGN and call(x=ODD) == ERR_ALIGN
    assert call(nws=1000) == ERR_WS and call(M=0) == 0

    def back(dy=P, lddy=N, mode=NONE, N=N, saved=P, gut=P, dnt=P, act=0, dx=P, dw=P, dd=P, dt=1, work=P, nws=ws):
        return L.zq_fp8_gated_ffn_backward(dy, lddy, mode, M, K, F, N, saved, gut, P, dnt, P, act, dx, dw, dd, dt, work, nws,
                                           None)

    assert back(mode=M2) == ERR_MODE and back(dt=3) == ERR_MODE
    assert back(N=40, lddy=40) == ERR_SHAPE and back(lddy=40) == ERR_SHAPE
    assert back(saved=NULL) == ERR_NULL and back(dw=NULL) == ERR_NULL and back(dx=NULL) == ERR_NULL
    assert back(dy=ODD) == ERR_ALIGN and back(dw=ODD) == ERR_ALIGN
    assert back(nws=binding.fp8_gated_ffn_workspace_bytes(M, K, F, N, False)) == ERR_WS


def test_size_queries(L):
    head = binding.fp8_block_linear_workspace_bytes(0, 0, 16)
    assert head >= 256 + 4 * 16384
    assert binding.fp8_block_linear_workspace_bytes(100, 0, 1040) >= head + 100 * 1040 + 9 * 100 * 4
    assert binding.fp8_gated_ffn_saved_bytes(10, 64, 32) >= 10 * 64 + 3 * 10 * 32 + 4 * 10 * 4
    for M in (1, 7, 100, 4095):
        assert binding.fp8_gated_ffn_workspace_bytes(M, 4096, 11008, 4096, True) <= \
            binding.fp8_gated_ffn_workspace_bytes(4096, 4096, 11008, 4096, True)
    # refused sizes
    assert binding.fp8_block_linear_workspace_bytes(4, 0, 24) == 0 and binding.fp8_block_linear_workspace_bytes(-1, 0, 64) == 0
    assert binding.fp8_gated_ffn_saved_bytes(4, 64, 24) == 0
    assert binding.fp8_gated_ffn_workspace_bytes(4, 64, 32, 40, True) == 0
    assert binding.fp8_gated_ffn_workspace_bytes(4, 64, 32, 40, False) > 0


def test_binding_refusals(L):
    u8, f32, bf = torch.uint8, torch.float32, torch.bfloat16
    w = binding.Fp8Weight(torch.zeros((32, 64), dtype=u8), torch.ones((1, 1)), 32, 64)
    with pytest.raises(ValueError):
        binding.Fp8Weight(torch.zeros((32, 64), dtype=u8), torch.ones((1, 2)), 32, 64)
    with pytest.raises(ValueError):
        binding.Fp8Weight(torch.zeros((64, 32), dtype=u8).t(), torch.ones((1, 1)), 32, 64)  # not contiguous
    with pytest.raises(ValueError):
        binding.quantize_fp8_block(torch.zeros((4, 64), dtype=f32))
    with pytest.raises(ValueError):
        binding.quantize_fp8_block(torch.zeros((64, 4), dtype=bf).t())
    with pytest.raises(ValueError):
        binding.fp8_block_linear(w)  # neither raw nor quantized
    with pytest.raises(ValueError):
        binding.fp8_block_linear(w, x=torch.zeros((4, 48), dtype=bf))
    q = binding.Fp8Block(torch.zeros((4, 64), dtype=u8), torch.ones((4, 1)))  # scales the wrong way round
    with pytest.raises(ValueError):
        binding.fp8_block_linear(w, q=q)
    with pytest.raises(ValueError):
        binding.fp8_gated_linear(w, x=torch.zeros((4, 64), dtype=bf))  # one projection, two are needed
    with pytest.raises(ValueError):
        binding.fp8_weight_grad(torch.zeros((5, 8), dtype=bf), binding.Fp8Block(torch.zeros((4, 64), dtype=u8), torch.ones((1, 4))))
    x = torch.zeros((4, 64), dtype=bf)  # fits, but in host memory
    for call in (lambda: binding.quantize_fp8_block(x), lambda: binding.fp8_block_linear(w, x=x),
                 lambda: binding.transpose_fp8_weight(w), lambda: binding.quantize_weight_fp8_block(torch.zeros((32, 64))),
                 lambda: binding.fp8_weight_grad(torch.zeros((4, 8), dtype=bf),
                                                 binding.Fp8Block(torch.zeros((4, 64), dtype=u8), torch.ones((1, 4))))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    gu = binding.Fp8Weight(torch.zeros((2, 32, 64), dtype=u8), torch.ones((2, 1, 1)), 32, 64, parts=2)
    with pytest.raises(ValueError):
        gated_ffn.GatedFfnFp8(gu, w)  # down has 64 features, the gated layer 32
    ffn = gated_ffn.GatedFfnFp8(gu, binding.Fp8Weight(torch.zeros((64, 32), dtype=u8), torch.ones((1, 1)), 64, 32))
    with pytest.raises(ValueError):
        ffn.backward(torch.zeros((4, 64), dtype=bf), torch.zeros(16, dtype=u8))  # not constructed for training


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def test_ref_codes_against_torch():
    """Every E4M3 value, and a spread of others, against torch's own cast."""
    rng = np.random.default_rng(0)
    v = np.concatenate([R.DEC[np.isfinite(R.DEC)], rng.standard_normal(20000) * 100, rng.standard_normal(20000) * 0.01,
                        np.arange(-448, 449, 0.5)]).astype(np.float32)
    t = torch.from_numpy(v).clamp(-448, 448).to(torch.float8_e4m3fn)
    assert np.array_equal(R.e4m3_round(v), t.view(torch.uint8).numpy())
    assert np.array_equal(R.DEC[R.e4m3_round(v)].astype(np.float32), t.float().numpy())


@pytest.mark.parametrize("mode", ["none", "M1"])
def test_ref_quantizer(mode):
    rng = np.random.default_rng(1)
    x = R.bf16(rng.standard_normal((5, 300)) * 3)
    x[2] = 0
    q, s = R.quantize_rows(x, mode)
    assert q.shape == (5, 300) and s.shape == (3, 5)
    v = R.rows_values(q, s)
    step = np.repeat(s.T.astype(np.float64), 128, 1)[:, :300] * 2.0 ** -10
    assert (np.abs(v - x) <= 2.0 ** -4 * np.abs(x) + step).all()
    assert (s[:, 2] == 1).all() and not q[2].any()
    if mode == "M1":
        assert (np.frexp(s)[0] == 0.5).all() and np.array_equal(R.bf16(v).astype(np.float64), v)
    else:
        assert np.abs(R.DEC[q]).max() == 448


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "relu"])
def test_ref_activation_derivative(kind):
    v = np.linspace(-8, 8, 401) + 0.003
    e = 1e-6
    fd = (R.act(v + e, kind)[0] - R.act(v - e, kind)[0]) / (2 * e)
    assert np.abs(fd - R.act(v, kind)[1]).max() < 1e-8


def test_promise_of_powers_of_two(L):
    """Where the promise may be made, and where it is refused."""
    P2 = binding.SCALES_POW2
    assert L.zq_quantize_fp8_block(P, 4, 64, 64, M1 | P2, P, P, None) == ERR_MODE      # nothing is given that has scales
    assert L.zq_quantize_weight_fp8_block(P, 4, 64, M1 | P2, P, P, None) == ERR_MODE
    ws = binding.fp8_block_linear_workspace_bytes(4, 8, 64)

    def call(mode, q=P, s=P, x=NULL, ldx=0, work=P, nws=ws):
        return L.zq_fp8_block_linear(q, s, x, ldx, mode, 1, 4, 8, 64, P, P, P, 0, 8, work, nws, None)

    raw = dict(q=NULL, s=NULL, x=P, ldx=64)
    assert call(M2 | P2) == ERR_MODE and call(P2 << 1) == ERR_MODE and call(-1) == ERR_MODE
    assert call(NONE | P2, **raw) == ERR_MODE                      # the call's own scales would not be powers of two
    # accepted as far as the mode goes: the next check answers
    assert call(M1 | P2, **raw, work=NULL) in (ERR_NULL, ERR_WS) and call(NONE | P2, work=NULL) in (ERR_NULL, ERR_WS)


def test_promise_of_the_binding():
    """The binding promises what it knows: of a weight on the CPU nothing."""
    codes = torch.zeros((128, 128), dtype=torch.uint8)
    assert binding.Fp8Weight(codes, torch.ones((1, 1)), 128, 128).pow2 is False
    w = binding.Fp8Weight(codes, torch.ones((1, 1)), 128, 128, pow2=True)
    assert binding._scales("M1", w, None) == M1 | binding.SCALES_POW2 and binding._scales("none", w, None) == NONE
    q = binding.Fp8Block(codes, torch.ones((1, 128)))
    assert binding._scales("M1", w, q) == M1                       # given activations of unknown scales
    q.pow2 = True
    assert binding._scales("none", w, q) == NONE | binding.SCALES_POW2
    w.pow2 = False
    assert binding._scales("M1", w, q) == M1
