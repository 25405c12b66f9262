"""How the FP8 operators are called: sizes one after the other without a workspace of the caller's, empty batches, results of
more bytes than 32 bits count, stream capture, threads, scales that change in place."""
import threading

import numpy as np
import pytest
import torch

import fp8_ref as R
from gpu_util import dev
from paper_2307_09782_b200 import binding, gated_ffn
from test_gpu_fp8_block import acts, bf16_tensor, check_values, sum_tol, weight

pytestmark = pytest.mark.gpu


def test_kept_workspace_over_sizes():
    """Raw activations of sizes whose needs are not ordered like M (K + 128)."""
    w = {K: binding.quantize_weight_fp8_block(torch.randn((48, K), device=dev())) for K in (256, 512, 1024, 4096)}
    with torch.cuda.stream(torch.cuda.Stream()):  # a stream that has no workspace yet
        for M, K in ((2048, 512), (300, 4096), (100, 1024), (27, 4096), (8192, 256), (700, 4096)):
            x = torch.randn((M, K), device=dev()).to(torch.bfloat16)
            y = binding.fp8_block_linear(w[K], x=x)
            assert torch.equal(y, binding.fp8_block_linear(w[K], q=binding.quantize_fp8_block(x))), (M, K)
        torch.cuda.synchronize()


def test_captured_calls():
    """A graph captured on a stream where the same calls ran before, replayed after those calls' workspaces have grown: it
    computes on new inputs, and writes to nothing but its own memory."""
    K, F, M = 512, 720, 24
    ffn = gated_ffn.GatedFfnFp8.from_weights(*[torch.randn(s, device=dev()) * 0.05 for s in ((F, K), (F, K), (K, F))], mode="M1")
    down = binding.quantize_weight_fp8_block(torch.randn((K, K), device=dev()) * 0.05)
    x = torch.randn((M, K), device=dev()).to(torch.bfloat16)
    big = torch.randn((3000, K), device=dev()).to(torch.bfloat16)
    s = torch.cuda.Stream()

    def both(v):
        return binding.fp8_block_linear(down, x=ffn.forward(v), out_dtype=torch.bfloat16)

    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both(x)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        y = both(x)
    with torch.cuda.stream(s):
        both(big)  # the kept workspaces grow: the old ones go back to the allocator
        fill = [torch.full((1 << 18,), 7, dtype=torch.uint8, device=dev()) for _ in range(64)]
    s.synchronize()
    for v in (x.clone(), torch.randn_like(x)):
        x.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, both(v))
    assert all(bool((f == 7).all()) for f in fill)


def test_threads_on_one_stream():
    """Two threads use one block on the same stream, each with its own tokens."""
    K, F, M = 512, 720, 40
    ffn = gated_ffn.GatedFfnFp8.from_weights(*[torch.randn(s, device=dev()) * 0.05 for s in ((F, K), (F, K), (K, F))])
    xs = [torch.randn((M, K), device=dev()).to(torch.bfloat16) for _ in range(2)]

    def call(x):
        y = ffn.forward(x)
        return y, binding.fp8_block_linear(ffn.down, x=torch.nn.functional.pad(y, (0, F - K)), out_dtype=torch.bfloat16)

    want = [call(x) for x in xs]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        for _ in range(200):
            got[i].append(call(xs[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 200
        assert all(torch.equal(a, b) for pair in got[i] for a, b in zip(pair, want[i]))


def test_scales_written_in_place():
    """Scales that were powers of two and are no more, and back: every call multiplies by the scales of its time."""
    M, K, N = 300, 528, 400
    x = acts(1, M, K)
    w, _ = weight(2, N, K, "M1")
    xv, xt = R.rows_values(*R.quantize_rows(x, "M1")), bf16_tensor(x)
    pow2 = w.scale.clone()
    first = binding.fp8_block_linear(w, x=xt, mode="M1", out_dtype=torch.bfloat16)
    for factor in (1.5, 0.3, 1.0):
        w.scale.copy_(pow2 * factor)
        wv = R.blocks_values(w.codes.cpu().numpy(), w.scale.cpu().numpy())
        y = binding.fp8_block_linear(w, x=xt, mode="M1", out_dtype=torch.bfloat16)
        check_values(y, xv @ wv.T, (132 * ((K + 127) // 128) + 2) * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T), True)
        assert w.pow2 is (factor == 1.0)
    assert torch.equal(y, first)


def test_scales_looked_up_late():
    """A weight wrapped under stream capture waits for nothing; its scales are looked at by the first eager call that asks."""
    M, K, N = 300, 528, 400
    w0, _ = weight(2, N, K, "M1")
    x = bf16_tensor(acts(1, M, K))
    want = binding.fp8_block_linear(w0, x=x, mode="M1")
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        w = binding.Fp8Weight(w0.codes, w0.scale, N, K)
        y = binding.fp8_block_linear(w, x=x, mode="M1")
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and w.pow2 is True


@pytest.mark.parametrize("bad", [1.5, -2.0, 2.0 ** -130, float("inf")])
def test_broken_promise_shows(bad):
    """A scale that is no power of two where one was promised: NaN in the results it belongs to, the others as they were."""
    M, K, N = 300, 528, 400
    w, _ = weight(2, N, K, "M1")
    q = binding.quantize_fp8_block(bf16_tensor(acts(1, M, K)), "M1")
    want = binding.fp8_block_linear(w, q=q, out_dtype=torch.bfloat16)
    q.scale[3, 70] = bad
    w.scale[1, 2] = bad
    q.pow2 = w.pow2 = True
    y = binding.fp8_block_linear(w, q=q, out_dtype=torch.bfloat16)
    rows, cols = torch.arange(M, device=dev()) == 70, torch.arange(N, device=dev()) // 128 == 1
    hit = rows[:, None] | cols[None, :]
    assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], want[~hit])


@pytest.mark.parametrize("mode", ["none", "M1"])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_no_tokens(mode, out):
    """An empty batch through every call: results without rows, weight gradients of zeros."""
    K, F, N = 144, 272, 160
    W = [torch.randn(s, device=dev()) for s in ((F, K), (F, K), (N, F))]
    ffn = gated_ffn.GatedFfnFp8.from_weights(*W, mode=mode, training=True)
    x, dy = (torch.empty((0, n), dtype=torch.bfloat16, device=dev()) for n in (K, N))
    assert ffn.forward(x, out_dtype=out).shape == (0, N)
    y, saved = ffn.forward_train(x, out_dtype=out)
    torch.full((1 << 16,), 7.0, device=dev())  # what the next results' memory may hold
    dx, dgu, dd = ffn.backward(dy, saved, out_dtype=out)
    assert y.shape == (0, N) and dx.shape == (0, K)
    assert dgu.shape == (2, F, K) and not dgu.any() and dd.shape == (N, F) and not dd.any()
    q = binding.quantize_fp8_block(x, mode)
    h, hq, gu = binding.fp8_gated_linear(ffn.gate_up, q=q, mode=mode, quantized=True, checkpoint=True)
    assert h.shape == (0, F) and hq.codes.shape == (0, F) and gu.codes.shape == (2, 0, F)
    d, dq = binding.fp8_gated_linear_backward(ffn.down_t, gu, dy=dy, mode=mode)
    assert d.shape == (2, 0, F) and dq.scale.shape == (2, 3, 0)
    dw = binding.fp8_weight_grad(d, q, out_dtype=out)
    assert dw.shape == (2, F, K) and not dw.any()
    assert binding.fp8_block_linear(ffn.gate_up_t, q=dq, out_dtype=out).shape == (0, K)


def test_weight_grad_of_one_token():
    """One token whose outputs are no multiple of eight, as a matrix and as a stack of one."""
    g = torch.randn((1, 20), device=dev()).to(torch.bfloat16)
    q = binding.quantize_fp8_block(torch.randn((1, 144), device=dev()).to(torch.bfloat16), "M1")
    dw = binding.fp8_weight_grad(g, q)
    assert torch.equal(dw, g.float().T @ q.values())  # one product each: exact
    assert torch.equal(binding.fp8_weight_grad(g[None], q), dw[None])


def test_outputs_beyond_32_bits_of_bytes():
    """2^29 outputs per token in FP32: the first ones, the last ones and those around multiples of 2^29 bytes are there."""
    M, K, N = 33, 16, (1 << 29) + 40
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 85 GB")
    probe = torch.tensor([0, 1, 127, 255, 256, 1 << 27, (1 << 28) + 3, (1 << 29) - 1, 1 << 29, N - 1], device=dev())
    codes = torch.full((N, K), 0x38, dtype=torch.uint8, device=dev())  # ones
    codes[probe] = torch.from_numpy(R.e4m3_round(np.random.default_rng(0).integers(-3, 4, (len(probe), K)).astype(np.float32))).to(dev())
    w = binding.Fp8Weight(codes, torch.ones(((N + 127) // 128, 1), device=dev()), N, K, pow2=False)
    q = binding.quantize_fp8_block(torch.randint(-3, 4, (M, K), device=dev()).to(torch.bfloat16), "M1")
    y = torch.full((M, N), -1000.0, device=dev())
    binding.fp8_block_linear(w, q=q, y=y)
    torch.cuda.synchronize()
    xv = q.values()
    assert torch.equal(y[:, probe], xv @ codes[probe].view(torch.float8_e4m3fn).float().T)
    step = 1 << 26
    row_sums = xv.sum(1)
    other = torch.ones(N, dtype=torch.bool, device=dev())
    other[probe] = False
    for n0 in range(0, N, step):
        part, keep = y[:, n0:n0 + step], other[n0:n0 + step]
        for m in (0, 7, 32):
            assert bool((part[m] == row_sums[m])[keep].all()), (m, n0)


def test_callers_workspace_refusals():
    """A workspace in host memory, of another type or not in one piece, in every call that takes one."""
    K, F, M = 144, 272, 8
    W = [torch.randn(s, device=dev()) for s in ((F, K), (F, K), (K, F))]
    ffn = gated_ffn.GatedFfnFp8.from_weights(*W, training=True)
    x = torch.randn((M, K), device=dev()).to(torch.bfloat16)
    y, saved = ffn.forward_train(x)
    q = binding.quantize_fp8_block(x)
    _, hq, gu = binding.fp8_gated_linear(ffn.gate_up, q=q, quantized=True, checkpoint=True)
    calls = [lambda ws: binding.fp8_block_linear(ffn.down, q=hq, workspace=ws),
             lambda ws: binding.fp8_gated_linear(ffn.gate_up, x=x, workspace=ws),
             lambda ws: binding.fp8_gated_linear_backward(ffn.down_t, gu, dy=x, workspace=ws),
             lambda ws: binding.fp8_weight_grad(x, q, workspace=ws),
             lambda ws: binding.fp8_gated_ffn(ffn.gate_up, ffn.down, x, workspace=ws),
             lambda ws: binding.fp8_gated_ffn_backward(ffn.gate_up_t, ffn.down_t, x, saved, workspace=ws)]
    n = 1 << 20
    for ws in (torch.zeros(n, dtype=torch.uint8), torch.zeros(n, device=dev()),
               torch.zeros(1, dtype=torch.uint8, device=dev()).expand(n), torch.zeros(n, dtype=torch.uint8, device=dev())[::2]):
        for call in calls:
            with pytest.raises(ValueError):
                call(ws)
    assert torch.equal(ffn.forward(x), y)
