"""Calls of the FP8 operators right behind the work whose results they read: nothing may be read before it is there.

The values are small integers with scales of one, so that every sum is exact and results are compared bit for bit."""
import numpy as np
import pytest
import torch

import fp8_ref as R
from gpu_util import dev
from paper_2307_09782_b200 import binding, gated_ffn

pytestmark = pytest.mark.gpu


def codes(rng, shape):
    return torch.from_numpy(R.e4m3_round(rng.integers(-3, 4, shape).astype(np.float32))).to(dev())


def values(c):
    return c.view(torch.float8_e4m3fn).float()


@pytest.mark.parametrize("M,raw", [(1, True), (16, False), (20, True), (200, False)])
@pytest.mark.parametrize("gated", [False, True])
def test_weights_rewritten_just_before(M, raw, gated):
    """Codes written in place by torch kernels directly ahead of the call (or ahead of its quantizer), many times over: each call
    multiplies by the codes of its own turn."""
    K, N, turns = 2048, 4096, 40
    rng = np.random.default_rng(M)
    parts = 2 if gated else 1
    shape = (2, N, K) if gated else (N, K)
    some = [codes(rng, shape) for _ in range(3)]
    x = torch.from_numpy(rng.integers(-3, 4, (M, K)).astype(np.float32)).to(dev())
    if raw:
        x[:, ::128] = 448.0  # a block's largest value makes its scale one
    q = R.e4m3_round(x.cpu().numpy())
    q = binding.Fp8Block(torch.from_numpy(q).to(dev()), torch.ones((K // 128, M), device=dev()))
    xb = x.to(torch.bfloat16)
    w = binding.Fp8Weight(some[0].clone(), torch.ones((*shape[:-2], N // 128, K // 128), device=dev()), N, K, parts, pow2=False)
    ws = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(M, N, K))

    def call():
        kw = dict(x=xb) if raw else dict(q=q)
        if gated:
            return binding.fp8_gated_linear(w, act="relu", workspace=ws, **kw)[0]
        return binding.fp8_block_linear(w, workspace=ws, **kw)

    want = []
    for c in some:
        w.codes.copy_(c)
        torch.cuda.synchronize()
        want.append(call())
        torch.cuda.synchronize()
        if not gated:
            assert torch.equal(want[-1].double(), x.double() @ values(c).double().T)
    got = []
    for i in range(turns):
        w.codes.copy_(some[i % 3])
        got.append(call())
    torch.cuda.synchronize()
    assert binding.device_status(ws) == (0, 0)
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 3]), i


@pytest.mark.parametrize("M", [1, 20, 200])
@pytest.mark.parametrize("mode", ["none", "M1"])
def test_calls_in_a_row(M, mode):
    """Training and serving passes of two blocks one after the other on the same buffers, each reading what the kernel just ahead
    wrote: the same bits as with the device waited for in between."""
    K, F = 512, 720
    gen = torch.Generator(device="cuda").manual_seed(M)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device=dev()) * std

    blocks = [gated_ffn.GatedFfnFp8.from_weights(normal(F, K, std=0.05), normal(F, K, std=0.05), normal(K, F, std=0.05), mode=mode,
                                                 training=True) for _ in range(2)]
    for b in blocks[1:]:
        b._workspaces = blocks[0]._workspaces  # one workspace for both: what a call leaves there the next one overwrites
    xs = [normal(M, K).to(torch.bfloat16) for _ in range(2)]

    def chain(wait):
        out = []
        for i in range(12):
            x = xs[i % 2]
            keep = []
            for b in blocks:
                x, saved = b.forward_train(x)
                keep.append(saved)
                wait()
            dy = x
            for b, saved in zip(reversed(blocks), reversed(keep)):
                dy, dgu, dd = b.backward(dy, saved)
                out += [dgu, dd]
                wait()
            out += [x, dy, blocks[0].forward(dy)]
            wait()
        torch.cuda.synchronize()
        return out

    want = chain(torch.cuda.synchronize)
    for i, (a, b) in enumerate(zip(want, chain(lambda: None))):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)), i
