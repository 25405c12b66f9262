"""Cases that measure the FP8 operators with block scales: the linear layer, the gated feed-forward block for serving
and for training, and weight gradients from 8-bit activation checkpoints.

Where ``own`` is false, ``run`` computes them in elementary torch operations in 32 bits; where it is true, through the
package's public calls.  Both take what ``prepare`` gives.
"""
import math

import torch

own = False

BLOCK = 128


# ---- cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a linear layer that serves one token of one user (7-billion-parameter attention projection)
        {"name": "linear-1-token", "op": "linear", "M": 1, "K": 4096, "N": 4096, "mode": "none", "out": "bf16"},
        # sizes that fill no tile: a projection head with an odd number of outputs, FP32 results
        {"name": "linear-ragged", "op": "linear", "M": 100, "K": 1040, "N": 1001, "mode": "M1", "out": "f32"},
        # a decoding batch of 32 through the widest layer of the 30-billion-parameter sweep
        {"name": "linear-32-tokens", "op": "linear", "M": 32, "K": 7168, "N": 28672, "mode": "none", "out": "bf16"},
        # prefill of 8192 tokens through the same layer
        {"name": "linear-prefill", "op": "linear", "M": 8192, "K": 7168, "N": 28672, "mode": "none", "out": "bf16"},
        # the whole gated block for one token
        {"name": "ffn-1-token", "op": "ffn", "M": 1, "K": 4096, "F": 11008, "mode": "none", "act": "silu"},
        # the whole gated block for an odd decoding batch of the larger model
        {"name": "ffn-33-tokens", "op": "ffn", "M": 33, "K": 6656, "F": 17920, "mode": "M1", "act": "silu"},
        # prefill of 2048 tokens
        {"name": "ffn-prefill", "op": "ffn", "M": 2048, "K": 4096, "F": 11008, "mode": "none", "act": "silu"},
        # one training step of a small block with ragged sizes
        {"name": "train-ragged", "op": "train", "M": 77, "K": 528, "F": 720, "mode": "M1", "act": "gelu_tanh"},
        # one training step, 2048 tokens
        {"name": "train-2048", "op": "train", "M": 2048, "K": 4096, "F": 11008, "mode": "M1", "act": "silu"},
        # one training step of the larger block, 4096 tokens
        {"name": "train-4096", "op": "train", "M": 4096, "K": 6656, "F": 17920, "mode": "M1", "act": "silu"},
        # weight gradient of a small projection from an 8-bit checkpoint, odd number of tokens
        {"name": "checkpoint-333", "op": "checkpoint", "M": 333, "K": 768, "N": 768, "mode": "M1", "out": "f32"},
        # the same for a long sequence
        {"name": "checkpoint-16384", "op": "checkpoint", "M": 16384, "K": 4096, "N": 4096, "mode": "M1", "out": "f32"},
    ]


def _log(rng, lo, hi, mult=1):
    """A whole number spread over the logarithm of [lo, hi], a multiple of `mult`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / mult)) * mult))


MOST_FLOPS = 8.0e12  # of a drawn case: below the largest listed one's


def draw(rng):
    while True:
        op = rng.choice(["linear", "linear", "ffn", "ffn", "train", "checkpoint"])
        if op == "linear":
            c = {"op": op, "M": _log(rng, 1, 8192), "K": _log(rng, 256, 28672, 16), "N": _log(rng, 64, 28672),
                 "mode": rng.choice(["none", "M1"]), "out": rng.choice(["bf16", "f32"])}
        elif op == "ffn":
            c = {"op": op, "M": _log(rng, 1, 4096), "K": _log(rng, 512, 8192, 16), "F": _log(rng, 512, 18432, 16),
                 "mode": rng.choice(["none", "M1"]), "act": rng.choice(["silu", "gelu_tanh", "relu"])}
        elif op == "train":
            c = {"op": op, "M": _log(rng, 48, 4096), "K": _log(rng, 512, 6656, 16), "F": _log(rng, 512, 17920, 16),
                 "mode": "M1", "act": rng.choice(["silu", "gelu_tanh", "relu"])}
        else:
            c = {"op": op, "M": _log(rng, 64, 16384), "K": _log(rng, 256, 8192, 16), "N": _log(rng, 256, 8192, 8),
                 "mode": "M1", "out": rng.choice(["bf16", "f32"])}
        if work(c)["flops"] <= MOST_FLOPS:
            return c


def work(case):
    op, M, K = case["op"], case["M"], case["K"]
    if op == "linear":
        N = case["N"]
        return {"bytes": 2 * M * K + N * K + M * N * (4 if case["out"] == "f32" else 2), "flops": 2 * M * N * K}
    if op == "checkpoint":
        N = case["N"]
        return {"bytes": 2 * M * K + 2 * M * N + M * K + N * K * (4 if case["out"] == "f32" else 2), "flops": 2 * M * N * K}
    F = case["F"]
    if op == "ffn":
        return {"bytes": 4 * M * K + 3 * F * K, "flops": 6 * M * F * K}
    # x, dy, y, dx in bf16; the weights and, for the gradients, their transposed codes; bf16 weight gradients
    return {"bytes": 8 * M * K + 6 * F * K + 6 * F * K, "flops": 18 * M * F * K}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _activations(gen, M, K, dev):
    """Near-normal activations with a few channels twenty times as large; in batches some padding tokens of zeros."""
    x = torch.randn((M, K), generator=gen, device=dev)
    ch = torch.randperm(K, generator=gen, device=dev)[: max(1, K // 100)]
    x[:, ch] *= 20.0
    if M >= 16:
        x[torch.randperm(M, generator=gen, device=dev)[: max(1, M // 64)]] = 0.0
    return x.to(torch.bfloat16)


def _blocks_of(w):
    """Weights [.., N, K] -> absolute maxima of their 128 x 128 blocks, [.., ceil(N / 128), ceil(K / 128)]."""
    n, k = w.shape[-2:]
    p = torch.nn.functional.pad(w, (0, -k % BLOCK, 0, -n % BLOCK))
    p = p.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, BLOCK))
    return p.abs().amax(dim=(-3, -1))


def _weight(gen, shape, dev, mode):
    """Quantized weights a program has loaded: E4M3 codes and the scales of their 128 x 128 blocks."""
    w = torch.randn(shape, generator=gen, device=dev) * 0.02
    s = _scale_of(_blocks_of(w), mode)
    q = w / _spread_w(s, shape)
    return q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), s


def _spread_w(s, shape):
    return s.repeat_interleave(BLOCK, -1)[..., : shape[-1]].repeat_interleave(BLOCK, -2)[..., : shape[-2], :]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    op, M, K, mode = case["op"], case["M"], case["K"], case["mode"]
    st = {"case": case, "x": _activations(gen, M, K, dev)}
    if op == "linear":
        st["w"], st["ws"] = _weight(gen, (case["N"], K), dev, mode)
    elif op == "checkpoint":
        st["dy"] = (torch.randn((M, case["N"]), generator=gen, device=dev) * 0.01).to(torch.bfloat16)
    else:
        F = case["F"]
        st["wgu"], st["wgus"] = _weight(gen, (2, F, K), dev, mode)
        st["wd"], st["wds"] = _weight(gen, (K, F), dev, mode)
        if op == "train":
            st["dy"] = (torch.randn((M, K), generator=gen, device=dev) * 0.01).to(torch.bfloat16)
    if own:
        from paper_2307_09782_b200 import binding, gated_ffn

        if op == "linear":
            st["handle"] = binding.Fp8Weight(st["w"].view(torch.uint8), st["ws"], case["N"], K)
            st["workspace"] = binding.make_workspace(binding.fp8_block_linear_workspace_bytes(M, case["N"], K))
        elif op != "checkpoint":
            st["handle"] = gated_ffn.GatedFfnFp8(
                binding.Fp8Weight(st["wgu"].view(torch.uint8), st["wgus"], case["F"], K, parts=2),
                binding.Fp8Weight(st["wd"].view(torch.uint8), st["wds"], K, case["F"]),
                act=case["act"], mode=mode, training=op == "train")
    return st


# ---- the plain form -----------------------------------------------------------------------------------------------
def _scale_of(a, mode):
    r = torch.clamp(a / torch.full_like(a, 448.0), min=2.0 ** -126)  # by a tensor: a true division, no reciprocal
    if mode == "M1":  # up to a power of two: carry into the exponent, drop the mantissa
        r = ((r.view(torch.int32) + 0x7FFFFF) & 0x7F800000).view(torch.float32)
    return torch.where(a == 0, torch.ones_like(r), r)


def _quantize(x, mode):
    """[.., M, K] -> E4M3 codes [.., M, K] and the scales of their 1 x 128 blocks [.., ceil(K / 128), M]."""
    x = x.float()
    k = x.shape[-1]
    p = torch.nn.functional.pad(x, (0, -k % BLOCK)).unflatten(-1, (-1, BLOCK))
    s = _scale_of(p.abs().amax(-1), mode)
    q = (p * (1.0 / s)[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return q.flatten(-2)[..., :k], s.transpose(-1, -2).contiguous()


def _values(q, s):
    """The values that codes and 1 x 128 scales stand for."""
    return q.float() * s.transpose(-1, -2).repeat_interleave(BLOCK, -1)[..., : q.shape[-1]]


def _weights(q, s):
    return q.float() * _spread_w(s, q.shape)


def _act(g, kind):
    """The activation and its derivative."""
    if kind == "silu":
        sg = 1.0 / (1.0 + torch.exp(-g))
        return g * sg, sg * (1.0 + g * (1.0 - sg))
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)
    return torch.clamp(g, min=0.0), (g > 0).to(g.dtype)


def _plain(st):
    case = st["case"]
    op, mode = case["op"], case["mode"]
    out = torch.float32 if case.get("out") == "f32" else torch.bfloat16
    q, s = _quantize(st["x"], mode)
    xv = _values(q, s)
    if op == "linear":
        return (xv @ _weights(st["w"], st["ws"]).T).to(out)
    if op == "checkpoint":
        return {"codes": q, "scales": s, "dw": (st["dy"].float().T @ xv).to(out)}
    w = _weights(st["wgu"], st["wgus"])
    wd = _weights(st["wd"], st["wds"])
    g, u = xv @ w[0].T, xv @ w[1].T
    h = _values(*_quantize(_act(g, case["act"])[0] * u, mode))
    y = (h @ wd.T).to(out)
    if op == "ffn":
        return y
    g, u = _values(*_quantize(g, mode)), _values(*_quantize(u, mode))  # as the checkpoints keep them
    dh = _values(*_quantize(st["dy"], mode)) @ wd
    a, da = _act(g, case["act"])
    db = torch.stack([dh * u * da, dh * a]).to(torch.bfloat16).float()  # the gradients of g and u are bf16 tensors
    dv = _values(*_quantize(db, mode))
    return {"y": y, "dx": (dv[0] @ w[0] + dv[1] @ w[1]).to(out), "dwgu": (db.transpose(1, 2) @ xv).to(out),
            "dwd": (st["dy"].float().T @ h).to(out)}


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(st):
    if not own:
        return _plain(st)
    from paper_2307_09782_b200 import binding

    case = st["case"]
    op = case["op"]
    out = torch.float32 if case.get("out") == "f32" else torch.bfloat16
    if op == "linear":
        return binding.fp8_block_linear(st["handle"], x=st["x"], mode=case["mode"], out_dtype=out, workspace=st["workspace"])
    if op == "checkpoint":
        q = binding.quantize_fp8_block(st["x"], mode=case["mode"])
        dw = binding.fp8_weight_grad(st["dy"], q, out_dtype=out)
        return {"codes": q.codes.view(torch.float8_e4m3fn), "scales": q.scale, "dw": dw}
    if op == "ffn":
        return st["handle"].forward(st["x"])
    y, saved = st["handle"].forward_train(st["x"])
    dx, dwgu, dwd = st["handle"].backward(st["dy"], saved)
    return {"y": y, "dx": dx, "dwgu": dwgu, "dwd": dwd}


# ---- 64 bits --------------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    D = torch.float64
    mode = case["mode"]

    def two_to(k):
        return ((k.to(torch.int64) + 1023) << 52).view(D)  # exactly; pow and exp2 need not be

    def pow2_up(r):
        m, e = torch.frexp(r)
        return two_to(torch.where(m > 0.5, e, e - 1))

    def fp8(x):
        """Values of the quantized form: scale and scaled element are FP32 by definition, the rounding is to the grid."""
        m, k = x.shape
        kb = -(-k // BLOCK)
        z = torch.zeros((m, kb * BLOCK), dtype=torch.float32, device=x.device)
        z[:, :k] = x.to(torch.float32)
        z = z.view(m, kb, BLOCK)
        a = z.abs().max(dim=2).values
        s = torch.true_divide(a, torch.tensor([448.0], device=a.device)).clamp_min(2.0 ** -126)
        if mode == "M1":
            s = pow2_up(s.to(D)).to(torch.float32)
        s[a == 0] = 1.0
        v = (z * s.reciprocal()[:, :, None]).to(D)
        step = two_to(torch.frexp(v.abs().clamp_min(2.0 ** -6))[1] - 4)
        c = (torch.round(v / step) * step).clamp(-448, 448)
        return c.view(m, -1)[:, :k], s, (c * s.to(D)[:, :, None]).view(m, -1)[:, :k]

    def weight(q, s):
        n, k = q.shape
        rows = torch.arange(n, device=q.device) // BLOCK
        cols = torch.arange(k, device=q.device) // BLOCK
        return q.to(D) * s.to(D)[rows][:, cols]

    codes, s, xv = fp8(st["x"])
    if case["op"] == "linear":
        return xv @ weight(st["w"], st["ws"]).T
    if case["op"] == "checkpoint":
        return {"codes": codes, "scales": s.to(D).T.contiguous(), "dw": st["dy"].to(D).T @ xv}
    wg, wu = weight(st["wgu"][0], st["wgus"][0]), weight(st["wgu"][1], st["wgus"][1])
    wd = weight(st["wd"], st["wds"])

    def value_and_slope(g):
        if case["act"] == "silu":
            p = torch.sigmoid(g)
            return g * p, p + g * p * (1 - p)
        if case["act"] == "relu":
            return torch.relu(g), torch.heaviside(g, torch.zeros((), dtype=D, device=g.device))
        r = math.sqrt(2 / math.pi)
        t = torch.tanh(r * (g + 0.044715 * g ** 3))
        return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t ** 2) * r * (1 + 0.134145 * g ** 2) / 2

    g, u = xv @ wg.T, xv @ wu.T
    h = fp8(value_and_slope(g)[0] * u)[2]
    y = h @ wd.T
    if case["op"] == "ffn":
        return y
    g, u = fp8(g)[2], fp8(u)[2]
    dh = fp8(st["dy"])[2] @ wd
    a, slope = value_and_slope(g)
    dg, du = [d.to(torch.float32).to(torch.bfloat16) for d in (dh * u * slope, dh * a)]  # bf16 tensors by definition
    dx = fp8(dg)[2] @ wg + fp8(du)[2] @ wu
    dwgu = torch.stack([dg.to(D).T @ xv, du.to(D).T @ xv])
    return {"y": y, "dx": dx, "dwgu": dwgu, "dwd": st["dy"].to(D).T @ h}
