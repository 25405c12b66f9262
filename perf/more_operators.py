"""Cases that measure the attention half of a decoder layer around an 8-bit cache: norms of queries and keys with the position
rotation (both directions), the paged E4M3 cache (written, read back) and attention over it.

Where ``own`` is false, ``run`` computes them in elementary torch operations in 32 bits; where it is true, through the
package's public calls.  Both take what ``prepare`` gives.
"""
import math

import torch

own = False


# ---- cases ------------------------------------------------------------------------------------------------------
# Attention and cache cases: B sequences, the longest of `ctx` tokens with the new ones, the most new ones `new` (see _lengths).
def listed():
    return [
        # one user's chat of 699 tokens, the smallest configuration (125 million parameters), one token
        {"name": "attn-1-token", "op": "attn", "B": 1, "new": 1, "ctx": 699, "Hq": 12, "H": 12, "D": 64, "page": 16,
         "mode": "none", "causal": True, "window": 0, "out": "bf16"},
        # a decoding batch of 64 users with contexts up to 8192 tokens, grouped heads
        {"name": "attn-64-tokens", "op": "attn", "B": 64, "new": 1, "ctx": 8192, "Hq": 32, "H": 8, "D": 128, "page": 64,
         "mode": "none", "causal": True, "window": 0, "out": "bf16"},
        # one token of one user over a very long document, an odd group of seven query heads
        {"name": "attn-1-long", "op": "attn", "B": 1, "new": 1, "ctx": 131071, "Hq": 56, "H": 8, "D": 128, "page": 64,
         "mode": "M1", "causal": True, "window": 0, "out": "bf16"},
        # chunks of prompts behind contexts of other lengths, a window, every head its own keys, FP32 results
        {"name": "attn-chunks", "op": "attn", "B": 3, "new": 777, "ctx": 6001, "Hq": 32, "H": 32, "D": 128, "page": 32,
         "mode": "none", "causal": True, "window": 4096, "out": "f32"},
        # a whole prompt of 8191 tokens
        {"name": "attn-prompt", "op": "attn", "B": 1, "new": 8191, "ctx": 8191, "Hq": 32, "H": 8, "D": 128, "page": 128,
         "mode": "M1", "causal": True, "window": 0, "out": "bf16"},
        # queries and keys of 33 decoded tokens
        {"name": "norm-33", "op": "norm", "T": 33, "Hq": 32, "H": 8, "D": 128, "rot": 128, "pairs": "halves", "far": 131072},
        # of a prompt batch
        {"name": "norm-16384", "op": "norm", "T": 16384, "Hq": 32, "H": 8, "D": 128, "rot": 128, "pairs": "halves",
         "far": 16384},
        # their gradients in a training step, half of each head rotated, neighbouring pairs
        {"name": "norm-grad-8192", "op": "norm_grad", "T": 8192, "Hq": 32, "H": 32, "D": 64, "rot": 32,
         "pairs": "neighbours", "far": 8192},
        # one new token of each of 64 users goes into pages that are mostly begun
        {"name": "write-64-tokens", "op": "write", "B": 64, "new": 1, "ctx": 8192, "H": 8, "D": 128, "page": 64,
         "mode": "none"},
        # prompts of five users
        {"name": "write-prompts", "op": "write", "B": 5, "new": 4099, "ctx": 5001, "H": 8, "D": 128, "page": 64,
         "mode": "M1"},
        # a prefix of 1000 tokens is read back
        {"name": "read-prefix", "op": "read", "B": 1, "ctx": 1000, "H": 8, "D": 128, "page": 16, "mode": "none",
         "out": "bf16"},
        # a batch of caches is read back in FP32
        {"name": "read-batch", "op": "read", "B": 16, "ctx": 4095, "H": 8, "D": 128, "page": 64, "mode": "none",
         "out": "f32"},
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MOST_FLOPS = 5.4e11  # of a drawn case: not above the largest listed one's
MOST_BYTES = 7.0e8


def draw(rng):
    while True:
        op = rng.choice(["attn", "attn", "attn", "norm", "norm_grad", "write", "read"])
        D, H = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 12, 32])
        paged = {"page": rng.choice([16, 32, 64, 128]), "mode": rng.choice(["none", "M1"])}
        if op == "attn":
            ctx = _log(rng, 1, 100000)
            c = {"op": op, "B": _log(rng, 1, 256), "new": 1 if rng.random() < 0.5 else _log(rng, 1, min(ctx, 8192)), "ctx": ctx,
                 "Hq": H * rng.choice([1, 1, 2, 4, 5, 8, 16]), "H": H, "D": D, **paged, "causal": rng.random() < 0.8,
                 "window": rng.choice([0, 0, 0, _log(rng, 1, 8192)]), "out": rng.choice(["bf16", "bf16", "f32"])}
            if not c["causal"]:
                c["window"] = 0
        elif op in ("norm", "norm_grad"):
            c = {"op": op, "T": _log(rng, 1, 16384), "Hq": H * rng.choice([1, 2, 4, 5]), "H": H, "D": D,
                 "rot": rng.choice([D, D, D // 2, 16]), "pairs": rng.choice(["halves", "neighbours"]),
                 "far": rng.choice([4096, 32768, 131072])}
        elif op == "write":
            ctx = _log(rng, 1, 32768)
            c = {"op": op, "B": _log(rng, 1, 256), "new": rng.choice([1, _log(rng, 1, ctx)]), "ctx": ctx, "H": H, "D": D, **paged}
        else:
            c = {"op": op, "B": _log(rng, 1, 64), "ctx": _log(rng, 1, 32768), "H": H, "D": D, **paged,
                 "out": rng.choice(["bf16", "f32"])}
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and _footprint(c) <= 2.0e9:
            return c


def _lengths(case):
    """(tokens of each sequence with the new ones, new ones of each): the first has the most of both, the others are spread
    between a quarter and the whole; with many new tokens some sequences have one only."""
    lens, new = [], []
    for b in range(case["B"]):
        f = 1.0 - 0.75 * ((b * 0.6180339887498949) % 1.0)
        L = max(1, int(round(case["ctx"] * f)))
        n = max(1, int(round(case.get("new", 1) * (1.0 - 0.75 * ((b * 0.7548776662466927) % 1.0)))))
        if b % 4 == 3:
            n = 1
        lens.append(L)
        new.append(min(n, L))
    return lens, new


def _footprint(case):
    """Bytes of the cache."""
    return 0 if "page" not in case else sum(L + case["page"] for L in _lengths(case)[0]) * 2 * case["H"] * case["D"]


def _visible(case):
    """(visible pairs of query and key, keys that some query sees), summed over the sequences."""
    pairs = keys = 0
    for L, n in zip(*_lengths(case)):
        if not case["causal"]:
            pairs += n * L
            keys += L
            continue
        w = case["window"] or L
        # row i sees min(L - n + i + 1, w) keys
        first, last = L - n + 1, L
        below = max(0, min(last, w) - first + 1)
        pairs += below * (first + first + below - 1) // 2 + (n - below) * w
        keys += L - max(0, first - w)
    return pairs, keys


def work(case):
    op, D, H = case["op"], case["D"], case["H"]
    if op == "attn":
        pairs, keys = _visible(case)
        rows = sum(_lengths(case)[1]) * case["Hq"]
        return {"bytes": keys * 2 * H * D + rows * D * (2 + (4 if case["out"] == "f32" else 2)),
                "flops": 4 * D * case["Hq"] * pairs}
    if op == "norm":
        e = case["T"] * (case["Hq"] + H) * D
        return {"bytes": 4 * e + 4 * case["T"] * case["rot"], "flops": 8 * e}
    if op == "norm_grad":
        e = case["T"] * (case["Hq"] + H) * D
        return {"bytes": 6 * e + 4 * case["T"] * case["rot"], "flops": 16 * e}
    lens, new = _lengths(case)
    if op == "write":
        e = sum(new) * 2 * H * D
        return {"bytes": 3 * e, "flops": 4 * e}
    e = sum(lens) * 2 * H * D
    return {"bytes": e * (1 + (4 if case["out"] == "f32" else 2)), "flops": e}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _heads(gen, T, H, D, dev):
    """Near-normal rows with a few features of each head five times as large; some rows of zeros (padding)."""
    x = torch.randn((T, H, D), generator=gen, device=dev)
    f = torch.randperm(D, generator=gen, device=dev)[: D // 32]
    x[:, :, f] *= 5.0
    if T >= 64:
        x[torch.randperm(T, generator=gen, device=dev)[: T // 64]] = 0.0
    return x.to(torch.bfloat16)


def _cache(case, gen, dev):
    """A pool of pages in use: codes, scales, the sequences' page tables (pages in no order), some pages nobody owns."""
    page, H, D = case["page"], case["H"], case["D"]
    lens, new = _lengths(case)
    per = [-(-L // page) for L in lens]
    total = sum(per) + max(1, sum(per) // 16)
    codes = torch.empty((total, 2, H, page, D), dtype=torch.uint8, device=dev)
    scale = torch.empty((total, 2, H), device=dev)
    step = max(1, (1 << 26) // (2 * H * page * D))
    for i in range(0, total, step):
        x = torch.randn((min(step, total - i), 2, H, page, D), generator=gen, device=dev)
        x[:, 0, :, :, :4] *= 4.0  # some features of the keys are larger
        x *= 0.5 + torch.rand((x.shape[0], 2, H, 1, 1), generator=gen, device=dev)
        s = _scale_of(x.abs().amax((3, 4)), case["mode"])
        codes[i:i + step] = (x * (1.0 / s)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scale[i:i + step] = s
    order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
    table = torch.full((len(lens), max(per)), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    cu = torch.zeros(len(lens) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(new), 0)
    return {"codes": codes, "scale": scale, "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device=dev),
            "cu": cu.to(dev)}


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    op, D = case["op"], case["D"]
    st = {"case": case}
    if op in ("norm", "norm_grad"):
        T, Hq, H = case["T"], case["Hq"], case["H"]
        qkv = torch.cat([_heads(gen, T, h, D, dev) for h in (Hq, H, H)], 1)  # as the projection leaves them
        st["q"], st["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + H]
        st["wq"], st["wk"] = (1.0 + 0.2 * torch.randn((2, D), generator=gen, device=dev)).unbind(0)
        angle = torch.arange(case["far"], dtype=torch.float64, device=dev)[:, None] \
            * 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=dev) / case["rot"])
        st["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        st["positions"] = torch.randint(0, case["far"], (T,), generator=gen, device=dev, dtype=torch.int32)
        if op == "norm_grad":
            st["dq"], st["dk"] = [(torch.randn((T, h, D), generator=gen, device=dev) * 0.01).to(torch.bfloat16) for h in (Hq, H)]
        return st
    st.update(_cache(case, gen, dev))
    rows = sum(_lengths(case)[1])
    if op == "attn":
        st["q"] = _heads(gen, rows, case["Hq"], D, dev)
    elif op == "write":
        st["k"], st["v"] = _heads(gen, rows, case["H"], D, dev), _heads(gen, rows, case["H"], D, dev)
    else:
        cu = torch.zeros(case["B"] + 1, dtype=torch.int32)
        cu[1:] = torch.cumsum(torch.tensor(_lengths(case)[0]), 0)
        st["cu"], st["rows"] = cu.to(dev), int(cu[-1])
    if own:
        from paper_2307_09782_b200 import binding

        st["cache"] = binding.Fp8KvCache(st["codes"], st["scale"])
        if op == "attn":
            st["workspace"] = binding.make_workspace(binding.kv_attention_workspace_bytes(rows, case["B"], case["Hq"], case["H"], D))
    return st


# ---- the plain form -----------------------------------------------------------------------------------------------
def _scale_of(a, mode):
    s = torch.clamp(a / torch.full_like(a, 448.0), min=2.0 ** -64)  # by a tensor: a true division, no reciprocal
    if mode == "M1":  # up to a power of two: carry into the exponent, drop the mantissa
        s = ((s.view(torch.int32) + 0x7FFFFF) & 0x7F800000).view(torch.float32)
    return torch.where(torch.isfinite(a), s, torch.full_like(s, float("nan")))


def _codes_of(x, s):
    """x [.., H, page, D], s [.., H] -> E4M3 codes (zeros where the scale is not a number)."""
    c = (x * (1.0 / s)[..., None, None]).clamp(-448.0, 448.0)
    return torch.where(torch.isnan(s)[..., None, None], torch.zeros_like(c), c).to(torch.float8_e4m3fn)


def _rotate(z, cos, sin, rot, pairs, back=False):
    """z [T, H, D]; cos, sin [T, rot / 2]."""
    cos, sin = cos[:, None], -sin[:, None] if back else sin[:, None]
    y = z.clone()
    a, b = (z[..., : rot // 2], z[..., rot // 2: rot]) if pairs == "halves" else (z[..., 0:rot:2], z[..., 1:rot:2])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    if pairs == "halves":
        y[..., : rot // 2], y[..., rot // 2: rot] = ya, yb
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = ya, yb
    return y


EPS = 1e-6


def _norm(st):
    case = st["case"]
    t = st["table"][st["positions"].long()]
    cos, sin = t[:, : case["rot"] // 2], t[:, case["rot"] // 2:]
    out = {}
    for name in ("q", "k"):
        x, w = st[name].float(), st["w" + name]
        r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * r
        if case["op"] == "norm":
            out[name] = _rotate(n * w, cos, sin, case["rot"], case["pairs"]).to(torch.bfloat16)
            continue
        g = _rotate(st["d" + name].float(), cos, sin, case["rot"], case["pairs"], back=True)
        u = g * w
        out["d" + name] = (r * (u - n * (u * n).mean(-1, keepdim=True))).to(torch.bfloat16)
        out["dw" + name] = (g.double() * n.double()).sum((0, 1)).float()  # a long sum
    return out


def _write(st):
    case = st["case"]
    page, H, D = case["page"], case["H"], case["D"]
    lens, new = _lengths(case)
    at = 0
    for b, (L, n) in enumerate(zip(lens, new)):
        first, off = (L - n) // page, (L - n) % page
        pages = st["table"][b, first: -(-L // page)].long()
        x = torch.zeros((2, pages.numel() * page, H, D), device=st["codes"].device)
        x[0, off:off + n], x[1, off:off + n] = st["k"][at:at + n].float(), st["v"][at:at + n].float()
        x = x.unflatten(1, (-1, page)).permute(1, 0, 3, 2, 4)  # [pages, 2, H, page, D]
        s = _scale_of(x.abs().amax((3, 4)), case["mode"])
        codes = st["codes"][pages]
        if off:
            old = st["scale"][pages[0]]
            s[0] = torch.maximum(old, s[0])
            kept = codes[0, :, :, :off].view(torch.float8_e4m3fn)
            again = _codes_of(kept.float() * old[..., None, None], s[0])
            grown = torch.isnan(s[0]) | (s[0] > old)
            codes[0, :, :, :off] = torch.where(grown[..., None, None], again.view(torch.uint8), kept.view(torch.uint8))
        fresh = _codes_of(x, s).view(torch.uint8)
        pos = torch.arange(pages.numel() * page, device=codes.device).view(-1, 1, 1, page, 1)
        st["codes"][pages] = torch.where((pos >= off) & (pos < off + n), fresh, codes)
        st["scale"][pages] = s
        at += n
    return {"codes": st["codes"].view(torch.float8_e4m3fn), "scale": st["scale"]}


def _gather(st, b, L):
    """Keys and values of a sequence's first L tokens, [2, H, L, D] in 32 bits."""
    page = st["case"]["page"]
    pages = st["table"][b, : -(-L // page)].long()
    x = st["codes"][pages].view(torch.float8_e4m3fn).float() * st["scale"][pages][..., None, None]
    return x.permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :L]


def _read(st):
    out = torch.float32 if st["case"]["out"] == "f32" else torch.bfloat16
    parts = [_gather(st, b, L).transpose(1, 2).to(out) for b, L in enumerate(_lengths(st["case"])[0])]
    return {"k": torch.cat([p[0] for p in parts]), "v": torch.cat([p[1] for p in parts])}


def _attn(st):
    case = st["case"]
    H, D, G = case["H"], case["D"], case["Hq"] // case["H"]
    out = torch.empty(st["q"].shape, dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device=st["q"].device)
    at = 0
    for b, (L, n) in enumerate(zip(*_lengths(case))):
        k, v = _gather(st, b, L)
        q = st["q"][at:at + n].float().view(n, H, G, D).permute(1, 2, 0, 3)  # [H, G, n, D]
        row = torch.arange(L - n, L, device=q.device)[:, None]
        col = torch.arange(L, device=q.device)[None]
        hidden = torch.zeros((n, L), dtype=torch.bool, device=q.device)
        if case["causal"]:
            hidden |= col > row
        if case["window"]:
            hidden |= col <= row - case["window"]
        per = max(1, (1 << 28) // (G * n * L))  # heads of the cache at a time
        for h in range(0, H, per):
            s = (q[h:h + per].flatten(1, 2) @ k[h:h + per].transpose(1, 2)).unflatten(1, (G, n)) * (1.0 / math.sqrt(D))
            s.masked_fill_(hidden, float("-inf"))
            s = torch.exp(s.sub_(s.amax(-1, keepdim=True)))
            o = (s.flatten(1, 2) @ v[h:h + per]).unflatten(1, (G, n)) / s.sum(-1, keepdim=True)
            out[at:at + n].view(n, H, G, D)[:, h:h + per] = o.permute(2, 0, 1, 3).to(out.dtype)
        at += n
    return out


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"norm": _norm, "norm_grad": _norm, "write": _write, "read": _read, "attn": _attn}[op](st)
    from paper_2307_09782_b200 import binding

    out = torch.float32 if case.get("out") == "f32" else torch.bfloat16
    if op == "norm":
        q, k = binding.qk_norm_rope(st["q"], st["k"], st["table"], st["positions"], wq=st["wq"], wk=st["wk"], eps=EPS,
                                    pairs=case["pairs"])
        return {"q": q, "k": k}
    if op == "norm_grad":
        dq, dk, dwq, dwk = binding.qk_norm_rope_backward(st["dq"], st["dk"], st["q"], st["k"], st["table"], st["positions"],
                                                         wq=st["wq"], wk=st["wk"], eps=EPS, pairs=case["pairs"])
        return {"dq": dq, "dwq": dwq, "dk": dk, "dwk": dwk}
    if op == "write":
        binding.kv_cache_write(st["cache"], st["k"], st["v"], st["table"], st["lens"], cu=None if case["new"] == 1 else st["cu"],
                               mode=case["mode"])
        return {"codes": st["codes"].view(torch.float8_e4m3fn), "scale": st["scale"]}
    if op == "read":
        k, v = binding.kv_cache_read(st["cache"], st["table"], st["cu"], st["rows"], out_dtype=out)
        return {"k": k, "v": v}
    return binding.kv_attention(st["cache"], st["q"], st["table"], st["lens"], cu=None if case["new"] == 1 else st["cu"],
                                causal=case["causal"], window=case["window"], out_dtype=out, workspace=st["workspace"])


# ---- 64 bits --------------------------------------------------------------------------------------------------------
def _two_to(k):
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)  # exactly; pow and exp2 need not be


def _to_e4m3(v):
    """The nearest E4M3 value (ties to the even mantissa) of a float64, at most 448 in size."""
    step = _two_to(torch.frexp(v.abs().clamp_min(2.0 ** -6))[1] - 4)
    return (torch.round(v / step) * step).clamp(-448, 448)


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    op, D, H = case["op"], case["D"], case["H"]
    lens, new = _lengths(case) if "page" in case else ([], [])
    if op in ("norm", "norm_grad"):
        R = case["rot"]
        half = torch.arange(R // 2, device=st["q"].device)
        first, second = (half, half + R // 2) if case["pairs"] == "halves" else (2 * half, 2 * half + 1)
        phase = torch.complex(*[st["table"].to(f64)[st["positions"].long()][:, None, c] for c in (slice(0, R // 2), slice(R // 2, R))])
        res = {}
        for x, w, name in ((st["q"], st["wq"], "q"), (st["k"], st["wk"], "k")):
            x, w = x.to(f64), w.to(f64)
            rms = torch.linalg.vector_norm(x, dim=2, keepdim=True).square().div(D).add(EPS).sqrt()
            if op == "norm":
                y = x / rms * w
                z = torch.complex(y[:, :, first], y[:, :, second]) * phase
                y[:, :, first], y[:, :, second] = z.real, z.imag
                res[name] = y
            else:
                g = st["d" + name].to(f64)
                z = torch.complex(g[:, :, first], g[:, :, second]) * phase.conj()
                g[:, :, first], g[:, :, second] = z.real, z.imag
                res["dw" + name] = torch.einsum("thd,thd->d", g, x / rms)
                inner = torch.einsum("thd,thd,d->th", g, x, w)[:, :, None]
                res["d" + name] = g * w / rms - x * inner / (D * rms ** 3)
        return {k: res[k] for k in (("q", "k") if op == "norm" else ("dq", "dwq", "dk", "dwk"))}

    page = case["page"]
    table = st["table"].tolist()
    if op == "write":
        if sum(new) > 100 * page + 20000:
            return None  # block by block it would take too long
        values, scale = st["codes"].view(torch.float8_e4m3fn).to(f64), st["scale"].clone()
        both = torch.stack([st["k"], st["v"]]).to(torch.float32)  # [2, rows, H, D]
        start = 0
        for b in range(case["B"]):
            pos, end = lens[b] - new[b], lens[b]
            while pos < end:
                stop = min(end, (pos // page + 1) * page)
                p, r0, r1 = table[b][pos // page], pos % page, (stop - 1) % page + 1
                x = both[:, start:start + stop - pos].transpose(1, 2)  # [2, H, rows, D]
                s = torch.true_divide(x.abs().flatten(2).max(2).values, torch.tensor([448.0], device=x.device)).clamp_min(2.0 ** -64)
                if case["mode"] == "M1":
                    m, e = torch.frexp(s.to(f64))
                    s = _two_to(torch.where(m > 0.5, e, e - 1)).to(torch.float32)
                if r0 > 0:
                    old = scale[p].clone()
                    s = torch.max(old, s)
                    again = ((values[p, :, :, :r0].to(torch.float32) * old[:, :, None, None]) * s.reciprocal()[:, :, None, None]).to(f64)
                    values[p, :, :, :r0] = torch.where((s > old)[:, :, None, None], _to_e4m3(again), values[p, :, :, :r0])
                values[p, :, :, r0:r1] = _to_e4m3((x * s.reciprocal()[:, :, None, None]).to(f64))
                scale[p] = s
                start += stop - pos
                pos = stop
        return {"codes": values, "scale": scale.to(f64)}

    def cached(b):
        c = torch.tensor(table[b][: (lens[b] + page - 1) // page], device=st["codes"].device)
        x = torch.einsum("pchtd,pch->chptd", st["codes"][c].view(torch.float8_e4m3fn).to(f64), st["scale"][c].to(f64))
        return x.reshape(2, H, -1, D)[:, :, : lens[b]]

    if op == "read":
        both = [cached(b).permute(0, 2, 1, 3) for b in range(case["B"])]
        return {"k": torch.cat([x[0] for x in both]), "v": torch.cat([x[1] for x in both])}
    if work(case)["flops"] > 1e13:
        return None
    G = case["Hq"] // H
    out = []
    start = 0
    for b in range(case["B"]):
        kv = cached(b)
        L, n = lens[b], new[b]
        o = torch.empty((n, case["Hq"], D), dtype=f64, device=kv.device)
        rows = max(1, (1 << 26) // L)
        for hq in range(case["Hq"]):
            for i in range(0, n, rows):
                at = torch.arange(i, min(n, i + rows), device=kv.device) + (L - n)
                logits = st["q"][start + i:start + min(n, i + rows), hq].to(f64)
                logits = logits @ kv[0, hq // G].T / math.sqrt(D)
                key = torch.arange(L, device=kv.device)
                if case["causal"]:
                    seen = key <= at[:, None]
                    if case["window"]:
                        seen &= key > at[:, None] - case["window"]
                    logits = torch.where(seen, logits, -math.inf)
                o[i:i + rows, hq] = torch.softmax(logits, 1) @ kv[1, hq // G]
        out.append(o)
        start += n
    return torch.cat(out)
