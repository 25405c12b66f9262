"""Plain 64-bit forms of the operators around the 8-bit cache, and random batches for their tests."""
import math

import torch

F64 = torch.float64


def norm_rope(x, w, table, positions, eps, pairs):
    """Forward pass in 64 bits (differentiable)."""
    rot = table.shape[1]
    z = x
    if w is not None:
        z = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    t = table.to(F64)[positions.long()]
    c, s = t[:, None, :rot // 2], t[:, None, rot // 2:]
    if pairs == "halves":
        a, b = z[..., :rot // 2], z[..., rot // 2:rot]
        y = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = z[..., 0:rot:2], z[..., 1:rot:2]
        y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([y, z[..., rot:]], -1)


def scale_of(a, mode):
    """Scale for largest absolute values (float32), by definition in FP32 steps."""
    s = torch.clamp(a / torch.tensor(448.0, device=a.device).expand_as(a), min=2.0 ** -64)
    if mode == "M1":
        m, e = torch.frexp(s.to(F64))
        s = torch.ldexp(torch.ones_like(m), torch.where(m > 0.5, e, e - 1)).float()
    return torch.where(torch.isfinite(a), s, torch.full_like(s, math.nan))


def codes_of(x, s):
    v = x.float() * (1.0 / s)
    return torch.where(torch.isnan(s).expand_as(v), torch.zeros_like(v), v.clamp(-448, 448)).to(torch.float8_e4m3fn).view(torch.uint8)


def write(codes, scale, k, v, table, lens, cu, mode):
    """Token by token's page: what kv_cache_write leaves in (copies of) codes and scale."""
    codes, scale = codes.clone(), scale.clone()
    page = codes.shape[3]
    for b in range(len(lens)):
        r, n = cu[b], cu[b + 1] - cu[b]
        pos, end = lens[b] - n, lens[b]
        if n <= 0 or pos < 0:
            continue
        while pos < end:
            stop = min(end, (pos // page + 1) * page)
            i = pos // page
            p = int(table[b, i]) if i < table.shape[1] else -1
            m = stop - pos
            if 0 <= p < codes.shape[0]:
                lo = pos % page
                for w, x in enumerate((k, v)):
                    for h in range(codes.shape[2]):
                        new = x[r:r + m, h].float()
                        s = scale_of(new.abs().max() if torch.isfinite(new).all() else torch.tensor(math.inf, device=x.device), mode)
                        old = scale[p, w, h].clone()
                        if lo > 0:
                            if torch.isnan(old) or s <= old:
                                s = old
                            else:
                                kept = codes[p, w, h, :lo].view(torch.float8_e4m3fn).float() * old
                                codes[p, w, h, :lo] = codes_of(kept, s)
                        codes[p, w, h, lo:lo + m] = codes_of(new, s)
                        scale[p, w, h] = s
            r += m
            pos = stop
    return codes, scale


def gather(codes, scale, table_row, L):
    """[2, H, L, D] of a sequence; NaN where the table names no page."""
    page = codes.shape[3]
    x = torch.full((2, codes.shape[2], -(-L // page) * page, codes.shape[4]), math.nan, dtype=F64, device=codes.device)
    for i in range(-(-L // page)):
        p = int(table_row[i]) if i < len(table_row) else -1
        if 0 <= p < codes.shape[0]:
            x[:, :, i * page:(i + 1) * page] = codes[p].view(torch.float8_e4m3fn).to(F64) * scale[p].to(F64)[..., None, None]
    return x[:, :, :L]


def attention(codes, scale, q, table, lens, cu, sm_scale, causal, window):
    """(o, lse, bound): `bound` is what errors multiply: sum of p |v|; the largest |q| . |k| of the row; the largest product of a
    probability and its value's scale times the sum of |codes|."""
    T, Hq, D = q.shape
    H = codes.shape[2]
    G = Hq // H
    o = torch.zeros((T, Hq, D), dtype=F64, device=q.device)
    pv = torch.zeros_like(o)
    lse = torch.full((T, Hq), -math.inf, dtype=F64, device=q.device)
    qk = torch.zeros((T, Hq), dtype=F64, device=q.device)
    low = torch.zeros_like(o)
    tab = table.tolist()
    for b in range(len(lens)):
        L, r0, n = lens[b], cu[b], cu[b + 1] - cu[b]
        if L <= 0 or n <= 0:
            continue
        kv = gather(codes, scale, tab[b], L)
        ones = torch.full_like(codes[:, :, :, :, :1], 0x38)  # E4M3's 1: the blocks' scales, token by token
        per_token = gather(ones, scale, tab[b], L)[1, :, :, 0].nan_to_num(nan=1.0)
        pos = torch.arange(L - n, L, device=q.device)[:, None]
        col = torch.arange(L, device=q.device)[None]
        seen = torch.ones((n, L), dtype=torch.bool, device=q.device)
        if causal:
            seen &= col <= pos
            if window:
                seen &= col > pos - window
        for hq in range(Hq):
            k, v = kv[0, hq // G], kv[1, hq // G]
            x = q[r0:r0 + n, hq].to(F64)
            s = (x @ k.T) * sm_scale
            s = torch.where(seen, s, -math.inf)
            any_ = seen.any(1)
            m = torch.where(any_, s.max(1).values, 0.0)
            e = torch.where(seen, torch.exp(s - m[:, None]), 0.0)
            z = e.sum(1, keepdim=True)
            # (0 x NaN: what is not seen has no influence)
            clean, bad = torch.nan_to_num(v, nan=0.0), torch.isnan(v).to(F64)
            poison = (seen.to(F64) @ bad) > 0
            o[r0:r0 + n, hq] = torch.where(any_[:, None], torch.where(poison, math.nan, e @ clean / z), 0.0)
            pv[r0:r0 + n, hq] = torch.where(any_[:, None], e @ clean.abs() / z, 0.0)
            sv = per_token[hq // G]
            top = (e / torch.where(z > 0, z, 1.0) * sv).max(1, keepdim=True).values
            low[r0:r0 + n, hq] = top * (seen.to(F64) @ (clean.abs() / torch.where(sv > 0, sv, 1.0)[:, None]))
            lse[r0:r0 + n, hq] = torch.where(any_, m + torch.log(z[:, 0]), -math.inf)
            kk = torch.nan_to_num(k, nan=0.0).abs()
            qk[r0:r0 + n, hq] = torch.where(seen, x.abs() @ kk.T, 0.0).max(1).values * sm_scale
    return o, lse, (pv, qk, low)


def batch(lens, new, H, D, page, seed=0, mode="none", spare=3, spread=1.0, dev="cuda"):
    """A cache in use for sequences of `lens` tokens: (codes, scale, table int32 [B, n], lens, cu lists).  Rows behind the sequences'
    ends and pages that nobody owns hold all bit patterns, NaN among them."""
    g = torch.Generator(device=dev).manual_seed(seed)
    per = [max(0, -(-L // page)) for L in lens]
    total = sum(per) + spare
    codes = torch.randint(0, 256, (total, 2, H, page, D), generator=g, device=dev, dtype=torch.uint8)
    scale = torch.rand((total, 2, H), generator=g, device=dev)
    scale[torch.randint(0, total, (1,), generator=g, device=dev)] = math.nan  # overwritten below where somebody owns it
    order = torch.randperm(total, generator=g, device=dev).tolist()
    table = torch.full((len(lens), max(per + [1])), -7, dtype=torch.int32)
    for b, n in enumerate(per):
        for i in range(n):
            p = order.pop()
            table[b, i] = p
            x = torch.randn((2, H, page, D), generator=g, device=dev) * torch.exp(spread * torch.randn((2, H, 1, 1), generator=g, device=dev))
            s = scale_of(x.abs().amax((2, 3)), mode)
            scale[p] = s
            rows = min(page, lens[b] - i * page)
            codes[p, :, :, :rows] = codes_of(x, s[..., None, None])[:, :, :rows]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return codes, scale, table.to(dev), list(lens), cu


def ints(x, dev="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def heads(T, H, D, seed=0, extra=0, dev="cuda"):
    """bf16 [T, H, D]; with `extra` a part of wider rows."""
    g = torch.Generator(device=dev).manual_seed(seed)
    x = torch.randn((T, H + extra, D), generator=g, device=dev)
    x[..., : max(1, D // 32)] *= 4
    return x.to(torch.bfloat16)[:, extra // 2: extra // 2 + H]
