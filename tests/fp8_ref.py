"""Plain 64-bit forms of the FP8 operators with block scales (include/zqfp.h), for the tests: written from the
definitions with numpy, sharing nothing with the package."""
import numpy as np

B = 128
F32 = np.float32


def e4m3_table():
    """Values of the 256 E4M3 codes."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        a = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = np.nan if (c & 127) == 127 else (-a if c & 128 else a)
    return v


DEC = e4m3_table()


def e4m3_round(v):
    """Codes of float32 values: nearest, ties to even, saturating; NaN -> NaN."""
    v = np.asarray(v, F32)
    a = np.minimum(np.abs(v.astype(np.float64)), 448.0)
    e = np.maximum(np.frexp(np.where(a > 0, a, 1.0))[1] - 1, -6)
    m = np.rint(a / np.exp2(e - 3.0))              # 0 .. 16, in units of the step; numpy's rint ties to even
    code = np.where(m < 8, m, np.where(m < 16, (e + 7) * 8 + (m - 8), (e + 8) * 8))
    code = np.where(np.isnan(v), 127, code).astype(np.int64)
    return (code | (np.signbit(v).astype(np.int64) << 7)).astype(np.uint8)


def scale_of(a, mode):
    a = np.asarray(a, F32)
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.maximum(a / F32(448.0), F32(2.0 ** -126)).astype(F32)
        if mode == "M1":
            m, e = np.frexp(s.astype(np.float64))
            s = np.exp2(np.where(m == 0.5, e - 1.0, e + 0.0)).astype(F32)
    s = np.where(a == 0, F32(1), s)
    return np.where(np.isfinite(a), s, F32(np.nan)).astype(F32)


def _pad(x, axes):
    w = [(0, 0)] * x.ndim
    for ax in axes:
        w[ax] = (0, -x.shape[ax] % B)
    return np.pad(x, w)


def amax(x, axis):
    """np.max, which hands NaN on."""
    return np.max(np.abs(x), axis=axis)


def quantize_rows(x, mode):
    """float32 [M, K] -> codes [M, K], scales [ceil(K / 128), M]."""
    M, K = x.shape
    p = _pad(np.asarray(x, F32), [1]).reshape(M, -1, B)
    s = scale_of(amax(p, 2), mode)
    with np.errstate(invalid="ignore", over="ignore"):
        q = e4m3_round((p * (F32(1) / s)[..., None]).astype(F32))
    return q.reshape(M, -1)[:, :K], np.ascontiguousarray(s.T)


def quantize_blocks(w, mode):
    N, K = w.shape
    p = _pad(np.asarray(w, F32), [0, 1])
    p = p.reshape(p.shape[0] // B, B, p.shape[1] // B, B)
    s = scale_of(amax(p, (1, 3)), mode)
    with np.errstate(invalid="ignore", over="ignore"):
        q = e4m3_round((p * (F32(1) / s)[:, None, :, None]).astype(F32))
    return q.reshape(p.shape[0] * B, -1)[:N, :K], s


def rows_values(q, s):
    return DEC[q] * np.repeat(s.T.astype(np.float64), B, 1)[:, :q.shape[1]]


def blocks_values(q, s):
    return DEC[q] * np.repeat(np.repeat(s.astype(np.float64), B, 0)[:q.shape[0]], B, 1)[:, :q.shape[1]]


def act(v, kind):
    """Value and derivative."""
    with np.errstate(over="ignore"):
        if kind == "silu":
            p = 1 / (1 + np.exp(-v))
            return v * p, p * (1 + v * (1 - p))
        if kind == "gelu_tanh":
            c = np.sqrt(2 / np.pi)
            t = np.tanh(c * (v + 0.044715 * v ** 3))
            return 0.5 * v * (1 + t), 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * c * (1 + 3 * 0.044715 * v * v)
    return np.maximum(v, 0), (v > 0) * 1.0


def bf16(v):
    """Nearest bf16 value (ties to even) of float32 values."""
    u = np.ascontiguousarray(v, F32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(F32)
