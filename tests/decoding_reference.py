"""The decoding operators from their definitions, in 64 bits on the host (test infrastructure)."""
import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_BF16 = 2.0 ** -8          # a bf16 rounding, relative
HALF_E4M3 = 2.0 ** -4
ADD = 2.0 ** -23               # an fp32 addition of the matrix instructions (rounded or cut)


def bf16(a) -> np.ndarray:
    """float64 -> the nearest bf16 values (ties to even), as float64."""
    u = np.asarray(a, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)


def device(a, dtype="bfloat16"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(getattr(torch, dtype))


def host(t) -> np.ndarray:
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------- MXFP4

def mx_quantize(x):
    """Values [R, K] (bf16-valued) -> (codes 0..15 [R, K], scale bytes [R, K/32])."""
    R, K = x.shape
    b = x.reshape(R, K // 32, 32)
    top = np.abs(b).max(-1)
    finite = np.isfinite(b).all(-1)
    with np.errstate(invalid="ignore"):
        e = np.where((top > 0) & finite, np.frexp(np.where(finite, top, 1.0))[1] - 1, -1000)
    E = np.maximum(e - 2, -127)
    a = np.abs(b) / np.exp2(E.astype(np.float64))[..., None]
    far = np.abs(a[..., None] - E2M1)
    far[..., 1::2] *= 1 + 1e-12            # a tie goes to the even code
    code = np.where(np.isnan(a), 0, far.argmin(-1)) + 8 * np.signbit(b)
    return code.reshape(R, K), np.where(finite, E + 127, 255).astype(np.uint8)


def mx_values(code, byte):
    R, K = code.shape
    v = np.where(code & 8, -1.0, 1.0) * E2M1[code & 7]
    s = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return (v.reshape(R, K // 32, 32) * s[..., None]).reshape(R, K)


def mx_pack(code, byte):
    """The library's layout: codes [K/32, R, 16], scales [ceil(K/128), R, 4]."""
    R, K = code.shape
    c = code.reshape(R, K // 32, 16, 2).astype(np.uint8)
    codes = np.ascontiguousarray((c[..., 0] | c[..., 1] << 4).transpose(1, 0, 2))
    words = -(-K // 128)
    s = np.zeros((R, words * 4), np.uint8)
    s[:, :K // 32] = byte
    return codes, np.ascontiguousarray(s.reshape(R, words, 4).transpose(1, 0, 2))


def gelu(y):
    return 0.5 * y * (1 + np.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))


def linear(a, w, bias=None, act=False):
    """(y, how far a correct bf16 result may be) for the values a [M, K], w [N, K]."""
    y, size = a @ w.T, np.abs(a) @ np.abs(w).T
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    far = (a.shape[1] + 8) * ADD * size
    if act:
        # slope of GELU below 1.13; its own fp32 steps: the exponent's argument, at
        # most 128, is off by 3 roundings
        y, far = gelu(y), 1.13 * far
        far = far + 128 * 3 * 2.0 ** -24 * np.abs(y) + 1e-30
    return y, HALF_BF16 * np.abs(y) + (1 + HALF_BF16) * far


# ------------------------------------------------------------------- rotary

def turns(freqs):
    """int64 frequencies -> turns a position as exact integers of 2^-64."""
    return [int(f) for f in np.asarray(freqs)]


def rotate(x, positions, freqs, layout, inverse=False, magnitude=1.0):
    """x [T, H, d] -> (y, how far an fp32 computation may be, before the output's rounding)."""
    y, far = x.copy(), np.zeros_like(x)
    half = len(freqs)
    for i, f in enumerate(turns(freqs)):
        phase = np.array([(int(p) * f) % (1 << 64) for p in positions], dtype=np.float64) / 2.0 ** 64
        c, s = np.cos(2 * np.pi * phase)[:, None], np.sin(2 * np.pi * phase)[:, None]
        s = -s if inverse else s
        j, k = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        a, b = x[..., j], x[..., k]
        y[..., j], y[..., k] = (a * c - b * s) * magnitude, (b * c + a * s) * magnitude
        # sine and cosine: 1.2e-7 from the instruction, 2e-7 from the angle's fp32 fraction of a
        # turn; three fp32 roundings
        far[..., j] = far[..., k] = (np.abs(a) + np.abs(b)) * abs(magnitude) * (3.2e-7 + 4 * 2.0 ** -24)
    return y, far


# ------------------------------------------------------------------- attention

def attention(q, k, v, scale):
    """One sequence and cache head: q [G, d], k, v [n, d] -> (o [G, d], how far it may be)."""
    n, d = k.shape
    if n == 0:
        return np.zeros_like(q), np.zeros_like(q)
    s = scale * (q @ k.T)
    size = abs(scale) * (np.abs(q) @ np.abs(k).T)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o, weight = p @ v, p @ np.abs(v)
    # a score is off by its sum's additions and three roundings of its product with the scale; a
    # weight by that (twice: itself and the sum it is divided by), the exponential, and its bf16
    # rounding (twice)
    off = ((d + 8) * ADD * size + 3 * 2.0 ** -24 * np.abs(s)).max(-1, keepdims=True)
    far = weight * (2 * HALF_BF16 + 2 * np.expm1(off) + 2.0 ** -20 + (n + 8) * ADD)
    return o, HALF_BF16 * np.abs(o) + (1 + HALF_BF16) * far + 1e-37
