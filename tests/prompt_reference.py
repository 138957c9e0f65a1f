"""The operators of prompts and drafted tokens from their definitions, in 64 bits on the host (test
infrastructure)."""
import math

import numpy as np

import decoding_reference as R

HALF_FP16 = 2.0 ** -11          # an fp16 rounding, relative


def rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def int32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def table(g, lengths, page, width=None, spare=2):
    """Shuffled pages for these lengths: (table with -1 where there is none, number of pages)."""
    need = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(need) + spare
    order = g.permutation(pages)
    width = max(max(need), 1) if width is None else width
    out, at = np.full((len(lengths), width), -1, np.int64), 0
    for b, n in enumerate(need):
        out[b, :n] = order[at:at + n]
        at += n
    return out, pages


def cache(g, pages, kv, page, d, fp8, size=1.0):
    import torch
    out = []
    for _ in range(2):
        t = torch.from_numpy(g.normal(0, size, (pages, kv, page, d))).cuda()
        out.append(t.to(torch.float8_e4m3fn if fp8 else torch.bfloat16))
    return out


def rows(t, tab, b, h, n, page):
    """Positions 0 .. n - 1 of sequence b and cache head h, NaN where there is no page."""
    out = np.full((n, t.shape[3]), np.nan)
    for j in range(-(-n // page)):
        if 0 <= tab[b, j] < len(t):
            part = t[tab[b, j], h][:n - j * page]
            out[j * page:j * page + len(part)] = part
    return out


def sight(new, length, window=0, prefix=None, bits=None):
    """Which keys the new tokens of a sequence see, [new, length]."""
    j, p = np.arange(length)[None], length - new + np.arange(new)[:, None]
    if bits is not None:
        node = j - (length - new) + np.zeros_like(p)
        inside = (node >= 0) & (node < bits.shape[1])
        own = np.take_along_axis(bits, np.clip(node, 0, bits.shape[1] - 1), 1)
        return (node < 0) | (inside & own)
    seen = j <= p
    if window:
        seen &= j > p - window
    if prefix is not None:
        seen |= j < prefix
    return seen


def attention(q, k, v, seen, scale, cap=0.0, slope=0.0, position=None, weight=HALF_FP16):
    """One sequence and query head: q [n, d], k, v [L, d], seen [n, L] -> (o [n, d], how far it may be).
    `weight`: the rounding of a weight."""
    n, L = seen.shape
    d = q.shape[1]
    if L == 0 or n == 0:
        return np.zeros((n, d)), np.zeros((n, d))
    any_seen = seen.any(0)
    k, v = np.where(any_seen[:, None], k, 0.0), np.where(any_seen[:, None], v, 0.0)
    s = scale * (q @ k.T)
    off = (d + 8) * R.ADD * abs(scale) * (np.abs(q) @ np.abs(k).T) + 4 * 2.0 ** -24 * (np.abs(s) + 1)
    if cap:
        # the exponential, its sum with one and the reciprocal: 4 steps of 2^-23 of a number up to 2
        s, off = cap * np.tanh(s / cap), off + cap * 8 * R.ADD
    if position is not None:
        far = slope * np.abs(np.arange(L)[None] - position[:, None])
        s, off = s - far, off + 4 * 2.0 ** -24 * (np.abs(far) + np.abs(s))
    # the argument of the exponential, in units of log2
    off = off + 4 * 2.0 ** -24 * (np.abs(s) + 1)
    s, off = np.where(seen, s, -np.inf), np.where(seen, off, 0.0).max(-1, keepdims=True)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdims=True)
    p = p / np.where(total > 0, total, 1.0)
    o, size = p @ v, p @ np.abs(v)
    # weights' and their sum's errors: the scores', the exponential (2^-20), their rounding; the
    # additions of either
    far = size * (2 * np.expm1(off) + 2 * weight + 2.0 ** -20 + 2 * (2 * L + 8) * R.ADD)
    # weights below fp16's normal range are off by 2^-32 of the largest, which is one in these units
    far = far + 2.0 ** -31 * (seen.astype(float) @ np.abs(v)) / np.where(total > 0, total, 1.0) + 2.0 ** -126
    return o, R.HALF_BF16 * np.abs(o) + (1 + R.HALF_BF16) * far


def check(o, q, k, v, tab, starts, lengths, page, scale=None, window=0, cap=0.0, slopes=None, prefix=None, bits=None,
          k_scale=1.0, v_scale=1.0, weight=HALF_FP16):
    """o and q [T, H, d], k and v [pages, kv, page, d] as float64."""
    T, H, d = q.shape
    kv = k.shape[1]
    scale = 1 / math.sqrt(d) if scale is None else scale
    worst = 0.0
    for b, length in enumerate(lengths):
        length = min(max(length, 0), tab.shape[1] * page)
        first, n = starts[b], starts[b + 1] - starts[b]
        if n == 0:
            continue
        node = None if bits is None else bits[first:first + n]
        seen = sight(n, length, window, None if prefix is None else prefix[b], node)
        for h in range(H):
            kk, vv = rows(k, tab, b, h // (H // kv), length, page), rows(v, tab, b, h // (H // kv), length, page)
            there = np.array([0 <= tab[b, j // page] < len(k) for j in range(length)], bool)
            position = None if slopes is None else length - n + np.arange(n)
            want, far = attention(q[first:first + n, h], kk * k_scale, vv * v_scale, seen & there[None], scale, cap,
                                  0.0 if slopes is None else slopes[h], position, weight)
            off = np.abs(o[first:first + n, h] - want)
            assert (off <= far).all(), (b, h, n, length, np.nanmax(off), np.unravel_index(np.argmax(~(off <= far)), off.shape),
                                        int((~(off <= far)).sum()))
            worst = max(worst, float((off / (far + 1e-300)).max()))
            nothing = ~(seen & there[None]).any(-1)
            assert (o[first:first + n, h][nothing] == 0).all()
    return worst


def starts_of(new):
    return [int(sum(new[:i])) for i in range(len(new) + 1)]


def random_tree(g, n):
    """Which nodes each of n nodes sees: itself and its ancestors."""
    seen = np.eye(n, dtype=bool)
    for i in range(1, n):
        seen[i] |= seen[g.integers(0, i)]
    return seen


def words(bits):
    """bool [T, nodes] -> int64 [T, words]."""
    T, n = bits.shape
    padded = np.zeros((T, max(1, -(-n // 64)) * 64), np.uint64)
    padded[:, :n] = bits
    return (padded.reshape(T, -1, 64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)


def head_norm(x, weight, eps):
    """(values, how far fp32 may be off, relative)."""
    if eps is None:
        return x, 0.0
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    # sums of squares (relative: a step each of the d terms at most), root, quotient, two products
    return y * (1.0 if weight is None else weight), (x.shape[-1] / 2 + 8) * 2.0 ** -24


def turned(x, far, positions, axes, freqs, layout, magnitude=1.0):
    """x [T, H, d] turned by positions [axes, T]; `far` relative to the inputs -> (y, how far)."""
    y, off = x.copy(), np.abs(x) * far
    half = len(freqs)
    for i, f in enumerate(R.turns(freqs)):
        p = positions[axes[i]] if 0 <= axes[i] < len(positions) else np.zeros(x.shape[0], int)
        phase = np.array([(int(t) * f) % (1 << 64) for t in p], dtype=np.float64) / 2.0 ** 64
        c, s = np.cos(2 * np.pi * phase)[:, None], np.sin(2 * np.pi * phase)[:, None]
        j, k = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        a, b = x[..., j], x[..., k]
        y[..., j], y[..., k] = (a * c - b * s) * magnitude, (b * c + a * s) * magnitude
        off[..., j] = off[..., k] = (np.abs(a) + np.abs(b)) * abs(magnitude) * (far + 3.2e-7 + 4 * 2.0 ** -24)
    return y, R.HALF_BF16 * np.abs(y) + (1 + R.HALF_BF16) * off + 1e-37
