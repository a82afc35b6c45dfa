"""Plain CPU implementation, in 64-bit numpy, of the operators around the GEMVs of a decoder layer:
the cache formats, the paged cache's writing and reading, attention over it, and the norms around a
block. It shares no code with the kernels or with the package.

Batches are given as Python lists: q_len[s] new tokens of sequence s, ctx_len[s] its length with
them, pages[s] its page numbers.
"""
from __future__ import annotations

import numpy as np

F16, FP8, FP4 = 0, 1, 2
BLOCK = 32


def e4m3_values() -> np.ndarray:
    """The 256 values of E4M3 by code (S.EEEE.MMM, bias 7, no infinity, S.1111.111 is NaN)."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if e == 15 and m == 7:
            v = np.nan
        out[b] = -v if b & 128 else v
    return out


def e2m1_values() -> np.ndarray:
    """The 16 values of E2M1 by code (S.EE.M, bias 1)."""
    out = []
    for b in range(16):
        e, m = b >> 1 & 3, b & 1
        v = m * 0.5 if e == 0 else (2 + m) * 2.0 ** (e - 2)
        out.append(-v if b & 8 else v)
    return np.array(out)


def _nearest(x, magnitudes):
    """Index of the nearest of ascending magnitudes to each x >= 0, ties to the even index."""
    hi = np.clip(np.searchsorted(magnitudes, x), 1, len(magnitudes) - 1)
    lo = hi - 1
    dl, dh = x - magnitudes[lo], magnitudes[hi] - x
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def encode(x, fmt):
    """Rows of fp32 values [..., D] as (codes, scale bytes): fp16 bits, E4M3 bytes or packed E2M1."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    if fmt == F16:
        return np.clip(x, -65504, 65504).astype(np.float16), None
    limit, e_max = (448.0, 7) if fmt == FP8 else (6.0, 13)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    top = np.fmax.reduce(np.abs(b), axis=-1)
    top = np.where(np.isnan(top), 0, top)
    e = np.full(top.shape, -14)
    for _ in range(e_max + 14):
        e = np.where((top > limit * 2.0 ** e) & (e < e_max), e + 1, e)
    v = b * (2.0 ** -e)[..., None]
    mag = np.minimum(np.abs(v), limit)
    if fmt == FP8:
        code = _nearest(mag, e4m3_values()[:127])
        code = np.where(np.isnan(v), 127, code | np.where(np.signbit(v), 128, 0))
        codes = code.reshape(x.shape).astype(np.uint8)
    else:
        code = _nearest(np.where(np.isnan(mag), 6.0, mag), e2m1_values()[:8])
        code = (code | np.where(np.signbit(v), 8, 0)).reshape(x.shape)
        codes = (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)
    return codes, (e + 127).astype(np.uint8)


def decode(codes, scale, fmt):
    """The values that a cache's rows stand for, in 64 bits."""
    if fmt == F16:
        return codes.astype(np.float64)
    if fmt == FP8:
        x = e4m3_values()[codes]
    else:
        x = np.stack((e2m1_values()[codes & 15], e2m1_values()[codes >> 4]), -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    return x * np.repeat(2.0 ** (scale.astype(np.float64) - 127), BLOCK, axis=-1)


def rms_norm(x, weight, eps):
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * weight


def prepare_heads(x, positions, weight=None, cos=None, sin=None, eps=1e-6):
    """Per-head norm and rotation of [tokens][heads][D] at each token's position, in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = rms_norm(x, np.asarray(weight, dtype=np.float64), eps)
    if cos is not None:
        at = np.clip(positions, 0, len(cos) - 1)
        c, s = (np.asarray(t, dtype=np.float64)[at][:, None] for t in (cos, sin))
        h = x.shape[-1] // 2
        a, b = x[..., :h], x[..., h:]
        x = np.concatenate((a * c - b * s, b * c + a * s), axis=-1)
    return x


def token_positions(q_len, ctx_len):
    return np.concatenate([np.arange(n - m, n) for m, n in zip(q_len, ctx_len)] or [np.zeros(0, int)]).astype(int)


def sequence_rows(pool, scales, fmt, pages, n):
    """The first n tokens of a sequence from pool [n_pages][heads][page][row]: [n][heads][D]."""
    page = pool.shape[2]
    rows = []
    for p in range(n):
        at = (pages[p // page], slice(None), p % page)
        rows.append(decode(pool[at], None if scales is None else scales[at], fmt))
    return np.stack(rows) if rows else np.zeros((0, pool.shape[1], 1))


def attention(q, k_of, v_of, q_len, ctx_len, scale, window=0):
    """q [tokens][Hq][D]; k_of[s], v_of[s]: sequence s's [ctx][Hkv][D]. Returns (out, lse, spread):
    spread[t][h][d] = sum_j p_j |v_j| / sum_j p_j, what rounding the weights acts on."""
    t_all, hq, d = q.shape
    out, spread, lse = np.zeros((t_all, hq, d)), np.zeros((t_all, hq, d)), np.full((t_all, hq), -np.inf)
    t = 0
    for s, (n, ctx) in enumerate(zip(q_len, ctx_len)):
        for i in range(n):
            pos = ctx - n + i
            lo = max(0, pos - window + 1) if window else 0
            if pos >= 0:
                group = hq // k_of[s].shape[1]
                for h in range(hq):
                    k, v = k_of[s][lo:pos + 1, h // group], v_of[s][lo:pos + 1, h // group]
                    z = scale * (k @ q[t, h].astype(np.float64))
                    p = np.exp(z - z.max())
                    out[t, h] = p @ v / p.sum()
                    spread[t, h] = p @ np.abs(v) / p.sum()
                    lse[t, h] = z.max() + np.log(p.sum())
            t += 1
    return out, lse, spread


def norm(h, weight=None, y=None, post_weight=None, gate=None, res_scale=1.0, eps=1e-6):
    """(h', x) of the norms around a block, in 64 bits; x is None without weight."""
    h = np.asarray(h, dtype=np.float64)
    if y is not None:
        t = np.asarray(y, dtype=np.float64)
        if post_weight is not None:
            t = rms_norm(t, np.asarray(post_weight, dtype=np.float64), eps)
        if gate is not None:
            t = t * np.asarray(gate, dtype=np.float64)
        h = h + res_scale * t
    return h, None if weight is None else rms_norm(h, np.asarray(weight, dtype=np.float64), eps)
