"""The operators' formulas in 64 bits on the CPU, in numpy, one row at a time where that is plainest."""
from __future__ import annotations

import numpy as np
import torch

GROUP = 32
SCALES = np.array([(8 + (b & 7)) * 2.0 ** ((b >> 3) - 21) for b in range(256)])


def rounded(x, dtype: str) -> np.ndarray:
    """x as the storage type holds it, in float64."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return (t.to(torch.bfloat16) if dtype == "bf16" else t).double().numpy()


def quantise(x: np.ndarray):
    """x [..., d] -> codes -7..7 and scale bytes [..., d / 32]."""
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    amax = np.abs(g).max(-1)
    byte = np.minimum(np.searchsorted(7 * SCALES, amax), 255)              # the least whose sevenfold reaches it
    code = np.clip(np.rint(g / SCALES[byte][..., None]), -7, 7)            # half to even; 24 by 4 bits: exact in 53
    return code.reshape(x.shape).astype(np.int64), byte.astype(np.int64)


def values(code: np.ndarray, byte: np.ndarray) -> np.ndarray:
    g = code.reshape(*code.shape[:-1], -1, GROUP) * SCALES[byte][..., None]
    return g.reshape(code.shape)


def pack(code: np.ndarray) -> np.ndarray:
    n = (code + 8).astype(np.uint8)
    return np.ascontiguousarray(n[..., 0::2] | (n[..., 1::2] << 4))


def unpack(codes: np.ndarray) -> np.ndarray:
    return np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1).astype(np.int64) - 8


def norm_rope(x: np.ndarray, w, eps: float, pos: np.ndarray, freq, interleaved: bool):
    """[n, H, d] -> the result, and |a| + |b| of every channel's pair, which its rounding errors scale with."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else w)
    rot = 2 * len(freq)
    out, size = y.copy(), np.abs(y)
    if rot:
        # the angle in turns, reduced before it is multiplied by 2 pi: longdouble keeps 64 bits of pos * f
        turns = np.asarray(pos, dtype=np.longdouble)[:, None] * (np.asarray(freq, dtype=np.longdouble) / (2 * np.longdouble(np.pi) + np.longdouble(2.4492935982947064e-16)))
        angle = ((turns - np.rint(turns)) * 2 * np.longdouble(np.pi)).astype(np.float64)[:, None]
        c, s = np.cos(angle), np.sin(angle)
        i = np.arange(rot // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, seen: np.ndarray, scale: float):
    """q [R, Hq, d], k, v [T, Hkv, d], seen [R, T] -> o, lse, sum p |v|, and the largest sum |q k| scale of a row."""
    R, hq, d = q.shape
    g = hq // k.shape[1]
    o, lse = np.zeros(q.shape), np.full((R, hq), -np.inf)
    weight, terms = np.zeros(q.shape), np.zeros((R, hq))
    for i in range(R):
        j = np.flatnonzero(seen[i])
        if len(j) == 0:
            continue
        for h in range(hq):
            kk, vv = k[j, h // g], v[j, h // g]
            t = kk @ q[i, h] * scale
            m = t.max()
            p = np.exp(t - m)
            z = p.sum()
            o[i, h], lse[i, h] = p @ vv / z, m + np.log(z)
            weight[i, h] = p @ np.abs(vv) / z
            terms[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * abs(scale)
    return o, lse, weight, terms


def window_mask(n: int, window: int, sink: int, causal: bool, rows=None) -> np.ndarray:
    """[rows, n]: which keys of a segment of n rows its rows see."""
    i = np.arange(n)[:, None] if rows is None else np.asarray(rows)[:, None]
    j = np.arange(n)
    seen = (np.abs(i - j) < window) | (j < sink)
    return seen & (j <= i) if causal else seen


def check_attention(o, lse, ref, dtype: str, what="", weights=None):
    """weights: the type that the softmax weights are stored in, where that is not the storage type.  Bounds by arithmetic.  A logit is a sum of fp32 products whose partial sums are rounded, or cut off by the tensor core, to 24
    bits, at most 2^-23 each over 8 + 2 steps, of the sum of magnitudes; the factor log2(e) and the subtraction of the reference add
    2 roundings of the logit: e_s = 2^-19 * terms.  A weight is off by e_s, by the exponential's 2^-21 and, where it is stored in
    bf16, by 2^-8 (in two bf16 parts, each to the nearest: the first leaves 2^-8, the second 2^-9 of that); the largest is what the row sum divides by, so both of numerator and denominator: twice that times sum p |v|.  The
    output is rounded by 2^-8 (bf16) or 2^-24 of itself.  Sums over keys and partials: 2^-19 of sum p |v|."""
    want_o, want_lse, weight, terms = ref
    e_s = 2.0 ** -19 * terms
    p_err = e_s + 2.0 ** -21 + {"bf16": 2.0 ** -8, "2 x bf16": 2.0 ** -17}.get(weights or dtype, 0.0)
    tol = (2 * p_err[..., None] + 2.0 ** -19) * weight + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want_o) + 1e-30
    assert np.isfinite(o).all(), what
    bad = np.abs(o - want_o) > tol
    assert not bad.any(), "%s: o off by %.3e where %.3e is allowed" % (what, np.abs(o - want_o)[bad].max(), tol[bad].min())
    if lse is not None:
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(lse), empty), what + ": empty rows"
        lim = e_s + 2.0 ** -19 + 2.0 ** -22 * np.where(empty, 0, np.abs(want_lse))
        err = np.where(empty, 0, np.abs(np.where(empty, 0, lse) - np.where(empty, 0, want_lse)))
        assert (err <= lim).all(), "%s: lse off by %.3e where %.3e is allowed" % (what, (err - lim).max(), lim.min())
