"""MXFP4 (OCP microscaling, E2M1 elements, E8M0 scales) and expert selection in plain numpy, 64 bits, from the definitions.

A block of 32 values shares a power of two 2^(s - 127); its codes are the nearest of {0, .5, 1, 1.5, 2, 3, 4, 6}, ties to the even
code, saturating.  Shares no code with csrc/.
"""
from __future__ import annotations

import math

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest_code(a: np.ndarray) -> np.ndarray:
    """Codes 0..7 of magnitudes a >= 0, by distance; of two equally near values the even code."""
    gap = np.abs(a[..., None] - VALUES)
    low = gap.min(-1, keepdims=True)
    near = gap == low
    first = near.argmax(-1)
    last = 7 - near[..., ::-1].argmax(-1)
    return np.where(first % 2 == 0, first, last).astype(np.uint8)


def quantize(x: np.ndarray):
    """x [rows, n] float64 (exact copies of fp32 or bf16 values) -> codes uint8 [rows, nb, 32] (0..15), scale bytes uint8 [rows, nb]."""
    rows, n = x.shape
    nb = -(-n // 32)
    v = np.zeros((rows, nb * 32))
    v[:, :n] = x
    v = v.reshape(rows, nb, 32)
    top = np.abs(v).max(2)
    fine = np.isfinite(v).all(2)
    exponent = np.frexp(np.where(fine, top, 1.0))[1] - 1
    s = np.where(fine, np.where(top > 0, np.maximum(exponent - 2, -127), -127) + 127, 255).astype(np.uint8)
    blk = np.where(fine[..., None], v, 0.0)
    step = np.ldexp(1.0, np.where(fine, s.astype(np.int64), 127) - 127)[..., None]
    codes = nearest_code(np.abs(blk) / step) + 8 * np.signbit(blk).astype(np.uint8)
    return codes, s


def values(codes: np.ndarray, s: np.ndarray, n: int) -> np.ndarray:
    """The values that codes [rows, nb, 32] and scale bytes stand for, [rows, n]."""
    scale = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 127))
    v = np.where(codes & 8, -1.0, 1.0) * VALUES[codes & 7] * scale[..., None]
    return v.reshape(v.shape[0], -1)[:, :n]


def store(codes: np.ndarray, s: np.ndarray):
    """The layout in memory: bytes [rows, 16 nb], scales [ceil(nb / 4), rows rounded up to 4, 4]."""
    rows, nb = s.shape
    packed = (codes[:, :, 0::2] | (codes[:, :, 1::2] << 4)).reshape(rows, 16 * nb)
    sc = np.zeros((-(-nb // 4), -(-rows // 4) * 4, 4), np.uint8)
    for b in range(nb):
        sc[b // 4, :rows, b % 4] = s[:, b]
    return packed, sc


def load(packed: np.ndarray, sc: np.ndarray, n: int) -> np.ndarray:
    """values() of a stored matrix."""
    rows, nb = packed.shape[0], -(-n // 32)
    codes = np.empty((rows, nb * 32), np.uint8)
    codes[:, 0::2], codes[:, 1::2] = packed & 15, packed >> 4
    s = np.stack([sc[b // 4, :rows, b % 4] for b in range(nb)], 1)
    return values(codes.reshape(rows, nb, 32), s, n)


def product(a: np.ndarray, w: np.ndarray, offsets, n_experts: int):
    """a [rows, n], w [E N, n] -> out [rows, N] (NaN in rows of no expert)."""
    N = w.shape[0] // n_experts
    out = np.full((a.shape[0], N), np.nan)
    for e in range(n_experts):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        out[lo:hi] = a[lo:hi] @ w[e * N:(e + 1) * N].T
    return out


def select(logits: np.ndarray, k: int, *, scoring="softmax", bias=None, groups=1, kept=1, group_top=1, renorm=True, scale=1.0):
    """Token by token.  Returns (idx [T, k], w [T, k])."""
    T, E = logits.shape
    per = E // groups
    idx, wts = np.zeros((T, k), np.int64), np.zeros((T, k))
    for t in range(T):
        l = [(-math.inf if math.isnan(v) else float(v)) for v in logits[t]]
        m = max(l)
        if scoring == "softmax":
            ex = [0.0 if v == -math.inf else 1.0 if v == m else math.exp(v - m) if m < math.inf else 0.0 for v in l]
            tot = math.fsum(ex)
            s = [v / tot if tot > 0 else 0.0 for v in ex]
        else:
            s = [0.0 if v < -700 else 1.0 / (1.0 + math.exp(-v)) for v in l]
        if bias is None and (groups == 1 or group_top == 1):
            key = list(l)
        else:
            key = [v + (0.0 if bias is None else float(bias[e])) for e, v in enumerate(s)]
        key = [-math.inf if l[e] == -math.inf else key[e] for e in range(E)]
        g = [sum(sorted(key[i * per:(i + 1) * per], reverse=True)[:group_top]) for i in range(groups)]
        stay = sorted(range(groups), key=lambda i: (-g[i], i))[:kept]
        left = [e for e in range(E) if e // per in stay]
        chosen = sorted(left, key=lambda e: (-key[e], e))[:k]
        w = [s[e] for e in chosen]
        tot = math.fsum(w)
        if renorm:
            w = [v / tot if tot > 0 else 0.0 for v in w]
        idx[t], wts[t] = chosen, [v * scale for v in w]
    return idx, wts


def experts(x: np.ndarray, gate: np.ndarray, up: np.ndarray, down: np.ndarray, idx: np.ndarray, wt: np.ndarray) -> np.ndarray:
    """The experts' FFN: x [T, d]; gate, up [E, f, d] and down [E, d, f] are the 4-bit matrices' values; rows and hidden rows are
    rounded to MXFP4 here."""
    xq = values(*quantize(x), x.shape[1])
    y = np.zeros_like(x)
    for t in range(x.shape[0]):
        for j in range(idx.shape[1]):
            e = int(idx[t, j])
            g, u = gate[e] @ xq[t], up[e] @ xq[t]
            h = (g / (1.0 + np.exp(-g)) * u)[None]
            y[t] += wt[t, j] * (down[e] @ values(*quantize(h), h.shape[1])[0])
    return y
