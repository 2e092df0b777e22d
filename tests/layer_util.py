"""A pruned layer's training step in 64 bits, and device buffers for its tests.

Nothing here uses the library: matrices are dense float64, derivatives are the formulas'."""
import math

import numpy as np
from scipy.special import erfc, expit

from synthetic import decode_f64, encode, make_weights, select_blocks

EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}    # half a step, relative
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}  # smallest positive value
_A = math.sqrt(2.0 / math.pi)


def act(name, z, lo=0.0, hi=0.0):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "clamp":
        return np.clip(z, lo, hi)
    if name == "gelu":
        return z * 0.5 * erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return z * expit(2.0 * _A * (z + 0.044715 * z ** 3))
    if name == "silu":
        return z * expit(z)
    return z.copy()


def act_slope(name, z, lo=0.0, hi=0.0):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "clamp":
        return ((z >= lo) & (z <= hi)).astype(np.float64)
    if name == "gelu":
        return 0.5 * erfc(-z / math.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        s = expit(2.0 * _A * (z + 0.044715 * z ** 3))
        return s + z * s * (1.0 - s) * 2.0 * _A * (1.0 + 3.0 * 0.044715 * z * z)
    if name == "silu":
        s = expit(z)
        return s + z * s * (1.0 - s)
    return np.ones_like(z)


def round_to(x, dtype):
    """Nearest values of a type, as float64 (through fp32 only where that rounds the same: x has 53 bits, so a tie in
    the second rounding may go the other way; callers compare within half a step)."""
    return decode_f64(encode(np.asarray(x, dtype=np.float32), dtype), dtype)


def half_step(v, dtype):
    """Half the distance to the next value of the type at |v|."""
    return np.maximum(np.abs(v) * EPS[dtype], TINY[dtype] / 2)


def layer(M, K, bh, bw, density, dtype, seed):
    """Blocks, encoded weights and the dense float64 matrix of the kept ones."""
    blocks = select_blocks(M, K, bh, bw, density, seed=seed) if density > 0 else np.zeros((0, 2), np.int32)
    W = make_weights(M, K, seed + 1, dtype)
    kept = np.zeros((M, K))
    for r, c in blocks:
        kept[r:r + bh, c:c + bw] = 1.0
    return blocks, W, decode_f64(W, dtype) * kept


def value_cells(blocks, bh, bw):
    """(row, column) of every kept weight in the packed order: blocks by (start row, column), columns, slots."""
    rows, cols = [], []
    for r, c in sorted(map(tuple, np.asarray(blocks).tolist())):
        for q in range(bw):
            for s in range(bh):
                rows.append(r + (s - r) % bh)
                cols.append(c + q)
    return np.asarray(rows, dtype=np.int64), np.asarray(cols, dtype=np.int64)


def e4m3_values():
    v = [k * 2.0 ** -9 for k in range(8)]
    for e in range(-6, 9):
        v += [(8 + k) * 2.0 ** (e - 3) for k in range(8)]
    return np.asarray(v[:-1])


def checkpoint_of(X, dtype):
    """The 8-bit codes, the exponent bytes and the values they stand for in X's type, from the rule alone: per 32 values of
    a row the smallest s >= -127 with all finite |x| <= 448 2^s; x / 2^s to the nearest e4m3 (ties to the even code), but
    never to 2^128 (fp16: 2^16); Inf and NaN to NaN."""
    table = e4m3_values()
    K, N = X.shape
    G = (N + 31) // 32
    codes = np.zeros((K, N), np.uint8)
    bytes_ = np.zeros((K, G), np.uint8)
    out = np.zeros((K, N))
    top_s = 8 if dtype == "f16" else 120
    for r in range(K):
        for g in range(G):
            x = X[r, 32 * g:32 * g + 32]
            fin = np.isfinite(x)
            top = np.abs(x[fin]).max() if fin.any() else 0.0
            s = -127
            if top > 0:
                s = max(-127, math.frexp(top)[1] - 12)
                while top > math.ldexp(448.0, s):
                    s += 1
            bytes_[r, g] = s + 127
            y = np.abs(np.where(fin, x, 0.0)) / math.ldexp(1.0, s)
            if s >= top_s:
                y = np.minimum(y, 240.0)
            i = np.searchsorted(table, y).clip(1, len(table) - 1)
            up, down = table[i] - y, y - table[i - 1]
            code = np.where((up < down) | ((up == down) & (i % 2 == 0)), i, i - 1)
            code = np.where(fin, code, 127)
            codes[r, 32 * g:32 * g + 32] = code | np.where(np.signbit(x), 128, 0)
            val = np.append(table, np.nan)[code] * math.ldexp(1.0, s)
            out[r, 32 * g:32 * g + 32] = np.copysign(val, x)
    return codes, bytes_, out
