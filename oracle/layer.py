"""The operators around the quantized attention in 64 bits, from their formulas -- test infrastructure only.

Arrays are numpy float64 unless said otherwise; [B, H, N, d] throughout.
"""
import math

import numpy as np

INTERLEAVED, HALF = "interleaved", "half"


# ----------------------------------------------------------------------------- norm and rotation
def frequencies(n, theta=10000.0, scaling="none", factor=1.0, original=0, fast=32.0, slow=1.0):
    """Radians per position of the n / 2 pairs of an axis."""
    out = []
    for i in range(n // 2):
        f = theta ** (-2.0 * i / n)
        if scaling == "linear":
            f /= factor
        elif scaling == "ntk" and n > 2:
            f = (theta * factor ** (n / (n - 2.0))) ** (-2.0 * i / n)
        elif scaling == "yarn":
            c = lambda b: n * math.log(original / (2.0 * math.pi * b)) / (2.0 * math.log(theta))
            lo, hi = max(math.floor(c(fast)), 0), min(math.ceil(c(slow)), n - 1)
            r = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = f * (1.0 - r) + f / factor * r
        out.append(f)
    return np.array(out)


def positions_of(grid, start=(0, 0, 0)):
    T, Y, X = grid
    n = np.arange(T * Y * X)
    return np.stack([start[0] + n // (Y * X), start[1] + n // X % Y, start[2] + n % X], axis=1)


def default_dims(d):
    side = 2 * (d // 6)
    return (d - 2 * side, side, side)


def pair_channels(dims, layout):
    """[(axis, i, a, b)]: pair i of an axis is channels (a, b)."""
    out, s = [], 0
    for axis, n in enumerate(dims):
        for i in range(n // 2):
            out.append((axis, i, s + 2 * i, s + 2 * i + 1) if layout == INTERLEAVED else (axis, i, s + i, s + n // 2 + i))
        s += n
    return out


def qk_norm_rope(x, weight=None, norm="none", eps=1e-6, layout=None, dims=None, pos=None, freqs=None, mult=1.0):
    """(y, size): size bounds what a channel of y is a sum of, |a| + |b| of its normed pair times mult."""
    B, H, N, d = x.shape
    y = x.astype(np.float64)
    if norm == "head":
        y = y / np.sqrt((y ** 2).mean(axis=3, keepdims=True) + eps)
        y = y * (1.0 if weight is None else weight.reshape(1, 1, 1, d))
    elif norm == "token":
        y = y / np.sqrt((y ** 2).mean(axis=(1, 3), keepdims=True) + eps)
        y = y * (1.0 if weight is None else weight.reshape(1, H, 1, d))
    out, size = y.copy(), np.abs(y)
    if layout is not None:
        p = np.broadcast_to(pos, (B, N, 3)) if pos.ndim == 2 else pos
        for axis, i, a, b in pair_channels(dims, layout):
            t = p[:, None, :, axis] * freqs[axis][i]
            c, s = mult * np.cos(t), mult * np.sin(t)
            out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
            size[..., a] = size[..., b] = mult * (np.abs(y[..., a]) + np.abs(y[..., b]))
    return out, size


# ----------------------------------------------------------------------------- attention to an encoder's states
def cross_attention(q, k, v, scale, kv_len=None, mask=None):
    """(o, lse) with the kept keys alone; rows without any are 0 and -inf."""
    B, H, Nq, d = q.shape
    Hkv, Nkv = k.shape[1:3]
    o, lse = np.zeros((B, H, Nq, d)), np.full((B, H, Nq), -np.inf)
    for b in range(B):
        keep = np.arange(Nkv) < (Nkv if kv_len is None else kv_len[b])
        if mask is not None:
            keep &= mask[b] != 0
        if not keep.any():
            continue
        for h in range(H):
            g = h // (H // Hkv)
            s = scale * (q[b, h] @ k[b, g][keep].T)
            top = s.max(axis=1, keepdims=True)
            e = np.exp(s - top)
            total = e.sum(axis=1, keepdims=True)
            o[b, h] = e / total @ v[b, g][keep]
            lse[b, h] = (top + np.log(total))[:, 0]
    return o, lse


# ----------------------------------------------------------------------------- E4M3 blocks and their product
def e4m3_values():
    """The value of every E4M3 byte (1 sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7f and 0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = m / 8.0 * 2.0 ** -6 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)
        out[c] = np.nan if c & 127 == 127 else (-v if c & 128 else v)
    return out


def round_e4m3(x):
    """Codes of float64 values within +-464, to nearest, ties to the even code."""
    grid = e4m3_values()[:127]
    mag = np.abs(x)
    hi = np.clip(np.searchsorted(grid, mag), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = mag - grid[lo], grid[hi] - mag
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    return code | np.where(np.signbit(x), 128, 0).astype(np.uint8)


def quant_fp8(x, block_rows):
    """(codes [rows, cols], scale [row blocks, column blocks]) of an fp32 matrix; the decisions are single fp32 operations."""
    rows, cols = x.shape
    codes = np.empty((rows, cols), np.uint8)
    scale = np.empty((-(-rows // block_rows), -(-cols // 128)), np.float32)
    x = x.astype(np.float32)
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            at = (slice(i * block_rows, (i + 1) * block_rows), slice(128 * j, 128 * j + 128))
            a = max(np.abs(x[at]).max(), np.float32(448.0 * 2.0 ** -100))
            scale[i, j] = a / np.float32(448.0)
            codes[at] = round_e4m3((x[at] * (np.float32(448.0) / a)).astype(np.float64))
    return codes, scale


def linear_fp8(x_codes, x_scale, w_codes, w_scale, bias=None):
    """(y, size): x_scale [column blocks, M], w_scale [N blocks, column blocks]; size is the sum of the products' magnitudes."""
    val = e4m3_values()
    M, K = x_codes.shape
    N = w_codes.shape[0]
    xs = np.repeat(x_scale.T.astype(np.float64), 128, axis=1)[:, :K]
    ws = np.repeat(np.repeat(w_scale.astype(np.float64), 128, axis=0)[:N], 128, axis=1)[:, :K]
    x, w = val[x_codes] * xs, val[w_codes] * ws
    y, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    return y, size
