"""The 8-bit operators in 64 bits on the CPU, written from their definitions.

TEST INFRASTRUCTURE ONLY, like the rest of this folder.  Codes are numpy uint8 arrays in the e4m3 format (sign, four exponent
bits with bias 7, three mantissa bits; 0x7f and 0xff are NaN, there are no infinities), scales float64.
"""
import numpy as np

BLOCK = 128
LARGEST = 448.0
SMALLEST_SCALE = 2.0 ** -100


def _table():
    values = np.empty(256)
    for code in range(256):
        sign, exponent, mantissa = -1.0 if code & 0x80 else 1.0, code >> 3 & 15, code & 7
        if exponent == 15 and mantissa == 7:
            values[code] = np.nan
        elif exponent == 0:
            values[code] = sign * mantissa * 2.0 ** -9
        else:
            values[code] = sign * (8 + mantissa) * 2.0 ** (exponent - 10)
    return values


E4M3 = _table()


def _columns(scales, cols):
    """[..., blocks] -> [..., cols]"""
    return np.repeat(scales, BLOCK, axis=-1)[..., :cols]


def activations(codes, scales):
    """codes [R, C], scales [blocks, R]"""
    return E4M3[codes] * _columns(scales.T, codes.shape[1])


def weights(codes, scales):
    """codes [N, K], scales [N blocks, K blocks]"""
    return E4M3[codes] * _columns(np.repeat(scales, BLOCK, axis=0)[:codes.shape[0]], codes.shape[1])


def scales_of(v, block_rows=1):
    """The scale of every block of v [R, C]: [blocks, R] (before activations' scales are rounded to bf16), or [R blocks, C
    blocks] for block_rows = 128."""
    R, C = v.shape
    cb = -(-C // BLOCK)
    a = np.zeros((R, cb * BLOCK))
    a[:, :C] = np.abs(v)
    a = a.reshape(R, cb, BLOCK).max(2)
    if block_rows != 1:
        rb = -(-R // BLOCK)
        full = np.zeros((rb * BLOCK, cb))
        full[:R] = a
        return np.maximum(full.reshape(rb, BLOCK, cb).max(1) / LARGEST, SMALLEST_SCALE)
    return np.maximum(a / LARGEST, SMALLEST_SCALE).T


def silu(x):
    return x / (1.0 + np.exp(-x))


def normalized(v, kind, eps):
    """kind: "rms" or "layer"; the factor it multiplies with comes second"""
    if kind == "layer":
        v = v - v.mean(1, keepdims=True)
    factor = 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    return v * factor, factor


def activation(g, act):
    return {"plain": lambda: g, "sigmoid": lambda: 1.0 / (1.0 + np.exp(-g)), "tanh": lambda: np.tanh(g)}[act]()
