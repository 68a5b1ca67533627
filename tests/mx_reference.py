"""The microscaled formats and the operators over them, plain numpy in 64 bits: written from the formats' definition and
shared by the tests only."""
import math

import numpy as np

GRID4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def encode(x, bits):
    """(codes [rows][K] as whole numbers, scale bytes [rows][blocks]) of x, float64 [rows][K]."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    blocks = -(-K // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :K] = x
    v = v.reshape(rows, blocks, 32)
    bad = ~np.isfinite(v).all(2)
    v = np.where(bad[:, :, None], 0, v)
    top = np.abs(v).max(2)
    s = np.clip(np.where(top == 0, -127, np.frexp(top)[1] - 1 - (2 if bits == 4 else 0)), -127, 127)
    t = np.ldexp(v, -s[:, :, None])
    if bits == 8:
        codes = np.clip(np.rint(64 * t), -127, 127).astype(np.int64)
    else:
        distance = np.abs(np.abs(t)[..., None] - GRID4)
        first = distance.argmin(-1)                              # the lower of two at the same distance
        above = np.minimum(first + 1, 7)
        tie = (above > first) & (np.take_along_axis(distance, above[..., None], -1) == np.take_along_axis(distance, first[..., None], -1))[..., 0]
        codes = np.where(tie & (first % 2 == 1), above, first) + 8 * np.signbit(t)
    codes = np.where(bad[:, :, None], 0, codes).reshape(rows, blocks * 32)
    scales = np.where(bad, 255, s + 127)
    return codes[:, :K], scales


def decode(codes, scales, bits):
    rows, K = codes.shape
    s = np.repeat(scales, 32, 1)[:, :K]
    v = (GRID4[codes & 7] * np.where(codes & 8, -1, 1)) if bits == 4 else codes / 64
    return np.where(s == 255, np.nan, np.ldexp(v, np.where(s == 255, 0, s - 127)))


def quantised(x, bits):
    return decode(*encode(x, bits), bits)


def store(codes, scales, bits, code_pitch, scale_pitch):
    """The two buffers as the header describes them."""
    rows, K = codes.shape
    c = np.zeros((rows, code_pitch * 8 // bits), np.int64)
    c[:, :K] = codes
    c = (c[:, ::2] | c[:, 1::2] << 4) if bits == 4 else c & 255
    s = np.zeros((rows, scale_pitch), np.int64)
    s[:, : scales.shape[1]] = scales
    return c.astype(np.uint8), s.astype(np.uint8)


_erf = np.vectorize(math.erf, otypes=[np.float64])
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1, e) / (1 + e)


def function(name, v):
    return v * sigmoid(v) if name == "silu" else 0.5 * v * _erfc(-v / math.sqrt(2))


def slope(name, v):
    if name == "silu":
        s = sigmoid(v)
        return s + v * s * sigmoid(-v)
    return 0.5 * _erfc(-v / math.sqrt(2)) + v * np.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)


def norm(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean, rstd


def norm_grad(dy, X, mean, rstd, gamma):
    h, d = (X - mean) * rstd, dy * gamma
    dx = rstd * (d - d.mean(1, keepdims=True) - h * (d * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)
