"""Plain statements, in 64 bits on the CPU, of 8-bit floating point, of products in it and of the root-mean-square norm, and the error bounds that go with fp32 sums.

numpy only; nothing here is shared with the library."""
import numpy as np
import torch

from stage_reference import DEPTH, HALF_ULP, SMALLEST, U, act8_encode

# What the bytes 0 ... 126 stand for: four exponent bits biased by 7, three fraction bits, subnormals; 127 is no number.
TABLE = np.array([(byte & 7) * 2.0 ** -9 if byte < 8 else (8 + (byte & 7)) * 2.0 ** (byte // 8 - 10) for byte in range(127)])
MIDDLES = (TABLE[1:] + TABLE[:-1]) / 2


def bytes_of(x):
    """Nearest bytes of float64 numbers of at most 448, ties to even."""
    a = np.abs(x)
    byte = np.searchsorted(MIDDLES, a, side="left")  # the first number whose upper border is not below
    tie = (byte < 126) & (a == MIDDLES[np.minimum(byte, 125)]) & (byte % 2 == 1)
    return (byte + tie + 128 * np.signbit(x)).astype(np.uint8)


def fp8_encode(x, tile=1):
    """(numbers [rows, blocks * 128], S [rows, blocks], values read back) of a float64 matrix; `tile` rows share a scale."""
    rows, cols = x.shape
    blocks = -(-cols // 128)
    q, S, back = np.zeros((rows, blocks * 128), dtype=np.uint8), np.zeros((rows, blocks), dtype=np.uint8), np.full((rows, cols), np.nan)
    for top in range(0, rows, tile):
        for b in range(blocks):
            part = x[top:top + tile, 128 * b:128 * b + 128]
            here = np.s_[top:top + tile, 128 * b:128 * b + 128]
            if not np.isfinite(part).all():
                q[here], S[top:top + tile, b] = 0x7F, 255
                continue
            m, exponent = np.frexp(np.abs(part).max())  # m * 2^exponent, m in [1/2, 1); 448 = 0.875 * 2^9
            scale = max(int(exponent) - 9 + (1 if m > 0.875 else 0), -126) if m > 0 else -126
            byte = bytes_of(np.ldexp(part, -scale))
            q[top:top + tile, 128 * b:128 * b + part.shape[1]] = byte
            S[top:top + tile, b] = scale + 127
            back[here] = np.where(byte > 127, -1.0, 1.0) * np.ldexp(TABLE[byte & 127], scale)
    return q, S, back


def fp8_layout(rows, cols):
    """(bytes from one row to the next, where the scales begin, bytes from one block's scales to the next, all bytes)."""
    pitch, high = -(-cols // 128) * 128, -(-rows // 256) * 256
    at = -(-(rows * pitch) // 256) * 256
    return pitch, at, high, at + pitch // 128 * high


def fp8_buffer(x, tile=1):
    """The buffer of a float64 matrix, as the library lays it out; what is nobody's is 0xA5."""
    rows, cols = x.shape
    q, S, _ = fp8_encode(x, tile)
    _, at, high, size = fp8_layout(rows, cols)
    buffer = np.full(size, 0xA5, dtype=np.uint8)
    buffer[:q.size] = q.reshape(-1)
    buffer[at:].reshape(-1, high)[:, :rows] = S.T
    return buffer


def fp8_split(buffer, rows, cols):
    """(numbers, S) of a buffer."""
    pitch, at, high, size = fp8_layout(rows, cols)
    return buffer[:rows * pitch].reshape(rows, pitch), buffer[at:size].reshape(-1, high)[:, :rows].T


def product_bound(x, w, y, dtype):
    """Products are exact; of the sums over a row (the matrix instruction's and those behind it) each may lose two units of what has been summed so far, and they do not
    all point one way.  For 16-bit results the 8-bit instruction is used, which cuts each of eight neighbouring products off at 2^-13 of the power of two at or
    below the largest of them: 8 * 2^-13 of that at most for the eight, and the largest product is at most the largest factors'."""
    steps = 2 * U * (8 + 2 * np.sqrt(x.shape[1]))
    bound = (np.abs(x) @ np.abs(w).T) * steps + 2 * U * np.abs(y) + HALF_ULP[dtype] * np.abs(y) * (1 + 2.0 ** -8) + SMALLEST[dtype]
    if dtype != torch.float32:
        most = [np.pad(np.abs(t), ((0, 0), (0, -t.shape[1] % 8))).reshape(t.shape[0], -1, 8).max(axis=2) for t in (x, w)]
        bound = bound + 2.0 ** -10 * (most[0] @ most[1].T)
    return bound


# ---------------------------------------------------------------- root-mean-square norm
def rmsnorm(x, weight, eps):
    """(y, rstd, h)."""
    rstd = 1.0 / np.sqrt((x * x).mean(axis=1) + eps)
    h = x * rstd[:, None]
    return h * weight, rstd, h


def rmsnorm_bounds(y, rstd, dtype):
    """(of y, rstd): the average is a 64-bit sum and 1 / sqrt good to 2^-45; h is rounded once to 32 bits and its product with the weight once more.  Below 2^-126 an
    rstd is held in steps of 2^-149, so it is off by up to 2^-150 whatever its size, and its parts hold it no better: h and y by 2^-150 / rstd of theirs."""
    coarse = np.where(rstd < 2.0 ** -102, 2.0 ** -150 / rstd, 0.0)[:, None]
    return np.abs(y) * (2 * U * (1 + 2 * U) + coarse + HALF_ULP[dtype] * (1 + 4 * U)) + SMALLEST[dtype] + 2.0 ** -148, rstd * (U + 2.0 ** -44) + 2.0 ** -150


def rmsnorm_backward(dy, h, rstd, weight, dsum):
    g = dy * weight
    return rstd[:, None] * (g - h * (g * h).mean(axis=1)[:, None]) + dsum, (dy * h).sum(axis=0)


def rmsnorm_backward_bounds(dy, h, d_h, rstd, weight, dsum, dx, dtype):
    """(of dx, dweight); d_h: what h itself may be off by (nothing where it was kept in 8 bits, a rounding of x * rstd otherwise)."""
    rows = dy.shape[0]
    g = np.abs(dy * weight)
    along = (g * np.abs(h)).mean(axis=1)[:, None]
    d = (DEPTH + 6) * U * np.abs(h) * along + 4 * U * g + d_h * along + np.abs(h) * (g * d_h).mean(axis=1)[:, None]
    depth = rows / 256 + 64  # additions one behind the other: a wavefront's rows, a workgroup's four, the parts
    return (rstd[:, None] * d + 2 * U * np.abs(dsum) + (HALF_ULP[dtype] + U) * np.abs(dx) + SMALLEST[dtype],
            depth * U * (np.abs(dy) * np.abs(h)).sum(axis=0) + (np.abs(dy) * d_h).sum(axis=0) + 1e-40)


__all__ = ["act8_encode", "bytes_of", "fp8_buffer", "fp8_encode", "fp8_layout", "fp8_split", "product_bound", "rmsnorm", "rmsnorm_backward", "rmsnorm_backward_bounds",
           "rmsnorm_bounds", "TABLE"]
