"""Plain statements, in 64 bits on the CPU, of the operators of a stage's training step, and the error bounds that go with fp32 arithmetic.

numpy only; nothing here is shared with the library.  Values of a type travel as float64 arrays that hold exactly representable numbers."""
import numpy as np
import torch

U = 2.0 ** -24  # unit roundoff of fp32
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # of a type, relative: 24, 8 and 11 significant bits
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def rounded(x, dtype):
    """float64 -> nearest value of the type (fp32 first: none of the tests' values lies near a tie of both)."""
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.float32).to(dtype).double().numpy()


def on_device(x, dtype, slack=0, offset=0):
    """A float64 matrix as a device tensor of the type: rows `slack` elements apart, the first one `offset` elements behind an allocation's start."""
    rows, cols = x.shape
    flat = torch.full((offset + rows * (cols + slack) + 8,), 7.0, dtype=dtype, device="cuda")
    view = flat[offset:offset + rows * (cols + slack)].view(rows, cols + slack)[:, :cols]
    view.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(dtype))
    return view


def host(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------- 8 bits
def act8_encode(x):
    """(numbers, exponents, values read back) of a float64 matrix, group by group."""
    rows, cols = x.shape
    groups = -(-cols // 32)
    q, e, back = np.zeros((rows, groups * 32), dtype=np.int8), np.zeros((rows, groups), dtype=np.uint8), np.full((rows, cols), np.nan)
    for g in range(groups):
        part = x[:, 32 * g:32 * g + 32]
        finite = np.isfinite(part).all(axis=1)
        amax = np.where(finite, np.abs(np.where(np.isfinite(part), part, 0.0)).max(axis=1), 1.0)
        exponent = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 1 + 127, 0)  # amax in [2^(exponent - 127), 2^(exponent - 126))
        E = np.maximum(exponent, 7)
        step = np.ldexp(1.0, E - 133)[:, None]
        number = np.clip(np.rint(np.where(finite[:, None], part, 0.0) / step), -127, 127)
        q[:, 32 * g:32 * g + part.shape[1]] = number
        e[:, g] = np.where(finite, E, 255)
        back[:, 32 * g:32 * g + 32] = np.where(finite[:, None], number * step + 0.0, np.nan)
    return q, e, back


def act8_buffer(x):
    """The buffer of a float64 matrix, as the library lays it out."""
    q, e, _ = act8_encode(x)
    at = -(-q.size // 256) * 256
    buffer = np.zeros(at + e.size, dtype=np.uint8)
    buffer[:q.size] = q.reshape(-1).view(np.uint8)
    buffer[at:] = e.reshape(-1)
    return buffer


def act8_split(buffer, rows, cols):
    """(numbers, exponents) of a buffer."""
    groups = -(-cols // 32)
    n = rows * groups * 32
    at = -(-n // 256) * 256
    return buffer[:n].view(np.int8).reshape(rows, groups * 32), buffer[at:at + rows * groups].reshape(rows, groups)


# ---------------------------------------------------------------- GELU
ROOT = np.sqrt(2.0 / np.pi)


def _phi(x):
    # (not 1 + erf, whose sum loses the lower tail)
    return 0.5 * torch.special.erfc(torch.from_numpy(-np.asarray(x, dtype=np.float64) / np.sqrt(2.0))).numpy()


def gelu(x, tanh):
    if tanh:
        with np.errstate(over="ignore"):
            return x / (1.0 + np.exp(-2.0 * ROOT * (x + 0.044715 * x ** 3)))
    return x * _phi(x)


def gelu_slope(x, tanh):
    if tanh:
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-2.0 * ROOT * (x + 0.044715 * x ** 3)))
        return s + x * s * (1.0 - s) * 2.0 * ROOT * (1.0 + 3 * 0.044715 * x ** 2)
    return _phi(x) + x * np.exp(-x * x / 2.0) / np.sqrt(2.0 * np.pi)


def gelu_bound(x, y, tanh, dtype):
    """Both forms are a product of x and a tail with relative errors: of the polynomial (eight steps, two units each), reciprocal, exponential and
    products, 30 units in all; the tanh form's exponent w has three roundings of its own, which the exponential turns into |w| ln 2 units each."""
    w = np.abs(2.0 * np.log2(np.e) * ROOT * (x + 0.044715 * x ** 3)) if tanh else 0.0
    return np.abs(y) * ((30.0 + 3.0 * np.log(2.0) * w) * U + HALF_ULP[dtype]) + SMALLEST[dtype] + np.abs(x) * 2.0 ** -125


def gelu_slope_bound(dy, out, dtype):
    """Slopes are sums of terms of at most 1.2 that carry the same relative errors (|w| times a term stays below 2): 40 units of dy."""
    return np.abs(dy) * 40 * U + np.abs(out) * HALF_ULP[dtype] + SMALLEST[dtype]


# ---------------------------------------------------------------- layer norm
def layernorm(x, weight, bias, eps):
    mean = x.mean(axis=1)
    var = ((x - mean[:, None]) ** 2).mean(axis=1)
    rstd = 1.0 / np.sqrt(var + eps)
    h = (x - mean[:, None]) * rstd[:, None]
    return h * weight + bias, mean, rstd, h


DEPTH = 64  # additions one behind the other in a sum over a row: 32 in a lane, 6 between lanes, 16 between wavefronts, and some


def layernorm_bounds(x, weight, bias, mean, rstd, h, y, dtype):
    """(of y, mean, rstd, h): a sum's error is DEPTH units of the magnitudes' average; the centred squares carry it once more."""
    d_mean = DEPTH * U * np.abs(x).mean(axis=1) + 2.0 ** -140
    r_rstd = (DEPTH + 6) * U + (d_mean * rstd) ** 2 + d_mean * rstd * np.abs(h).mean(axis=1) * 2
    d_h = (d_mean * rstd)[:, None] + U * np.abs(x - mean[:, None]) * rstd[:, None] + np.abs(h) * (r_rstd[:, None] + 3 * U)
    d_y = np.abs(weight) * d_h + 3 * U * (np.abs(h * weight) + np.abs(bias)) + HALF_ULP[dtype] * (np.abs(y) + np.abs(weight) * d_h) + SMALLEST[dtype]
    return d_y, d_mean, r_rstd * rstd, d_h


def layernorm_backward(dy, h, rstd, weight, dsum):
    g = dy * weight
    dx = rstd[:, None] * (g - g.mean(axis=1)[:, None] - h * (g * h).mean(axis=1)[:, None])
    return dx + dsum, (dy * h).sum(axis=0), dy.sum(axis=0)


def layernorm_backward_bounds(dy, h, d_h, rstd, weight, dsum, dx, dtype):
    """(of dx, dweight, dbias); d_h: what h itself may be off by (nothing where it was kept in 8 bits)."""
    rows, cols = dy.shape
    g = np.abs(dy * weight)
    level, along = g.mean(axis=1)[:, None], (g * np.abs(h)).mean(axis=1)[:, None]
    d = (DEPTH + 6) * U * (level + np.abs(h) * along) + 6 * U * g + d_h * along + np.abs(h) * (g * d_h).mean(axis=1)[:, None]
    d_dx = rstd[:, None] * d + 2 * U * np.abs(dsum) + HALF_ULP[dtype] * np.abs(dx) + U * np.abs(dx) + SMALLEST[dtype]
    depth = rows / 256 + 64  # additions one behind the other: a wavefront's rows, a workgroup's four, the parts
    return d_dx, depth * U * (np.abs(dy) * np.abs(h)).sum(axis=0) + (np.abs(dy) * d_h).sum(axis=0) + 1e-40, depth * U * np.abs(dy).sum(axis=0) + 1e-40


# ---------------------------------------------------------------- weight gradient
def weight_grad(dy, x, weight=None, bias=None):
    if weight is not None:
        x = x * weight
    if bias is not None:
        x = x + bias
    return dy.T @ x, dy.sum(axis=0)


def weight_grad_bounds(dy, x, weight=None, bias=None):
    """Products are exact; each of the additions loses at most two units of what has been summed so far, and they do not all point one way."""
    steps = 2 * U * (8 + 2 * np.sqrt(dy.shape[0]))
    w = 1.0 if weight is None else np.abs(weight)
    total = np.abs(dy).sum(axis=0)
    d = (np.abs(dy).T @ np.abs(x)) * w * steps
    if bias is not None:
        d = d + np.outer(total, np.abs(bias)) * steps
    return d + 1e-40, total * steps + 1e-40
