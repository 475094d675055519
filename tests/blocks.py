"""Plain forms in 64 bits of the operators on blocks [n][B] (layer norm, activations in 8 bits) and of a net's backward pass from
kept activations, for the tests: numpy, and nothing of the library's."""
import numpy as np

HALF = 2.0 ** -24  # what a rounding to fp32 moves a value by, relative to it
TINY = 2.0 ** -149


# ---- activations in 8 bits ---------------------------------------------------------------------------------------

def bf16_up(v):
    """The smallest floats of 8 significant bits (of fp32's exponents, subnormal ones among them) that are >= v >= 0."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(v)
    unit = np.ldexp(1.0, np.maximum(e - 8, -133))
    return np.ceil(v / unit) * unit


def pack8(x, cap):
    """(codes, scales as 16 bits, values) of a block.  The cap is an fp32 number."""
    cap = float(np.float32(cap))
    flat = np.asarray(x, np.float32).ravel()
    groups = -(-flat.size // 128)
    v = np.zeros(groups * 128, np.float64)
    v[:flat.size] = flat
    v = v.reshape(groups, 128)
    with np.errstate(invalid="ignore"):
        live = (v > 0) & (v < cap) if cap > 0 else np.isfinite(v)
    size = np.where(live, np.abs(v), 0.0)
    most = 253.0 if cap > 0 else 127.0
    t = bf16_up(size.max(axis=1, keepdims=True) / most)
    t = np.where(t * most < size.max(axis=1, keepdims=True), bf16_up(np.nextafter(t, np.inf)), t)  # the division was rounded down
    quotient = np.divide(size, t, out=np.zeros_like(size), where=t > 0)
    count = np.floor(quotient + 0.5)
    if cap > 0:
        below = float(np.nextafter(np.float32(cap), np.float32(0)))
        code = np.where(live, np.maximum(count, 1), 0)
        value = np.where(live, np.minimum(code * t, below), 0.0)
        with np.errstate(invalid="ignore"):
            full, nan = v >= cap, np.isnan(v)
        code, value = np.where(full, 255, code), np.where(full, cap, value)
        code, value = np.where(nan, 254, code), np.where(nan, np.nan, value)
    else:
        signed = np.where(v < 0, -count, count)
        code = np.where(live, signed, -128) % 256
        value = np.where(live, signed * t, np.nan)
    scales = (t[:, 0].astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return code.astype(np.uint8).ravel(), scales, value.ravel()[:flat.size].reshape(np.shape(x))


def packed_bytes(n, b):
    return -(-130 * -(-n * b // 128) // 256) * 256


def split_packed(data, n, b):
    """(codes, scales) of a packed block's bytes."""
    groups = -(-n * b // 128)
    return data[:128 * groups], data[128 * groups:130 * groups].view(np.uint16)


# ---- layer norm --------------------------------------------------------------------------------------------------

def norm(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    n, b = x.shape
    gamma = np.ones(n) if gamma is None else np.asarray(gamma, np.float64)
    beta = np.zeros(n) if beta is None else np.asarray(beta, np.float64)
    mean = x[0] + (x - x[0]).mean(axis=0, dtype=np.longdouble).astype(np.float64)
    var = ((x - mean) ** 2).mean(axis=0, dtype=np.longdouble).astype(np.float64)
    rstd = 1.0 / np.sqrt(var + eps)
    return (x - mean) * rstd * gamma[:, None] + beta[:, None], np.stack([mean, rstd])


def norm_backward(dy, x, stats, gamma):
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    n, b = x.shape
    gamma = np.ones(n) if gamma is None else np.asarray(gamma, np.float64)
    mean, rstd = stats
    h = (x - mean) * rstd
    d = gamma[:, None] * dy
    p, q, dgamma, dbeta = (v.astype(np.float64) for v in (d.mean(axis=0, dtype=np.longdouble), (d * h).mean(axis=0, dtype=np.longdouble),
                                                          (dy * h).sum(axis=1, dtype=np.longdouble), dy.sum(axis=1, dtype=np.longdouble)))
    return rstd * (d - p - h * q), dgamma, dbeta


# ---- a net's backward pass ---------------------------------------------------------------------------------------

def dense(layer):
    w = np.zeros((layer.n_out, layer.n_in))
    rows = np.repeat(np.arange(layer.n_out), np.diff(layer.row_ptr))
    w[rows, layer.col_idx] = layer.values
    return w, rows


def forward(layers, x, cap, activation):
    """X_0 .. X_L in 64 bits."""
    xs = [np.asarray(x, np.float64)]
    for y in layers:
        z = dense(y)[0] @ xs[-1] + (0.0 if y.bias is None else np.asarray(y.bias, np.float64)[:, None])
        xs.append(1.0 / (1.0 + np.exp(-z)) if activation == "sigmoid" else np.clip(z, 0.0, cap))
    return xs


def backward(layers, xs, dloss, cap, activation):
    """(gradients of entries and biases layer by layer, dX_0), each with a bound of what fp32 storage of the Deltas may move it by.

    A Delta is rounded once where it is stored: relative HALF of itself, and of what the Deltas above it were moved by; sums in 64 bits
    add nothing that matters; a gradient may be the rounded sum of two rounded halves (two more).  So a value that has gone through k
    roundings is off by at most k HALF (to first order; 1.01 covers the rest) of the same sums taken over absolute values."""
    back, size, stores, out = np.asarray(dloss, np.float64), np.abs(np.asarray(dloss, np.float64)), 0, []
    for y, below, above in zip(layers[::-1], xs[-2::-1], xs[:0:-1]):
        slope = above * (1 - above) if activation == "sigmoid" else ((above > 0) & (above < cap)).astype(np.float64)
        delta, size = back * slope, size * slope
        stores += 1
        w, rows = dense(y)
        g, bound = (delta @ below.T)[rows, y.col_idx], (size @ np.abs(below).T)[rows, y.col_idx]
        out.insert(0, [(g, 1.01 * (stores + 2) * HALF * bound + TINY), (delta.sum(1), 1.01 * (stores + 2) * HALF * size.sum(1) + TINY)])
        back, size = w.T @ delta, np.abs(w).T @ size
    return out, (back, 1.01 * (stores + 1) * HALF * size + TINY)


def close(got, want, bound, what=""):
    err = np.abs(np.asarray(got, np.float64) - want)
    assert np.all(err <= bound), f"{what}: off by {np.max(err - bound):.3e} more than may be, at {np.argmax(err - bound)}"
