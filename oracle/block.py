"""What stands around a layer of experts in 64 bits, from the definitions (numpy; test infrastructure only)."""
import numpy as np


def layernorm(x, gamma=None, beta=None, eps=1e-5):
    """y, mean, rstd."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    c = x - mean[:, None]
    with np.errstate(divide="ignore"):
        rstd = 1 / np.sqrt((c * c).mean(1) + eps)
    with np.errstate(invalid="ignore"):
        y = c * rstd[:, None]
    return y * (1 if gamma is None else gamma) + (0 if beta is None else beta), mean, rstd


def layernorm_bwd(dy, x, mean, rstd, gamma=None):
    """dx, dgamma, dbeta from the forward pass's mean and rstd."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    mean, rstd = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    h, g = (x - mean) * rstd, dy * (1 if gamma is None else np.asarray(gamma, np.float64))
    dx = rstd * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def probabilities(logits):
    """softmax of each row, zeros where all are masked, and which rows are not."""
    x = np.asarray(logits, np.float64)
    there = ~(x == -np.inf).all(1) if x.shape[1] else np.zeros(len(x), bool)
    p = np.zeros_like(x)
    with np.errstate(invalid="ignore"):
        z = np.exp(x[there] - x[there].max(1, keepdims=True))
        p[there] = z / z.sum(1, keepdims=True)
    return p, there


def balance(logits, ids):
    """loss, counts, shares, rows."""
    E = np.shape(logits)[1]
    p, there = probabilities(logits)
    counts = np.array([(np.asarray(ids) == e).sum() for e in range(E)], np.int64)
    rows = int(there.sum())
    shares = p.sum(0) / rows if rows else np.zeros(E)
    f = counts / counts.sum() if counts.sum() else np.zeros(E)
    return E * np.dot(f, shares), counts, shares, rows


def balance_bwd(logits, counts, rows, dloss=1.0):
    E = np.shape(logits)[1]
    p, _ = probabilities(logits)
    f = np.asarray(counts, np.float64) / counts.sum() if np.sum(counts) else np.zeros(E)
    return dloss * E / max(rows, 1) * p * (f - (p * f).sum(1, keepdims=True))


def total_norm(tensors):
    return np.sqrt(sum((np.asarray(t, np.float64) ** 2).sum() for t in tensors))


def clipped(tensors, max_norm):
    norm = total_norm(tensors)
    factor = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, [np.asarray(t, np.float64) * factor for t in tensors]


MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx4_codes(x):
    """Codes [...][KB * 32] and scale bytes [...][KB], value by value: the nearest of the eight magnitudes, of two the one with the even code."""
    x = np.asarray(x, np.float64)
    K = x.shape[-1]
    x = np.concatenate([x, np.zeros((*x.shape[:-1], -K % 128))], -1)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(-1)
    broken = ~np.isfinite(top)
    with np.errstate(divide="ignore", invalid="ignore"):
        exponent = np.where(broken, 0, np.frexp(top)[1] - 1)                    # floor(log2): 1/2 <= mantissa < 1
    b = np.where(top > 0, np.maximum(exponent - 2, -127), -127) + 127
    with np.errstate(invalid="ignore"):
        r = np.abs(blocks) / np.exp2(b - 127.0)[..., None]
        away = np.abs(r[..., None] - MAGNITUDES)
    # of two that are equally far the one with the even code
    code = np.argmin(np.where(np.arange(8) % 2 == 0, away, np.nextafter(away, np.inf)), -1) + 8 * np.signbit(blocks)
    code = np.where(broken[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(broken, 255, b).astype(np.uint8)


def mx4_pack(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def mx4_values(q, scales, K=None):
    """The values that packed codes and scales stand for."""
    codes = np.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], -1)
    v = np.where(codes & 8, -1.0, 1.0) * MAGNITUDES[codes & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v * np.repeat(s, 32, -1))[..., :K]
