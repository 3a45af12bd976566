"""Operators of a training step in 64 bits, from their definitions: the 8-bit copy of an activation, GroupNorm with an
activation and FiLM vectors, its gradients, the weight gradient of a projection or convolution (the backward side of
`nets.group_norm`, `nets.mish`, `nets.conv1d_k5`).

Pins: the gradients against central differences of the forward functions, the copy against its definition on chosen values."""
import numpy as np


# ------------------------------------------------------------------------------------------- 8-bit copies
def pack(x):
    """(q int8, scale uint8) of x [rows, C]: blocks of 32 channels, q 2^(scale - 127), the smallest scale in 1 .. 248 for which
    no rounded magnitude exceeds 127; 255 for a block with a value that is not finite."""
    x = np.asarray(x, dtype=np.float64)
    rows, C = x.shape
    q = np.zeros((rows, C), dtype=np.int8)
    scale = np.zeros((rows, -(-C // 32)), dtype=np.uint8)
    for r in range(rows):
        for j in range(scale.shape[1]):
            v = x[r, 32 * j:32 * j + 32]
            if not np.isfinite(v).all():
                scale[r, j] = 255
                continue
            lo, hi = 1, 248                                # the largest rounded magnitude falls with the scale
            while lo < hi:
                mid = (lo + hi) // 2
                if np.rint(np.max(np.abs(v)) * 2.0 ** (127 - mid)) <= 127:
                    hi = mid
                else:
                    lo = mid + 1
            scale[r, j] = lo
            q[r, 32 * j:32 * j + 32] = np.clip(np.rint(v * 2.0 ** (127 - lo)), -127, 127)
    return q, scale


def unpack(q, scale):
    step = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return q.astype(np.float64) * np.repeat(step, 32, axis=1)[:, :q.shape[1]]


# ------------------------------------------------------------------------------------------- activations
def _logistic(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


def act(name, z):
    """(act(z), act'(z))"""
    if name == "none":
        return z, np.ones_like(z)
    s = _logistic(z)
    if name == "silu":
        return z * s, s + z * s * (1.0 - s)
    if name == "gelu":                                     # tanh form
        k = np.sqrt(2.0 / np.pi)
        t = np.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * z * z)
    t = np.tanh(np.log1p(np.exp(-np.abs(z))) + np.maximum(z, 0.0))
    return z * t, t + z * (1.0 - t * t) * s


# ------------------------------------------------------------------------------------------- GroupNorm
def group_norm(x, gamma, beta, groups, name="mish", film=None, eps=1e-5):
    """(y, mean, rstd) of x [N, L, C]; film [N, 2C]: scale, bias."""
    N, L, C = x.shape
    v = x.reshape(N, L, groups, C // groups)
    mean = v.mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3)) + eps)
    h = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(N, L, C)
    a = act(name, h * gamma + beta)[0]
    if film is not None:
        a = film[:, None, :C] * a + film[:, None, C:]
    return a, mean, rstd


def group_norm_grad(dy, x, gamma, beta, groups, mean, rstd, name="mish", film=None):
    """(dx, dgamma, dbeta, dfilm) for given statistics: dx takes them as functions of x."""
    N, L, C = x.shape
    w = C // groups
    wide = lambda t: np.repeat(t, w, axis=1)[:, None, :]  # noqa: E731
    h = (x - wide(mean)) * wide(rstd)
    a, da = act(name, h * gamma + beta)
    dz = dy * da if film is None else dy * film[:, None, :C] * da
    dfilm = np.concatenate([(dy * a).sum(1), dy.sum(1)], axis=1)
    dh = dz * gamma
    of_group = lambda t: wide(t.reshape(N, L, groups, w).mean(axis=(1, 3)))  # noqa: E731
    dx = wide(rstd) * (dh - of_group(dh) - h * of_group(dh * h))
    return dx, (dz * h).sum((0, 1)), dz.sum((0, 1)), dfilm


# ------------------------------------------------------------------------------------------- weight gradient
def weight_grad(x, dy, taps, length):
    """(dW [taps, K, O], db [O]) of x [rows, K], dy [rows, O]; sequences of `length` rows, zeros beyond their ends."""
    K = x.shape[1]
    xs = x.reshape(-1, length, K)
    side = np.zeros((xs.shape[0], taps // 2, K))
    xp = np.concatenate([side, xs, side], axis=1)
    return np.stack([xp[:, j:j + length].reshape(-1, K).T @ dy for j in range(taps)]), dy.sum(0)
