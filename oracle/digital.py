"""Plain float64 definitions (test infrastructure) of the digital operators beside the crossbar layers: group normalisation with an
activation, low-rank adapters, global gradient norm, clipping and the clipped step."""
import numpy as np


def act(z, kind):
    return z if kind == "none" else np.where(z > 0, z, 0.0) if kind == "relu" else z / (1.0 + np.exp(-z))


def act_slope(z, kind):
    if kind == "none":
        return np.ones_like(z)
    if kind == "relu":
        return (z > 0).astype(np.float64)
    s = 1.0 / (1.0 + np.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _spread(stat, x, groups):
    """[batch][groups] to the shape of x."""
    b, c = x.shape[0], x.shape[-1]
    return np.repeat(stat, c // groups, axis=1).reshape((b,) + (1,) * (x.ndim - 2) + (c,))


def gn_stats(x, groups, eps):
    b, c = x.shape[0], x.shape[-1]
    rows = x.astype(np.float64).reshape(b, -1, groups, c // groups)
    mean = rows.mean((1, 3))
    var = ((rows - mean[:, None, :, None]) ** 2).mean((1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def gn_z(x, gamma, beta, mean, invstd, skip=None):
    """(xhat, z) from given statistics."""
    groups = mean.shape[1]
    xhat = (x.astype(np.float64) - _spread(mean, x, groups)) * _spread(invstd, x, groups)
    z = xhat * gamma.astype(np.float64) + beta.astype(np.float64)
    return xhat, z if skip is None else z + skip


def gn_bwd(x, dy, gamma, beta, mean, invstd, kind, skip=None, slope_dy=None):
    """(dx, dgamma, dbeta, dskip); slope_dy: the error behind the activation, where it is known already."""
    b, c, groups = x.shape[0], x.shape[-1], mean.shape[1]
    xhat, z = gn_z(x, gamma, beta, mean, invstd, skip)
    g = act_slope(z, kind) * dy if slope_dy is None else slope_dy
    axes = tuple(range(x.ndim - 1))
    grouped = lambda t: t.reshape(b, -1, groups, c // groups).mean((1, 3))
    gg = g * gamma
    dx = _spread(invstd, x, groups) * (gg - _spread(grouped(gg), x, groups) - xhat * _spread(grouped(gg * xhat), x, groups))
    return dx, (g * xhat).sum(axes), g.sum(axes), g


def adapter_fwd(rows, base, X, A, B, scale):
    """(Y, T)."""
    base, X, A, B, scale = (np.asarray(t, dtype=np.float64) for t in (base, X, A, B, scale))
    Y, T = base.copy(), np.zeros((X.shape[0], A.shape[1]))
    for m, a in enumerate(rows):
        if 0 <= a < A.shape[0]:
            T[m] = A[a] @ X[m]
            Y[m] += scale[a] * (T[m] @ B[a])
    return Y, T


def adapter_bwd(rows, base, dY, X, T, A, B, scale):
    """(dX, dA, dB, dT)."""
    base, dY, X, T, A, B, scale = (np.asarray(t, dtype=np.float64) for t in (base, dY, X, T, A, B, scale))
    dX, dA, dB, dT = base.copy(), np.zeros_like(A), np.zeros_like(B), np.zeros_like(T)
    for m, a in enumerate(rows):
        if 0 <= a < A.shape[0]:
            dT[m] = scale[a] * (B[a] @ dY[m])
            dX[m] += dT[m] @ A[a]
            dA[a] += np.outer(dT[m], X[m])
            dB[a] += scale[a] * np.outer(T[m], dY[m])
    return dX, dA, dB, dT


def grad_norm(grads):
    return float(np.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads)))


def clip_factor(norm, max_norm):
    """None: nothing moves."""
    return None if not np.isfinite(norm) else max_norm / norm if norm > max_norm else 1.0
