"""Plain numpy oracle, in float64, of the operators around a large layer (test
infrastructure only): tensors in 8-bit integers with a scale for each row and their
grouped product, layer norm and its gradients, gradients clipped by their norm.
Written from the definitions in include/lsgd.h.
"""
import numpy as np


def up(n, m):
    return -(-n // m) * m


def quantise_rows(X):
    """(q, scale) of X [G][M][N] (float64 holding fp32 values): integers in the padded
    layout, and the scales as fp32 numbers."""
    G, M, N = X.shape
    q, s = np.zeros((G, M, up(N, 128))), np.empty((G, M))
    for g, m in np.ndindex(G, M):
        row = X[g, m]
        if not np.isfinite(row).all():
            s[g, m] = np.nan
            continue
        top = np.abs(row).max()
        s[g, m] = 1.0 if top == 0 else float(np.float32(max(top / 127.0, 2.0 ** -126)))
        # (the quotient of two fp32 numbers is no nearer to the middle of two integers than
        # 2^-48 of it, unless it lies there)
        q[g, m, :N] = np.rint(row / s[g, m])
    return q, s


def product(qa, sa, qb, sb, bias=None):
    """C[g] = A[g] B[g]^T + bias[g], the integers' sums exact."""
    C = (qa @ qb.transpose(0, 2, 1)) * sa[:, :, None] * sb[:, None, :]
    return C if bias is None else C + bias[:, None, :]


def layer_norm(X, w, b, eps):
    """(y, mean, rstd) of X [G][M][N], w and b [G][N]."""
    mean = X.mean(2, keepdims=True)
    d = X - mean
    rstd = 1.0 / np.sqrt((d * d).mean(2, keepdims=True) + float(np.float32(eps)))
    return d * rstd * w[:, None] + b[:, None], mean[..., 0], rstd[..., 0]


def layer_norm_backward(dY, X, mean, rstd, w):
    """(dx, dw, db)."""
    rstd = rstd[..., None]
    n = (X - mean[..., None]) * rstd
    e = dY * w[:, None]
    dx = rstd * (e - e.mean(2, keepdims=True) - n * (e * n).mean(2, keepdims=True))
    return dx, (dY * n).sum(1), dY.sum(1)


def clip(tensors, bound):
    """(norms [K], clipped tensors) of tensors [K][...]."""
    K = tensors[0].shape[0]
    norm = np.sqrt(sum((t.reshape(K, -1) ** 2).sum(1) for t in tensors))
    with np.errstate(divide="ignore", invalid="ignore"):
        f = np.where((norm > bound) & np.isfinite(norm), bound / norm, 1.0)
    out = []
    for t in tensors:
        by = f.reshape((K,) + (1,) * (t.ndim - 1))
        out.append(np.where(by == 1.0, t, t * by))
    return norm, out
