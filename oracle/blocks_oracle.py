"""Plain numpy oracle of the large-layer operators, in float64 (test
infrastructure only): tensors in 8-bit blocks, their grouped product, and the
orthogonalised momentum update. Written from the definitions in include/lsgd.h.
"""
import numpy as np

# largest value, mantissa bits, smallest normal exponent
FORMATS = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}


def up(n, m):
    return -(-n // m) * m


def round_format(x, fmt):
    """x (float64) to the nearest value of the format, ties to even; no
    overflow. Infinities: kept for e5m2, NaN for e4m3."""
    _, bits, low = FORMATS[fmt]
    with np.errstate(invalid="ignore", over="ignore"):
        _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
        step = np.ldexp(1.0, np.maximum(e - 1, low) - bits)
        q = np.where(np.isfinite(x), np.rint(x / step) * step, x)
    if fmt == "e4m3":
        q = np.where(np.isinf(q), np.nan, q)
    return q


def quantise(X, fmt):
    """(q, scale) of X [G][M][N]: float64 values in the padded layout, and the
    scales 2^e (1 in the padding)."""
    top = FORMATS[fmt][0]
    G, M, N = X.shape
    nb = up(N, 128) // 128
    x = np.zeros((G, M, nb * 128))
    x[:, :, :N] = X
    x = x.reshape(G, M, nb, 128)
    amax = np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=3)
    e = np.zeros(amax.shape, int)
    for at in np.ndindex(amax.shape):
        if amax[at] > 0:
            k = -127
            while amax[at] > np.ldexp(top, k):
                k += 1
            e[at] = min(k, 127)
    q = round_format(np.ldexp(x, -e[..., None]), fmt).reshape(G, M, nb * 128)
    s = np.ones((G, M, up(nb, 4)))
    s[:, :, :nb] = np.ldexp(1.0, e)
    return q, s


def values(q, s):
    """What blocks stand for, padding included."""
    return q * np.repeat(s[:, :, :q.shape[2] // 128], 128, axis=2)


def newton_schulz(X, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    a, b, c = (float(np.float32(v)) for v in coefficients)
    out = np.empty(X.shape)
    for g in range(X.shape[0]):
        x = X[g].astype(np.float64)
        flip = x.shape[0] > x.shape[1]
        x = x.T if flip else x
        x = x / (np.sqrt((x * x).sum()) + float(np.float32(eps)))
        for _ in range(steps):
            A = x @ x.T
            x = a * x + (b * A + c * (A @ A)) @ x
        out[g] = x.T if flip else x
    return out


def _pieces(x, scale, n):
    """x in n fp16 pieces of x * scale, as float32."""
    x = (x * np.float32(scale)).astype(np.float32)
    with np.errstate(over="ignore"):
        hi = x.astype(np.float16).astype(np.float32)
        lo = (x - hi).astype(np.float16).astype(np.float32)
    return [hi, lo][:n]


def newton_schulz_rounded(X, n, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    """The same with the roundings of a computation in n fp16 pieces per
    operand (X itself in two) and fp32 sums: how far such a computation lands from
    the exact one says what a kernel of that precision may be off by."""
    a, b, c = (np.float32(v) for v in coefficients)
    f = np.float32

    def product(p, q):
        r = p[0] @ q[0]
        return r if n == 1 else r + (p[0] @ q[1] + p[1] @ q[0])

    out = np.empty(X.shape)
    for g in range(X.shape[0]):
        x = X[g].astype(np.float64)
        flip = x.shape[0] > x.shape[1]
        x = x.T if flip else x
        x = (x / (np.sqrt((x * x).sum()) + float(f(eps)))).astype(f)
        S = f(2.0 ** np.floor(np.log2(np.sqrt(x.size))))
        Sa, Sb = f(2.0 ** 15), f(2.0 ** 14)
        X2 = _pieces(x, S, 2)
        for _ in range(steps):
            A = product(X2, [p.T for p in X2]) * (Sa / S / S)
            Ap = _pieces(A, 1.0, n)
            B = (b * sum(Ap) + c * (product(Ap, Ap) / Sa)) / Sa
            y = product(_pieces(B, Sb, n), X2) / Sb + a * sum(X2)
            X2 = _pieces(y, 1.0, 2)
        y = y.astype(np.float64) / S
        out[g] = y.T if flip else y
    return out


def orthogonal_update(W, U, G, lr, momentum, weight_decay, nesterov, scale, **kw):
    f = lambda v: float(np.float32(v))  # noqa: E731  (arguments arrive as fp32)
    U = f(momentum) * U + G
    d = G + f(momentum) * U if nesterov else U
    O = newton_schulz(d, **kw)
    return W - f(lr) * (f(weight_decay) * W + f(scale) * O), U, O
