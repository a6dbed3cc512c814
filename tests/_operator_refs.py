"""Group norm with an activation and the orthogonalised update direction from their definitions, in 64 bits."""
import numpy as np

A, B, C = 3.4445, -4.7750, 2.0315


def act(z, kind):
    return np.maximum(z, 0) if kind == "relu" else z / (1 + np.exp(-z)) if kind == "silu" else z


def act_slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def gn_forward(x, gamma, beta, groups, eps, kind):
    """x [G][B][P][C], gamma and beta [G][C]: y, mean and rstd [G][B][groups], z before the activation."""
    G, Bn, P, Ch = x.shape
    v = x.astype(np.float64).reshape(G, Bn, P, groups, Ch // groups)
    mean = v.mean((2, 4), keepdims=True)
    rstd = 1 / np.sqrt(((v - mean) ** 2).mean((2, 4), keepdims=True) + eps)
    z = ((v - mean) * rstd).reshape(x.shape) * gamma[:, None, None] + beta[:, None, None]
    return act(z, kind), mean[:, :, 0, :, 0], rstd[:, :, 0, :, 0], z


def gn_backward(x, dy, gamma, beta, mean, rstd, groups, kind, positive=None):
    """dx, dgamma, dbeta; `positive` replaces ReLU's z > 0 (the stored output's sign)."""
    G, Bn, P, Ch = x.shape
    shape = (G, Bn, P, groups, Ch // groups)
    m, r = mean.astype(np.float64)[:, :, None, :, None], rstd.astype(np.float64)[:, :, None, :, None]
    xh = (x.astype(np.float64).reshape(shape) - m) * r
    z = xh.reshape(x.shape) * gamma[:, None, None] + beta[:, None, None]
    slope = positive.astype(np.float64) if kind == "relu" and positive is not None else act_slope(z, kind)
    dz = dy.astype(np.float64) * slope
    t = (dz * gamma[:, None, None]).reshape(shape)
    m1, m2 = t.mean((2, 4), keepdims=True), (t * xh).mean((2, 4), keepdims=True)
    dx = (r * (t - m1 - xh * m2)).reshape(x.shape)
    return dx, (dz * xh.reshape(x.shape)).sum((1, 2)), dz.sum((1, 2)), dz, xh.reshape(x.shape)


def direction(x, steps):
    """`steps` quintic steps on x / ||x||_F for each matrix of x [G][rows][cols]."""
    out = np.zeros(x.shape)
    for k, m in enumerate(x.astype(np.float64)):
        n = np.linalg.norm(m)
        X = m / n if n > 0 else m
        for _ in range(steps):
            M = X @ X.T if X.shape[0] <= X.shape[1] else X.T @ X
            P = B * M + C * M @ M
            X = A * X + (P @ X if X.shape[0] <= X.shape[1] else X @ P)
        out[k] = X
    return out
