"""Low-rank adapters beside a shared projection in float64, sequence by sequence from the definition: test infrastructure only.

x [T][B][K], dy [T][B][N], W [N][K], b [N], A [count][r][K], Bm [count][N][r], ids [B]; an id of NONE has no adapter, any other outside [0, count) gives NaN."""
import numpy as np

NONE = -1


def forward(W, b, A, Bm, ids, x, scale):
    """y [T][B][N] and t [T][B][r]."""
    y = np.einsum("tbk,nk->tbn", x, W) + (0.0 if b is None else b)
    t = np.zeros((*x.shape[:2], A.shape[1]))
    for s, a in enumerate(ids):
        if 0 <= a < len(A):
            t[:, s] = x[:, s] @ A[a].T
            y[:, s] += scale * t[:, s] @ Bm[a].T
        elif a != NONE:
            y[:, s] = t[:, s] = np.nan
    return y, t


def backward(W, A, Bm, ids, x, t, dy, scale):
    """dx, dA, dB, dW, db."""
    dx = np.einsum("tbn,nk->tbk", dy, W)
    dA, dB = np.zeros(A.shape), np.zeros(Bm.shape)
    for s, a in enumerate(ids):
        if 0 <= a < len(A):
            q = dy[:, s] @ Bm[a]
            dx[:, s] += scale * q @ A[a]
            dA[a] += scale * q.T @ x[:, s]
            dB[a] += scale * dy[:, s].T @ t[:, s]
        elif a != NONE:
            dx[:, s] = np.nan
    return dx, dA, dB, np.einsum("tbn,tbk->nk", dy, x), dy.sum((0, 1))
