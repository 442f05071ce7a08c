"""The orthogonalised update in float64, from its definition: test infrastructure only.

Matrices are [R][C]; X <- G / |G|, then five times X <- a X + b S X + c S^2 X with S = X X^T (of a matrix with more rows than columns:
the same of its transpose)."""
import numpy as np

A, B, C = 3.4445, -4.7750, 2.0315
STEPS = 5


def orthogonalize(G):
    G = np.asarray(G, dtype=np.float64)
    if G.shape[0] > G.shape[1]:
        return orthogonalize(G.T).T
    size = np.sqrt((G * G).sum())
    if size == 0.0:
        return np.zeros_like(G)
    X = G / size
    for _ in range(STEPS):
        S = X @ X.T
        X = A * X + B * (S @ X) + C * (S @ (S @ X))
    return X


def matrices_step(theta, grad, velocity, lr, momentum, weight_decay, nesterov):
    """theta' and velocity' of a batch [count][R][C]."""
    v = momentum * velocity + grad
    d = grad + momentum * v if nesterov else v
    R, C = theta.shape[1:]
    O = np.stack([orthogonalize(m) for m in d])
    return (1 - lr * weight_decay) * theta - lr * np.sqrt(max(1.0, R / C)) * O, v


def matrices(layout, gates, softmax):
    """(offset, rows, cols) of what is orthogonalised, from (name, offset, shape) of every tensor of the flat vector."""
    out = []
    for name, at, shape in layout:
        if name.startswith(("Wx", "Uh")) or name == "Wp" or (name == "Ws" and softmax):
            parts = 4 if gates and name.startswith(("Wx", "Uh")) else 1
            R, C = shape[0] // parts, shape[1]
            out += [(at + k * R * C, R, C) for k in range(parts)]
    return out


def step(layout, theta, grad, velocity, lr, lr_rest, momentum, weight_decay, nesterov, gates, softmax):
    """theta' and velocity' of a model's flat vector."""
    v = momentum * velocity + grad
    d = grad + momentum * v if nesterov else v
    new = theta - lr_rest * d
    for at, R, C in matrices(layout, gates, softmax):
        part = slice(at, at + R * C)
        X = orthogonalize(d[part].reshape(R, C)).reshape(-1)
        new[part] = (1 - lr * weight_decay) * theta[part] - lr * np.sqrt(max(1.0, R / C)) * X
    return new, v
