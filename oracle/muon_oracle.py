"""Plain fp64 definitions of the Newton-Schulz orthogonalisation and the Muon
step (numpy, CPU): test infrastructure only, shares no code with the GPU
path."""
import numpy as np

COEFS = (3.4445, -4.7750, 2.0315)


def orthogonalize(x, steps=5, coefs=COEFS, eps=1e-7):
    x = np.asarray(x, np.float64)
    if x.shape[-2] > x.shape[-1]:
        return np.swapaxes(orthogonalize(np.swapaxes(x, -1, -2), steps, coefs, eps), -1, -2)
    a, b, c = coefs
    x = x / np.maximum(np.sqrt((x * x).sum((-1, -2), keepdims=True)), eps)
    for _ in range(steps):
        g = x @ np.swapaxes(x, -1, -2)
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


def singular_map(s, steps=5, coefs=COEFS):
    """What the steps make of singular values s."""
    a, b, c = coefs
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


def muon_step(param, grad, momentum, swa, *, lr, momentum_decay, nesterov, weight_decay, swa_decay, update_scale=1.0,
              grad_scale=1.0, steps=5, coefs=COEFS, eps=1e-7):
    """(param, momentum, swa) of one matrix after the step."""
    p, g, m = (np.asarray(v, np.float64) for v in (param, grad, momentum))
    g = g * grad_scale
    m = momentum_decay * m + (1 - momentum_decay) * g
    u = (1 - momentum_decay) * g + momentum_decay * m if nesterov else m
    p = (1 - lr * weight_decay) * p - lr * update_scale * orthogonalize(u, steps, coefs, eps)
    w = None if swa is None else swa_decay * np.asarray(swa, np.float64) + (1 - swa_decay) * p
    return p, m, w
