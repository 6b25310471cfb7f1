"""Plain fp64 definition of the gated attention of queries to states of another
length, forward and backward (numpy, CPU): test infrastructure only, shares no
code with the GPU path."""
import numpy as np


def _parts(q, k, bias, mask, rpb, n, head, group):
    d = q.shape[3]
    x = q[n, :, head] @ k[n, :, head // group].T / np.sqrt(d)
    if bias is not None:
        x = x + bias[n // rpb, head]
    if mask is not None:
        x = np.where(mask[n][None, :] != 0, x, -np.inf)
    return np.where(x > -1e30, x, -np.inf)


def forward(q, k, v, gate=None, bias=None, mask=None, rpb=None):
    """out [N, Lq, H, d], lse [N, H, Lq], probabilities [N, H, Lq, Lk]."""
    N, Lq, H, d = q.shape
    Lk, Hk = k.shape[1:3]
    rpb = rpb or max(N, 1)
    if mask is not None:  # what masked keys hold does not matter
        k, v = (np.where((mask != 0)[:, :, None, None], t, 0.0) for t in (k, v))
        if bias is not None:
            bias = bias if np.isfinite(bias).all() else np.where(np.isnan(bias), 0.0, bias)
    out, lse, prob = np.zeros(q.shape), np.full((N, H, Lq), -np.inf), np.zeros((N, H, Lq, Lk))
    for n in range(N):
        for h in range(H):
            x = _parts(q, k, bias, mask, rpb, n, h, H // Hk)
            if Lk:
                top = np.max(x, 1, keepdims=True)
                top = np.where(np.isfinite(top), top, 0.0)
                e = np.exp(x - top)
                s = e.sum(1, keepdims=True)
                prob[n, h] = np.where(s > 0, e / np.where(s > 0, s, 1.0), 0.0)
                lse[n, h] = np.where(s[:, 0] > 0, np.log(np.where(s[:, 0] > 0, s[:, 0], 1.0)) + top[:, 0], -np.inf)
            out[n, :, h] = prob[n, h] @ v[n, :, h // (H // Hk)]
    if gate is not None:
        out = out / (1 + np.exp(-gate))
    return out, lse, prob


def backward(q, k, v, gate, bias, mask, dout, rpb=None):
    """(dq, dk, dv, dgate, dbias): the chain rule through the definitions."""
    N, Lq, H, d = q.shape
    Hk = k.shape[2]
    rpb = rpb or max(N, 1)
    if mask is not None:
        k, v = (np.where((mask != 0)[:, :, None, None], t, 0.0) for t in (k, v))
    a, _, prob = forward(q, k, v, None, bias, mask, rpb)
    sig = 1 / (1 + np.exp(-gate)) if gate is not None else 1.0
    da = dout * sig
    dgate = dout * a * sig * (1 - sig) if gate is not None else None
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    dbias = np.zeros(bias.shape) if bias is not None else None
    for n in range(N):
        for h in range(H):
            j, p = h // (H // Hk), prob[n, h]
            dp = da[n, :, h] @ v[n, :, j].T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            dq[n, :, h] = ds @ k[n, :, j] / np.sqrt(d)
            dk[n, :, j] += ds.T @ q[n, :, h] / np.sqrt(d)
            dv[n, :, j] += p.T @ da[n, :, h]
            if bias is not None:
                dbias[n // rpb, h] += ds
    return dq, dk, dv, dgate, dbias
