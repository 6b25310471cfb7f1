"""Plain fp64 definition of the learned relative position bias and its table's
gradient (numpy, CPU): test infrastructure only, shares no code with the GPU
path."""
import numpy as np


def buckets(pos_i, pos_j, edges, seg_i=None, seg_j=None):
    """Bucket of every pair [B, Li, Lj]: how many edges the difference reaches."""
    d = np.asarray(pos_i, np.int64)[:, :, None] - np.asarray(pos_j, np.int64)[:, None, :]
    n = np.zeros(d.shape, np.int64)
    for e in np.asarray(edges, np.int64):
        n += d >= e
    if seg_i is not None:
        n[np.asarray(seg_i)[:, :, None] != np.asarray(seg_j)[:, None, :]] = len(edges) + 1
    return n


def forward(pos_i, pos_j, edges, table, base=None, seg_i=None, seg_j=None):
    """[B, H, Li, Lj]"""
    n = buckets(pos_i, pos_j, edges, seg_i, seg_j)
    out = np.moveaxis(np.asarray(table, np.float64)[:, n], 0, 1)
    return out if base is None else out + np.asarray(base, np.float64)


def backward(pos_i, pos_j, edges, dbias, seg_i=None, seg_j=None):
    """Gradient [H, buckets] of the table."""
    n = buckets(pos_i, pos_j, edges, seg_i, seg_j)
    k = len(edges) + 1 + (seg_i is not None)
    g = np.asarray(dbias, np.float64)
    return np.stack([np.bincount(n.reshape(-1), g[:, h].reshape(-1), k) for h in range(g.shape[1])])
