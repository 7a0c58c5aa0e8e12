"""Rows of an embedding by token id and the gradient of the embedding, in fp64, row by row."""
import numpy as np

F = 2.0 ** -24                  # half a step of fp32


def embed(ids, E, scale=1.0):
    out = np.zeros((len(ids), E.shape[1]))
    for r, i in enumerate(np.asarray(ids)):
        if 0 <= i < E.shape[0]:
            out[r] = np.asarray(E[i], np.float64) * scale
    return out


def embed_backward(dout, ids, V, scale=1.0, dE=None):
    """(dE [V, H], a limit on the error of sums in fp32: of m rows, m - 1 additions, the scale and (where there is a dE to add to) one more, each F
    of the sum of magnitudes at most)."""
    dout = np.asarray(dout, np.float64)
    total, size, count = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros((V, 1))
    for r, i in enumerate(np.asarray(ids)):
        if 0 <= i < V:
            total[i] += dout[r] * scale
            size[i] += np.abs(dout[r] * scale)
            count[i] += 1
    if dE is not None:
        dE = np.asarray(dE, np.float64)
        touched = count > 0
        return total + dE, np.where(touched, (count + 2) * F * (size + np.abs(dE)), 0.0)
    return total, (count + 1) * F * size
