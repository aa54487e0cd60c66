"""The layers in 64 bits on the CPU, from their definitions (include/bridger.h), with tolerances
counted from the roundings to 32 bits; operators_ref adds those to an output's type."""
import numpy as np

from operators_ref import U, np64


def entries(ids, offsets, n_entries):
    """The entry that each slot reads [n, k], -1 for an empty one."""
    ids = ids.cpu().numpy().astype(np.int64)
    ids = ids.reshape(len(ids), -1)
    if offsets is None:
        at, end = ids, n_entries
    else:
        off = offsets.cpu().numpy()
        at, end = ids + off[:-1], np.minimum(off[1:], n_entries)
    return np.where((ids >= 0) & (at < end), at, -1)


def embed(ids, table, scale=1.0, offsets=None):
    """(output, tolerance before the rounding to its type)."""
    t = np64(table)
    at = entries(ids, offsets, len(t))
    out, size = np.zeros((len(at), t.shape[1])), np.zeros((len(at), t.shape[1]))
    with np.errstate(all="ignore"):
        for s in range(at.shape[1]):
            ok = at[:, s] >= 0
            out[ok] += t[at[ok, s]]
            size[ok] += np.abs(t[at[ok, s]])
        # each sum is off by U of a partial sum, the scale and its product by U each
        return out * scale, np.nan_to_num((at.shape[1] + 1) * U * size * abs(scale), posinf=0)


def embed_grad(ids, grad, n_entries, scale=1.0, offsets=None):
    g = np64(grad)
    at = entries(ids, offsets, n_entries)
    out, size = np.zeros((n_entries, g.shape[1])), np.zeros((n_entries, g.shape[1]))
    count = np.zeros(n_entries)
    with np.errstate(all="ignore"):
        for s in range(at.shape[1]):
            ok = at[:, s] >= 0
            np.add.at(out, at[ok, s], g[ok])
            np.add.at(size, at[ok, s], np.abs(g[ok]))
            np.add.at(count, at[ok, s], 1)
        tol = (count[:, None] + 1) * U * size * abs(scale)
        return out * scale, np.nan_to_num(tol, posinf=0)
