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


def random_words(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 on uint64 arrays that hold words of 32 bits."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, np.uint64) for v in (c0, c1, c2, c3)]
    k0, k1 = int(k0), int(k1)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        s = np.uint64(32)
        c = [(b >> s) ^ c[1] ^ np.uint64(k0), b & low, (a >> s) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    return c


def kept(n, w, p, seed, layer):
    """Which elements dropout keeps, bool [n, w]."""
    s0, step = (int(v) % 2 ** 64 for v in seed)
    unit, row = np.meshgrid(np.arange((w + 7) // 8, dtype=np.uint64), np.arange(n, dtype=np.uint64))
    half = []
    for low in (0, 1):
        words = random_words(unit, row, np.full_like(unit, step % 2 ** 32),
                             np.full_like(unit, 2 * layer + low), s0 % 2 ** 32, s0 >> 32)
        parts = [h for v in words for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))]
        half.append(np.stack(parts, 2).reshape(n, -1)[:, :w])
    number = half[0] << np.uint64(16) | half[1]
    return number.astype(np.float64) >= np.rint(p * 2.0 ** 32)


def dropout(x, p, seed, residual=None, layer=0):
    x = np64(x)
    up = 1 / (1 - p) if p < 1 else 0.0
    with np.errstate(all="ignore"):
        out = np.where(kept(*x.shape, p, seed.tolist(), layer), x * up, 0.0)
        tol = 2 * U * np.abs(out)                      # the factor, and the product
        if residual is not None:
            out = out + np64(residual)
            tol = tol + U * np.abs(out)
    return out, np.where(np.isfinite(tol), tol, 0.0)


# A lane adds at most 32 values in a row, a row's lanes in at most 10 steps more.
ADDS = 42


def _norm(t, eps):
    """h, 1 / std, and how far h may be off."""
    n = t.shape[1]
    mean = t.mean(1, keepdims=True)
    c = t - mean
    r = 1 / np.sqrt((c * c).sum(1, keepdims=True) / n + eps)
    h = c * r
    # the mean is off by the sum of t - m (each off by U) and its quotient; 1 / std by half the sum
    # of squares' error, the root and the quotient; the differences and their product by 4 U
    er = (ADDS + 4) / 2 * U + 3 * U
    eh = np.abs(h) * (er + 4 * U) + (ADDS + 3) * U * np.abs(c).mean(1, keepdims=True) * r
    return h, r, eh, er


def layer_norm(t, weight=None, bias=None, eps=1e-5):
    """The norm of t (the sum, already rounded) and its tolerance."""
    with np.errstate(all="ignore"):
        h, _, eh, _ = _norm(np64(t), eps)
        w = 1.0 if weight is None else np64(weight)
        y, tol = h * w, eh * np.abs(w) + U * np.abs(h * w)
        if bias is not None:
            y = y + np64(bias)
            tol = tol + U * np.abs(y)
    return y, np.where(np.isfinite(tol), tol, 0.0)


def layer_norm_grad(grad, t, weight=None, grad_total=None, eps=1e-5):
    """((dx, dweight, dbias), their tolerances)."""
    with np.errstate(all="ignore"):
        g = np64(grad)
        h, r, eh, er = _norm(np64(t), eps)
        s = g if weight is None else g * np64(weight)
        mean, along = s.mean(1, keepdims=True), (s * h).mean(1, keepdims=True)
        size = np.abs(s).mean(1, keepdims=True)
        dx = r * (s - mean - h * along)
        e_mean = (ADDS + 3) * U * size
        e_along = (np.abs(s) * eh).mean(1, keepdims=True) + \
            (ADDS + 4) * U * np.abs(s * h).mean(1, keepdims=True)
        terms = np.abs(s) + np.abs(mean) + np.abs(h * along)
        tol = r * (e_mean + np.abs(h) * e_along + np.abs(along) * eh + 4 * U * terms) \
            + (er + 2 * U) * np.abs(dx)
        if grad_total is not None:
            dx = dx + np64(grad_total)
            tol = tol + U * np.abs(dx)
        # a workgroup adds its share of the rows, then up to 256 groups of lanes; the rest in double
        adds = len(g) / 512 + 300
        dw, db = (g * h).sum(0), g.sum(0)
        tw = (np.abs(g) * eh).sum(0) + (adds + 2) * U * np.abs(g * h).sum(0)
        tb = (adds + 2) * U * np.abs(g).sum(0)
    return (dx, dw, db), [np.where(np.isfinite(v), v, 0.0) for v in (tol, tw, tb)]


def sample_row(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(class, log of its share, the classes that stay, how far the draw and the cut by top_p are from
    another answer: the smallest distance of a sum from its limit, relative to the sum of all)."""
    z = np.asarray(z, np.float64)
    cls = np.flatnonzero(z > -np.inf)
    cls = cls[np.argsort(-z[cls], kind="stable")]
    if len(cls) == 0:
        return -1, -np.inf, cls, 1.0
    top = z[cls[0]]
    if not temperature >= 1e-6 or top_p <= 0:
        return cls[0], 0.0, cls[:1], 1.0
    temperature = min(temperature, 1e6)
    if top_k > 0:
        cls = cls[:top_k]
    with np.errstate(all="ignore"):
        w = np.where(z[cls] == top, 1.0, np.exp((z[cls] - top) / temperature))
    sums = np.cumsum(w)
    gap, stay = 1.0, len(cls)
    if top_p < 1:
        limit = top_p * sums[-1]
        before = np.concatenate([[0.0], sums[:-1]])
        stay = int((before < limit).sum())
        near = np.abs(before[1:] - limit) if len(before) > 1 else np.ones(1)
        exact = np.all(w == 1.0)                 # whole numbers: no rounding, so no doubt
        gap = 1.0 if exact else near.min() / sums[-1]
    if min_p > 0:
        stay = min(stay, int((z[cls] >= top + temperature * np.log(min(min_p, 1.0))).sum()))
    order = np.argsort(cls[:stay], kind="stable")
    cls, w = cls[:stay][order], w[:stay][order]
    sums = np.cumsum(w)
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    at = min(int((sums <= u * sums[-1]).sum()), len(sums) - 1)
    if not np.all(w == 1.0):
        gap = min(gap, np.abs(sums[:-1] - u * sums[-1]).min() / sums[-1] if len(sums) > 1 else 1.0)
    return cls[at], np.log(w[at] / sums[-1]), cls, gap
