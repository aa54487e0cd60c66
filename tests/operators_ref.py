"""The row operators in 64 bits on the CPU, from their definitions (include/bridger.h), and how far
an output in 32 bits, rounded once to its type, may be from them."""
import numpy as np
import torch

U = 2.0 ** -24                     # half a step of float32, relative
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {t: torch.finfo(t).tiny * torch.finfo(t).eps for t in HALF}   # the smallest step of a type
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def np64(t):
    return t.detach().double().cpu().numpy()


def top_k(scores, k):
    """(values float64 [n, k], ids [n, k]): stable order, NaN after every number."""
    s = np64(scores)
    n, c = s.shape
    key = np.where(np.isnan(s), np.inf, -s)
    key = np.where(key == 0, 0.0, key)
    # NaN after -infinity: order by (is NaN, -score), both stable
    order = np.lexsort((np.broadcast_to(np.arange(c), s.shape), key, np.isnan(s)), axis=1)[:, :k]
    v = np.full((n, k), -np.inf)
    i = np.full((n, k), -1, np.int64)
    m = min(k, c)
    i[:, :m] = order
    v[:, :m] = np.take_along_axis(s, order, 1)
    return v, i


def distill(logits, ids, teacher, T, weight=None):
    """loss, gradient and their tolerances before the rounding of the gradient to its type."""
    z, t, ids = np64(logits), np64(teacher), ids.cpu().numpy().astype(np.int64)
    n, c = z.shape
    k = ids.shape[1]
    w = np.ones(n) if weight is None else np64(weight)
    loss, grad = np.zeros(n), np.zeros((n, c))
    loss_tol, grad_tol = np.zeros(n), np.zeros((n, c))
    # one thread adds at most c / 8 + 64 values in a row, in float
    adds = c / 64 + 64
    for r in range(n):
        ok = (ids[r] >= 0) & (ids[r] < c)
        if not ok.any() or (t[r, ok] == -np.inf).all():
            continue
        with np.errstate(all="ignore"):
            u = (t[r, ok] - np.max(np.where(np.isnan(t[r, ok]), -np.inf, t[r, ok]))) / T
            p = np.exp(u) / np.exp(u).sum()
            logp = u - np.log(np.exp(u).sum())
            most = np.max(np.where(np.isnan(z[r]), -np.inf, z[r]))
            most = 0.0 if most == -np.inf else most
            x = (z[r] - most) / T
            mass = np.exp(x).sum()
            q = np.exp(x) / mass if mass > 0 else np.exp(x)
            logq = np.where(np.isneginf(x), -np.inf, x - np.log(mass))
            term = np.where(p == 0, 0.0, p * (logp - logq[ids[r, ok]]))
        loss[r] = T * T * term.sum()
        g = q.copy()
        pj = np.zeros(c)
        np.add.at(pj, ids[r, ok], p)
        grad[r] = T * w[r] * (g - pj)
        # exponent of e^x: the quotient and the product with log2(e) (and that constant) are each
        # off by U |x|; the exponential itself by 2 steps.  |x| e^x is weighed by the distribution.
        fx = np.where(np.isfinite(x), np.abs(x), 0.0)
        fu = np.where(np.isfinite(u), np.abs(u), 0.0)
        d_mass = (3 * np.nansum(q * fx) + 4 + adds) * U
        d_p = (3 * np.nansum(p * fu) + 4 + k) * U
        used = np.where(p == 0, 0.0, 3 * fu + 3 * fx[ids[r, ok]] + 8)
        reach = np.where(p == 0, 0.0, np.abs(logp) + np.abs(np.where(np.isfinite(logq), logq, 0)[ids[r, ok]]))
        # log p, log q and their difference, p itself, k products and sums
        with np.errstate(all="ignore"):
            loss_tol[r] = T * T * np.nansum(p * ((used + 4 * reach) * U + d_mass + d_p
                                                 + reach * (3 * fu * U + d_p + (k + 4) * U)))
        grad_tol[r] = T * abs(w[r]) * (q * ((3 * fx + 8) * U + d_mass)
                                       + pj * ((3 * fu.max() + 8 + k) * U + d_p))
    return loss, grad, loss_tol, grad_tol


def assert_near(got, ref, tol, dtype, what=""):
    """|got - ref| within tol and the type's rounding; equal infinities and NaN."""
    got = np64(got)
    ref = np.asarray(ref, np.float64)
    top = torch.finfo(dtype).max
    special = ~np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN differ"
    assert np.array_equal(got[special & ~np.isnan(ref)], ref[special & ~np.isnan(ref)]), what
    ok = ~special
    err = np.abs(got[ok] - ref[ok])
    most = np.broadcast_to(tol, ref.shape)[ok] * (1 + HALF[dtype]) + HALF[dtype] * np.abs(ref[ok]) + TINY[dtype]
    bad = ~(err <= most)
    bad &= ~((np.abs(ref[ok]) > top * (1 - HALF[dtype])) & np.isinf(got[ok]))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} values, worst {np.max(err[bad] / most[bad])} times the bound"


def check_rmsnorm(x, weight, residual, eps, q, scale, total, what=""):
    """Every output of rmsnorm_q8 against the definition."""
    s = np64(x)
    if residual is not None:
        s = s + np64(residual)
    w = np.ones(s.shape[1]) if weight is None else np64(weight)
    dtype = x.dtype
    qn, sc = q.cpu().numpy().astype(np.float64), np64(scale)
    with np.errstate(all="ignore"):
        y = s * w / np.sqrt((s * s).mean(1, keepdims=True) + eps)
        y = np.where(s == 0, np.where(np.isfinite(w) | (s != 0), 0.0, np.nan), y)
    # what float cannot hold counts as infinite
    broken = ~np.isfinite(y).all(1) | (np.abs(s) > torch.finfo(torch.float32).max).any(1) | \
        (np.abs(np.where(np.isfinite(y), y, 0)).max(1) > torch.finfo(torch.float32).max)
    assert np.array_equal(np.isnan(sc), broken), f"{what}: rows with a NaN scale"
    assert (qn[broken] == 0).all(), what
    y, qn, sc = y[~broken], qn[~broken], sc[~broken]
    most = np.abs(y).max(1) if y.size else np.zeros(len(y))
    # s, its product with the weight and with the row's factor, and the quotient by 127: 8 roundings
    assert (np.abs(sc - most / 127) <= 8 * U * most / 127 + 2.0 ** -149).all(), f"{what}: scale"
    assert (qn[most == 0] == 0).all() and (np.abs(qn) <= 127).all(), what
    live = most > 127 * 2.0 ** -126
    t = y[live] * 127 / most[live, None]
    off = np.abs(qn[live] - t).max() if t.size else 0
    # half a step, and 8 roundings of a value of up to 127
    assert off <= 0.5 + 127 * 8 * U, f"{what}: 8-bit values off by {off}"
    if total is not None:
        # the sum is rounded to float, then to its type
        assert_near(total, s, U * np.abs(np.where(np.isfinite(s), s, 0)), dtype, f"{what}: total")


def check_matmul(a, a_scale, b, b_scale, bias, out, what=""):
    acc = a.cpu().numpy().astype(np.float64) @ b.cpu().numpy().astype(np.float64).T   # exact
    with np.errstate(all="ignore"):
        ref = acc * np64(a_scale)[:, None] * np64(b_scale)[None, :]
        tol = 3 * U * np.abs(ref)          # the integer, and two products
        if bias is not None:
            ref = ref + np64(bias)[None, :]
            tol = tol + U * np.abs(ref)
    assert_near(out, ref, np.where(np.isfinite(tol), tol, 0), out.dtype, what)
