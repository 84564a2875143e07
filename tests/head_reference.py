"""sample, logit_error and orthogonalize from their definitions, in numpy and 64 bits (see include/sage.h)."""
import math

import numpy as np

UNIT = 2.0 ** 42
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def weights(z, T):
    """Whole-number weights of a row (float64) relative to its maximum."""
    with np.errstate(over="ignore", invalid="ignore"):
        x = (z - z.max()) / T
    w = np.rint(np.exp(np.where(z == -np.inf, -1e9, x)) * UNIT)
    return w.astype(np.int64)


def kept_classes(z, T, top_k, top_p, min_p):
    """The classes that a row's settings keep, in the order of the classes."""
    n = len(z)
    w = weights(z, T)
    order = np.lexsort((np.arange(n), -z))
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        before = np.concatenate([[0], np.cumsum(w[order])[:-1]])
        need = math.ceil(top_p * float(w[order].sum()))
        order = order[:max(1, int((before < need).sum()))]
    if min_p > 0:
        border = T * math.log(min(min_p, 1.0))
        order = order[(np.arange(len(order)) == 0) | (z[order] - z.max() >= border)]
    return np.sort(order), w


def sample_row(z, u, T, top_k, top_p, min_p):
    """(label, log-probability) of one row; all arguments widened to float64 from what the call takes."""
    z = z + 0.0  # (both zeros are one value)
    if np.isnan(z).any() or not np.isfinite(z.max()):
        return -1, math.nan
    if not T > 0:
        return int(z.argmax()), 0.0
    kept, w = kept_classes(z, T, top_k, top_p, min_p)
    c = np.cumsum(w[kept])
    S = int(c[-1])
    t = min(int(min(max(u, 0.0), 1.0) * float(S)) if u == u else 0, S - 1)
    j = int(kept[np.searchsorted(c, t, side="right")])
    return j, (z[j] - z.max()) / T - math.log(float(S) / UNIT)


def logit_error(z, y, w):
    """(E, loss, 1 - p of the label) of rows, float64."""
    n, C = z.shape
    E, loss, miss = np.zeros((n, C)), np.zeros(n), np.zeros(n)
    for i in range(n):
        if y[i] < 0:
            continue
        if y[i] >= C or np.isnan(z[i]).any() or z[i].max() == np.inf:
            E[i], loss[i] = np.nan, np.nan
            continue
        if z[i].max() == -np.inf:
            loss[i] = np.inf
            continue
        e = np.exp(z[i] - z[i].max())
        ey = e[y[i]]
        e[y[i]] = 0.0
        R = math.fsum(e)
        E[i] = w[i] * e / (R + ey)
        E[i, y[i]] = -w[i] * R / (R + ey)
        loss[i] = math.log1p(R / ey) if ey > 0 else (math.log(R) - (z[i, y[i]] - z[i].max()))
        miss[i] = R / (R + ey)
    return E, loss, miss


def orthogonalize(G, triples, eps, scale):
    """(result, norms of X at the beginning of each step), float64."""
    X = G / (math.sqrt(float((G * G).sum())) + eps) if G.any() else G * 0.0
    norms = []
    for a, b, c in triples:
        norms.append(float(np.linalg.norm(X)))
        if X.shape[0] <= X.shape[1]:
            A = X @ X.T
            X = a * X + b * (A @ X) + c * (A @ (A @ X))
        else:
            A = X.T @ X
            X = a * X + b * (X @ A) + c * ((X @ A) @ A)
    return scale * X, norms


def orthogonalize_bound(norms, triples, scale, entries):
    """How far the Frobenius norm of the error may go: a step's three terms have each a relative error of about 2^-22 (two fp16 parts
    22 bits or more, lo * lo left out, sums in fp32), on singular values of at most 1.25, and what a step begins with is
    stretched by the slopes of those after it, at most |a| + 3 |b| 1.25^2 + 5 |c| 1.25^4 and, near 0, |a|; for the polynomials
    in use (decreasing slopes) |a|. Entries are scaled so that singular values of 1 (what the norm with eps leaves at most) become 2^14 or
    more; the spacing of the low part ends at 2^-24 there: each of the entries is off by up to 2^-25 / 2^14 = 2^-39 of the
    singular values' bound (1.25 here) however small it is, in every step."""
    total = 2.0 ** -24 * norms[0]
    for n, (a, b, c) in zip(norms, triples):
        total = (total + math.sqrt(entries) * 1.25 * 2.0 ** -39) * max(abs(a), 1.0) + n * (abs(a) + 2 * abs(b) + 4 * abs(c)) * 2.0 ** -22
    return total * abs(scale)
