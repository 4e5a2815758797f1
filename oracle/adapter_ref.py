"""fp64 restatement of the low-rank adapters beside a shared projection, row by row's own adapter:

    out[t,o] = sum_i x[t,i] w[o,i] + sum_r h[t,r] b[a,o,r],   h[t,r] = scale[a] sum_i x[t,i] a[a,r,i],   a = row_adapter[t]

and its gradients, and of clipping gradients by their global norm."""
import numpy as np


def hidden(x, a, scale, row_adapter):
    h = np.zeros((x.shape[0], a.shape[1]))
    for n in range(a.shape[0]):
        rows = np.nonzero(row_adapter == n)[0]
        h[rows] = scale[n] * (x[rows] @ a[n].T)
    return h


def adapter_fwd(x, w, a, b, scale, row_adapter):
    h = hidden(x, a, scale, row_adapter)
    out = x @ w.T
    for n in range(a.shape[0]):
        rows = np.nonzero(row_adapter == n)[0]
        out[rows] += h[rows] @ b[n].T
    return {"out": out, "hidden": h}


def adapter_bwd(x, w, a, b, scale, row_adapter, dout):
    h = hidden(x, a, scale, row_adapter)
    dx, da, db, g = dout @ w, np.zeros_like(a), np.zeros_like(b), np.zeros_like(h)
    for n in range(a.shape[0]):
        rows = np.nonzero(row_adapter == n)[0]
        g[rows] = scale[n] * (dout[rows] @ b[n])
        dx[rows] += g[rows] @ a[n]
        da[n] = g[rows].T @ x[rows]
        db[n] = dout[rows].T @ h[rows]
    return {"dx": dx, "da": da, "db": db, "dhidden": g}


def clip(grads, max_norm):
    """norm, clipped gradients."""
    with np.errstate(all="ignore"):
        norm = np.sqrt(np.float64(sum(float(np.sum(np.square(g))) for g in grads)))
        by = np.float64(max_norm) / (norm + 1e-6)
        by = by if not by > 1.0 and max_norm < np.inf else 1.0     # an infinite max_norm is no bound, also where the norm is not finite
        return norm, [g * by for g in grads]
