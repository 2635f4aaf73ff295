"""64-bit forms of the routing, expert-row and head-loss operators, from their definitions (numpy),
with bounds on how far fp32 sums and bf16 outputs may lie from them."""
import numpy as np

U32 = 2.0 ** -24  # half a unit in the last place of fp32 at 1
U16 = 2.0 ** -8   # the same of bf16 (7 fraction bits: half a unit at 1 is 2^-8)


def route(z, k, normalize, valid=None):
    """experts [T, k] (-1: none) and weights; NaN and -inf are never chosen, +inf is the largest fp32."""
    z = np.asarray(z, dtype=np.float64)
    T, E = z.shape
    z = np.minimum(np.where(np.isnan(z), -np.inf, z), np.finfo(np.float32).max)
    experts = np.full((T, k), -1, dtype=np.int64)
    weights = np.zeros((T, k))
    for t in range(T):
        if valid is not None and not valid[t]:
            continue
        order = sorted((e for e in range(E) if z[t, e] > -np.inf), key=lambda e: (-z[t, e], e))
        if not order:
            continue
        p = np.exp(z[t] - z[t, order[0]])
        chosen = order[:k]
        total = p[chosen].sum() if normalize else p[np.isfinite(z[t])].sum()
        experts[t, :len(chosen)] = chosen
        weights[t, :len(chosen)] = p[chosen] / total
    return experts, weights


def route_grad(z, experts, dweights, normalize):
    """(dlogits, magnitude of the terms they are sums of)."""
    z = np.asarray(z, dtype=np.float64)
    z = np.minimum(np.where(np.isnan(z), -np.inf, z), np.finfo(np.float32).max)
    out, size = np.zeros_like(z), np.zeros_like(z)
    for t in range(z.shape[0]):
        at = [int(e) for e in experts[t] if 0 <= e < z.shape[1]]
        if not at:
            continue
        q = np.zeros(z.shape[1])
        over = at if normalize else [e for e in range(z.shape[1]) if z[t, e] > -np.inf]
        p = np.exp(z[t, over] - z[t, over].max())
        q[over] = p / p.sum()
        dw = np.zeros(z.shape[1])
        dw[at] = [dweights[t, j] for j, e in enumerate(experts[t]) if 0 <= e < z.shape[1]]
        out[t] = q * (dw - (q * dw).sum())
        size[t] = q * (np.abs(dw) + (q * np.abs(dw)).sum())
    return out, size


def sort(experts, E):
    flat = np.asarray(experts).reshape(-1)
    n = len(flat)
    on = (flat >= 0) & (flat < E)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[on], minlength=E))]).astype(np.int64)
    slots = [i for e in range(E) for i in np.nonzero(flat == e)[0]] if E <= 16 else list(
        np.argsort(np.where(on, flat, E), kind="stable")[:offsets[E]])
    slot_of = np.full(n, -1, dtype=np.int64)
    slot_of[:len(slots)] = slots
    row_of = np.full(n, -1, dtype=np.int64)
    row_of[slots] = np.arange(len(slots))
    return offsets, row_of.reshape(np.asarray(experts).shape), slot_of


def dispatch(X, slot_of, k, R):
    out = np.zeros((R, X.shape[1]))
    for r in range(R):
        if slot_of[r] >= 0:
            out[r] = X[slot_of[r] // k]
    return out


def combine(Ys, row_of, weights):
    """(Y, sum of the magnitudes of its terms)."""
    T, k = row_of.shape
    Y, size = np.zeros((T, Ys.shape[1])), np.zeros((T, Ys.shape[1]))
    for t in range(T):
        for j in range(k):
            r = row_of[t, j]
            if 0 <= r < len(Ys):
                term = (1.0 if weights is None else float(weights[t, j])) * Ys[r]
                Y[t] += term
                size[t] += np.abs(term)
    return Y, size


def combine_grad(dY, Ys, row_of, slot_of, weights):
    """(dYs, dweights, magnitude of dweights' terms)."""
    T, k = row_of.shape
    dYs = np.zeros_like(Ys)
    dw, size = np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            r = row_of[t, j]
            if 0 <= r < len(Ys):
                dYs[r] = float(weights[t, j]) * dY[t]
                dw[t, j] = (dY[t] * Ys[r]).sum()
                size[t, j] = np.abs(dY[t] * Ys[r]).sum()
    return dYs, dw, size


def head_loss(X, W, labels, dloss=None):
    """loss, lse, dX (None without dloss) and the bounds of each, element by element."""
    T, D = X.shape
    V = len(W)
    z = X @ W.T
    # a logit's fp32 sum: at most one rounding (or truncation) of a partial sum per product
    dz = 2 * (D + 4) * U32 * (np.abs(X) @ np.abs(W).T)
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    total = e.sum(1, keepdims=True)
    p = e / total
    lse = (top + np.log(total))[:, 0]
    on = (labels >= 0) & (labels < V)
    at = np.where(on, labels, 0)
    rows = np.arange(T)
    loss = lse - z[rows, at]
    err_z = dz.max(1)
    # log-sum-exp moves by at most the largest logit error; 2^x and the fp32 sum add their own:
    # the exponent's rounding (|x| <= 256 where it counts), the 2^-22 of the exponential, V terms
    err = 2 * err_z + 512 * U32 + 2 ** -21 + (V + 16) * U32
    out = {"loss": np.where(on, loss, 0.0), "lse": np.where(on, lse, 0.0)}
    out["loss_err"] = np.where(on, err + 4 * U32 * np.abs(loss), 0.0)
    out["lse_err"] = np.where(on, err + 4 * U32 * np.abs(lse), 0.0)
    if dloss is not None:
        d = p.copy()
        d[rows, at] -= 1.0
        d *= dloss[:, None]
        dX = d @ W
        # every exponential rounded to bf16, its logit off by dz, the sum's own rounding; then bf16
        size = (p * np.abs(dloss)[:, None]) @ np.abs(W) + np.abs(dloss * (1 - p[rows, at]))[:, None] * np.abs(W[at])
        out["dX"] = np.where(on[:, None], dX, 0.0)
        out["dX_err"] = np.where(on[:, None], size * (U16 + 4 * err + 2 * (V + 16) * U32)[:, None] + 1.01 * U16 * np.abs(dX), 0.0) + 1e-38
    return out
