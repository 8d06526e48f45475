"""64-bit references of distillation from a teacher's lists and of the best
tokens under rules (numpy), with the bounds that the GPU tests hold the kernels
to (no test functions here).

Bounds are first-order worst cases of the stated arithmetic, as in
token_reference: U = 2^-24 per float32 operation, 2^-20 for an exponential with
the rounding of its argument (and U per unit of the argument beyond), 2^-16 for a
value kept as a bf16 pair."""
import numpy as np

from token_reference import U


def logits(X, W, bias, node):
    """(z, its bound, x) of the chosen rows."""
    n, H = X.shape
    node = np.asarray(node, np.int64)
    inside = (node >= 0) & (node < n)
    x = np.where(inside[:, None], X[np.where(inside, node, 0)], 0.0)
    b = np.zeros(W.shape[0]) if bias is None else np.where(bias <= -1e30, -np.inf, bias)
    z = x @ W.T + b
    dz = (H + 4) * U * (np.abs(x) @ np.abs(W).T + np.where(np.isfinite(b), np.abs(b), 0.0))
    return z, dz, x, inside


def log_sum(z, dz):
    """Rows' log sums of exponentials of z, whose bound is dz, and their bound."""
    top = np.where(np.isfinite(z.max(1)), z.max(1), 0.0)
    s = np.exp(z - top[:, None]).sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(s > 0, top + np.log(s), -np.inf)
    live = np.where(np.isfinite(z), dz, 0.0).max(1)
    fin = np.where(np.isfinite(lse), lse, 0.0)
    return lse, live + 2.0 ** -21 + z.shape[1] / 2 * U + 8 * U * (1 + np.abs(fin) + np.abs(top))


def distill(X, W, bias, node, t_id, t_logit, t_lse, tau, weight, scale, dt):
    """Losses, log sums and gradients, with a bound for each."""
    n, H = X.shape
    V, (R, K) = W.shape[0], t_id.shape
    z, dz, x, inside = logits(X, W, bias, node)
    z, dz = z / tau, dz / tau + 4 * U * np.abs(np.where(np.isfinite(z), z, 0.0)) / tau
    lse, lse_tol = log_sum(z, dz)
    node = np.asarray(node, np.int64)
    here = (t_id >= 0) & inside[:, None]
    t = np.where(here, np.where(here, t_logit, 0.0) / tau, -np.inf)
    bad = (here & ((t_id >= V) | ~(t < np.inf))).any(1)
    some = (t > -np.inf).any(1)
    if t_lse is not None:
        bad |= some & ~np.isfinite(np.where(some, t_lse, 0.0))
    t = np.where(bad[:, None], -np.inf, t)
    top = np.where(some & ~bad, t.max(1), 0.0)
    fin = np.where(np.isfinite(t), t, 0.0)
    with np.errstate(divide="ignore"):
        own = top + np.log(np.exp(t - top[:, None]).sum(1))
    T = own if t_lse is None else np.asarray(t_lse, np.float64)
    T = np.where(some & ~bad, T, 0.0)
    q = np.where(np.isfinite(t), np.exp(t - T[:, None]), 0.0)
    T_tol = (2 * U * np.abs(fin).max(1) + 2.0 ** -20 + (K + 4) * U * (1 + np.abs(T))) if t_lse is None else np.zeros(R)
    # of a q, relative: the listed logits' rounding, the exponential with its argument, the sum
    eq = (4 * U * np.abs(fin) + T_tol[:, None] + 2 * U * np.abs(T)[:, None] + 2.0 ** -20 + 4 * U * np.abs(fin - T[:, None])
          + (K + 4) * U)
    s = q.sum(1)
    ok = some & ~bad
    r, k = np.nonzero(here & ok[:, None] & (q > 0))
    v = t_id[r, k]
    loss, loss_tol = np.zeros(R), np.zeros(R)
    with np.errstate(invalid="ignore"):
        a = t[r, k] - z[r, v] + lse[r] - T[r]
        a = np.where(np.isneginf(z[r, v]), np.inf, a)
    np.add.at(loss, r, q[r, k] * a)
    size = np.abs(t[r, k]) + np.where(np.isfinite(z[r, v]), np.abs(z[r, v]), 0) + np.abs(T[r]) + np.where(
        np.isfinite(lse[r]), np.abs(lse[r]), 0)
    step = dz[r, v] + lse_tol[r] + T_tol[r] + 8 * U * size
    np.add.at(loss_tol, r, q[r, k] * (np.where(np.isfinite(a), np.abs(a), 0.0) * (eq[r, k] + K * U) + step))
    loss[ok & np.isneginf(lse)] = np.inf
    loss[bad] = np.nan
    # gradients
    live = ok & np.isfinite(lse)
    g = np.where(live, scale * (np.ones(R) if weight is None else weight) / tau, 0.0)
    P = np.where(live[:, None], np.exp(z - np.where(live, lse, 0.0)[:, None]), 0.0)
    Q, Qe = np.zeros((R, V)), np.zeros((R, V))
    np.add.at(Q, (r, v), q[r, k])
    np.add.at(Qe, (r, v), q[r, k] * eq[r, k])
    D = g[:, None] * (s[:, None] * P - Q)
    pair = 2.0 ** -16 if dt == "bf16" else 0.0
    far = np.where(P > 0, np.abs(z - np.where(live, lse, 0.0)[:, None]), 0.0) + np.where(live, np.abs(lse), 0.0)[:, None]
    live_dz = np.where(np.isfinite(dz), dz, 0.0).max(1)
    eps = (2 * live_dz + lse_tol + eq.max(1) + 2.0 ** -20 + pair)[:, None] + 6 * U * far
    ag = np.abs(g)[:, None]
    dense, sparse = ag * s[:, None] * P, ag * Q
    big = dense + sparse
    rel = dense * eps + ag * Qe + 8 * U * big
    dX, dX_tol = np.zeros((n, H)), np.zeros((n, H))
    dX[node[inside]] = (D @ W)[inside]
    dX_tol[node[inside]] = ((rel + (V + K) * U * big) @ np.abs(W))[inside]
    tolw = rel + (R + 8) * U * big
    return dict(loss=loss, loss_tol=loss_tol, lse=lse, lse_tol=lse_tol, dX=dX, dX_tol=dX_tol, dW=D.T @ x,
                dW_tol=tolw.T @ np.abs(x), db=D.sum(0), db_tol=tolw.sum(0))


def apply_rules(z, rules):
    """Logits [R][V] after the rules (a dict as NodeTokens takes them, lists per row), in 64 bits."""
    z = np.array(z, np.float64)
    R, V = z.shape
    for r in range(R):
        seen = np.asarray(rules["seen"][r] if rules.get("seen") else [], np.int64)
        seen = seen[(seen >= 0) & (seen < V)]
        tok, times = np.unique(seen, return_counts=True)
        v = z[r, tok]
        rho = rules.get("repetition", 1.0)
        v = np.where(v > 0, v / rho, v * rho)
        z[r, tok] = v - (rules.get("presence", 0.0) + rules.get("frequency", 0.0) * times)
        for t, a in (rules["add"][r] if rules.get("add") else []):
            if 0 <= t < V:
                z[r, t] += a
        mask, of = rules.get("mask"), rules.get("mask_of")
        m = -1 if mask is None else (r if of is None else int(of[r]))
        if mask is not None and 0 <= m < len(mask):
            z[r, ~np.asarray(mask[m], bool)] = -np.inf
    return z


def best(z, K):
    """(ids, logits): the K largest of each row, equal ones by the lower id; -1 and -inf beyond."""
    R, V = z.shape
    o = np.argsort(-np.where(np.isnan(z), -np.inf, z), axis=1, kind="stable")[:, :K]
    zk = np.take_along_axis(z, o, 1)
    gone = ~(zk > -np.inf)
    ids, zk = np.where(gone, -1, o), np.where(gone, -np.inf, zk)
    pad = ((0, 0), (0, K - ids.shape[1]))
    return np.pad(ids, pad, constant_values=-1).astype(np.int64), np.pad(zk, pad, constant_values=-np.inf)
