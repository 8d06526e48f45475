"""64-bit references of the token operators (numpy), with the bounds that the
GPU tests hold the kernels to (no test functions here).

Bounds are first-order worst cases of the stated arithmetic: u = 2^-24 per
float32 operation, 2^-16 for a value kept as a bf16 pair (8 significant bits:
2^-8 of the value for the first, 2^-8 of that for the second) and 2^-21 for an
exponential (argument and hardware function).  A result rounded to bf16 has to
be the rounding of some value within the float32 bound."""
import numpy as np

U = 2.0 ** -24
LOWEST = float(np.finfo(np.float32).min)


def philox7(block, offset, seed):
    """[n, 4] uint32 words of the 7-round Philox4x32 blocks at counters (block, offset) under key seed."""
    u = np.uint64
    lo = u(0xFFFFFFFF)
    block = np.asarray(block, np.uint64)
    c = [block & lo, block >> u(32), np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(7):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        k0, k1 = u((k[0] + r * 0x9E3779B9) & 0xFFFFFFFF), u((k[1] + r * 0xBB67AE85) & 0xFFFFFFFF)
        c = [(b >> u(32)) ^ c[1] ^ k0, b & lo, (a >> u(32)) ^ c[3] ^ k1, a & lo]
    return np.stack(c, 1).astype(np.uint32)


def keep_factor(first, count, p, seed, offset):
    """1 / (1 - p) where element first .. first + count - 1 stays, else 0."""
    cut = min(round(p * 65536), 65535)
    b0, b1 = first // 8, (first + count + 7) // 8
    w = philox7(np.arange(b0, b1, dtype=np.uint64), offset, seed)
    h = np.stack([w & 0xFFFF, w >> 16], 2).reshape(-1)[first - 8 * b0:][:count]
    return np.where(h >= cut, 65536.0 / (65536 - cut), 0.0)


def lists(n, tok_ptr, n_tok):
    """(row, position) of every listed token, in order, and the lists' lengths."""
    if tok_ptr is None:
        k = np.arange(n_tok)
        return k, k, (np.arange(n) < n_tok).astype(np.int64)
    lens = np.diff(np.asarray(tok_ptr, np.int64))
    return np.repeat(np.arange(n), lens), np.arange(tok_ptr[0], tok_ptr[-1]), lens


def embed(table, n, tok_ptr, tok, n_tok, scale, mean, p, seed, offset):
    """(X, sum of the terms' magnitudes, list lengths)."""
    V, H = table.shape
    row, pos, lens = lists(n, tok_ptr, n_tok)
    ids = np.asarray(tok, np.int64)[pos]
    ok = (ids >= 0) & (ids < V)
    X, A = np.zeros((n, H)), np.zeros((n, H))
    np.add.at(X, row[ok], table[ids[ok]])
    np.add.at(A, row[ok], np.abs(table[ids[ok]]))
    c = (scale / np.maximum(lens, 1) if mean else np.full(n, scale))[:, None]
    k = keep_factor(0, n * H, p, seed, offset).reshape(n, H)
    return X * c * k, A * np.abs(c) * k, lens


def embed_grad(dX, V, tok_ptr, tok, n_tok, scale, mean, p, seed, offset):
    """(dtable, sum of the terms' magnitudes, listings of each token)."""
    n, H = dX.shape
    row, pos, lens = lists(n, tok_ptr, n_tok)
    ids = np.asarray(tok, np.int64)[pos]
    ok = (ids >= 0) & (ids < V)
    c = (scale / np.maximum(lens, 1) if mean else np.full(n, scale))[:, None]
    G = dX * c * keep_factor(0, n * H, p, seed, offset).reshape(n, H)
    D, A = np.zeros((V, H)), np.zeros((V, H))
    np.add.at(D, ids[ok], G[row[ok]])
    np.add.at(A, ids[ok], np.abs(G[row[ok]]))
    return D, A, np.bincount(ids[ok], minlength=V)


def vocab(X, W, bias, node, target, weight, scale, dt):
    """Losses, lse, best entries and gradients of the chosen nodes, with a bound for each floating result."""
    n, H = X.shape
    V = W.shape[0]
    node, target = np.asarray(node, np.int64), np.asarray(target, np.int64)
    R = len(node)
    inside = (node >= 0) & (node < n)
    x = np.where(inside[:, None], X[np.where(inside, node, 0)], 0.0)
    b = np.zeros(V) if bias is None else np.where(bias <= -1e30, -np.inf, bias)
    z = x @ W.T + b
    dz = (H + 4) * U * (np.abs(x) @ np.abs(W).T + np.where(np.isfinite(b), np.abs(b), 0.0))   # of a logit
    best = np.where(np.isfinite(z).any(1), np.argmax(z, 1), -1)
    top = np.where(np.isfinite(z.max(1)), z.max(1), 0.0)
    e = np.exp(z - top[:, None])
    s = e.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(s > 0, top + np.log(s), -np.inf)
    live = np.where(np.isfinite(z), dz, 0.0).max(1)
    fin = np.where(np.isfinite(lse), lse, 0.0)
    lse_tol = live + 2.0 ** -21 + V / 2 * U + 8 * U * (1 + np.abs(fin) + np.abs(top))
    has = inside & (target >= 0) & (target < V)
    t = np.where(has, target, 0)
    zt = z[np.arange(R), t]
    loss = np.where(has, np.where(s > 0, lse - np.where(np.isfinite(zt), zt, -np.inf), np.inf), 0.0)
    loss[inside & (target >= V)] = np.nan
    loss_tol = lse_tol + dz[np.arange(R), t] + 4 * U * np.abs(np.where(np.isfinite(zt), zt, 0.0))
    # gradients
    g = np.where(has & (s > 0), scale * (np.ones(R) if weight is None else weight), 0.0)
    P = np.where((s > 0)[:, None], e / np.maximum(s, 1e-300)[:, None], 0.0)
    one = np.zeros_like(P)
    one[np.arange(R), t] = 1.0
    D = g[:, None] * (P - one)
    pair = 2.0 ** -16 if dt == "bf16" else 0.0
    eps = (2 * live + lse_tol + 2.0 ** -20 + pair)[:, None]   # relative, of a probability
    big = np.abs(g)[:, None] * (P + one)
    dX = np.zeros((n, H))
    dX_tol = np.zeros((n, H))
    dX[node[inside]] = (D @ W)[inside]
    dX_tol[node[inside]] = ((np.abs(g)[:, None] * P * (eps + (V + 8) * U) + 8 * U * big) @ np.abs(W))[inside]
    dW = D.T @ x
    dW_tol = (big * (eps + (R + 8) * U)).T @ np.abs(x)
    db = D.sum(0)
    db_tol = (big * (eps + (R + 8) * U)).sum(0)
    return dict(loss=loss, loss_tol=loss_tol, lse=lse, lse_tol=lse_tol, best=best, dX=dX, dX_tol=dX_tol, dW=dW,
                dW_tol=dW_tol, db=db, db_tol=db_tol)


def within_rounded(got, want, tol, dt):
    """within(), for a result stored in dt: rounding is monotone, so it lies between the roundings of the bound's ends."""
    if dt == "f32":
        return within(got, want, tol)
    from ggnn_synth import round_bf16
    got = np.asarray(got, np.float64)
    assert np.all(np.isfinite(got)) and np.all(got >= round_bf16(want - tol)) and np.all(got <= round_bf16(want + tol))


def within(got, want, tol):
    """Where finite, |got - want| <= tol; elsewhere the same infinity or NaN."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    err = np.abs(got - want)[fin]
    tol = np.broadcast_to(tol, want.shape)[fin]
    assert np.all(np.isfinite(got[fin]))
    bad = err > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.size} outside, worst {float((err / np.maximum(tol, 1e-300)).max()):.3g} of the bound"
