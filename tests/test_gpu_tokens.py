"""Token operators on the GPU against 64-bit references: dropout bit for bit,
the token table's lookup and gradient, the cross entropy over a vocabulary
and its gradients, at the sizes and values where tiles, lists and masks end."""
import numpy as np
import pytest

import token_reference as R
from gpu_helpers import dev, host, round_to, say, torch_dt

capi = pytest.importorskip("paper_1906_11786_amd.capi")
torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def scratch(nbytes):
    """Workspace filled with a pattern: nothing may depend on what it held."""
    return torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------- dropout

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("count", [1, 7, 8, 9, 2047, 2048, 2049, 100003])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99999])
def test_dropout_is_the_generators_mask(dt, count, p):
    say(f"dropout dt={dt} count={count} p={p}")
    rng = np.random.default_rng(count)
    seed, offset = int(rng.integers(0, 2**64, dtype=np.uint64)), int(rng.integers(0, 2**64, dtype=np.uint64))
    x = rng.standard_normal(count)
    X = dev(round_to(dt, x), dt)
    Y = torch.full((count + 8,), 7.0, device="cuda").to(torch_dt(dt))
    capi.ggnn_dropout(dt, count, X, p, seed, offset, Y)
    k = torch.from_numpy(R.keep_factor(0, count, p, seed, offset).astype(np.float32)).cuda()
    want = torch.where(k > 0, X.float() * k, 0.0).to(torch_dt(dt))
    assert torch.equal(Y[:count], want)
    assert torch.equal(Y[count:].float(), torch.full((8,), 7.0, device="cuda"))   # nothing beyond the count
    capi.ggnn_dropout(dt, count, X, p, seed, offset, X)   # in place
    assert torch.equal(X, want)


def test_dropout_drops_what_is_not_finite_and_keeps_its_share():
    n = 1 << 20
    X = torch.full((n,), float("nan"), device="cuda")
    Y = torch.empty_like(X)
    capi.ggnn_dropout("f32", n, X, 0.25, 3, 4, Y)
    kept = torch.isnan(Y)
    assert torch.equal(Y[~kept], torch.zeros_like(Y[~kept]))
    # binomial, 6 standard deviations
    assert abs(float(kept.double().mean()) - 0.75) < 6 * (0.25 * 0.75 / n) ** 0.5
    Z = torch.ones((n,), device="cuda")
    capi.ggnn_dropout("f32", n, Z, 0.25, 3, 5, Z)      # another offset: another mask
    other = Z > 0
    agree = float((other == kept).double().mean())
    assert abs(agree - (0.75**2 + 0.25**2)) < 6 * (0.625 * 0.375 / n) ** 0.5


def test_dropout_numbers_elements_past_32_bits():
    n = (1 << 32) + 21
    X = torch.ones((n,), dtype=torch.bfloat16, device="cuda")
    capi.ggnn_dropout("bf16", n, X, 0.5, 11, 12, X)
    for first in (0, (1 << 32) - 16, (1 << 32) + 5):
        k = R.keep_factor(first, 16, 0.5, 11, 12)
        assert np.array_equal(host(X[first:first + 16]), k)


# -------------------------------------------------------------------- lookup

def bags(rng, n, most, V, wild):
    """tok_ptr, tok: lists of 0 .. most tokens (frequent ones first), some ids out of range when wild."""
    lens = rng.integers(0, most + 1, n)
    lens[rng.random(n) < 0.2] = 0
    ptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    tok = np.minimum((V ** rng.random(max(int(ptr[-1]), 1))).astype(np.int64) - 1, V - 1)
    tok = np.maximum(tok, 0)
    if wild:
        at = rng.random(len(tok)) < 0.1
        tok[at] = rng.choice([-1, V, V + 5, 2**31 - 1, -2**31], size=int(at.sum()))
    return ptr, tok.astype(np.int32)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H", [32, 64, 128, 256])
@pytest.mark.parametrize("n,most,V,p,mean", [(1, 1, 1, 0.0, False), (33, 5, 7, 0.3, True), (1000, 9, 401, 0.1, True),
                                            (257, 40, 50, 0.0, False)])
def test_lookup_of_lists(dt, H, n, most, V, p, mean):
    say(f"embed dt={dt} H={H} n={n} V={V}")
    rng = np.random.default_rng(n + H)
    ptr, tok = bags(rng, n, most, V, wild=V > 1)
    table = round_to(dt, rng.standard_normal((V, H)))
    X = torch.full((n, H), 9.0, device="cuda").to(torch_dt(dt))
    seed, offset = 2**63 + 5, 2**40 + 1
    capi.ggnn_embed(dt, n, H, V, dev(table, dt), ints(ptr), ints(tok), int(ptr[-1]), 1.5, mean, p, seed, offset, X)
    want, mag, lens = R.embed(table, n, ptr, tok, int(ptr[-1]), 1.5, mean, p, seed, offset)
    R.within_rounded(host(X), want, (lens[:, None] + 4) * R.U * mag, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,n_tok", [(1, 1), (1, 0), (100, 93), (4096, 4096)])
def test_lookup_of_one_token_a_node(dt, n, n_tok):
    rng = np.random.default_rng(n)
    H, V = 64, 90
    tok = rng.integers(-2, V + 2, max(n_tok, 1)).astype(np.int32)
    table = round_to(dt, rng.standard_normal((V, H)))
    X = torch.full((n, H), 9.0, device="cuda").to(torch_dt(dt))
    capi.ggnn_embed(dt, n, H, V, dev(table, dt), None, ints(tok), n_tok, -0.5, True, 0.1, 1, 2, X)
    want, mag, _ = R.embed(table, n, None, tok, n_tok, -0.5, True, 0.1, 1, 2)
    R.within_rounded(host(X), want, 4 * R.U * mag, dt)


def test_lookup_with_dropout_is_lookup_then_dropout():
    rng = np.random.default_rng(0)
    n, H, V = 500, 128, 77
    ptr, tok = bags(rng, n, 6, V, wild=False)
    table = dev(rng.standard_normal((V, H)))
    A, B = torch.empty((n, H), device="cuda"), torch.empty((n, H), device="cuda")
    capi.ggnn_embed("f32", n, H, V, table, ints(ptr), ints(tok), int(ptr[-1]), 2.0, True, 0.4, 9, 8, A)
    capi.ggnn_embed("f32", n, H, V, table, ints(ptr), ints(tok), int(ptr[-1]), 2.0, True, 0.0, 9, 8, B)
    capi.ggnn_dropout("f32", n * H, B, 0.4, 9, 8, B)
    assert torch.equal(A, B)


def embed_bwd(n, H, V, ptr, tok, n_tok, scale, mean, p, seed, offset, dX, dtable):
    need = capi.ggnn_embed_bwd_workspace_bytes(n, H, V, n_tok)
    capi.ggnn_embed_bwd(n, H, V, None if ptr is None else ints(ptr), ints(tok), n_tok, scale, mean, p, seed, offset,
                        dX, dtable, scratch(need), need)


def check_embed_bwd(n, H, V, ptr, tok, n_tok, mean, p, seed=0):
    rng = np.random.default_rng(seed)
    dX = round_to("f32", rng.standard_normal((n, H)))
    start = round_to("f32", rng.standard_normal((V, H)))
    got = [dev(start) for _ in range(2)]
    for d in got:
        embed_bwd(n, H, V, ptr, tok, n_tok, 0.75, mean, p, 21, 22, dev(dX), d)
    assert torch.equal(got[0], got[1])   # same bits again
    want, mag, cnt = R.embed_grad(dX, V, ptr, tok, n_tok, 0.75, mean, p, 21, 22)
    R.within(host(got[0]), start + want, (cnt[:, None] + 6) * R.U * (mag + np.abs(start)))
    rest = cnt == 0
    assert np.array_equal(host(got[0])[rest], start[rest])


@pytest.mark.parametrize("H", [32, 64, 128, 256])
@pytest.mark.parametrize("n,V,p", [(1, 1, 0.0), (50, 3, 0.5), (700, 255, 0.0), (700, 256, 0.1), (1500, 70001, 0.1)])
def test_table_gradient_of_lists(H, n, V, p):
    say(f"embed_bwd H={H} n={n} V={V}")
    rng = np.random.default_rng(V)
    ptr, tok = bags(rng, n, 7, V, wild=V > 1)
    if ptr[-1] == 0:
        ptr[-1] = 1
    check_embed_bwd(n, H, V, ptr, tok, int(ptr[-1]), True, p)


@pytest.mark.parametrize("n_tok", [1, 31, 32, 33, 63, 64, 65, 2047, 2048, 2049, 9001])
@pytest.mark.parametrize("kind", ["same", "two", "many"])
def test_table_gradient_of_runs(n_tok, kind):
    """Runs that end at, before and after the ends of chunks and tiles; one token on every node."""
    say(f"embed_bwd n_tok={n_tok} {kind}")
    rng = np.random.default_rng(n_tok)
    V = {"same": 5, "two": 5, "many": 300000}[kind]
    tok = {"same": np.full(n_tok, 4), "two": rng.integers(0, 2, n_tok) * 3,
           "many": rng.integers(0, V, n_tok)}[kind].astype(np.int32)
    check_embed_bwd(n_tok + 3, 64, V, None, tok, n_tok, False, 0.0)


def test_table_gradient_of_long_runs():
    """A few tokens on most of 200,000 nodes (a run over thousands of chunks), at the widest rows too."""
    rng = np.random.default_rng(1)
    for H, n in ((32, 200000), (256, 60000)):
        say(f"embed_bwd long runs H={H}")
        tok = np.where(rng.random(n) < 0.7, 3, rng.integers(0, 40, n)).astype(np.int32)
        check_embed_bwd(n, H, 40, None, tok, n, False, 0.1)


def test_table_gradient_ignores_tokens_that_no_list_holds():
    n, H, V = 10, 32, 6
    ptr = np.array([2, 2, 4, 4, 4, 5, 5, 5, 5, 7, 7], np.int32)   # positions 0, 1 and 7, 8 are in no list
    tok = np.array([0, 1, 2, 3, 2, 5, 5, 1, 0], np.int32)
    check_embed_bwd(n, H, V, ptr, tok, 9, True, 0.0)


def test_table_gradient_matches_differences():
    """<dtable, D> against the change of the forward call's <X, G> along D: the map is linear, so one difference is
    exact up to rounding."""
    rng = np.random.default_rng(2)
    n, H, V = 300, 64, 50
    ptr, tok = bags(rng, n, 6, V, wild=True)
    G, D = rng.standard_normal((n, H)), rng.standard_normal((V, H))
    X = torch.empty((n, H), device="cuda")
    args = (int(ptr[-1]), 1.25, True, 0.2, 5, 6)
    capi.ggnn_embed("f32", n, H, V, dev(D), ints(ptr), ints(tok), *args, X)
    dt = torch.zeros((V, H), device="cuda")
    embed_bwd(n, H, V, ptr, tok, *args, dev(G), dt)
    G32, D32 = round_to("f32", G), round_to("f32", D)
    lhs, rhs = float((host(X) * G32).sum()), float((host(dt) * D32).sum())
    size = float((np.abs(host(X)) * np.abs(G32)).sum())
    assert abs(lhs - rhs) <= 64 * R.U * size


# ---------------------------------------------------------- vocabulary loss

def vocab_case(rng, dt, n, H, V, rows, bias, spread=2.0):
    X = round_to(dt, rng.standard_normal((n, H)))
    W = round_to(dt, rng.standard_normal((V, H)) * (spread / np.sqrt(H)))
    node = rng.permutation(n)[:rows].astype(np.int32)
    target = rng.integers(0, V, rows).astype(np.int32)
    b = round_to("f32", rng.standard_normal(V)) if bias else None
    return X, W, node, target, b


def run_vocab(dt, X, W, b, node, target, weight=None, scale=1.0, grad=True, best=False):
    n, H = X.shape
    V, rows = W.shape[0], len(target)
    dX_, dW_ = torch.full((n, H), 5.0, device="cuda"), torch.ones((V, H), device="cuda")
    db_ = torch.ones((V,), device="cuda")
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    bst = torch.full((rows,), -7, dtype=torch.int32, device="cuda") if best else None
    need = capi.ggnn_vocab_workspace_bytes(dt, H, rows, V, grad)
    common = (dt, n, H, rows, V, dev(X, dt), dev(W, dt), None if b is None else dev(b),
              None if node is None else ints(node), ints(target))
    if grad:
        capi.ggnn_vocab_loss_grad(*common, None if weight is None else dev(weight), scale, loss, lse, dX_, dW_, db_,
                                  scratch(need), need)
    else:
        capi.ggnn_vocab_loss(*common, loss, lse, bst, scratch(need), need)
    out = dict(loss=host(loss), lse=host(lse))
    if best:
        out["best"] = bst.cpu().numpy()
    if grad:
        out.update(dX=host(dX_), dW=host(dW_) - 1.0, db=host(db_) - 1.0)
    return out


def check_vocab(dt, X, W, b, node, target, weight=None, scale=1.0):
    want = R.vocab(X, W, b, np.arange(len(target)) if node is None else node, target, weight, scale, dt)
    plain = run_vocab(dt, X, W, b, node, target, grad=False)
    got = run_vocab(dt, X, W, b, node, target, weight, scale)
    again = run_vocab(dt, X, W, b, node, target, weight, scale)
    for k in got:
        assert np.array_equal(got[k], again[k], equal_nan=True), k
    for o in (plain, got):
        R.within(o["lse"], want["lse"], want["lse_tol"])
        R.within(o["loss"], want["loss"], want["loss_tol"])
    R.within(got["dX"], want["dX"], want["dX_tol"])
    for k in ("dW", "db"):   # added to ones
        R.within(got[k], want[k], want[k + "_tol"] + 4 * R.U * (1 + np.abs(want[k])))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H", [32, 64, 128, 256])
@pytest.mark.parametrize("rows,V", [(1, 1), (1, 1000), (5, 31), (31, 63), (32, 64), (33, 65), (127, 127), (129, 129),
                                    (300, 5003), (700, 300)])
def test_vocab_loss_and_gradients(dt, H, rows, V):
    say(f"vocab dt={dt} H={H} rows={rows} V={V}")
    rng = np.random.default_rng(rows * 7 + V)
    X, W, node, target, b = vocab_case(rng, dt, rows + 13, H, V, rows, bias=rows % 2 == 1)
    check_vocab(dt, X, W, b, node, target, scale=1.0 / rows)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_vocab_ignored_rows_weights_and_ids_out_of_range(dt):
    rng = np.random.default_rng(4)
    X, W, node, target, b = vocab_case(rng, dt, 400, 64, 777, 200, bias=True)
    target[::3] = -1
    target[5] = -2**31
    target[7], target[8] = 777, 2**31 - 1
    node[10], node[11] = -1, 400
    weight = round_to("f32", rng.standard_normal(200))   # negative ones and a zero among them
    weight[20] = 0.0
    check_vocab(dt, X, W, b, node, target, weight, scale=-0.5)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_vocab_without_a_node_list_takes_the_first_rows(dt):
    rng = np.random.default_rng(5)
    X, W, _, target, b = vocab_case(rng, dt, 150, 32, 200, 140, bias=False)
    check_vocab(dt, X, W, b, None, target)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 130])
@pytest.mark.parametrize("low", [-np.inf, R.LOWEST, -1e30])
def test_vocab_masked_entries(dt, rows, low):
    """Entries taken out by their bias, a masked target among them; then all but one; then every entry."""
    rng = np.random.default_rng(6)
    X, W, node, target, b = vocab_case(rng, dt, 140, 64, 300, rows, bias=True)
    b[rng.random(300) < 0.5] = low
    b[250:] = low            # whole tiles too
    target[0], target[1] = 250, int(np.argmax(b))
    check_vocab(dt, X, W, b, node, target)
    b[:] = low
    b[77] = 0.25
    target[2] = 77
    check_vocab(dt, X, W, b, node, target)
    b[77] = low
    check_vocab(dt, X, W, b, node, target)
    assert np.all(run_vocab(dt, X, W, b, node, target, grad=False, best=True)["best"] == -1)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [2, 200])
def test_vocab_large_logits(dt, rows):
    """Logits of several hundred, growing along the vocabulary: the running maximum moves often."""
    rng = np.random.default_rng(7)
    X, W, node, target, b = vocab_case(rng, dt, 210, 128, 900, rows, bias=True, spread=60.0)
    b += np.linspace(-300, 300, 900)
    b = round_to("f32", b)
    check_vocab(dt, X, W, b, node, target)


@pytest.mark.parametrize("rows", [1, 200])
def test_vocab_nan_stays_in_its_row(rows):
    rng = np.random.default_rng(8)
    X, W, node, target, b = vocab_case(rng, "f32", 210, 64, 500, 200, bias=False)
    node, target = node[:rows], target[:rows]
    X[node[0], 3] = np.nan
    o = run_vocab("f32", X, W, None, node, target, grad=False)
    assert np.isnan(o["loss"][0]) and np.isnan(o["lse"][0])
    assert np.all(np.isfinite(o["loss"][1:])) and np.all(np.isfinite(o["lse"][1:]))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("weighted", [False, True])
def test_vocab_ignored_rows_may_hold_anything(dt, weighted):
    """NaN and infinite states, and NaN weights, of rows without a target leave every gradient as if they were zero."""
    rng = np.random.default_rng(10)
    X, W, node, target, b = vocab_case(rng, dt, 400, 64, 500, 300, bias=True)
    weight = round_to("f32", rng.standard_normal(300)) if weighted else None
    target[::5] = -1
    out = np.arange(0, 300, 5)
    X[node[out]] = 0.0
    want = R.vocab(X, W, b, node, target, weight, 0.5, dt)
    X[node[out[::2]], 3], X[node[out[1::2]], 60] = np.nan, np.inf
    if weighted:
        weight[out] = np.nan
    got = run_vocab(dt, X, W, b, node, target, weight, 0.5)
    keep = np.delete(np.arange(300), out)
    R.within(got["loss"], want["loss"], want["loss_tol"])
    R.within(got["lse"][keep], want["lse"][keep], want["lse_tol"][keep])
    R.within(got["dX"], want["dX"], want["dX_tol"])
    for k in ("dW", "db"):   # added to ones
        R.within(got[k], want[k], want[k + "_tol"] + 4 * R.U * (1 + np.abs(want[k])))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H", [32, 256])
@pytest.mark.parametrize("rows,V", [(1, 40), (32, 3000), (33, 3000), (300, 1001)])
def test_vocab_best_entry_ties_go_to_the_lowest(dt, H, rows, V):
    """Small whole numbers: every logit is exact and many are equal."""
    rng = np.random.default_rng(9)
    X = rng.integers(-1, 2, (rows + 5, H)).astype(np.float64)
    W = rng.integers(-1, 2, (V, H)).astype(np.float64)
    W[V // 2:] = W[:V - V // 2]          # every entry has an equal one
    node = rng.permutation(rows + 5)[:rows].astype(np.int32)
    b = rng.integers(-3, 4, V).astype(np.float64)
    b[V // 2:] = b[:V - V // 2]
    b[rng.random(V) < 0.3] = -np.inf
    o = run_vocab(dt, X, W, b, node, np.zeros(rows, np.int32), grad=False, best=True)
    assert np.array_equal(o["best"], np.argmax(X[node] @ W.T + b, 1))


def test_vocab_no_rows_and_no_targets():
    X, W = torch.randn((40, 32), device="cuda"), torch.randn((90, 32), device="cuda")
    dX, dW = torch.ones((40, 32), device="cuda"), torch.ones((90, 32), device="cuda")
    capi.ggnn_vocab_loss_grad("f32", 40, 32, 0, 90, X, W, None, None, None, None, 1.0, None, None, dX, dW, None, None, 0)
    assert not dX.any() and torch.equal(dW, torch.ones_like(dW))
    capi.ggnn_vocab_loss("f32", 40, 32, 0, 90, X, W, None, None, None, None, None, None, None, 0)
    lse, best = torch.empty((40,), device="cuda"), torch.empty((40,), dtype=torch.int32, device="cuda")
    need = capi.ggnn_vocab_workspace_bytes("f32", 32, 40, 90, False)
    capi.ggnn_vocab_loss("f32", 40, 32, 40, 90, X, W, None, None, None, None, lse, best, scratch(need), need)
    z = host(X) @ host(W).T
    R.within(host(lse), np.log(np.exp(z).sum(1)), 1e-4)
    assert np.array_equal(best.cpu().numpy(), np.argmax(z, 1))


def test_vocab_gradients_match_differences():
    """Central differences of the summed loss along random directions of X, W and the bias: the loss is off by at most
    its bound, the quotient by the third derivative too (|d3 loss| <= 8 |dz|^3 along a line)."""
    rng = np.random.default_rng(10)
    X, W, node, target, b = vocab_case(rng, "f32", 60, 64, 211, 50, bias=True)
    got = run_vocab("f32", X, W, b, node, target)
    want = R.vocab(X, W, b, node, target, None, 1.0, "f32")
    h = 1.0 / 64
    for name in ("X", "W", "b"):
        D = rng.standard_normal({"X": X, "W": W, "b": b}[name].shape)
        D = round_to("f32", D / np.abs(D).max())
        up, dn = [], []
        for sgn, out in ((1, up), (-1, dn)):
            q = {"X": X, "W": W, "b": b}
            q[name] = round_to("f32", q[name] + sgn * h * D)
            out.append(run_vocab("f32", q["X"], q["W"], q["b"], node, target, grad=False)["loss"].sum())
        diff = (up[0] - dn[0]) / (2 * h)
        dot = float((got["d" + name] * D).sum())
        dz = np.abs(D[node] @ W.T if name == "X" else X[node] @ D.T if name == "W" else D).max()
        rounding = float((np.abs(got["d" + name]) * R.U * (1 + np.abs({"X": X, "W": W, "b": b}[name]))).sum()) / h
        tol = want["loss_tol"].sum() / h + 50 * 8 * dz**3 * h**2 / 6 + rounding
        say(f"differences along {name}: {diff:.6g} against {dot:.6g}, bound {tol:.3g}")
        assert abs(diff - dot) <= tol


# ------------------------------------------------------- streams and graphs

def test_token_calls_in_a_captured_graph_on_a_side_stream():
    """Lookup, dropout, loss with gradients and the table's gradient recorded once and replayed with other work in
    between: every replay gives the eager bits."""
    rng = np.random.default_rng(11)
    n, H, V, rows = 640, 64, 901, 150
    ptr, tok = bags(rng, n, 5, V, wild=False)
    ptr_d, tok_d, n_tok = ints(ptr), ints(tok), int(ptr[-1])
    table = dev(round_to("bf16", rng.standard_normal((V, H)) * 0.3), "bf16")
    node, target = ints(rng.permutation(n)[:rows]), ints(rng.integers(0, V, rows))
    X = torch.empty((n, H), dtype=torch.bfloat16, device="cuda")
    Y = torch.empty_like(X)
    dX, dT = torch.empty((n, H), device="cuda"), torch.empty((V, H), device="cuda")
    loss, lse = torch.empty((rows,), device="cuda"), torch.empty((rows,), device="cuda")
    w1, w2 = capi.ggnn_vocab_workspace_bytes("bf16", H, rows, V, True), capi.ggnn_embed_bwd_workspace_bytes(n, H, V, n_tok)
    ws1, ws2 = scratch(w1), scratch(w2)

    def step():
        dT.zero_()
        capi.ggnn_embed("bf16", n, H, V, table, ptr_d, tok_d, n_tok, 1.0, True, 0.1, 1, 2, X)
        capi.ggnn_dropout("bf16", n * H, X, 0.2, 1, 3, Y)
        capi.ggnn_vocab_loss_grad("bf16", n, H, rows, V, Y, table, None, node, target, None, 1.0 / rows, loss, lse, dX,
                                  dT, None, ws1, w1)
        capi.ggnn_dropout("f32", n * H, dX, 0.2, 1, 3, dX)
        capi.ggnn_embed_bwd(n, H, V, ptr_d, tok_d, n_tok, 1.0, True, 0.1, 1, 2, dX, dT, ws2, w2)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (X, Y, dX, dT, loss, lse)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    for i in range(4):
        for t in (X, Y, dX, loss, lse):
            t.fill_(float(i))
        torch.randn((1000, 1000), device="cuda").sum().item()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((X, Y, dX, dT, loss, lse), want):
            assert torch.equal(t, w)


# ------------------------------------- sizes that start the other large forms

def large_reference(X, W, b, node, target, weight, scale, dt):
    """R.vocab's results and bounds (dX, dW, db, lse) in float64 on the GPU."""
    f = (lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float64)).cuda())
    x, Wd, t = f(X[node]), f(W), torch.from_numpy(target.astype(np.int64)).cuda()
    H, V, rows = X.shape[1], W.shape[0], len(node)
    Wt = Wd.t().contiguous()
    z = torch.mm(x, Wt) + (0.0 if b is None else f(b))
    dz = (H + 4) * R.U * (torch.mm(x.abs(), Wt.abs()).amax(1) + (0.0 if b is None else float(np.abs(b).max())))
    lse = torch.logsumexp(z, 1)
    lse_tol = dz + 2.0**-21 + V / 2 * R.U + 16 * R.U * (1 + lse.abs() + z.abs().amax(1))
    has = t >= 0
    g = torch.where(has, scale * (torch.ones(rows, device="cuda").double() if weight is None else f(weight)), 0.0)
    P = torch.exp(z - lse[:, None])
    del z
    D = g[:, None] * P
    at = (torch.arange(rows, device="cuda"), t.clamp(min=0))
    eps = 2 * dz + lse_tol + 2.0**-20 + (2.0**-16 if dt == "bf16" else 0.0)
    dX_tol = torch.mm(D.abs() * (eps[:, None] + (V + 8) * R.U), Wd.abs())
    big = D.abs()
    D[at] -= g
    big[at] += g.abs()
    dX_tol += 8 * R.U * torch.mm(big, Wd.abs())
    big *= (eps + (rows + 8) * R.U)[:, None]
    bigT, DT = big.t().contiguous(), D.t().contiguous()
    c = (lambda a: a.cpu().numpy())
    return dict(lse=c(lse), lse_tol=c(lse_tol), dX=c(torch.mm(D, Wd)), dX_tol=c(dX_tol), dW=c(torch.mm(DT, x)),
                dW_tol=c(torch.mm(bigT, x.abs())), db=c(D.sum(0)), db_tol=c(big.sum(0)))


@pytest.mark.parametrize("dt,H,rows,V,bias,weighted", [
    ("bf16", 256, 33500, 333, True, False),    # whole 128-tiles of rows for every worker, then the rest
    ("bf16", 256, 300, 33500, False, False),   # and of entries
    ("f32", 128, 300, 33500, True, True),
    ("bf16", 256, 33100, 4900, True, False),   # rows sorted by target
    ("bf16", 64, 65600, 9800, False, True),
    ("f32", 256, 33100, 4900, False, True),
    ("bf16", 64, 65600, 24500, True, True),
    ("bf16", 128, 33100, 12300, False, False),
])
def test_vocab_large_forms(dt, H, rows, V, bias, weighted):
    say(f"vocab large dt={dt} H={H} rows={rows} V={V}")
    rng = np.random.default_rng(V)
    X, W, node, target, b = vocab_case(rng, dt, rows + 100, H, V, rows, bias)
    target = np.where(rng.random(rows) < 0.3, 5, target).astype(np.int32)   # a frequent target
    target[::9] = -1
    weight = round_to("f32", rng.standard_normal(rows)) if weighted else None
    want = large_reference(X, W, b, node, target, weight, 2.0 / rows, dt)
    got = run_vocab(dt, X, W, b, node, target, weight, 2.0 / rows)
    again = run_vocab(dt, X, W, b, node, target, weight, 2.0 / rows)
    for k in got:
        assert np.array_equal(got[k], again[k]), k
    R.within(got["lse"], want["lse"], want["lse_tol"])
    R.within(got["dX"][node], want["dX"], want["dX_tol"])
    rest = np.ones(len(X), bool)
    rest[node] = False
    assert not got["dX"][rest].any()
    for k in ("dW", "db"):   # added to ones
        R.within(got[k], want[k], want[k + "_tol"] + 4 * R.U * (1 + np.abs(want[k])))
    plain = run_vocab(dt, X, W, b, node, target, grad=False)
    R.within(plain["lse"], want["lse"], want["lse_tol"])


def check_large(dt, H, rows, V, bias, weighted=False):
    """As test_vocab_large_forms, the losses too."""
    rng = np.random.default_rng(V)
    X, W, node, target, b = vocab_case(rng, dt, rows + 100, H, V, rows, bias)
    target[::9] = -1
    weight = round_to("f32", rng.standard_normal(rows)) if weighted else None
    want = large_reference(X, W, b, node, target, weight, 2.0 / rows, dt)
    has = target >= 0
    t = np.where(has, target, 0)
    zt = (X[node] * W[t]).sum(1) + (0.0 if b is None else b[t])
    zt_tol = (H + 4) * R.U * ((np.abs(X[node]) * np.abs(W[t])).sum(1) + (0.0 if b is None else np.abs(b[t])))
    loss = np.where(has, want["lse"] - zt, 0.0)
    loss_tol = want["lse_tol"] + zt_tol + 4 * R.U * np.abs(zt)
    got = run_vocab(dt, X, W, b, node, target, weight, 2.0 / rows)
    plain = run_vocab(dt, X, W, b, node, target, grad=False)
    for o in (got, plain):
        R.within(o["lse"], want["lse"], want["lse_tol"])
        R.within(o["loss"], loss, loss_tol)
    R.within(got["dX"][node], want["dX"], want["dX_tol"])
    rest = np.ones(len(X), bool)
    rest[node] = False
    assert not got["dX"][rest].any()
    for k in ("dW", "db"):   # added to ones
        R.within(got[k], want[k], want[k + "_tol"] + 4 * R.U * (1 + np.abs(want[k])))


@pytest.mark.parametrize("dt,H,rows,V", [
    ("bf16", 256, 256 * 128 + 5, 2570),    # one 128-tile of rows more than there are workgroups, cut into many shares
    ("bf16", 256, 300, 256 * 128 + 3),     # and of entries
    ("f32", 256, 256 * 128 + 1, 333),
    ("f32", 128, 1000, 256 * 128 + 130),
    ("bf16", 64, 768 * 128 + 9, 1500),
])
def test_vocab_one_left_over_tile(dt, H, rows, V):
    say(f"vocab left-over tile dt={dt} H={H} rows={rows} V={V}")
    check_large(dt, H, rows, V, bias=True)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 130])
@pytest.mark.parametrize("low", [-3e9, -1e10, -7.7e10, -1e15, -1e20, -9.9e29])
def test_vocab_very_low_logits_have_no_weight(dt, rows, low):
    """Biases far below the others, short of those that take an entry out, on the first entries and scattered: the
    results are those without these entries, whose exponentials vanish."""
    rng = np.random.default_rng(12)
    for H in (64, 256):
        X, W, node, target, b = vocab_case(rng, dt, 140, H, 300, rows, bias=True)
        far = rng.random(300) < 0.3
        far[:70] = True
        target[far[target]] = 299
        far[299] = False
        b[far] = np.float32(low) * (1 + rng.random(int(far.sum()))).astype(np.float32)
        b[3] = low
        b = np.maximum(round_to("f32", b), -9.9e29)
        want = R.vocab(X, W, np.where(far, -np.inf, b), node, target, None, 1.0, dt)
        got = run_vocab(dt, X, W, b, node, target)
        plain = run_vocab(dt, X, W, b, node, target, grad=False, best=True)
        for o in (got, plain):
            R.within(o["lse"], want["lse"], want["lse_tol"])
            R.within(o["loss"], want["loss"], want["loss_tol"])
        assert np.array_equal(plain["best"], want["best"])
        R.within(got["dX"], want["dX"], want["dX_tol"])
        for k in ("dW", "db"):   # added to ones
            R.within(got[k], want[k], want[k + "_tol"] + 4 * R.U * (1 + np.abs(want[k])))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 130])
@pytest.mark.parametrize("size", [-1e8, 1e8, -7.7e10, 7.7e10, -1e20, 1e20, -9e29])
def test_vocab_logits_of_any_size(dt, rows, size):
    """Every logit of one size, up to a few float32 steps: their log sum is theirs, to the same steps, and dX is the
    mean row of W over equal entries less the target's."""
    rng = np.random.default_rng(13)
    X, W, node, target, b = vocab_case(rng, dt, 140, 64, 300, rows, bias=True)
    b[:] = size
    b[200:] = size if size in (-1e8, 1e8) else size - 40 * abs(size) * 2.0**-23
    b = round_to("f32", b)
    X *= 2.0**-10 if abs(size) == 1e8 else 1.0
    top = 300 if abs(size) == 1e8 else 200
    want = R.vocab(X, W, b, node, target, None, 1.0, dt)
    got = run_vocab(dt, X, W, b, node, target)
    plain = run_vocab(dt, X, W, b, node, target, grad=False, best=True)
    for o in (got, plain):
        R.within(o["lse"], want["lse"], want["lse_tol"])
        R.within(o["loss"], want["loss"], want["loss_tol"])
    assert np.all((plain["best"] >= 0) & (plain["best"] < top))
    dX = np.zeros_like(X)
    dX[node] = W[:top].mean(0) - W[target]
    R.within(got["dX"], dX, 1e-4 * np.abs(W).max())


@pytest.mark.parametrize("H", [32, 256])
@pytest.mark.parametrize("n_tok", [1, 7, 300, 2049])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_lists_are_cut_at_n_tok_both_ways(H, n_tok, p):
    """Offsets that pass n_tok, and some before 0: the lookup takes the mean over the tokens that remain, and the
    gradient divides by as many."""
    rng = np.random.default_rng(n_tok)
    n, V = 700, 50
    ptr = np.concatenate([[0], np.cumsum(rng.integers(0, 9, n))]).astype(np.int32) - 3
    ptr[0] = -3
    assert ptr[-1] > n_tok
    tok = rng.integers(0, V, n_tok).astype(np.int32)
    cut = np.clip(ptr, 0, n_tok)
    table = round_to("f32", rng.standard_normal((V, H)))
    X = torch.empty((n, H), device="cuda")
    capi.ggnn_embed("f32", n, H, V, dev(table), ints(ptr), ints(tok), n_tok, 1.5, True, p, 3, 4, X)
    want, mag, lens = R.embed(table, n, cut, tok, n_tok, 1.5, True, p, 3, 4)
    R.within(host(X), want, (lens[:, None] + 4) * R.U * mag)
    dX = round_to("f32", rng.standard_normal((n, H)))
    got = torch.zeros((V, H), device="cuda")
    embed_bwd(n, H, V, ptr, tok, n_tok, 1.5, True, p, 3, 4, dev(dX), got)
    want, mag, cnt = R.embed_grad(dX, V, cut, tok, n_tok, 1.5, True, p, 3, 4)
    R.within(host(got), want, (cnt[:, None] + 6) * R.U * mag)


def sparse_lists(kind, n, n_tok, V, rng):
    """n_tok tokens on a few of n nodes: the first ones, the first and the last ones, or ones spread over all."""
    lens = np.zeros(n, np.int64)
    if kind == "spread":
        lens[np.sort(rng.permutation(n)[:n_tok])] = 1
    else:
        half = n_tok if kind == "first" else n_tok // 2
        lens[:half] = 1
        lens[n - (n_tok - half):] += 1 if half < n_tok else 0
    ptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return ptr, rng.integers(0, V, n_tok).astype(np.int32)


@pytest.mark.parametrize("kind", ["first", "ends", "spread"])
@pytest.mark.parametrize("n,n_tok", [(300000, 3000), (300000, 5), (40000, 9000), (20000, 2048)])
def test_table_gradient_of_few_lists_among_many_nodes(kind, n, n_tok):
    say(f"embed_bwd {kind} n={n} n_tok={n_tok}")
    ptr, tok = sparse_lists(kind, n, n_tok, 77, np.random.default_rng(n_tok))
    check_embed_bwd(n, 32, 77, ptr, tok, n_tok, True, 0.1)


@pytest.mark.parametrize("kind", ["first", "ends", "spread"])
def test_table_gradient_takes_no_longer_for_nodes_without_tokens(kind):
    """3,000 tokens among 1M nodes against the same tokens on 3,008 nodes: no workgroup passes over all rows by itself
    (that took a barrier per 1,024 of them, hundreds of microseconds).  Medians of calls in turn."""
    H, V, n_tok = 32, 997, 3000
    rng = np.random.default_rng(3)
    cases = []
    for n, k in ((3008, "first"), (1 << 20, kind)):
        ptr, tok = sparse_lists(k, n, n_tok, V, rng)
        need = capi.ggnn_embed_bwd_workspace_bytes(n, H, V, n_tok)
        cases.append((n, ints(ptr), ints(tok), torch.zeros((n, H), device="cuda"), torch.zeros((V, H), device="cuda"),
                      scratch(need), need))
    us = [[], []]
    for i in range(40):
        for c, (n, ptr, tok, dX, dT, ws, need) in enumerate(cases):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(4):
                capi.ggnn_embed_bwd(n, H, V, ptr, tok, n_tok, 1.0, True, 0.0, 0, 0, dX, dT, ws, need)
            b.record()
            torch.cuda.synchronize()
            us[c].append(a.elapsed_time(b) * 250)
    few, many = np.median(us[0][10:]), np.median(us[1][10:])
    say(f"  3,008 nodes {few:.1f} us, 1M nodes {many:.1f} us")
    assert many <= 2 * few + 20


@pytest.mark.parametrize("V,p", [(70001, 0.1), (501, 0.0)])
def test_table_gradient_of_many_lists(V, p):
    """Above 524,288 listings (the scan of the tiles' counts takes more than one turn) in lists with long stretches of
    empty ones; three digits of token numbers, and two."""
    say(f"embed_bwd many lists V={V}")
    rng = np.random.default_rng(V)
    n = 400000
    lens = rng.integers(0, 6, n)
    lens[rng.random(n) < 0.2] = 0
    for at, size in ((0, 3000), (100000, 40000), (200000, 900), (n - 5000, 5000)):
        lens[at:at + size] = 0
    ptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    assert ptr[-1] > 524288
    tok = np.minimum((V ** rng.random(int(ptr[-1]))).astype(np.int64) - 1, V - 1).astype(np.int32)
    tok[rng.random(len(tok)) < 0.01] = V
    check_embed_bwd(n, 32, V, ptr, tok, int(ptr[-1]), True, p)


@pytest.mark.parametrize("dt,H,rows,V", [("bf16", 64, 300, 901), ("f32", 64, 300, 901), ("bf16", 256, 33100, 300),
                                         ("bf16", 256, 300, 33100), ("f32", 128, 300, 33100), ("bf16", 256, 33100, 4900)])
def test_vocab_gradients_without_the_biases_gradient(dt, H, rows, V):
    """dbias NULL, in every deal of the columns pass: what else is written has the same bits as with it."""
    rng = np.random.default_rng(rows)
    X, W, node, target, b = vocab_case(rng, dt, rows + 20, H, V, rows, bias=True)
    want = run_vocab(dt, X, W, b, node, target, scale=0.25)
    n = rows + 20
    dX, dW = torch.full((n, H), 5.0, device="cuda"), torch.ones((V, H), device="cuda")
    loss, lse = torch.empty((rows,), device="cuda"), torch.empty((rows,), device="cuda")
    need = capi.ggnn_vocab_workspace_bytes(dt, H, rows, V, True)
    capi.ggnn_vocab_loss_grad(dt, n, H, rows, V, dev(X, dt), dev(W, dt), dev(b), ints(node), ints(target), None, 0.25,
                              loss, lse, dX, dW, None, scratch(need), need)
    for got, k in ((loss, "loss"), (lse, "lse"), (dX, "dX"), (dW, "dW")):
        assert np.array_equal(host(got) - (1.0 if k == "dW" else 0.0), want[k]), k


@pytest.mark.parametrize("dt,H", [("bf16", 256), ("f32", 256), ("bf16", 128)])
def test_vocab_best_entry_where_a_workgroup_has_several_runs(dt, H):
    """More 128-tiles of rows than workgroups; small whole numbers, so that every logit is exact and many are equal."""
    rng = np.random.default_rng(14)
    rows, V = (256 if H == 256 else 768) * 128 + 300, 301
    X = rng.integers(-1, 2, (rows, H)).astype(np.float64)
    W = rng.integers(-1, 2, (V, H)).astype(np.float64)
    W[V // 2:] = W[:V - V // 2]
    b = rng.integers(-3, 4, V).astype(np.float64)
    b[V // 2:] = b[:V - V // 2]
    b[rng.random(V) < 0.3] = -np.inf
    o = run_vocab(dt, X, W, b, None, np.zeros(rows, np.int32), grad=False, best=True)
    assert np.array_equal(o["best"], np.argmax(X.astype(np.float32) @ W.T.astype(np.float32) + b, 1))
