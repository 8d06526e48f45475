"""The best entries of chosen rows over a vocabulary on the GPU, plain and under
rules, against 64-bit references: entry for entry where every logit is exact,
within the rounding of a float32 sum elsewhere."""
import numpy as np
import pytest

import logit_reference as L
import token_reference as R
from gpu_helpers import dev, host, round_to, say

capi = pytest.importorskip("paper_1906_11786_amd.capi")
torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def scratch(nbytes):
    """Workspace filled with a pattern: nothing may depend on what it held."""
    return torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device="cuda")


def packed(mask, words):
    """Bits of a boolean [masks][V] as int32 words."""
    bits = np.zeros((mask.shape[0], 32 * words), np.uint8)
    bits[:, :mask.shape[1]] = mask
    return np.packbits(bits, axis=1, bitorder="little").view("<i4")


def csr(lists):
    ptr = np.concatenate([[0], np.cumsum([len(x) for x in lists])])
    return ptr, [y for x in lists for y in x]


def struct(rules, V, extra=0):
    """(token_rules, tensors to keep, listed) of a rules dict."""
    keep, kw, listed = [], {}, 0

    def up(a, f=ints):
        keep.append(f(np.asarray(a)))
        return keep[-1]

    if rules.get("mask") is not None:
        words = -(-V // 32) + extra
        kw.update(mask=up(packed(np.asarray(rules["mask"], bool), words)), n_masks=len(rules["mask"]), mask_words=words)
        if rules.get("mask_of") is not None:
            kw["mask_of"] = up(rules["mask_of"])
    if rules.get("seen"):
        ptr, ids = csr(rules["seen"])
        if len(ids):
            kw.update(seen_ptr=up(ptr), seen=up(ids), n_seen=len(ids))
        kw.update({k: rules[k] for k in ("repetition", "presence", "frequency") if k in rules})
        listed += len(ids)
    if rules.get("add"):
        ptr, ids = csr(rules["add"])
        if len(ids):
            kw.update(add_ptr=up(ptr), add=up([t for t, _ in ids]), value=up([a for _, a in ids], dev), n_add=len(ids))
        listed += len(ids)
    return capi.token_rules(**kw), keep, listed


def run(dt, X, W, b, node, K, tau=1.0, rules=None, with_lse=True, rows=None):
    n, H = X.shape
    V = W.shape[0]
    rows = len(node) if rows is None else rows
    top, logit = torch.full((rows, K), -7, dtype=torch.int32, device="cuda"), torch.full((rows, K), 9.0, device="cuda")
    lse = torch.full((rows,), 9.0, device="cuda") if with_lse else None
    ru, keep, listed = (None, None, 0) if rules is None else struct(rules, V)
    need = capi.ggnn_vocab_top_workspace_bytes(dt, H, rows, V, K, listed)
    ws = scratch(need)
    capi.ggnn_vocab_top(dt, n, H, rows, V, dev(X, dt), dev(W, dt), None if b is None else dev(b),
                        None if node is None else ints(node), ru, tau, K, top, logit, lse, ws, need)
    torch.cuda.synchronize()
    return top.cpu().numpy().astype(np.int64), host(logit), None if lse is None else host(lse)


def exact_case(H, rows, V, seed, ties=False, n=None):
    """States, rows and biases on eight-bit grids: every logit is exact whatever the order of its sum."""
    rng = np.random.default_rng(seed)
    n = n or rows + 5
    sx, sw = (1.0, 1 / 2) if ties else (1 / 16, 1 / 64)
    grid = (lambda a, s: np.clip(np.round(a / s), -127, 127) * s)
    X = grid(rng.standard_normal((n, H)), sx)
    W = grid(rng.standard_normal((V, H)) * 1.5 / H ** 0.5, sw)
    b = grid(rng.standard_normal(V) * 0.5, sw)
    node = rng.permutation(n)[:rows]
    return X, W, b, node


def lse_bound(z, dz, tau):
    return L.log_sum(z / tau, dz / tau + 4 * R.U * np.abs(np.where(np.isfinite(z), z, 0.0)) / tau)


def check_exact(dt, X, W, b, node, K, tau=1.0, rules=None):
    z, dz, _, _ = L.logits(X, W, b, node)
    if rules is not None:
        z = L.apply_rules(z, rules)
    ids, zk = L.best(z, K)
    top, logit, lse = run(dt, X, W, b, node, K, tau, rules)
    np.testing.assert_array_equal(top, ids)
    # a division, a product and two sums of the penalties, each rounded
    R.within(logit, zk, 8 * R.U * (np.abs(np.where(np.isfinite(zk), zk, 0.0)) + 8))
    want, tol = lse_bound(z, dz, tau)
    R.within(lse, want, tol)
    t2, l2, _ = run(dt, X, W, b, node, K, tau, rules, with_lse=False)
    np.testing.assert_array_equal(t2, top)
    np.testing.assert_array_equal(l2, logit)


SIZES = [(1, 1, 1), (1, 17, 4), (3, 400, 64), (32, 1000, 8), (33, 33, 40), (64, 2049, 5), (65, 515, 64), (130, 4100, 16),
         (257, 129, 33), (300, 1, 2), (2100, 700, 12)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H", [32, 64, 128, 256])
@pytest.mark.parametrize("rows,V,K", SIZES)
def test_the_same_entries(dt, H, rows, V, K):
    say(f"top dt={dt} H={H} rows={rows} V={V} K={K}")
    X, W, b, node = exact_case(H, rows, V, seed=rows + V)
    check_exact(dt, X, W, b if H != 64 else None, node, K, tau=2.0)


@pytest.mark.parametrize("dt,V", [("bf16", 8000), ("bf16", 16001), ("bf16", 30011), ("bf16", 60013), ("f32", 60013)])
def test_many_rows_over_vocabularies_of_all_sizes(dt, V):
    """Enough pairs of rows and blocks to be sorted; block maxima that registers hold, all or a part."""
    say(f"top dt={dt} V={V}")
    rows = 450
    X, W, b, node = exact_case(256, rows, V, seed=V)
    check_exact(dt, X, W, b, node, 64, tau=2.0)
    rng = np.random.default_rng(V)
    check_exact(dt, X, W, None, node, 64, 1.0, random_rules(rng, rows, V, 4, 60, 9, repetition=1.25, presence=0.5))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,K", [(2, 3000, 64), (70, 3000, 33), (2100, 3000, 64)])
def test_equal_logits_go_to_the_lower_entry(dt, rows, V, K):
    say(f"ties dt={dt} rows={rows}")
    X, W, b, node = exact_case(32, rows, V, seed=2, ties=True)
    check_exact(dt, X, W, b, node, K)
    check_exact(dt, np.zeros_like(X), W, None, node, K)                       # all equal: 0 .. K - 1
    W[1::2] = W[::2]
    check_exact(dt, X, W, np.repeat(b[::2], 2), node, K)                      # each twice


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 40, 200, 2100])
def test_rising_and_falling_logits(dt, rows):
    """Every block beats the one before, or none does."""
    V, H = 5000, 32
    W = np.zeros((V, H))
    W[:, 0] = np.arange(V) // 20        # 250 different values, exact in bf16
    X = np.zeros((rows, H))
    X[:, 0] = np.where(np.arange(rows) % 2 == 0, 1.0, -1.0)
    check_exact(dt, X, W, None, np.arange(rows), 50, tau=3.0)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,rows,V,K", [(64, 20, 999, 9), (128, 150, 3001, 32), (256, 300, 2000, 64)])
def test_ordinary_values(dt, H, rows, V, K):
    say(f"top dt={dt} H={H} rows={rows} V={V}")
    rng = np.random.default_rng(H)
    X, W = round_to(dt, rng.standard_normal((rows, H))), round_to(dt, rng.standard_normal((V, H)) * 0.2)
    b = rng.standard_normal(V).astype(np.float32).astype(np.float64)
    z, dz, _, _ = L.logits(X, W, b, np.arange(rows))
    top, logit, lse = run(dt, X, W, b, np.arange(rows), K, 0.5)
    want, tol = lse_bound(z, dz, 0.5)
    R.within(lse, want, tol)
    r = np.arange(rows)[:, None]
    R.within(logit, z[r, top], dz[r, top])
    assert np.all(np.diff(logit, axis=1) <= 0)
    assert all(len(set(t)) == K for t in top)
    left = z.copy()
    left[r, top] = -np.inf
    # what is left lies below the last one, but for the rounding of the two sums that put it there and back
    assert np.all(left.max(1) <= z[r, top].min(1) + 4 * dz.max(1))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 50, 90, 2100])
def test_entries_and_nodes_taken_out(dt, rows):
    X, W, b, node = exact_case(64, rows, 300, seed=3)
    b[::2], b[1::4] = -np.inf, LOWEST
    b[3] = -1e30
    node[0], node[1] = -1, len(X) + 3
    check_exact(dt, X, W, b, node, 64)         # 75 entries are left
    b[:250] = -np.inf
    check_exact(dt, X, W, b, node, 20)         # fewer than K
    b[:] = -np.inf
    check_exact(dt, X, W, b, node, 3)          # none


def random_rules(rng, rows, V, masks, seen, adds, wild=True, **kw):
    rules = dict(kw)
    if masks:
        share = np.array([0.97, 0.5, 0.1, 0.01, 0.0])[np.arange(masks) % 5]
        rules["mask"] = rng.random((masks, V)) < share[:, None]
        rules["mask_of"] = rng.integers(-1, masks + (1 if wild else 0), rows)
    draw = (lambda n: np.maximum((V ** rng.random(n)).astype(np.int64) - 1, 0))
    if seen:
        rules["seen"] = [list(draw(rng.integers(0, seen + 1))) for _ in range(rows)]
        rules["seen"][0] = list(draw(seen))
        if wild:
            for s in rules["seen"]:
                for i in range(0, len(s), 7):
                    s[i] = int(rng.choice([-1, V, 2**31 - 1, -2**31]))
    if adds:
        val = (lambda n: np.where(rng.random(n) < 0.1, -np.inf, np.round(rng.standard_normal(n) * 8) / 8))
        rules["add"] = [list(zip(draw(k).tolist(), val(k).tolist())) for k in rng.integers(0, adds + 1, rows)]
        if wild and rules["add"][0]:
            rules["add"][0][0] = (V, 3.0)
    return rules


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H", [32, 64, 128, 256])
@pytest.mark.parametrize("rows,V,K", [(1, 100, 5), (30, 1999, 64), (50, 33, 20), (140, 4100, 9), (2100, 257, 4)])
def test_rules(dt, H, rows, V, K):
    say(f"rules dt={dt} H={H} rows={rows} V={V} K={K}")
    rng = np.random.default_rng(rows + H)
    X, W, b, node = exact_case(H, rows, V, seed=rows)
    for masks, seen, adds, kw in ((7, 0, 0, {}), (0, 40, 0, dict(repetition=1.25, presence=0.5, frequency=0.25)),
                                  (0, 0, 12, {}), (5, 30, 9, dict(repetition=1.5, presence=-0.25, frequency=0.125))):
        say(f"  masks={masks} seen={seen} adds={adds}")
        check_exact(dt, X, W, b, node, K, 2.0, random_rules(rng, rows, V, masks, seen, adds, **kw))


@pytest.mark.parametrize("rows,V,seen", [(3, 5000, 1500), (40, 3000, 1100), (1, 9000, 40000), (1100, 2500, 1030)])
def test_rules_with_long_lists(rows, V, seen):
    """Lists on both sides of what a hash table holds, passed over in parts by one workgroup or several."""
    say(f"long lists rows={rows} V={V} seen={seen}")
    rng = np.random.default_rng(seen)
    X, W, b, node = exact_case(64, rows, V, seed=rows)
    rules = random_rules(rng, rows, V, 3, seen if rows < 1000 else 0, 20, repetition=1.25, presence=0.5, frequency=0.25)
    if rows >= 1000:
        rules["seen"] = [[] for _ in range(rows)]
        for r in range(0, rows, 100):
            rules["seen"][r] = list(rng.integers(0, V, seen))
    check_exact("bf16", X, W, b, node, 16, 1.0, rules)


@pytest.mark.parametrize("rows,adds", [(2, 300), (90, 40), (1, 9000)])
def test_biases_of_one_entry_are_added_in_list_order(rows, adds):
    """Values whose float sum depends on the order: the list's own, term by term."""
    rng = np.random.default_rng(adds)
    H, V = 32, 1500
    W, X = np.zeros((V, H)), np.zeros((rows, H))
    tok = rng.integers(0, 20, (rows, adds)) * 70
    val = (rng.standard_normal((rows, adds)) * 10.0 ** rng.integers(-4, 4, (rows, adds))).astype(np.float32)
    top, logit, _ = run("f32", X, W, None, np.arange(rows), 64, 1.0, dict(add=[list(zip(a, b)) for a, b in zip(tok, val)]))
    for r in range(rows):
        want = {}
        for t, v in zip(tok[r].tolist(), val[r]):
            want[t] = np.float32(want.get(t, np.float32(0)) + v)
        got = dict(zip(top[r].tolist(), logit[r].tolist()))
        for t, v in want.items():
            if v > 0:
                assert got[t] == float(v)


def test_logits_of_any_size():
    """From 2^-100 to 2^100: the same entries, and log sums by the largest."""
    for dt in ("f32", "bf16"):
        for rows in (3, 150):
            X, W, b, node = exact_case(32, rows, 700, seed=12)
            for power in (-100, 20, 31, 60, 100):
                s = 2.0 ** power
                z, _, _, _ = L.logits(X * s, W, b * s, node)
                for tau in (1.0, 0.3, 7.0):
                    top, logit, lse = run(dt, X * s, W, b * s, node, 9, tau)
                    ids, zk = L.best(z, 9)
                    np.testing.assert_array_equal(top, ids)
                    np.testing.assert_array_equal(logit, zk)
                    want = L.log_sum(z / tau, np.zeros_like(z))[0]
                    # the rounding of 1 / tau and of two products; a sum of equals and its logarithm
                    R.within(lse, want, 8 * R.U * np.abs(want) + 2.0 ** -20 + 700 * R.U)


def test_a_mask_of_its_own_for_each_row_and_wider_words():
    rng = np.random.default_rng(1)
    X, W, b, node = exact_case(64, 80, 700, seed=4)
    mask = rng.random((60, 700)) < 0.3          # rows 60 .. 79 have none
    check_exact("bf16", X, W, b, node, 10, 1.0, dict(mask=mask))
    ru, keep, _ = struct(dict(mask=mask), 700, extra=5)
    got = run("bf16", X, W, b, node, 10, 1.0, dict(mask=mask))
    top, logit = torch.empty((80, 10), dtype=torch.int32, device="cuda"), torch.empty((80, 10), device="cuda")
    need = capi.ggnn_vocab_top_workspace_bytes("bf16", 64, 80, 700, 10, 0)
    capi.ggnn_vocab_top("bf16", len(X), 64, 80, 700, dev(X, "bf16"), dev(W, "bf16"), dev(b), ints(node), ru, 1.0, 10, top,
                        logit, None, scratch(need), need)
    np.testing.assert_array_equal(top.cpu().numpy(), got[0])
    assert keep


def test_a_token_seen_named_and_masked_at_once():
    """One row: every combination of the rules on a handful of entries."""
    H, V = 32, 40
    W = np.zeros((V, H))
    W[:, 0] = np.arange(V) / 4 - 4
    X = np.zeros((1, H))
    X[0, 0] = 1.0
    rules = dict(seen=[[39, 39, 39, 2, 2, 30, 31, 16]], repetition=2.0, presence=0.5, frequency=0.25,
                 add=[[(39, 1.0), (39, 0.5), (30, -np.inf), (31, 100.0), (5, 8.0), (2, 0.25), (7, 0.0)]],
                 mask=[[v != 31 and v != 38 for v in range(V)]], mask_of=[0])
    check_exact("f32", X, W, None, np.zeros(1, np.int64), 40, 1.0, rules)
    top, logit, _ = run("f32", X, W, None, np.zeros(1, np.int64), 40, 1.0, rules)
    got = dict(zip(top[0].tolist(), logit[0].tolist()))
    assert got[39] == (39 / 4 - 4) / 2 - (0.5 + 3 * 0.25) + 1.5 and got[2] == (2 / 4 - 4) * 2 - 1.0 + 0.25
    assert got[16] == -0.75 and got[5] == 5 / 4 - 4 + 8 and 30 not in got and 31 not in got and 38 not in got


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K", [(4, 9), (60, 9), (150, 9), (2100, 64)])
def test_what_stands_in_masked_rows_does_not_matter(dt, rows, K):
    X, W, b, node = exact_case(32, rows, 3000, seed=13)
    rng = np.random.default_rng(3)
    mask = rng.random((1, 3000)) < 0.6
    mask[0, 0] = False
    rules = dict(mask=mask, mask_of=np.zeros(rows, np.int64), seen=[[0, 5, 7, 2999]] * rows, repetition=1.25, presence=0.5)
    want = run(dt, X, W, b, node, K, 1.0, rules)
    for value in (np.nan, np.inf, -np.inf):
        W2 = W.copy()
        W2[~mask[0]] = value
        for got, w in zip(run(dt, X, W2, b, node, K, 1.0, rules), want):
            np.testing.assert_array_equal(got, w)


def test_two_calls_at_once_on_two_streams():
    X, W, b, node = exact_case(64, 700, 5000, seed=14)
    rng = np.random.default_rng(4)
    rules = random_rules(rng, 700, 5000, 3, 40, 8, repetition=1.25, presence=0.5)
    want = run("bf16", X, W, b, node, 16, 1.0, rules)
    ru, keep, listed = struct(rules, 5000)
    args = dev(X, "bf16"), dev(W, "bf16"), dev(b), ints(node)
    outs = []
    torch.cuda.synchronize()
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        top, logit = torch.empty((700, 16), dtype=torch.int32, device="cuda"), torch.empty((700, 16), device="cuda")
        lse, ws = torch.empty((700,), device="cuda"), scratch(capi.ggnn_vocab_top_workspace_bytes("bf16", 64, 700, 5000, 16, listed))
        torch.cuda.synchronize()
        outs.append((s, top, logit, lse, ws))
    for _ in range(5):
        for s, top, logit, lse, ws in outs:
            capi.ggnn_vocab_top("bf16", len(X), 64, 700, 5000, *args, ru, 1.0, 16, top, logit, lse, ws, ws.numel(), stream=s)
    torch.cuda.synchronize()
    for _, top, logit, lse, _ in outs:
        np.testing.assert_array_equal(top.cpu().numpy(), want[0])
        np.testing.assert_array_equal(host(logit), want[1])
        np.testing.assert_array_equal(host(lse), want[2])
    assert keep


def test_logits_that_are_not_finite():
    """NaN and infinite biases: NaN entries are not answered and make the log sum NaN, +inf is the best."""
    for rows in (3, 100):
        X, W, b, node = exact_case(32, rows, 200, seed=6)
        b[17], b[40] = np.nan, np.inf
        top, logit, lse = run("bf16", X, W, b, node, 5)
        assert np.all(top[:, 0] == 40) and np.all(np.isinf(logit[:, 0])) and not np.any(top == 17)
        assert np.all(np.isnan(lse))
        z, _, _, _ = L.logits(X, W, np.where(np.isfinite(b), b, -np.inf), node)
        np.testing.assert_array_equal(top[:, 1:], L.best(z, 4)[0])


@pytest.mark.parametrize("dt,H,rows", [("bf16", 64, 10), ("bf16", 128, 500), ("f32", 64, 300)])
def test_same_bits_every_time(dt, H, rows):
    rng = np.random.default_rng(H)
    X, W = round_to(dt, rng.standard_normal((rows, H))), round_to(dt, rng.standard_normal((3000, H)) * 0.2)
    rules = random_rules(rng, rows, 3000, 3, 300, 40, repetition=1.3, presence=0.21, frequency=0.13)
    a = run(dt, X, W, None, np.arange(rows), 20, 1.7, rules)
    for _ in range(3):
        for p, q in zip(a, run(dt, X, W, None, np.arange(rows), 20, 1.7, rules)):
            np.testing.assert_array_equal(p, q)


def test_best_of_one_is_the_losses_best_entry():
    X, W, b, node = exact_case(128, 333, 2500, seed=7)
    best, lse = torch.empty((333,), dtype=torch.int32, device="cuda"), torch.empty((333,), device="cuda")
    need = capi.ggnn_vocab_workspace_bytes("bf16", 128, 333, 2500, False)
    capi.ggnn_vocab_loss("bf16", len(X), 128, 333, 2500, dev(X, "bf16"), dev(W, "bf16"), dev(b), ints(node), None, None, lse,
                         best, scratch(need), need)
    top, _, mine = run("bf16", X, W, b, node, 1)
    np.testing.assert_array_equal(top[:, 0], best.cpu().numpy())
    z, dz, _, _ = L.logits(X, W, b, node)
    R.within(mine - host(lse), np.zeros(333), 2 * lse_bound(z, dz, 1.0)[1])


def test_captured_and_replayed():
    dt, H, rows, V, K = "bf16", 64, 90, 1203, 12
    rng = np.random.default_rng(0)
    X0, W0, b0, node0 = exact_case(H, rows, V, seed=8)
    X, W, b, node = dev(X0, dt), dev(W0, dt), dev(b0), ints(node0)
    rules = random_rules(rng, rows, V, 4, 50, 10, repetition=1.25, presence=0.5, frequency=0.25)
    ru, keep, listed = struct(rules, V)
    top, logit = torch.empty((rows, K), dtype=torch.int32, device="cuda"), torch.empty((rows, K), device="cuda")
    lse = torch.empty((rows,), device="cuda")
    ws = scratch(capi.ggnn_vocab_top_workspace_bytes(dt, H, rows, V, K, listed))

    def call():
        capi.ggnn_vocab_top(dt, len(X0), H, rows, V, X, W, b, node, ru, 2.0, K, top, logit, lse, ws, ws.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (9, 8, 10):
        X1, W1, b1, node1 = exact_case(H, rows, V, seed=seed)
        X.copy_(dev(X1, dt)), W.copy_(dev(W1, dt)), b.copy_(dev(b1)), node.copy_(ints(node1))
        want = run(dt, X1, W1, b1, node1, K, 2.0, rules)
        ws.fill_(0xAB)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(top.cpu().numpy(), want[0])
        np.testing.assert_array_equal(host(logit), want[1])
        np.testing.assert_array_equal(host(lse), want[2])
    assert keep


def test_block_maxima_past_32_bits():
    """400,000 rows over 60,000 entries: 6 GB of block maxima; the first answers are the loss's best entries."""
    n, V, H, K = 400000, 60000, 32, 2
    g = torch.Generator(device="cuda").manual_seed(5)
    X = (torch.randn((n, H), generator=g, device="cuda") * 16).round_().clamp_(-127, 127).div_(16).bfloat16()
    W = (torch.randn((V, H), generator=g, device="cuda") * 16).round_().clamp_(-127, 127).div_(64).bfloat16()
    need = capi.ggnn_vocab_top_workspace_bytes("bf16", H, n, V, K, 0)
    assert need > 1 << 32
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")
    top, logit = torch.empty((n, K), dtype=torch.int32, device="cuda"), torch.empty((n, K), device="cuda")
    capi.ggnn_vocab_top("bf16", n, H, n, V, X, W, None, None, None, 1.0, K, top, logit, None, ws, need)
    best, lse = torch.empty((n,), dtype=torch.int32, device="cuda"), torch.empty((n,), device="cuda")
    capi.ggnn_vocab_loss("bf16", n, H, n, V, X, W, None, None, None, None, lse, best, ws, need)
    assert torch.equal(top[:, 0], best)
    for at in (0, 123457, n - 100):   # the second ones of a few rows, the lower entry of equals
        z = X[at:at + 100].float() @ W.float().t()
        want = torch.sort(z, dim=1, descending=True, stable=True)
        assert torch.equal(top[at:at + 100], want.indices[:, :2].int())
        assert torch.equal(logit[at:at + 100], want.values[:, :2])
