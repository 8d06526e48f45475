"""Ends of what the operators on a vocabulary's logits take: masked rows of W at the
vocabulary's end, logits of many temperatures, the most rows."""
import numpy as np
import pytest

import logit_reference as L
import test_gpu_distill as D
import token_reference as R
from gpu_helpers import dev, host, round_to, say
from test_gpu_top import exact_case, ints, scratch, struct

capi = pytest.importorskip("paper_1906_11786_amd.capi")
torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")


def top(dt, X, W, b, node, K, rules, padding):
    """ggnn_vocab_top under a mask whose bits past the vocabulary are `padding`."""
    n, H = X.shape
    V, rows = W.shape[0], len(node)
    ru, keep, listed = struct(rules, V, extra=2)
    bits = np.full(32 * (-(-V // 32) + 2), padding, np.uint8)
    bits[:V] = 0
    keep[0] |= torch.from_numpy(np.packbits(bits, bitorder="little").view("<i4")).cuda()   # (the same tensor)
    token, logit = torch.empty((rows, K), dtype=torch.int32, device="cuda"), torch.empty((rows, K), device="cuda")
    lse = torch.empty((rows,), device="cuda")
    need = capi.ggnn_vocab_top_workspace_bytes(dt, H, rows, V, K, listed)
    capi.ggnn_vocab_top(dt, n, H, rows, V, dev(X, dt), dev(W, dt), dev(b), ints(node), ru, 2.0, K, token, logit, lse,
                        scratch(need), need)
    torch.cuda.synchronize()
    return token.cpu().numpy(), host(logit), host(lse)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K", [(5, 9), (50, 9), (90, 9), (2100, 64)])
@pytest.mark.parametrize("V", [40, 96, 2976, 3001])
@pytest.mark.parametrize("lists", [False, True])
def test_what_stands_in_masked_rows_at_the_end_does_not_matter(dt, rows, K, V, lists):
    """A vocabulary padded with rows that no mask lets through: the same answers and log sums, bit for bit."""
    say(f"masked end dt={dt} rows={rows} V={V} lists={lists}")
    X, W, b, node = exact_case(32, rows, V, seed=V)
    mask = np.random.default_rng(V).random((2, V)) < 0.7
    mask[:, 32 * ((V - 1) // 32)] = True      # (an entry of the last mask word that is let through)
    mask[:, V - 2:] = False
    rules = dict(mask=mask, mask_of=np.arange(rows) % 2)
    if lists:
        rules.update(seen=[[0, 3, V - 1]] * rows, repetition=1.25, presence=0.5, add=[[(V - 2, 1.0), (7, 0.5)]] * rows)
    want = top(dt, X, W, b, node, K, rules, 0)
    assert np.all(np.isfinite(want[2]))
    gone = ~mask.any(0)
    for value in (np.nan, np.inf, -np.inf):
        W2 = W.copy()
        W2[gone] = value
        for padding in (0, 1):
            for got, w in zip(top(dt, X, W2, b, node, K, rules, padding), want):
                np.testing.assert_array_equal(got, w)


def two_rows(dt, tau, size, rng, far):
    """Row 0 is sure of the first half of the entries and row 1 of the second, with logits of about `size` temperatures
    that are exact in float32 in any order of their sums.  Within a half they lie at most four temperatures apart
    (far: one entry's is twice the others')."""
    H, V, K = 32, 70, 4
    W = np.zeros((V, H))
    W[:, 0] = np.where(np.arange(V) < V // 2, 200.0, -200.0)
    c = float(round_to("bf16", np.array([size * tau / 200]))[0])
    X = np.zeros((2, H))
    X[:, 0] = c, -c
    b = None
    if far:
        W[:, 0] /= 2
        W[[3, V - 3], 0] *= 2
    else:
        step = 2.0 ** (np.ceil(np.log2(tau)) - 6)   # a 24-bit logit of up to 2^17 tau has it as a place
        b = np.floor(rng.random(V) * 4 * tau / step) * step
    t_id = np.stack([rng.permutation(V)[:K] for _ in range(2)])
    return dict(n=2, X=X, W=W, b=b, node=np.arange(2), t_id=t_id, t_logit=(tau * rng.standard_normal((2, K))).astype(
        np.float32).astype(np.float64)), abs(c)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [0.3, 0.7, 1.0, 3.0, 7.0, 50.0])
@pytest.mark.parametrize("far", [False, True])
def test_gradients_of_logits_of_many_temperatures(dt, tau, far):
    """dW and dbias from probabilities exp(z / tau - lse) whose log sum is rounded once, to float: with exact logits a
    probability is off by half a step of it, exp(U |lse|) - 1; the exponential and its argument's factor, the pair of
    bf16 and the teacher's probabilities by 2^-15 together.  (far: one entry has all of it, and its logit is the log
    sum.)"""
    rng = np.random.default_rng(int(10 * tau))
    t32 = float(np.float32(tau))   # what the call gets: at 2^29 temperatures the rest of 0.7 would be many units of z / tau
    for i in range(12):
        size = 2.0 ** rng.uniform(29.2, 60) if far else 2.0 ** rng.uniform(14, 16.9)
        c, x = two_rows(dt, tau, size, rng, far)
        t_lse = None
        if i % 2:   # probabilities that do not add up to 1
            t_lse = (np.log(np.exp(c["t_logit"] / tau).sum(1)) + 0.5).astype(np.float32).astype(np.float64)
        got = D.run(dt, c, t32, t_lse, scale=0.7)
        want = L.distill(c["X"], c["W"], c["b"], c["node"], c["t_id"], c["t_logit"], t_lse, t32, None, 0.7, dt)
        z = (c["X"] @ c["W"].T + (0.0 if c["b"] is None else c["b"])) / t32
        P = np.exp(z - want["lse"][:, None])
        t = np.exp(c["t_logit"] / t32)
        q = t / t.sum(1)[:, None] if t_lse is None else t / np.exp(t_lse)[:, None]
        Q = np.zeros_like(P)
        np.add.at(Q, (np.arange(2)[:, None], c["t_id"]), q)
        off = np.zeros(2) if far else np.expm1(R.U * np.abs(want["lse"]))
        tol = (0.7 / tau * (q.sum(1)[:, None] * P * (off[:, None] + 2.0 ** -15) + Q * 2.0 ** -15)).sum(0)
        R.within(host(got["dW"])[:, 0], want["dW"][:, 0], tol * x)
        if c["b"] is not None:
            R.within(host(got["db"]), want["db"], tol)


@pytest.mark.parametrize("K,lists", [(1, True), (64, False)])
def test_the_most_rows(K, lists):
    """2^24 rows, the most there may be, of 64 nodes: lists of a few rows' own, and 2^30 pairs of rows and blocks."""
    rows, V, H = 1 << 24, 40, 32
    free = torch.cuda.mem_get_info()[0]
    need = capi.ggnn_vocab_top_workspace_bytes("bf16", H, rows, V, K, 3 if lists else 0)
    if free < need + 24 * rows * K + (4 << 30):
        pytest.skip(f"{need >> 30} GB of workspace")
    X, W, b, _ = exact_case(H, 64, V, seed=20, n=64)
    z, _, _, _ = L.logits(X, W, b, np.arange(64))
    node = torch.arange(rows, dtype=torch.int32, device="cuda") % 64
    ru, seen_ptr, seen = None, None, None
    listed = (0, 1 << 23, rows - 1)
    if lists:   # each of these rows has seen its best entry
        seen_ptr = torch.zeros((rows + 1,), dtype=torch.int32, device="cuda")
        for r in listed:
            seen_ptr[r + 1:] += 1
        seen = ints([int(np.argmax(z[r % 64])) for r in listed])
        ru = capi.token_rules(seen_ptr=seen_ptr, seen=seen, n_seen=3, presence=100.0)
    top, logit = torch.empty((rows, K), dtype=torch.int32, device="cuda"), torch.empty((rows, K), device="cuda")
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")
    capi.ggnn_vocab_top("bf16", 64, H, rows, V, dev(X, "bf16"), dev(W, "bf16"), dev(b), node, ru, 1.0, K, top, logit, None, ws,
                        need)
    ids, zk = L.best(z, K)
    same = torch.ones((rows,), dtype=torch.bool, device="cuda")
    if lists:
        for r in listed:
            same[r] = False
            penalised = z[r % 64:r % 64 + 1].copy()
            penalised[0, seen[listed.index(r)].item()] -= 100.0
            want = L.best(penalised, K)
            np.testing.assert_array_equal(top[r].cpu().numpy(), want[0][0])
            np.testing.assert_array_equal(host(logit[r]), want[1][0])
    view = (lambda a: a.view(-1, 64 * K))
    wrong = (view(top) != ints(ids).view(1, -1)) | (view(logit) != dev(zk).view(1, -1))
    assert not bool((wrong.view(rows, K).any(1) & same).any())
    del ws, top, logit, wrong
    torch.cuda.empty_cache()


def test_defaults_of_answers_and_of_training_on_them_fit():
    """top() and setup_training() as they are: the student's temperature is that of the teacher's log sums."""
    from test_gpu_node_tokens import setup
    _, teacher, *_, node, target, _ = setup("bf16", 64)
    m, student, *_ = setup("bf16", 64)
    out = teacher.top(node, 6)
    student.setup_training(node, target, teacher=out)
    student.gradients(1)
    want = L.distill(host(student.XT), host(student.table), host(student.bias), node, out["token"].cpu().numpy(),
                     host(out["logit"]), host(out["lse"]), 1.0, None, 1.0, "bf16")
    R.within(host(student.soft_loss), want["loss"], want["loss_tol"])
    with pytest.raises(ValueError, match="log sums are at temperature 1, not 2"):
        student.setup_training(node, target, teacher=out, temperature=2.0)
