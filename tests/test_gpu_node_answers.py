"""NodeTokens: answers with the best tokens under rules, and training on a
teacher's answers, against the 64-bit references of the operators."""
import os
import sys

import numpy as np
import pytest

import logit_reference as L
import oracle as O
import token_reference as R
from gpu_helpers import TOL, host, relerr, say

capi = pytest.importorskip("paper_1906_11786_amd.capi")
torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_1906_11786_amd.tokens import TokenRules  # noqa: E402
from test_gpu_node_tokens import setup  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")


def lists(seed, rows, V, K):
    """A teacher's lists: distinct tokens, short ones and an empty one among them."""
    rng = np.random.default_rng(seed)
    token = np.stack([rng.permutation(V)[:K] for _ in range(rows)])
    token[1::5, K // 2:] = -1
    token[3] = -1
    logit = (2 * rng.standard_normal((rows, K))).astype(np.float32)
    return token, logit


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("soft,whole", [(0.25, False), (1.0, True)])
def test_training_step_with_a_teacher_against_the_oracle(dt, soft, whole):
    H, tau = 64, 2.0
    say(f"teacher dt={dt} soft={soft}")
    m, t, comp, params, ptr, tok, table, bias, node, target, (B, T, V, p) = setup(dt, H)
    n, sc, step, K = comp.n_pad, float(np.sqrt(H)), 3, 7
    token, logit = lists(0, 60, V, K)
    lse = None
    if whole:
        lse = (np.log(np.where(token >= 0, np.exp(logit / tau), 0.0).sum(1) + 0.5)).astype(np.float32)
    teacher = dict(token=torch.from_numpy(token).cuda(), logit=logit, **({} if lse is None else {"lse": lse}))
    t.setup_training(node, target, lr=0.125, momentum=0.5, teacher=teacher, temperature=tau, soft=soft)
    t.step = step
    t.gradients(step)
    got = dict(loss=host(t.loss), soft_loss=host(t.soft_loss), dtable=host(t.dtable), dbias=host(t.dbias), dW=host(m.dW),
               dWi=host(m.dWi), dU=host(m.dU), db=host(m.db))
    X0, _, _ = R.embed(table, n, ptr, tok, int(ptr[-1]), sc, True, p, t.seed, 2 * step)
    X0 = host(m.X[0]) if dt == "bf16" else X0
    out = O.propagate(n, B, comp.src, comp.dst, comp.etype, X0, params.W, params.Wi, params.U, params.b, T,
                      bias=params.bias)
    keep = R.keep_factor(0, n * H, p, t.seed, 2 * step + 1).reshape(n, H)
    x = out["X"][-1] * keep
    v = R.vocab(x, table, bias, node, target, None, (1 - soft) / int((target >= 0).sum()), dt)
    d = L.distill(x, table, bias, node, token, logit.astype(np.float64), None if lse is None else lse.astype(np.float64), tau,
                  None, soft * tau ** 2 / int((token >= 0).any(1).sum()), dt)
    out = O.propagate(n, B, comp.src, comp.dst, comp.etype, X0, params.W, params.Wi, params.U, params.b, T,
                      G=(v["dX"] + d["dX"]) * keep, bias=params.bias)
    dT, _, _ = R.embed_grad(out["dX0"], V, ptr, tok, int(ptr[-1]), sc, True, p, t.seed, 2 * step)
    want = dict(loss=v["loss"], soft_loss=d["loss"], dtable=v["dW"] + d["dW"] + dT, dbias=v["db"] + d["db"], dW=out["dW"],
                dWi=out["dWi"], dU=out["dU"], db=out["db"])
    for k, w in want.items():
        e = relerr(got[k], w)
        say(f"  {k}: {e:.2e}")
        assert e <= TOL[dt], k
    before = t.master.clone()
    t.train_step()
    assert torch.equal(t.master, before - 0.125 * t.grad)


def test_without_a_teacher_again():
    m, t, *_, node, target, (_, _, V, _) = setup("bf16", 64)
    t.setup_training(node, target)
    t.gradients(2)
    want = t.grad.clone(), m.grad_buf.clone()
    token, logit = lists(1, 60, V, 5)
    t.setup_training(node, target, teacher=dict(token=token, logit=logit))
    t.gradients(2)
    assert not torch.equal(t.grad, want[0])
    t.setup_training(node, target)
    t.gradients(2)
    assert torch.equal(t.grad, want[0]) and torch.equal(m.grad_buf, want[1])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_answers_under_rules(dt):
    m, t, comp, *_, node, target, (_, _, V, _) = setup(dt, 64)
    rng = np.random.default_rng(5)
    rows = 40
    seen = [list(rng.integers(0, V, rng.integers(0, 9))) for _ in range(rows)]
    bias = [{int(v): float(a) for v, a in zip(rng.integers(0, V, 4), rng.integers(-8, 9, 4) / 4)} for _ in range(rows)]
    bias[3] = [(5, 1.0), (5, 0.5), (6, -np.inf)]
    allowed = rng.random((3, V)) < np.array([0.9, 0.3, 0.0])[:, None]
    of = rng.integers(-1, 3, rows)
    kw = dict(repetition=1.5, presence=0.5, frequency=0.25)
    cases = [(None, {}), (dict(seen=seen, **kw), dict(seen=seen, **kw)),
             (dict(allowed=allowed, allowed_of=of), dict(mask=allowed, mask_of=of)),
             (dict(allowed=allowed, allowed_of=of, seen=seen, bias=bias, **kw),
              dict(mask=allowed, mask_of=of, seen=seen, add=[list(b.items()) if isinstance(b, dict) else b for b in bias],
                   **kw))]
    for given, plain in cases:
        out = t.top(node[:rows], 9, None if given is None else t.rules(rows, **given), temperature=2.0)
        z0, dz, _, _ = L.logits(host(m.X[m.T]), host(t.table), host(t.bias), node[:rows])
        z = L.apply_rules(z0, plain)
        token, logit = out["token"].cpu().numpy(), host(out["logit"])
        want_token, want_logit = L.best(z, 9)
        tol = 2 * 1.5 * dz.max() + 8 * R.U * (np.abs(z0).max() + 8)   # of a logit after the rules: 1.5 at most
        np.testing.assert_array_equal(token >= 0, want_token >= 0)
        live = token >= 0
        assert np.all(np.abs(logit - want_logit)[live] <= tol)
        assert np.all(np.abs(np.take_along_axis(z, np.maximum(token, 0), 1) - logit)[live] <= tol)
        want, lse_tol = L.log_sum(z / 2.0, np.full_like(z, tol))
        R.within(host(out["lse"]), want, lse_tol)


def test_a_teachers_answers_teach_a_student():
    """top() of one model as the lists of another: shapes, temperatures and log sums fit."""
    _, teacher, *_, node, target, _ = setup("bf16", 128)
    m, student, *_ = setup("bf16", 64)
    out = teacher.top(node, 6, temperature=3.0)
    for given in (out, {k: v.cpu().numpy() for k, v in out.items()}, {k: out[k] for k in ("token", "logit")}):
        student.setup_training(node, target, teacher=given, temperature=3.0, soft=0.5)
        student.gradients(1)
        want = L.distill(host(student.XT), host(student.table), host(student.bias), node, out["token"].cpu().numpy(),
                         host(out["logit"]), host(out["lse"]) if "lse" in given else None, 3.0, None, 1.0, "bf16")
        R.within(host(student.soft_loss), want["loss"], want["loss_tol"])


def test_a_captured_training_step_with_a_teacher():
    """Captured once, replayed with the program's own eager work between."""
    m, t, *_, node, target, (_, _, V, _) = setup("bf16", 64)
    token, logit = lists(2, 60, V, 9)
    t.setup_training(node, target, teacher=dict(token=token, logit=logit))
    t.gradients(4)
    want = t.grad.clone(), m.grad_buf.clone(), t.soft_loss.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        t.gradients(4)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.gradients(4)
    for i in range(3):
        t.gradients(5 + i)
        t.top(node[:10], 4, t.rules(10, seen=[[1, 2]] * 10, presence=1.0))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t.grad, want[0]) and torch.equal(m.grad_buf, want[1]) and torch.equal(t.soft_loss, want[2])


def test_all_of_a_call_runs_on_the_given_stream():
    m, t, *_, node, target, (_, _, V, _) = setup("bf16", 64)
    rules = t.rules(60, seen=[[1, 2, 2]] * 60, presence=1.0, allowed=np.ones((1, V), bool), allowed_of=np.zeros(60, int))
    want = t.top(node, 5, rules)
    a = torch.randn((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            a = torch.mm(a, a).mul_(1.0 / 4096)
    m.X[0].zero_()
    got = t.top(node, 5, rules, stream=side)
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k])


def test_refusals():
    m, t, comp, *_, node, target, (_, _, V, _) = setup("f32", 64)
    token, logit = lists(3, 60, V, 4)
    with pytest.raises(ValueError, match="k=65"):
        t.top(node, 65)
    with pytest.raises(ValueError, match="node ids"):
        t.top([comp.n_pad], 3)
    with pytest.raises(ValueError, match="rules for 3 rows"):
        t.top(node[:4], 3, t.rules(3))
    with pytest.raises(ValueError, match="rules for 4 rows over 9"):
        t.top(node[:4], 3, TokenRules(9, 4))
    with pytest.raises(ValueError, match="below V"):
        t.setup_training(node, target, teacher=dict(token=np.full((60, 4), V), logit=logit))
    with pytest.raises(ValueError, match="shapes"):
        t.setup_training(node, target, teacher=dict(token=token[:5], logit=logit))
    with pytest.raises(ValueError, match="shapes"):
        t.setup_training(node, target, teacher=dict(token=token, logit=logit[:, :3]))
    with pytest.raises(ValueError, match="log sums"):
        t.setup_training(node, target, teacher=dict(token=token, logit=logit, lse=np.zeros(3)))
    with pytest.raises(ValueError, match="soft"):
        t.setup_training(node, target, teacher=dict(token=token, logit=logit), soft=1.5)
    with pytest.raises(ValueError, match="temperature"):
        t.setup_training(node, target, teacher=dict(token=token, logit=logit), temperature=0.0)


def test_example_runs():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import distill_tokens
    losses, free, ruled, masked = distill_tokens.main(steps=3)
    assert len(losses) == 3 and np.all(np.isfinite(losses))
    assert bool((masked["token"] < 250).all()) and bool((free["token"] >= 0).all())
    for out in (free, ruled, masked):
        assert bool((out["logit"].diff(dim=1) <= 0).all())
