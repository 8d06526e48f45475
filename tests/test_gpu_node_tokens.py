"""NodeTokens: one training step's losses, gradients and update against the
oracle's propagation with the 64-bit references of the token operators; the
example learns; serving answers with the largest logit."""
import os
import sys

import numpy as np
import pytest

import oracle as O
import token_reference as R
from ggnn_synth import backbone_graph, draw_params, scramble_graph
from gpu_helpers import TOL, host, relerr, round_to, say

capi = pytest.importorskip("paper_1906_11786_amd.capi")
torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_1906_11786_amd.driver import BandedGGNN, compile_graphs  # noqa: E402
from paper_1906_11786_amd.tokens import NodeTokens, token_lists  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")


def setup(dt, H, n=400, B=64, E=3, T=2, V=173, p=0.25):
    rng = np.random.default_rng(H)
    g = scramble_graph(9, 0, backbone_graph(9, 0, n, E, span_mean=6.0, max_span=B))[0]
    comp = compile_graphs([g], B, E, reorder=True)
    params = draw_params(9, comp.n_real, comp.n_pad, H, E, dt, with_bias=True)
    lists = [list(rng.integers(0, V, rng.integers(0, 5))) for _ in range(n)]
    ptr, tok = token_lists(lists, comp.n_pad)
    table = round_to(dt, rng.standard_normal((V, H)) / np.sqrt(H))
    bias = round_to("f32", 0.3 * rng.standard_normal(V))
    m = BandedGGNN(comp, H, T, dt, params)
    t = NodeTokens(m, table, ptr, tok, bias=bias, scale=float(np.sqrt(H)), p_in=p, p_out=p, seed=2**40 + 3)
    node = rng.permutation(n)[:60]
    target = rng.integers(0, V, 60)
    target[::7] = -1
    return m, t, comp, params, ptr, tok, table, bias, node, target, (B, T, V, p)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H", [64, 128])
def test_training_step_against_the_oracle(dt, H):
    say(f"node tokens dt={dt} H={H}")
    m, t, comp, params, ptr, tok, table, bias, node, target, (B, T, V, p) = setup(dt, H)
    n, sc, step = comp.n_pad, float(np.sqrt(H)), 3
    t.setup_training(node, target, lr=0.125, momentum=0.5)
    t.step = step
    t.gradients(step)
    got = dict(loss=host(t.loss), dtable=host(t.dtable), dbias=host(t.dbias), dW=host(m.dW), dWi=host(m.dWi),
               dU=host(m.dU), db=host(m.db))
    # the same step in 64 bits; the first states are the stored (rounded) ones
    X0, _, _ = R.embed(table, n, ptr, tok, int(ptr[-1]), sc, True, p, t.seed, 2 * step)
    X0 = host(m.X[0]) if dt == "bf16" else X0
    out = O.propagate(n, B, comp.src, comp.dst, comp.etype, X0, params.W, params.Wi, params.U, params.b, T,
                      bias=params.bias)
    keep = R.keep_factor(0, n * H, p, t.seed, 2 * step + 1).reshape(n, H)
    live = int((target >= 0).sum())
    v = R.vocab(out["X"][-1] * keep, table, bias, node, target, None, 1.0 / live, dt)
    out = O.propagate(n, B, comp.src, comp.dst, comp.etype, X0, params.W, params.Wi, params.U, params.b, T,
                      G=v["dX"] * keep, bias=params.bias)
    dT, _, _ = R.embed_grad(out["dX0"], V, ptr, tok, int(ptr[-1]), sc, True, p, t.seed, 2 * step)
    want = dict(loss=v["loss"], dtable=v["dW"] + dT, dbias=v["db"], dW=out["dW"], dWi=out["dWi"], dU=out["dU"],
                db=out["db"])
    for k, w in want.items():
        e = relerr(got[k], w)
        say(f"  {k}: {e:.2e}")
        assert e <= TOL[dt], k
    # the update: velocities start at zero, so parameter -= lr * gradient
    before = t.master.clone()
    t.train_step()
    assert t.step == step + 1
    assert torch.equal(t.master, before - 0.125 * t.grad)
    if dt == "bf16":
        assert torch.equal(t.compute_copy, t.master.to(torch.bfloat16))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_serving_answers_with_the_largest_logit(dt):
    m, t, comp, params, ptr, tok, table, bias, node, target, _ = setup(dt, 64)
    out = t.evaluate(node[:5], target[:5])
    x = host(m.X[m.T])[node[:5]]
    z = x @ host(t.table).T + host(t.bias)
    top = np.sort(z, 1)
    assert np.all(top[:, -1] - top[:, -2] > 1e-3)    # no near ties in these five rows
    assert np.array_equal(out["best"].cpu().numpy(), np.argmax(z, 1))
    one = t.evaluate(node[:1])
    assert torch.equal(one["best"], out["best"][:1]) and "loss" not in one
    lse = np.log(np.exp(z).sum(1))
    assert np.max(np.abs(host(out["lse"]) - lse)) <= 1e-4
    want = np.where(target[:5] >= 0, lse - z[np.arange(5), np.maximum(target[:5], 0)], 0.0)
    assert np.max(np.abs(host(out["loss"]) - want)) <= 1e-4


@pytest.mark.parametrize("as_handle", [False, True])
def test_all_of_a_call_runs_on_the_given_stream(as_handle):
    """Three calls behind a stream that is still busy: the fills between them wait for it as the kernels do."""
    m, t, *_, node, target, _ = setup("bf16", 64)
    t.setup_training(node, target)
    t.gradients(2)
    want = (t.grad.clone(), m.grad_buf.clone(), t.loss.clone())
    best = t.evaluate(node)["best"]
    a = torch.randn((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            a = torch.mm(a, a).mul_(1.0 / 4096)
    given = side.cuda_stream if as_handle else side
    t.gradients(1, stream=given)
    t.gradients(2, stream=given)
    got = t.evaluate(node, stream=given)["best"]
    torch.cuda.synchronize()
    assert torch.equal(t.grad, want[0]) and torch.equal(m.grad_buf, want[1]) and torch.equal(t.loss, want[2])
    assert torch.equal(got, best)


def test_refusals():
    m, t, comp, params, ptr, tok, table, bias, node, target, (_, _, V, _) = setup("f32", 64)
    with pytest.raises(ValueError, match="table"):
        NodeTokens(m, table[:, :32], ptr, tok)
    with pytest.raises(ValueError, match="tok_ptr"):
        NodeTokens(m, table, ptr[:-1], tok)
    with pytest.raises(ValueError, match="more than once"):
        t.setup_training([3, 3], [0, 1])
    with pytest.raises(ValueError, match="node ids"):
        t.evaluate([comp.n_pad])
    with pytest.raises(ValueError, match="targets"):
        t.setup_training([3, 4], [0, V])
    with pytest.raises(RuntimeError, match="setup_training"):
        t.train_step()


def test_example_learns():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import hidden_tokens
    losses = hidden_tokens.main(steps=40)
    assert losses[0] > 5.0                       # about log 500 at the start
    assert np.mean(losses[-5:]) < 0.5 * losses[0]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-np.inf, R.LOWEST, -1e30])
@pytest.mark.parametrize("weight_decay", [0.0, 0.125])
def test_masked_tokens_stay_masked_in_training(dt, low, weight_decay):
    """Tokens that the bias takes out: their bias stays, what is updated stays finite, and after three steps the log
    sums are those over the other tokens."""
    m, t, comp, params, ptr, tok, table, bias, node, target, (_, _, V, _) = setup(dt, 64)
    out = np.arange(V) % 3 == 0
    bias[out] = low
    t = NodeTokens(m, table, ptr, tok, bias=bias, scale=8.0, p_in=0.25, p_out=0.25, seed=5)
    target = np.where(out[np.maximum(target, 0)], -1, target)
    t.setup_training(node, target, lr=0.125, momentum=0.5, weight_decay=weight_decay)
    start = t.bias.clone()
    for _ in range(3):
        t.train_step()
        assert bool(torch.isfinite(t.loss).all()) and bool(torch.isfinite(m.master).all())
    assert bool((t.bias[torch.from_numpy(out).cuda()] <= -1e30).all())
    keep = torch.from_numpy(~out).cuda()
    assert bool(torch.isfinite(t.table).all()) and bool(torch.isfinite(t.bias[keep]).all())
    assert not torch.equal(t.bias[keep], start[keep])
    got = t.evaluate(node[:50], target[:50])
    z = (host(m.X[m.T])[node[:50]] @ host(t.table).T + np.where(out, 0.0, host(t.bias)))[:, ~out]
    assert np.max(np.abs(host(got["lse"]) - np.log(np.exp(z).sum(1)))) <= 1e-4
    assert not np.any(out[got["best"].cpu().numpy()])
