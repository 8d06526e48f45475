"""Operators on a vocabulary's logits on the CPU: refusals (checked before
anything reaches the device), workspace sizes, and the references that the GPU
tests use against differences."""
import numpy as np
import pytest

import logit_reference as L

capi = pytest.importorskip("paper_1906_11786_amd.capi")

P, Q, S = 1 << 20, 1 << 30, 1 << 34   # 16-byte aligned stand-in addresses; nothing is launched
NAN = float("nan")


def refused(status, text, fn, *args):
    with pytest.raises(capi.GGNNError) as e:
        fn(*args, stream=0)
    assert e.value.status_name == status, str(e.value)
    assert text in str(e.value), str(e.value)


DISTILL = dict(dt="bf16", n_nodes=100, H=64, n_rows=50, V=1000, X=P, W=Q, bias=None, node=S, K=8, teacher_id=S,
               teacher_logit=S, teacher_lse=None, temperature=2.0)
DISTILL_BAD = [(dict(dt=5), "dtype"), (dict(n_nodes=0), "n_nodes"), (dict(H=16), "H="), (dict(n_rows=-1), "n_rows"),
               (dict(node=None, n_rows=101), "n_rows=101 exceeds"), (dict(V=0), "V="), (dict(X=None), "X is NULL"),
               (dict(bias=P + 2), "bias is not"), (dict(node=P + 4), "node is not"), (dict(K=0), "K=0"),
               (dict(K=65), "K=65"), (dict(n_rows=(1 << 24) - 1, n_nodes=1 << 24, K=64, teacher_id=None), "teacher_id"),
               (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(n_rows=1 << 24, n_nodes=1 << 24, K=64, V=-1), "V="),
               (dict(teacher_id=None), "teacher_id is NULL"), (dict(teacher_logit=None), "teacher_logit is NULL"),
               (dict(teacher_logit=S + 4), "teacher_logit is not"), (dict(teacher_lse=S + 8), "teacher_lse is not"),
               (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"),
               (dict(temperature=NAN), "temperature"), (dict(temperature=2000.0), "temperature"),
               (dict(loss=None), "loss is NULL"), (dict(lse=None), "lse is NULL")]


@pytest.mark.parametrize("kw,text", DISTILL_BAD)
def test_distillation_refuses(kw, text):
    a = dict(DISTILL, loss=S, lse=S, workspace=S, workspace_bytes=1 << 40)
    a.update(kw)
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_vocab_distill, *a.values())


@pytest.mark.parametrize("kw,text", DISTILL_BAD + [
    (dict(dX=None), "dX is NULL"), (dict(dW=None), "dW is NULL"), (dict(dbias=P + 4), "dbias is not"),
    (dict(weight=P + 4), "weight is not"), (dict(scale=float("inf")), "scale"), (dict(dX=P + 16), "dX overlaps"),
    (dict(dW=Q + 16), "dW overlaps"), (dict(dW=S + (1 << 30)), "dW overlaps")])
def test_distillation_gradients_refuse(kw, text):
    a = dict(DISTILL, weight=None, scale=1.0, add=False, loss=S, lse=S, dX=S + (1 << 30), dW=S + (2 << 30), dbias=None,
             workspace=S, workspace_bytes=1 << 40)
    a.update(kw)
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_vocab_distill_grad, *a.values())


def test_distillation_wants_its_workspace():
    head = tuple(DISTILL.values())
    for grad in (False, True):
        need = capi.ggnn_vocab_distill_workspace_bytes("bf16", 64, 50, 1000, 8, grad)
        assert need > 0
        for ws, size in ((None, need), (S, need - 1), (S + 8, need)):
            if grad:
                refused("GGNN_ERR_WORKSPACE", f"{need} bytes", capi.ggnn_vocab_distill_grad, *head, None, 1.0, False, S, S,
                        S + (1 << 30), S + (2 << 30), None, ws, size)
            else:
                refused("GGNN_ERR_WORKSPACE", f"{need} bytes", capi.ggnn_vocab_distill, *head, S, S, ws, size)
        for bad in ((64, 0, 1000, 8), (48, 50, 1000, 8), (64, 50, 1 << 25, 8), (64, 50, 1000, 0), (64, 50, 1000, 65)):
            assert capi.ggnn_vocab_distill_workspace_bytes("bf16", *bad, grad) == 0


def test_distillation_without_rows_succeeds_without_a_device():
    a = dict(DISTILL, n_rows=0, teacher_id=None, teacher_logit=None)
    capi.ggnn_vocab_distill(*a.values(), None, None, None, 0, stream=0)
    capi.ggnn_vocab_distill_grad(*a.values(), None, 1.0, True, None, None, S + (1 << 30), S + (2 << 30), None, None, 0,
                                 stream=0)   # add: nothing is cleared either


TOP = dict(dt="bf16", n_nodes=100, H=64, n_rows=50, V=1000, X=P, W=Q, bias=None, node=S, rules=None, temperature=1.0, K=8,
           top=S, logit=S, lse=None, workspace=S, workspace_bytes=1 << 40)


def rules(**kw):
    a = dict(mask=P, n_masks=3, mask_words=32, mask_of=Q, seen_ptr=P, seen=Q, n_seen=5, repetition=1.2, presence=0.1,
             frequency=0.1, add_ptr=P, add=Q, value=P, n_add=4)
    a.update(kw)
    return dict(rules=capi.token_rules(**a))


@pytest.mark.parametrize("kw,text", [
    (dict(dt=5), "dtype"), (dict(n_nodes=0), "n_nodes"), (dict(H=16), "H="), (dict(n_rows=-1), "n_rows"),
    (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(node=None, n_rows=101), "n_rows=101 exceeds"), (dict(V=0), "V="),
    (dict(V=1 << 25), "V="), (dict(X=None), "X is NULL"), (dict(W=None), "W is NULL"), (dict(bias=P + 2), "bias is not"),
    (dict(node=P + 4), "node is not"), (dict(K=0), "K=0"), (dict(K=65), "K=65"), (dict(temperature=0.0), "temperature"),
    (dict(temperature=NAN), "temperature"), (dict(top=None), "top is NULL"), (dict(top=S + 4), "top is not"),
    (dict(logit=None), "logit is NULL"), (dict(lse=S + 8), "lse is not"), (rules(n_masks=-1), "n_masks"),
    (rules(mask=None), "mask is NULL"), (rules(mask_words=31), "mask_words=31"), (rules(mask_of=P + 4), "mask_of is not"),
    (rules(n_seen=-1), "n_seen"), (rules(n_add=-2), "n_add"), (rules(n_seen=1 << 30), "2^30"),
    (rules(seen_ptr=None), "seen_ptr is NULL"), (rules(seen=None), "seen is NULL"), (rules(repetition=0.0), "repetition"),
    (rules(repetition=float("inf")), "repetition"), (rules(presence=NAN), "presence"),
    (rules(frequency=float("inf")), "frequency"), (rules(add_ptr=None), "add_ptr is NULL"), (rules(add=None), "add is NULL"),
    (rules(value=None), "value is NULL"), (rules(value=P + 8), "value is not")])
def test_top_refuses(kw, text):
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_vocab_top, *dict(TOP, **kw).values())


def test_top_wants_its_workspace():
    for ru, listed in ((None, 0), (rules()["rules"], 9), (rules(n_seen=0)["rules"], 4), (rules(n_add=0)["rules"], 5)):
        need = capi.ggnn_vocab_top_workspace_bytes("bf16", 64, 50, 1000, 8, listed)
        assert need > 0
        for ws, size in ((None, need), (S, need - 1), (S + 8, need)):
            refused("GGNN_ERR_WORKSPACE", f"{need} bytes", capi.ggnn_vocab_top,
                    *dict(TOP, rules=ru, workspace=ws, workspace_bytes=size).values())
    for bad in ((64, 0, 1000, 8, 0), (48, 50, 1000, 8, 0), (64, 50, 1 << 25, 8, 0), (64, 50, 1000, 65, 0),
                (64, 50, 1000, 8, -1), (64, 50, 1000, 8, (1 << 30) + 1)):
        assert capi.ggnn_vocab_top_workspace_bytes("bf16", *bad) == 0


def test_top_without_rows_succeeds_without_a_device():
    capi.ggnn_vocab_top(*dict(TOP, n_rows=0, top=None, logit=None, workspace=None, workspace_bytes=0).values(), stream=0)


def test_rules_reference():
    z = np.array([[2.0, -2.0, 1.0, 0.5]])
    out = L.apply_rules(z, dict(seen=[[0, 1, 1, 9]], repetition=2.0, presence=0.5, frequency=0.25, add=[[(2, 1.0), (2, -3.0)]],
                                mask=[[1, 1, 1, 0]]))
    np.testing.assert_array_equal(out, [[1.0 - 0.75, -4.0 - 1.0, -1.0, -np.inf]])
    ids, zk = L.best(out, 5)
    np.testing.assert_array_equal(ids, [[0, 2, 1, -1, -1]])
    np.testing.assert_array_equal(zk, [[0.25, -1.0, -5.0, -np.inf, -np.inf]])


def test_distillation_reference_against_differences():
    rng = np.random.default_rng(0)
    n, H, V, rows, K = 9, 5, 13, 6, 4
    X, W, b = rng.standard_normal((n, H)), rng.standard_normal((V, H)), rng.standard_normal(V)
    node = rng.permutation(n)[:rows]
    t_id = np.stack([rng.permutation(V)[:K] for _ in range(rows)])
    t_id[1, 2:], t_id[2], t_id[3, 0] = -1, -1, t_id[3, 1]
    t_logit = rng.standard_normal((rows, K))
    t_lse = np.log(np.exp(t_logit / 3.0).sum(1) + 1.0)
    weight = rng.random(rows)
    for T in (None, t_lse):
        def total(X, W, b):
            r = L.distill(X, W, b, node, t_id, t_logit, T, 3.0, weight, 0.7, "f32")
            return 0.7 * float((weight * r["loss"]).sum())
        r = L.distill(X, W, b, node, t_id, t_logit, T, 3.0, weight, 0.7, "f32")
        h = 1e-6
        for name, a, i in (("dX", 0, (int(node[0]), 2)), ("dX", 0, (int(node[3]), 0)), ("dX", 0, (int(node[2]), 1)),
                           ("dW", 1, (int(t_id[0, 0]), 1)), ("dW", 1, (int(t_id[3, 0]), 4)), ("db", 2, (3,))):
            lo, hi = [X.copy(), W.copy(), b.copy()], [X.copy(), W.copy(), b.copy()]
            lo[a][i] -= h
            hi[a][i] += h
            assert abs((total(*hi) - total(*lo)) / (2 * h) - r[name][i]) < 1e-8


def test_rules_of_rows_as_they_are_uploaded():
    from paper_1906_11786_amd.tokens import TokenRules
    V = 70
    allowed = np.zeros((2, V), bool)
    allowed[0, [0, 31, 32, 69]] = True
    allowed[1] = True
    r = TokenRules(V, 3, allowed=allowed, allowed_of=[1, -1, 0], seen=[[5, 5, 2**40], [], [7]], repetition=1.5,
                   bias=[{3: 1.0}, [(4, -np.inf), (4, 2.0)], []], device="cpu")
    mask, of, sp, seen, ap, add, value = [x.numpy() for x in r.tensors]
    np.testing.assert_array_equal(mask.view(np.uint32), [[0x80000001, 1, 0x20], [0xFFFFFFFF, 0xFFFFFFFF, 0x3F]])
    np.testing.assert_array_equal(of, [1, -1, 0])
    np.testing.assert_array_equal(sp, [0, 3, 3, 4])
    np.testing.assert_array_equal(seen, [5, 5, -1, 7])
    np.testing.assert_array_equal(ap, [0, 1, 3, 3])
    np.testing.assert_array_equal(add, [3, 4, 4])
    np.testing.assert_array_equal(value, np.float32([1.0, -np.inf, 2.0]))
    assert r.n_listed == 7 and r.struct.n_masks == 2 and r.struct.mask_words == 3 and r.struct.repetition == 1.5
    empty = TokenRules(V, 2, seen=[[], []], bias=[{}, []], device="cpu")
    assert empty.n_listed == 0 and empty.struct.n_seen == 0 and empty.struct.seen_ptr is None


@pytest.mark.parametrize("kw,text", [
    (dict(allowed=np.zeros((2, 5), bool)), "allowed"), (dict(allowed=np.zeros((2, 6))), "allowed"),
    (dict(allowed=np.zeros((2, 6), bool), allowed_of=[0]), "allowed_of"), (dict(allowed_of=[0, 0, 0]), "without allowed"),
    (dict(seen=[[1]]), "1 seen lists for 3 rows"), (dict(bias=[{}] * 4), "4 bias lists for 3 rows"),
    (dict(repetition=0.0), "penalties"), (dict(presence=float("nan")), "penalties"),
    (dict(frequency=float("inf")), "penalties")])
def test_rules_of_rows_refuse(kw, text):
    from paper_1906_11786_amd.tokens import TokenRules
    with pytest.raises(ValueError, match=text):
        TokenRules(6, 3, device="cpu", **kw)


def test_a_teachers_log_sums_at_another_temperature_are_refused():
    """top()'s dict holds its temperature: the student takes it, or is refused one that the log sums do not fit."""
    torch = pytest.importorskip("torch")
    from test_host_tokens import node_tokens
    t = node_tokens()
    lists = dict(token=torch.tensor([[3, 4], [5, -1]]), logit=torch.tensor([[2.0, 1.0], [0.5, 0.0]]))
    out = dict(lists, lse=torch.tensor([3.0, 4.0]), temperature=torch.tensor(1.0, dtype=torch.float64))
    for told in (out, {k: v.numpy() for k, v in out.items()}, dict(out, temperature=1.0)):
        t.setup_training([0, 2], [1, 2], teacher=told)
        assert t.teacher["temperature"] == 1.0 and t.teacher["scale"] == 0.5 / 2
        t.setup_training([0, 2], [1, 2], teacher=told, temperature=1)
        for other in (2.0, 0.999):
            with pytest.raises(ValueError, match="log sums are at temperature 1, not"):
                t.setup_training([0, 2], [1, 2], teacher=told, temperature=other)
    t.setup_training([0, 2], [1, 2], teacher=dict(out, temperature=0.3), temperature=float(np.float32(0.3)))
    t.setup_training([0, 2], [1, 2], teacher=dict(lists, temperature=1.0), temperature=2.0)   # lists alone: any
    assert t.teacher["temperature"] == 2.0
    for plain in (lists, dict(lists, lse=out["lse"])):   # nothing told: what is asked for, or 2
        t.setup_training([0, 2], [1, 2], teacher=plain, temperature=3.0)
        assert t.teacher["temperature"] == 3.0
        t.setup_training([0, 2], [1, 2], teacher=plain)
        assert t.teacher["temperature"] == 2.0 and t.teacher["scale"] == 0.5 * 4 / 2
    with pytest.raises(ValueError, match="temperature"):
        t.setup_training([0, 2], [1, 2], teacher=dict(lists, temperature=0.0))


@pytest.mark.parametrize("kw", [
    dict(teacher=dict(token=np.full((3, 2), 20), logit=np.zeros((3, 2)))), dict(teacher=dict(token=np.zeros((2, 2), int),
    logit=np.zeros((2, 2)))), dict(teacher=dict(token=np.zeros((3, 2), int), logit=np.zeros((3, 2)), lse=np.zeros(2))),
    dict(teacher=dict(token=np.zeros((3, 2), int), logit=np.zeros((3, 2))), soft=2.0), dict(target=[1, 2, 20])])
def test_a_refused_set_up_leaves_the_one_before_it(kw):
    from test_host_tokens import node_tokens
    t = node_tokens()
    teacher = dict(token=np.array([[3, 4], [5, -1]]), logit=np.zeros((2, 2)))
    t.setup_training([0, 2], [1, -1], teacher=teacher, lr=0.5)
    t.step = 7
    before = dict(vars(t))
    with pytest.raises(ValueError):
        t.setup_training(**dict(dict(node=[1, 2, 3], target=[1, 2, 3]), **kw))
    assert vars(t).keys() == before.keys() and all(vars(t)[k] is before[k] for k in before)


def test_rules_on_another_device_are_refused():
    from paper_1906_11786_amd.tokens import TokenRules
    from test_host_tokens import node_tokens
    t = node_tokens()
    for kw in (dict(seen=[[1], [2]]), dict(bias=[{1: 2.0}, {}]), dict(allowed=np.ones((2, 20), bool))):
        with pytest.raises(ValueError, match="rules on meta, the model is on cpu"):
            t.top([0, 2], 3, TokenRules(20, 2, device="meta", **kw))
