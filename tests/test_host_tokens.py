"""Token operators on the CPU: refusals (checked before anything reaches the
device) and the generator's published structure."""
import numpy as np
import pytest

import token_reference as R

capi = pytest.importorskip("paper_1906_11786_amd.capi")

P, Q, S = 1 << 20, 1 << 30, 1 << 34   # 16-byte aligned stand-in addresses; nothing is launched
NAN = float("nan")


def refused(status, text, fn, *args):
    with pytest.raises(capi.GGNNError) as e:
        fn(*args, stream=0)
    assert e.value.status_name == status, str(e.value)
    assert text in str(e.value), str(e.value)


@pytest.mark.parametrize("args,text", [
    ((7, 8, P, 0.1, 0, 0, Q), "dtype"),
    (("f32", -1, P, 0.1, 0, 0, Q), "count"),
    (("f32", (1 << 34) + 1, P, 0.1, 0, 0, Q), "count"),
    (("f32", 8, P, 1.0, 0, 0, Q), "p="),
    (("f32", 8, P, -0.1, 0, 0, Q), "p="),
    (("f32", 8, P, NAN, 0, 0, Q), "p="),
    (("f32", 8, None, 0.1, 0, 0, Q), "X is NULL"),
    (("f32", 8, P, 0.1, 0, 0, Q + 4), "Y is not 16-byte aligned"),
    (("f32", 800, P, 0.1, 0, 0, P + 16), "overlap"),
])
def test_dropout_refuses(args, text):
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_dropout, *args)


def embed_args(**kw):
    a = dict(dt="bf16", n=10, H=64, V=20, table=P, tok_ptr=Q, tok=Q, n_tok=30, scale=1.0, mean=True, p=0.1, seed=0,
             offset=0, X=S)
    a.update(kw)
    return list(a.values())


EMBED_BAD = [(dict(n=-1), "n="), (dict(H=48), "H="), (dict(V=0), "V="), (dict(n_tok=-1), "n_tok"),
             (dict(n_tok=(1 << 30) + 1), "n_tok"), (dict(tok_ptr=None), "n_tok=30 exceeds n=10"),
             (dict(scale=NAN), "scale"), (dict(p=1.5), "p="), (dict(tok=None), "tok is NULL"),
             (dict(tok_ptr=Q + 4), "tok_ptr is not"), (dict(n=1 << 29, H=256), "2^34")]


@pytest.mark.parametrize("kw,text", EMBED_BAD + [(dict(dt=9), "dtype"), (dict(table=None), "table is NULL"),
                                                 (dict(X=None), "X is NULL"), (dict(X=P + 64), "overlaps")])
def test_lookup_refuses(kw, text):
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_embed, *embed_args(**kw))


@pytest.mark.parametrize("kw,text", EMBED_BAD + [(dict(dX=None), "dX is NULL"), (dict(dtable=None), "dtable is NULL"),
                                                 (dict(dtable=P + 64), "overlaps")])
def test_table_gradient_refuses(kw, text):
    a = dict(n=10, H=64, V=20, tok_ptr=Q, tok=Q, n_tok=30, scale=1.0, mean=True, p=0.1, seed=0, offset=0, dX=P,
             dtable=S, workspace=Q, workspace_bytes=1 << 30)
    a.update(kw)
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_embed_bwd, *a.values())


def test_table_gradient_wants_its_workspace():
    need = capi.ggnn_embed_bwd_workspace_bytes(10, 64, 20, 30)
    assert need > 0
    for ws, size in ((None, need), (Q, need - 1), (Q + 8, need)):
        refused("GGNN_ERR_WORKSPACE", f"{need} bytes", capi.ggnn_embed_bwd, 10, 64, 20, Q, Q, 30, 1.0, True, 0.0, 0, 0, P,
                S, ws, size)
    assert capi.ggnn_embed_bwd_workspace_bytes(10, 48, 20, 30) == 0
    assert capi.ggnn_embed_bwd_workspace_bytes(10, 64, 20, -1) == 0


VOCAB_BAD = [(dict(dt=5), "dtype"), (dict(n_nodes=0), "n_nodes"), (dict(H=16), "H="), (dict(n_rows=-1), "n_rows"),
             (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(node=None, n_rows=101), "n_rows=101 exceeds"),
             (dict(V=0), "V="), (dict(V=1 << 25), "V="), (dict(X=None), "X is NULL"), (dict(W=None), "W is NULL"),
             (dict(bias=P + 2), "bias is not"), (dict(node=P + 4), "node is not"), (dict(target=P + 4), "target is not"),
             (dict(lse=None), "lse is NULL"), (dict(loss=None), "loss is NULL")]


@pytest.mark.parametrize("kw,text", VOCAB_BAD + [(dict(best=P + 8), "best is not")])
def test_vocab_loss_refuses(kw, text):
    a = dict(dt="bf16", n_nodes=100, H=64, n_rows=50, V=1000, X=P, W=Q, bias=None, node=S, target=S, loss=S, lse=S,
             best=None, workspace=S, workspace_bytes=1 << 40)
    a.update(kw)
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_vocab_loss, *a.values())


@pytest.mark.parametrize("kw,text", VOCAB_BAD + [
    (dict(target=None), "target is NULL"), (dict(dX=None), "dX is NULL"), (dict(dW=None), "dW is NULL"),
    (dict(dbias=P + 4), "dbias is not"), (dict(weight=P + 4), "weight is not"), (dict(scale=float("inf")), "scale"),
    (dict(dX=P + 16), "dX overlaps"), (dict(dW=Q + 16), "dW overlaps"), (dict(dW=S + (1 << 30)), "dW overlaps")])
def test_vocab_gradients_refuse(kw, text):
    a = dict(dt="bf16", n_nodes=100, H=64, n_rows=50, V=1000, X=P, W=Q, bias=None, node=S, target=S, weight=None,
             scale=1.0, loss=S, lse=S, dX=S + (1 << 30), dW=S + (2 << 30), dbias=None, workspace=S,
             workspace_bytes=1 << 40)
    a.update(kw)
    refused("GGNN_ERR_INVALID_ARG", text, capi.ggnn_vocab_loss_grad, *a.values())


def test_vocab_wants_its_workspace():
    for grad in (False, True):
        need = capi.ggnn_vocab_workspace_bytes("bf16", 64, 50, 1000, grad)
        assert need > 0
        head = ("bf16", 100, 64, 50, 1000, P, Q, None, S, S)
        for ws, size in ((None, need), (S, need - 1), (S + 8, need)):
            if grad:
                refused("GGNN_ERR_WORKSPACE", f"{need} bytes", capi.ggnn_vocab_loss_grad, *head, None, 1.0, S, S,
                        S + (1 << 30), S + (2 << 30), None, ws, size)
            else:
                refused("GGNN_ERR_WORKSPACE", f"{need} bytes", capi.ggnn_vocab_loss, *head, S, S, None, ws, size)
        assert capi.ggnn_vocab_workspace_bytes("bf16", 64, 0, 1000, grad) == 0
        assert capi.ggnn_vocab_workspace_bytes("bf16", 48, 50, 1000, grad) == 0
        assert capi.ggnn_vocab_workspace_bytes("bf16", 64, 50, 1 << 25, grad) == 0


def test_calls_without_work_succeed_without_a_device():
    capi.ggnn_dropout("f32", 0, None, 0.1, 0, 0, None, stream=0)
    capi.ggnn_dropout("f32", 100, P, 0.0, 0, 0, P, stream=0)   # nothing dropped, in place
    capi.ggnn_embed("f32", 0, 32, 5, None, None, None, 0, 1.0, False, 0.0, 0, 0, None, stream=0)
    capi.ggnn_embed_bwd(10, 32, 5, None, None, 0, 1.0, False, 0.0, 0, 0, None, None, None, 0, stream=0)
    capi.ggnn_vocab_loss("f32", 10, 32, 0, 5, P, Q, None, None, None, None, None, None, None, 0, stream=0)


def test_generator_words_are_spread_evenly():
    """The reference generator of the GPU tests: 16-bit words over 64 bins, chi-square within 6 standard deviations;
    another key or offset changes about half of all bits."""
    w = R.philox7(np.arange(1 << 16, dtype=np.uint64), 5, 2**40 + 9)
    h = np.stack([w & 0xFFFF, w >> 16], 2).reshape(-1)
    n = np.bincount(h >> 10, minlength=64)
    e = len(h) / 64
    chi = float(((n - e) ** 2 / e).sum())
    assert abs(chi - 63) < 6 * (2 * 63) ** 0.5
    for other in (R.philox7(np.arange(1 << 16, dtype=np.uint64), 6, 2**40 + 9),
                  R.philox7(np.arange(1 << 16, dtype=np.uint64), 5, 2**40 + 8)):
        bits = np.unpackbits((w ^ other).view(np.uint8)).mean()
        assert abs(bits - 0.5) < 6 * 0.5 / (w.size * 32) ** 0.5


def test_token_lists_layout():
    tokens = pytest.importorskip("paper_1906_11786_amd.tokens")
    ptr, tok = tokens.token_lists([[3, 1], [], [2]], 5)
    assert ptr.tolist() == [0, 2, 2, 3, 3, 3] and tok.tolist() == [3, 1, 2]
    assert ptr.dtype == np.int32 and tok.dtype == np.int32
    ptr, tok = tokens.token_lists([[], []], 4)
    assert ptr.tolist() == [0, 0, 0, 0, 0] and len(tok) == 1
    with pytest.raises(ValueError, match="3 token lists for 2 nodes"):
        tokens.token_lists([[], [], []], 2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H", [32, 64, 128, 256])
def test_vocab_workspace_grows_with_its_rows_and_entries(dt, H):
    """One row, or one entry, more than the workgroups take in whole tiles costs shares of that tile only: every tile
    dealt whole has one share, and the others of a pass at most four per workgroup."""
    workers = 256 * {32: 4, 64: 3, 128: 3, 256: 1}[H]          # that the compute units hold, at most
    share = 128 * (4 * H + 16)                                  # O (or dW), maximum, sum, best entry
    up = (lambda x: -(-x // 128) * 128)

    def bound(rows, V, grad):
        per_row = 16 + (4 * H + 6 * H + 64 + H * H // 1024 if grad else 0)   # shares; state, sort and its partial sums
        return up(rows) * per_row + (6 * V * H if dt == "f32" else 0) + (2 if grad else 1) * 4 * workers * share + (1 << 20)

    most = ((1 << 31) - 1) // H
    sizes = [(128 * w * k + d, 50021) for w in (256, 512, 768, 1024) for k in (1, 3) for d in (-1, 0, 1, 129)]
    sizes += [(r, 128 * w + d) for r in (33, 3001, 30000) for w in (256, 512, 768, 1024, 2048) for d in (0, 2, 200)]
    sizes += [(1 << 24, 50021), ((1 << 24) - 32767, 50021), (3001, most), (3001, most - 127)]
    for rows, V in sizes:
        if V > most:
            continue
        for grad in (False, True):
            need = capi.ggnn_vocab_workspace_bytes(dt, H, rows, V, grad)
            assert 0 < need <= bound(rows, V, grad), (rows, V, grad, need, bound(rows, V, grad))


def test_table_gradient_of_nothing_needs_no_workspace():
    assert capi.ggnn_embed_bwd_workspace_bytes(10, 64, 20, 0) == 0
    assert capi.ggnn_embed_bwd_workspace_bytes(0, 64, 20, 30) == 0
    capi.ggnn_embed_bwd(10, 64, 20, Q, None, 0, 1.0, True, 0.0, 0, 0, P, S, None, 0, stream=0)
    capi.ggnn_embed_bwd(0, 64, 20, Q, Q, 30, 1.0, True, 0.0, 0, 0, P, S, None, 0, stream=0)


def node_tokens(n=4, H=32, V=20, **kw):
    """NodeTokens on host buffers (nothing is launched)."""
    import types
    torch = pytest.importorskip("torch")
    tokens = pytest.importorskip("paper_1906_11786_amd.tokens")
    model = types.SimpleNamespace(comp=types.SimpleNamespace(n_pad=n), H=H, T=1, dt="f32", device="cpu",
                                  X=torch.zeros((2, n, H)), master=torch.zeros((64,)))
    a = dict(table=np.zeros((V, H)), tok_ptr=[0, 2, 5, 5, 6], tok=[1, 2, 3, 4, 5, 6])
    a.update(kw)
    return tokens.NodeTokens(model, **a)


@pytest.mark.parametrize("wide", [2**32 + 5, 2**31 + 7, 2**40, -2**32 + 3, -2**63])
def test_node_tokens_of_ids_past_32_bits_are_no_tokens(wide):
    """An id outside the table adds nothing; its low 32 bits would name another token."""
    t = node_tokens(tok=np.array([1, wide, 3, 4, 5, 6], np.int64))
    got = t.tok.tolist()
    assert got[0] == 1 and got[2:] == [3, 4, 5, 6] and not 0 <= got[1] < 20
    tokens = pytest.importorskip("paper_1906_11786_amd.tokens")
    _, tok = tokens.token_lists([np.array([3, wide], np.int64), [wide], [2]], 4)
    assert tok.dtype == np.int32 and tok[[0, 3]].tolist() == [3, 2] and tok[1] == tok[2] and not 0 <= tok[1] < 2**31 - 1


@pytest.mark.parametrize("target", [-2**32, -2**33 + 4, -2**63])
def test_node_tokens_targets_below_32_bits_stay_negative(target):
    t = node_tokens()
    t.setup_training([0, 2], np.array([3, target], np.int64))
    assert t.target[0].item() == 3 and t.target[1].item() < 0 and t.n_live == 1


def test_node_tokens_counts_past_32_bits_are_refused():
    tokens = pytest.importorskip("paper_1906_11786_amd.tokens")
    with pytest.raises(ValueError, match="2\\^30"):
        tokens.token_lists([range(1 << 30), range(5)], 4)
    with pytest.raises(ValueError, match="2\\^30"):
        tokens.token_lists([range(1 << 31), range(1 << 31), [1]], 4)


@pytest.mark.parametrize("bias", [0.5, [0.5], np.zeros(19), np.zeros(21), np.zeros((20, 1)), np.zeros((2, 20))])
def test_node_tokens_bias_of_another_shape_is_refused(bias):
    with pytest.raises(ValueError, match="bias"):
        node_tokens(bias=bias)
    assert node_tokens(bias=np.arange(20.0)).bias.tolist() == list(range(20))
