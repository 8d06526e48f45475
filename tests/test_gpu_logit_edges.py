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
