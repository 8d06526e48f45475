"""Timing cases of the token operators: node states from a token table and the table's gradient, dropout with a
mask that is never stored, and the cross entropy of chosen nodes over a vocabulary with its gradient.

A graph's nodes carry labels made of (sub)tokens: a node's first state is the scaled sum or mean of its tokens' table
rows, with dropout; after propagation, chosen nodes (hidden ones in training, one asked-for node in serving) answer
with a token of the vocabulary.  The cases cover that range on this package's graph sizes (512, 20,000, 100,000 and
1,048,576 nodes; H = 32 .. 256; float32 and bfloat16), with vocabularies from a few hundred to 50,021 tokens.

`own = False` computes the operators in elementary torch operations in float32; `own = True` calls the package.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ES = {"f32": 4, "bf16": 2}

LISTED = [
    # one small graph's node labels, one token each: the launch is all there is
    dict(name="embed tiny f32", op="embed", dt="f32", n=512, real=512, H=32, V=997, bag=0, p=0.0),
    # a 20,000-node program graph (padded to whole blocks), each label the mean of its subtokens, with dropout
    dict(name="embed bags 20k bf16", op="embed", dt="bf16", n=20096, real=20000, H=64, V=10007, bag=6, p=0.1),
    # the 1M-node batch, one token per node
    dict(name="embed 1M bf16", op="embed", dt="bf16", n=1048576, real=1047000, H=256, V=50021, bag=0, p=0.1),
    # their gradients: the 20,000-node graph's, and the 1M-node batch's with subtokens
    dict(name="embed grad bags 20k", op="embed_grad", dt="f32", n=20096, real=20000, H=64, V=10007, bag=6, p=0.1),
    dict(name="embed grad bags 1M", op="embed_grad", dt="f32", n=1048576, real=1047000, H=256, V=50021, bag=4, p=0.1),
    # dropout's reverse on one graph's float32 gradient (an odd count), and its forward on the 1M-node states
    dict(name="dropout grad 20k f32", op="dropout", dt="f32", count=20000 * 64 - 3, p=0.1),
    dict(name="dropout 1M bf16", op="dropout", dt="bf16", count=1048576 * 256, p=0.1),
    # serving: the loss of one node's token
    dict(name="vocab one node bf16", op="vocab", dt="bf16", n=20096, rows=1, H=64, V=10007, bias=True),
    # evaluation: held-out nodes of a 20,000-node graph against the large vocabulary
    dict(name="vocab eval 3k bf16", op="vocab", dt="bf16", n=20096, rows=2999, H=128, V=50021, bias=False),
    # a training step's loss and gradients: hidden nodes of one 20,000-node graph; the same in float32 on a smaller
    # vocabulary; and hidden nodes of the 1M-node batch
    dict(name="vocab grad 3k bf16", op="vocab_grad", dt="bf16", n=20096, rows=3001, H=64, V=10007, bias=True),
    dict(name="vocab grad 1k f32", op="vocab_grad", dt="f32", n=8192, rows=1229, H=128, V=4999, bias=True),
    dict(name="vocab grad 60k bf16", op="vocab_grad", dt="bf16", n=1048576, rows=60001, H=256, V=50021, bias=False),
]


def listed():
    return [dict(c) for c in LISTED]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges: each operator, type and width, sizes spread over their logarithm."""
    op = rng.choice(["embed", "embed_grad", "dropout", "vocab", "vocab_grad"])
    dt = rng.choice(["f32", "bf16"])
    p = rng.choice([0.0, 0.1, 0.25, 0.5])
    if op == "dropout":
        return dict(op=op, dt=dt, count=_log_int(rng, 1000, 1 << 27), p=max(p, 0.1))
    H = rng.choice([32, 64, 128, 256])
    V = _log_int(rng, 300, 50021)
    if op in ("embed", "embed_grad"):
        real = _log_int(rng, 200, (1 << 28) // H // 4)
        n = -(-real // 32) * 32
        return dict(op=op, dt="f32" if op == "embed_grad" else dt, n=n, real=real, H=H, V=V, bag=rng.choice([0, 3, 6]), p=p)
    rows = _log_int(rng, 1, 30000 if dt == "bf16" else 6000)
    n = -(-max(rows * rng.randint(1, 8), 32) // 32) * 32
    return dict(op=op, dt=dt, n=n, rows=rows, H=H, V=V, bias=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

def _tokens(g, count, V):
    """Token ids whose frequency falls with the id, as a vocabulary sorted by frequency has it."""
    u = torch.rand((count,), generator=g, device="cuda")
    return (torch.exp(u * math.log(V + 1.0)) - 1.0).to(torch.int32).clamp_(0, V - 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case, seed=(int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), offset=int(seed) % 1000)
    op = case["op"]
    if op == "dropout":
        s["X"] = normal(case["count"]).to(DT[case["dt"]])
        s["Y"] = torch.empty_like(s["X"])
        return s
    H, V, n = case["H"], case["V"], case["n"]
    td = DT[case["dt"]]
    if op in ("embed", "embed_grad"):
        real, bag = case["real"], case["bag"]
        if bag:   # 0 .. bag subtokens a node, none for the padding nodes
            lens = torch.randint(0, bag + 1, (real,), generator=g, device="cuda", dtype=torch.int32)
            s["tok_ptr"] = torch.zeros((n + 1,), dtype=torch.int32, device="cuda")
            s["tok_ptr"][1:real + 1] = torch.cumsum(lens, 0)
            s["tok_ptr"][real + 1:] = s["tok_ptr"][real]
            s["n_tok"] = int(s["tok_ptr"][real])
        else:
            s["tok_ptr"], s["n_tok"] = None, real
        s["tok"] = _tokens(g, max(s["n_tok"], 1), V)
        s["scale"] = math.sqrt(H)
        if op == "embed":
            s["table"] = (normal(V, H) / math.sqrt(H)).to(td)
            s["X"] = torch.empty((n, H), dtype=td, device="cuda")
        else:
            s["dX"] = normal(n, H) * 1e-3
            s["dtable"] = torch.empty((V, H), device="cuda")
        return s
    # chosen nodes' final states: noise and a part of the target's row, so that some nodes know their token and
    # some do not; every 16th target is left out (no loss)
    rows = case["rows"]
    W = normal(V, H) * (1.5 / math.sqrt(H))
    s["node"] = torch.randperm(n, generator=g, device="cuda")[:rows].to(torch.int32)
    s["target"] = _tokens(g, rows, V)
    knows = 2.5 * torch.rand((rows, 1), generator=g, device="cuda")
    X = normal(n, H)
    X[s["node"].long()] += knows * W[s["target"].long()]
    s["target"][15::16] = -1
    s["X"], s["W"] = X.to(td), W.to(td)
    s["b"] = 0.5 * normal(V) if case["bias"] else None
    if op == "vocab_grad":
        s["scale"] = 1.0 / rows
        s["dX"] = torch.empty((n, H), device="cuda")
        s["dW"] = torch.empty((V, H), device="cuda")
        s["db"] = torch.empty((V,), device="cuda") if case["bias"] else None
    s["loss"] = torch.empty((rows,), device="cuda")
    s["lse"] = torch.empty((rows,), device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    op = s["op"]
    if op == "dropout":
        return _drop(s["X"].float(), 0, s).to(s["X"].dtype)
    if op == "embed":
        return _embed_plain(s)
    if op == "embed_grad":
        return _embed_grad_plain(s)
    return _vocab_plain(s, op == "vocab_grad")


def _workspace(s, need):
    """The call's scratch memory, kept with the buffers of the state."""
    if "ws" not in s:
        s["ws"] = torch.empty((max(need, 16),), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own(s):
    from paper_1906_11786_amd import capi

    op, dt = s["op"], s["dt"]
    if op == "dropout":
        capi.ggnn_dropout(dt, s["count"], s["X"], s["p"], s["seed"], s["offset"], s["Y"])
        return s["Y"]
    n, H, V = s["n"], s["H"], s["V"]
    if op == "embed":
        capi.ggnn_embed(dt, n, H, V, s["table"], s["tok_ptr"], s["tok"], s["n_tok"], s["scale"], True, s["p"],
                        s["seed"], s["offset"], s["X"])
        return s["X"]
    if op == "embed_grad":
        need = capi.ggnn_embed_bwd_workspace_bytes(n, H, V, s["n_tok"])
        ws = _workspace(s, need)
        s["dtable"].zero_()
        capi.ggnn_embed_bwd(n, H, V, s["tok_ptr"], s["tok"], s["n_tok"], s["scale"], True, s["p"], s["seed"],
                            s["offset"], s["dX"], s["dtable"], ws, ws.numel())
        return s["dtable"]
    ws = _workspace(s, capi.ggnn_vocab_workspace_bytes(dt, H, s["rows"], V, op == "vocab_grad"))
    if op == "vocab":
        capi.ggnn_vocab_loss(dt, n, H, s["rows"], V, s["X"], s["W"], s["b"], s["node"], s["target"], s["loss"],
                             s["lse"], None, ws, ws.numel())
        return {"loss": s["loss"], "lse": s["lse"]}
    s["dW"].zero_()
    if s["db"] is not None:
        s["db"].zero_()
    capi.ggnn_vocab_loss_grad(dt, n, H, s["rows"], V, s["X"], s["W"], s["b"], s["node"], s["target"], None,
                              s["scale"], s["loss"], s["lse"], s["dX"], s["dW"], s["db"], ws, ws.numel())
    out = {"loss": s["loss"], "lse": s["lse"], "dX": s["dX"], "dW": s["dW"]}
    if s["db"] is not None:
        out["db"] = s["db"]
    return out


# ---- plain forms, float32 throughout

M32 = 0xFFFFFFFF


def _philox_round(state, i):
    """Round i of Philox4x32 (Salmon et al. 2011) on int64 tensors that hold 32-bit words."""
    c0, c1, c2, c3, k0, k1 = state
    a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57   # mod 2^64: bits 32 .. 63 are those of the full product
    return ((b >> 32) & M32) ^ c1 ^ k0, b & M32, ((a >> 32) & M32) ^ c3 ^ k1, a & M32, (k0 + 0x9E3779B9) & M32, \
        (k1 + 0xBB67AE85) & M32


def _drop(x, first, s):
    """Dropout of a flat float32 tensor whose elements are numbers first, first + 1, ... of the whole: element e takes
    16-bit word e % 8 of the 7-round Philox4x32 block at counter (e / 8, offset) under the key `seed`, and stays where
    that is at least p * 2^16."""
    cut = round(s["p"] * 65536)
    if cut == 0:
        return x
    count = x.numel()
    b = torch.arange(first // 8, (first + count + 7) // 8, device=x.device)
    zero = torch.zeros_like(b)
    start = (b & M32, b >> 32, zero + (s["offset"] & M32), zero + (s["offset"] >> 32), s["seed"] & M32, s["seed"] >> 32)
    w = torch.stack(functools.reduce(_philox_round, range(7), start)[:4], 1)
    u = torch.stack((w & 0xFFFF, w >> 16), 2).reshape(-1)[first % 8:first % 8 + count]
    return torch.where(u >= cut, x.reshape(-1) * (65536.0 / (65536 - cut)), 0.0).view(x.shape)


def _row_of_token(s):
    """(row of each listed token, factor of each row): scale / length of the row's list."""
    n, real = s["n"], s["real"]
    if s["tok_ptr"] is None:
        return torch.arange(s["n_tok"], device="cuda"), torch.full((n, 1), s["scale"], device="cuda")
    lens = s["tok_ptr"].diff()
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), lens.long(), output_size=s["n_tok"])
    return row, (s["scale"] / lens.clamp(min=1).float())[:, None]


def _embed_plain(s):
    row, factor = _row_of_token(s)
    tok = s["tok"][:s["n_tok"]].long()
    X = torch.zeros((s["n"], s["H"]), device="cuda").index_add_(0, row, s["table"][tok].float()) * factor
    return _drop(X, 0, s).to(DT[s["dt"]])


def _embed_grad_plain(s):
    row, factor = _row_of_token(s)
    G = _drop(s["dX"], 0, s) * factor
    return torch.zeros((s["V"], s["H"]), device="cuda").index_add_(0, s["tok"][:s["n_tok"]].long(), G[row])


def _vocab_plain(s, grad):
    node, target = s["node"].long(), s["target"].long()
    x, W = s["X"][node].float(), s["W"].float()
    z = x @ W.t()
    if s["b"] is not None:
        z += s["b"]
    top = z.amax(1, keepdim=True)
    has = target >= 0
    t = target.clamp(min=0)[:, None]
    zt = z.gather(1, t)
    e = z.sub_(top).exp_()
    total = e.sum(1, keepdim=True)
    lse = top + total.log()
    out = {"loss": torch.where(has, (lse - zt)[:, 0], 0.0), "lse": lse[:, 0]}
    if not grad:
        return out
    g = torch.where(has, s["scale"], 0.0)[:, None]
    dz = e.mul_(g / total)
    dz.scatter_add_(1, t, -g)
    out["dX"] = torch.zeros((s["n"], s["H"]), device="cuda").index_copy_(0, node, dz @ W)
    out["dW"] = dz.t() @ x
    if s["b"] is not None:
        out["db"] = dz.sum(0)
    return out


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]

    def kept(count):
        """1 / keep probability where element e of `count` stays, else 0, in float64.  The generator's 32 x 32 bit
        products are put together from 16-bit halves."""
        cut = round(s["p"] * 65536)
        if cut == 0:
            return None

        def product(c, m):
            lo, hi = c % 65536, c // 65536
            ml, mh = m % 65536, m // 65536
            low = lo * ml
            mid = lo * mh + low // 65536
            mid2 = hi * ml + mid % 65536
            return hi * mh + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + low % 65536

        blocks = -(-count // 8)
        e = torch.arange(blocks, device="cuda")
        words = [e % (1 << 32), e // (1 << 32), torch.full_like(e, s["offset"] % (1 << 32)),
                 torch.full_like(e, s["offset"] // (1 << 32))]
        key = [s["seed"] % (1 << 32), s["seed"] // (1 << 32)]
        for r in range(7):
            h0, l0 = product(words[0], 0xD2511F53)
            h1, l1 = product(words[2], 0xCD9E8D57)
            words = [h1 ^ words[1] ^ ((key[0] + r * 0x9E3779B9) % (1 << 32)), l1,
                     h0 ^ words[3] ^ ((key[1] + r * 0xBB67AE85) % (1 << 32)), l0]
        keep = torch.empty((blocks, 8), dtype=torch.float64, device="cuda")
        for k in range(8):
            u = words[k // 2] // (65536 if k % 2 else 1) % 65536
            keep[:, k] = (u >= cut).double() * (65536.0 / (65536.0 - cut))
        return keep.view(-1)[:count]

    if op == "dropout":
        return s["X"].double() * kept(case["count"])
    n, H, V = case["n"], case["H"], case["V"]
    if op in ("embed", "embed_grad"):
        ids = s["tok"].long()[:s["n_tok"]]
        if s["tok_ptr"] is None:
            first = torch.arange(n, device="cuda").clamp(max=s["n_tok"])
            last = torch.arange(1, n + 1, device="cuda").clamp(max=s["n_tok"])
        else:
            first, last = s["tok_ptr"][:-1].long(), s["tok_ptr"][1:].long()
        length = last - first
        keep = kept(n * H)
        c = s["scale"] / length.clamp(min=1).double()
        # the k-th token of every row that has one, for k = 0, 1, ...
        if op == "embed":
            T, X = s["table"].double(), torch.zeros((n, H), dtype=torch.float64, device="cuda")
            for k in range(int(length.max())):
                r = torch.nonzero(length > k)[:, 0]
                X[r] += T[ids[first[r] + k]]
            X *= c[:, None]
            return X if keep is None else X * keep.view(n, H)
        G = s["dX"].double() * c[:, None]
        if keep is not None:
            G *= keep.view(n, H)
        dT = torch.zeros((V, H), dtype=torch.float64, device="cuda")
        for k in range(int(length.max())):
            r = torch.nonzero(length > k)[:, 0]
            dT.index_add_(0, ids[first[r] + k], G[r])
        return dT
    # vocabulary: blocks of rows
    rows, grad = case["rows"], op == "vocab_grad"
    W = s["W"].double()
    loss = torch.empty((rows,), dtype=torch.float64, device="cuda")
    lse = torch.empty_like(loss)
    dX = torch.zeros((n, H), dtype=torch.float64, device="cuda") if grad else None
    dW = torch.zeros((V, H), dtype=torch.float64, device="cuda") if grad else None
    db = torch.zeros((V,), dtype=torch.float64, device="cuda") if grad else None
    for lo in range(0, rows, 8192):
        at = slice(lo, min(rows, lo + 8192))
        node, tgt = s["node"][at].long(), s["target"][at].long()
        x = s["X"][node].double()
        z = torch.mm(x, W.t().contiguous())
        if s["b"] is not None:
            z += s["b"].double()
        lse[at] = torch.logsumexp(z, 1)
        live = torch.nonzero(tgt >= 0)[:, 0]
        loss[at] = 0.0
        loss[lo + live] = lse[at][live] - z[live, tgt[live]]
        if grad:
            P = torch.exp(z - lse[at][:, None])
            P[live, tgt[live]] -= 1.0
            P[tgt < 0] = 0.0
            P *= s["scale"]
            dX[node] = torch.mm(P, W)
            dW += torch.mm(P.t().contiguous(), x)
            db += P.sum(0)
    out = {"loss": loss, "lse": lse}
    if grad:
        out.update(dX=dX, dW=dW)
        if s["b"] is not None:
            out["db"] = db
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "dropout":
        return {"bytes": 2 * case["count"] * ES[case["dt"]], "flops": case["count"]}
    n, H, V, es = case["n"], case["H"], case["V"], ES[case["dt"]]
    if op in ("embed", "embed_grad"):
        n_tok = case["real"] * case["bag"] // 2 if case["bag"] else case["real"]
        lists = 4 * n_tok + (4 * (n + 1) if case["bag"] else 0)
        if op == "embed":
            return {"bytes": lists + min(V, n_tok) * H * es + n * H * es, "flops": n_tok * H + n * H}
        return {"bytes": lists + case["real"] * H * 4 + V * H * 4, "flops": n_tok * H + n * H}
    rows = case["rows"]
    bias = 4 * V if case["bias"] else 0
    read = rows * H * es + V * H * es + bias + 16 * rows
    if op == "vocab":
        return {"bytes": read, "flops": 2 * rows * V * H}
    # logits, the gradient of the states and the gradient of the vocabulary's rows: one product each
    return {"bytes": read + n * H * 4 + V * H * 4 + bias, "flops": 6 * rows * V * H}
