"""Timing cases of the operators around a vocabulary's logits: the best tokens of chosen nodes with their logits, the same
under rules (grammar masks, penalties of repeated tokens, biases), and the distillation loss from a teacher's top logits
with its gradients.

Chosen nodes of a graph answer with tokens of a vocabulary.  Serving asks for the best few of one node or of many, under
rules that say which tokens fit the place and which were used already; a teacher model leaves its top logits for
every hidden node of a training set, and a student is trained on them.  The cases cover that range on this package's graph
sizes (512 to 1,048,576 nodes, H = 32 .. 256, float32 and bfloat16) and vocabularies from 997 to 50,021 tokens.

`own = False` computes the operators in elementary torch operations in float32; `own = True` calls the package.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ES = {"f32": 4, "bf16": 2}
INF = float("inf")

LISTED = [
    # serving: the eight best tokens of one node; latency is all there is
    dict(name="top one node bf16", op="top", dt="bf16", n=20096, rows=1, H=64, V=10007, K=8, bias=True, tau=1.0),
    # a float32 teacher's lists on a small vocabulary
    dict(name="top 1k f32", op="top", dt="f32", n=8192, rows=1229, H=128, V=4999, K=16, bias=True, tau=2.0),
    # evaluation: ranked answers of held-out nodes of a 20,000-node graph against the large vocabulary
    dict(name="top eval 3k bf16", op="top", dt="bf16", n=20096, rows=2999, H=128, V=50021, K=32, bias=False, tau=1.0),
    # a teacher's lists for hidden nodes of the large batch
    dict(name="top teacher 12k bf16", op="top", dt="bf16", n=131072, rows=12001, H=256, V=50021, K=32, bias=False, tau=2.0),
    # serving under rules: one node with a mask and a short list of used tokens; a batch of requests with long lists;
    # evaluation of many nodes
    dict(name="rules one node bf16", op="rules", dt="bf16", n=20096, rows=1, H=256, V=50021, K=8, bias=True, tau=1.0,
         masks=7, seen=40, adds=8, repetition=1.25, presence=0.5, frequency=0.25),
    dict(name="rules 64 nodes bf16", op="rules", dt="bf16", n=20096, rows=64, H=128, V=50021, K=1, bias=False, tau=1.0,
         masks=64, seen=1500, adds=64, repetition=1.5, presence=0.0, frequency=0.125),
    dict(name="rules 3k bf16", op="rules", dt="bf16", n=20096, rows=3001, H=64, V=10007, K=16, bias=True, tau=1.0,
         masks=7, seen=100, adds=16, repetition=1.25, presence=0.25, frequency=0.0),
    # a step's distillation on a small graph: latency; the loss alone on held-out nodes; a training step's loss and
    # gradients in bfloat16 and in float32; and hidden nodes of the large batch
    dict(name="distill grad tiny f32", op="distill_grad", dt="f32", n=512, rows=101, H=32, V=997, K=4, bias=True, tau=2.0,
         whole=False),
    dict(name="distill eval 3k bf16", op="distill", dt="bf16", n=20096, rows=2999, H=128, V=50021, K=32, bias=False,
         tau=2.0, whole=False),
    dict(name="distill grad 3k bf16", op="distill_grad", dt="bf16", n=20096, rows=3001, H=64, V=10007, K=16, bias=True,
         tau=2.0, whole=False),
    dict(name="distill grad 1k f32", op="distill_grad", dt="f32", n=8192, rows=1229, H=128, V=4999, K=8, bias=True,
         tau=1.0, whole=True),
    dict(name="distill grad 16k bf16", op="distill_grad", dt="bf16", n=131072, rows=16001, H=256, V=50021, K=32,
         bias=False, tau=2.0, whole=False),
]


def listed():
    return [dict(c) for c in LISTED]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges: each operator, type and width, sizes spread over their logarithm."""
    op = rng.choice(["top", "rules", "distill", "distill_grad"])
    dt = rng.choice(["f32", "bf16"])
    H = rng.choice([32, 64, 128, 256])
    V = _log_int(rng, 300, 50021)
    rows = _log_int(rng, 1, {"top": 8000, "rules": 2500, "distill": 8000, "distill_grad": 8000}[op] if dt == "bf16" else 2000)
    n = -(-max(rows * rng.randint(1, 8), 32) // 32) * 32
    K = min(_log_int(rng, 1, 64), V)
    c = dict(op=op, dt=dt, n=n, rows=rows, H=H, V=V, K=K, bias=rng.random() < 0.5, tau=rng.choice([1.0, 2.0, 4.0]))
    if op == "rules":
        c.update(masks=rng.choice([0, 1, 7, rows]), seen=rng.choice([0, 10, 100, 1500 if rows <= 300 else 200]),
                 adds=rng.choice([0, 8, 64]), repetition=rng.choice([1.0, 1.25, 1.5]),
                 presence=rng.choice([0.0, 0.25, 0.5]), frequency=rng.choice([0.0, 0.125, 0.25]))
    elif op != "top":
        c["whole"] = rng.random() < 0.5
    return c


# ------------------------------------------------------------------ inputs

def _tokens(g, shape, V):
    """Token ids whose frequency falls with the id, as a vocabulary sorted by frequency has it."""
    u = torch.rand(shape, generator=g, device="cuda")
    return (torch.exp(u * math.log(V + 1.0)) - 1.0).to(torch.int32).clamp_(0, V - 1)


def _grid(x, step):
    """Rounded to an eight-bit fixed point: seven bits and a sign at steps of `step`."""
    return (x / step).round_().clamp_(-127, 127) * step


def _lists(g, rows, most, V):
    """0 .. most tokens a row: (offsets, tokens, their count)."""
    lens = torch.randint(0, most + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
    lens[-1] = most
    ptr = torch.zeros((rows + 1,), dtype=torch.int32, device="cuda")
    ptr[1:] = torch.cumsum(lens, 0)
    total = int(ptr[-1])
    return ptr, _tokens(g, max(total, 1), V), total


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case)
    n, rows, H, V, K, td = case["n"], case["rows"], case["H"], case["V"], case["K"], DT[case["dt"]]
    # chosen nodes' final states: noise and a part of one token's row, so that some nodes know their token and some
    # do not
    s["node"] = torch.randperm(n, generator=g, device="cuda")[:rows].to(torch.int32)
    node, fits = s["node"].long(), _tokens(g, (rows,), V).long()
    knows = 2.5 * torch.rand((rows, 1), generator=g, device="cuda")
    W = normal(V, H) * (1.5 / math.sqrt(H))
    X = normal(n, H)
    X[node] += knows * W[fits]
    b = 0.5 * normal(V)
    if case["op"] in ("top", "rules"):
        # a quantised model's states, rows and biases: every logit is an exact float32 whatever the order of its
        # sum, so that which tokens are the best, equal ones among them, has one answer
        W, X, b = _grid(W, 1 / 64), _grid(X, 1 / 16), _grid(b, 1 / 64)
        s["top"] = torch.empty((rows, K), dtype=torch.int32, device="cuda")
        s["logit"] = torch.empty((rows, K), device="cuda")
    s["X"], s["W"] = X.to(td), W.to(td)
    s["b"] = b if case["bias"] else None
    s["lse"] = torch.empty((rows,), device="cuda")
    if case["op"] == "rules":
        masks = case["masks"]
        words = -(-V // 32)
        s["mask"] = s["mask_of"] = None
        if masks:   # from nearly all tokens to a handful, and one that leaves none
            share = torch.tensor([0.98, 0.5, 0.1, 0.98, 0.01, 0.7, 0.0], device="cuda")[torch.arange(masks, device="cuda") % 7]
            s["mask"] = torch.empty((masks, words), dtype=torch.int32, device="cuda")
            weight = (1 << torch.arange(32, device="cuda", dtype=torch.int64))
            for m in range(masks):
                bits = torch.rand((words, 32), generator=g, device="cuda") < share[m]
                word = (bits * weight).sum(1)
                s["mask"][m] = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
            s["mask_of"] = torch.randint(0, masks, (rows,), generator=g, device="cuda", dtype=torch.int32)
            s["mask_of"][5::8] = -1   # rows that may answer with any token
            if rows == 1:
                s["mask_of"][:] = 0
        s["seen_ptr"], s["seen"], s["n_seen"] = _lists(g, rows, case["seen"], V)
        s["add_ptr"], s["add"], s["n_add"] = _lists(g, rows, case["adds"], V)
        s["value"] = _grid(normal(max(s["n_add"], 1)), 1 / 8)
        s["value"][3::11] = -INF   # tokens taken out
    if case["op"] in ("distill", "distill_grad"):
        # the teacher knows every node's token better; every 16th node has no list, every 5th one a short one
        Xt = normal(rows, H) + 2.0 * W[fits]
        s["t_id"] = torch.empty((rows, K), dtype=torch.int32, device="cuda")
        s["t_logit"] = torch.empty((rows, K), device="cuda")
        s["t_lse"] = torch.empty((rows,), device="cuda") if case["whole"] else None
        for at in _blocks(rows, V):
            z = Xt[at] @ W.t()
            best = z.topk(K, dim=1)
            s["t_id"][at], s["t_logit"][at] = best.indices.to(torch.int32), best.values
            if case["whole"]:
                s["t_lse"][at] = torch.logsumexp(z / case["tau"], 1)
        s["t_id"][4::5, (K + 1) // 2:] = -1
        s["t_id"][15::16] = -1
        s["loss"] = torch.empty((rows,), device="cuda")
    if case["op"] == "distill_grad":
        s["scale"] = case["tau"] ** 2 / rows
        s["dX"] = torch.empty((n, H), device="cuda")
        s["dW"] = torch.empty((V, H), device="cuda")
        s["db"] = torch.empty((V,), device="cuda") if case["bias"] else None
    return s


def _blocks(rows, V, most=1 << 27):
    """Rows in blocks of at most `most` logits."""
    step = max(1, most // V)
    return [slice(lo, min(rows, lo + step)) for lo in range(0, rows, step)]


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    return _top_plain(s) if s["op"] in ("top", "rules") else _distill_plain(s, s["op"] == "distill_grad")


def _workspace(s, need):
    """The call's scratch memory, kept with the buffers of the state."""
    if "ws" not in s:
        s["ws"] = torch.empty((max(need, 16),), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own(s):
    from paper_1906_11786_amd import capi

    op, dt, n, H, rows, V, K = s["op"], s["dt"], s["n"], s["H"], s["rows"], s["V"], s["K"]
    if op in ("top", "rules"):
        rules, listed_tokens = None, 0
        if op == "rules":
            listed_tokens = s["n_seen"] + s["n_add"]
            rules = capi.token_rules(mask=s["mask"], n_masks=s["masks"], mask_words=-(-V // 32), mask_of=s["mask_of"],
                                     seen_ptr=s["seen_ptr"], seen=s["seen"], n_seen=s["n_seen"],
                                     repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                                     add_ptr=s["add_ptr"], add=s["add"], value=s["value"], n_add=s["n_add"])
        ws = _workspace(s, capi.ggnn_vocab_top_workspace_bytes(dt, H, rows, V, K, listed_tokens))
        capi.ggnn_vocab_top(dt, n, H, rows, V, s["X"], s["W"], s["b"], s["node"], rules, s["tau"], K, s["top"], s["logit"],
                            s["lse"], ws, ws.numel())
        return {"top": s["top"], "logit": s["logit"], "lse": s["lse"]}
    ws = _workspace(s, capi.ggnn_vocab_distill_workspace_bytes(dt, H, rows, V, K, op == "distill_grad"))
    if op == "distill":
        capi.ggnn_vocab_distill(dt, n, H, rows, V, s["X"], s["W"], s["b"], s["node"], K, s["t_id"], s["t_logit"], s["t_lse"],
                                s["tau"], s["loss"], s["lse"], ws, ws.numel())
        return {"loss": s["loss"], "lse": s["lse"]}
    s["dW"].zero_()
    if s["db"] is not None:
        s["db"].zero_()
    capi.ggnn_vocab_distill_grad(dt, n, H, rows, V, s["X"], s["W"], s["b"], s["node"], K, s["t_id"], s["t_logit"],
                                 s["t_lse"], s["tau"], None, s["scale"], False, s["loss"], s["lse"], s["dX"], s["dW"],
                                 s["db"], ws, ws.numel())
    out = {"loss": s["loss"], "lse": s["lse"], "dX": s["dX"], "dW": s["dW"]}
    if s["db"] is not None:
        out["db"] = s["db"]
    return out


# ---- plain forms, float32 throughout

def _log_sum(z):
    """Log of the rows' sums of exponentials; -inf where all are -inf."""
    top = z.amax(1, keepdim=True)
    top = torch.where(top == -INF, 0.0, top)
    return (top + (z - top).exp_().sum(1, keepdim=True).log())[:, 0]


def _listings(ptr, tok, count, at):
    """(row within the block, token, position) of the listings of the rows `at`."""
    lens = ptr.diff()
    row = torch.repeat_interleave(torch.arange(lens.numel(), device="cuda"), lens.long(), output_size=count)
    pos = torch.nonzero((row >= at.start) & (row < at.stop))[:, 0]
    return row[pos] - at.start, tok[pos].long(), pos


def _top_plain(s):
    V, K = s["V"], s["K"]
    W = s["W"].float().t()
    top, logit, lse = torch.empty_like(s["top"]), torch.empty_like(s["logit"]), torch.empty_like(s["lse"])
    low = (1 << 32) - 1 - torch.arange(V, device="cuda")
    for at in _blocks(s["rows"], V, 1 << 25):
        z = s["X"][s["node"][at].long()].float() @ W
        if s["b"] is not None:
            z += s["b"]
        if s["op"] == "rules":
            row, tok, _ = _listings(s["seen_ptr"], s["seen"], s["n_seen"], at)
            c = torch.zeros_like(z).index_put_((row, tok), torch.ones((), device="cuda"), accumulate=True)
            z = torch.where(c > 0, torch.where(z > 0, z / s["repetition"], z * s["repetition"])
                            - (s["presence"] + s["frequency"] * c), z)
            row, tok, pos = _listings(s["add_ptr"], s["add"], s["n_add"], at)
            z = z + torch.zeros_like(z).index_put_((row, tok), s["value"][pos], accumulate=True)
            if s["mask"] is not None:
                bits = (s["mask"][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
                bits = bits.view(s["masks"], -1)[:, :V].bool()
                m = s["mask_of"][at].long()
                may = bits[m.clamp(min=0)] | (m < 0)[:, None]
                z = torch.where(may, z, -INF)
        lse[at] = _log_sum(z / s["tau"])
        # one whole number per token that orders by value, then by the lower id
        bits = (z + 0.0).view(torch.int32).long()
        key = (torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF) - 1) << 32) + low
        best = key.topk(K, dim=1).values
        ids = ((1 << 32) - 1 - (best & 0xFFFFFFFF))
        zk = z.gather(1, ids)
        top[at], logit[at] = torch.where(zk == -INF, -1, ids).to(torch.int32), zk
    return {"top": top, "logit": logit, "lse": lse}


def _distill_plain(s, grad):
    tau = s["tau"]
    node, ids = s["node"].long(), s["t_id"].long()
    W, x = s["W"].float(), s["X"][s["node"].long()].float()
    here = ids >= 0
    some = here.any(1)
    t = torch.where(here, s["t_logit"] / tau, -INF)
    L = _log_sum(t) if s["t_lse"] is None else s["t_lse"]
    L = torch.where(some, L, 0.0)[:, None]
    q = (t - L).exp()
    mass = q.sum(1)
    loss, lse = torch.empty_like(s["loss"]), torch.empty_like(s["lse"])
    if grad:
        dX = torch.zeros((s["n"], s["H"]), device="cuda")
        dW = torch.zeros_like(W)
        db = torch.zeros((s["V"],), device="cuda")
    for at in _blocks(s["rows"], s["V"]):
        z = x[at] @ W.t()
        if s["b"] is not None:
            z += s["b"]
        z /= tau
        lse[at] = _log_sum(z)
        logp = z.gather(1, ids[at].clamp(min=0)) - lse[at][:, None]
        loss[at] = torch.where(here[at], q[at] * (t[at] - L[at] - logp), 0.0).sum(1)
        if grad:
            g = s["scale"] / tau
            dz = z.sub_(lse[at][:, None]).exp_().mul_((mass[at] * g)[:, None])
            dz.scatter_add_(1, ids[at].clamp(min=0), torch.where(here[at], -g * q[at], 0.0))
            dX[node[at]] = dz @ W
            dW += dz.t() @ x[at]
            db += dz.sum(0)
    out = {"loss": loss, "lse": lse}
    if grad:
        out.update(dX=dX, dW=dW)
        if s["b"] is not None:
            out["db"] = db
    return out


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    rows, V, K, H, n, tau = case["rows"], case["V"], case["K"], case["H"], case["n"], case["tau"]
    Wt = s["W"].double().t().contiguous()
    f64 = dict(dtype=torch.float64, device="cuda")
    lse = torch.empty((rows,), **f64)
    if case["op"] in ("top", "rules"):
        ids = torch.full((rows, K), -1, dtype=torch.int32, device="cuda")
        logit = torch.full((rows, K), -INF, **f64)
        if case["op"] == "rules":
            seen, add = s["seen"].cpu().numpy(), s["add"].cpu().numpy()
            seen_ptr, add_ptr, value = s["seen_ptr"].cpu().numpy(), s["add_ptr"].cpu().numpy(), s["value"].cpu().numpy()
            mask = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint32)
            mask_of = None if s["mask"] is None else s["mask_of"].cpu().numpy()
        for at in _blocks(rows, V, 1 << 26):
            z = torch.mm(s["X"][s["node"][at].long()].double(), Wt)
            if s["b"] is not None:
                z += s["b"].double()
            if case["op"] == "rules":
                for r in range(at.start, at.stop):   # row by row, as the rules read
                    zr = z[r - at.start].cpu().numpy()
                    tok, times = np.unique(seen[seen_ptr[r]:seen_ptr[r + 1]], return_counts=True)
                    v = zr[tok]
                    v = np.where(v > 0, v / case["repetition"], v * case["repetition"])
                    zr[tok] = v - case["presence"] - case["frequency"] * times
                    np.add.at(zr, add[add_ptr[r]:add_ptr[r + 1]], value[add_ptr[r]:add_ptr[r + 1]].astype(np.float64))
                    if mask is not None and mask_of[r] >= 0:
                        may = np.unpackbits(mask[mask_of[r]].astype("<u4").view(np.uint8), bitorder="little")[:V]
                        zr[may == 0] = -np.inf
                    z[r - at.start] = torch.from_numpy(zr).cuda()
            lse[at] = torch.logsumexp(z / tau, 1)
            least = z.topk(K, dim=1).values[:, -1:]
            r, v = torch.nonzero((z >= least) & (z > -INF), as_tuple=True)   # by row, then by token
            zv = z[r, v]
            o = torch.argsort(zv, descending=True, stable=True)
            o = o[torch.argsort(r[o], stable=True)]
            r, v, zv = r[o], v[o], zv[o]
            place = torch.arange(r.numel(), device="cuda") - torch.searchsorted(r, r)
            keep = place < K
            ids[at.start + r[keep], place[keep]] = v[keep].to(torch.int32)
            logit[at.start + r[keep], place[keep]] = zv[keep]
        return {"top": ids, "logit": logit, "lse": lse}
    grad = case["op"] == "distill_grad"
    loss = torch.zeros((rows,), **f64)
    dX, dW, db = (torch.zeros((n, H), **f64), torch.zeros((V, H), **f64), torch.zeros((V,), **f64)) if grad else [None] * 3
    W = s["W"].double()
    for at in _blocks(rows, V, 1 << 26):
        node = s["node"][at].long()
        x = s["X"][node].double()
        z = torch.mm(x, Wt)
        if s["b"] is not None:
            z += s["b"].double()
        z /= tau
        lse[at] = torch.logsumexp(z, 1)
        # the teacher's probabilities as a matrix over the vocabulary
        r, k = torch.nonzero(s["t_id"][at] >= 0, as_tuple=True)
        v = s["t_id"][at][r, k].long()
        t = torch.full((at.stop - at.start, K), -INF, **f64)
        t[r, k] = s["t_logit"][at][r, k].double() / tau
        total = torch.logsumexp(t, 1) if s["t_lse"] is None else s["t_lse"][at].double()
        q = torch.zeros_like(z)
        q[r, v] = torch.exp(t[r, k] - total[r])
        logp = z - lse[at][:, None]
        loss[at] = torch.where(q > 0, q * (torch.log(q) - logp), 0.0).sum(1)
        if grad:
            D = (torch.exp(logp) * q.sum(1, keepdim=True) - q) * (s["scale"] / tau)
            dX[node] = torch.mm(D, W)
            dW += torch.mm(D.t().contiguous(), x)
            db += D.sum(0)
    out = {"loss": loss, "lse": lse}
    if grad:
        out.update(dX=dX, dW=dW)
        if s["b"] is not None:
            out["db"] = db
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    n, rows, H, V, K, es = case["n"], case["rows"], case["H"], case["V"], case["K"], ES[case["dt"]]
    bias = 4 * V if case["bias"] else 0
    common = rows * H * es + V * H * es + bias + 4 * rows + 4 * rows   # states, rows, biases; nodes and log sums
    if case["op"] in ("top", "rules"):
        extra = 0
        if case["op"] == "rules":
            extra = case["masks"] * V // 8 + (4 * rows if case["masks"] else 0) + 8 * (rows + 1)
            extra += 4 * rows * (case["seen"] // 2) + 8 * rows * (case["adds"] // 2)
        return {"bytes": common + 8 * rows * K + extra, "flops": 2 * rows * V * H}
    read = common + 8 * rows * K + 4 * rows + (4 * rows if case["whole"] else 0)
    if case["op"] == "distill":
        return {"bytes": read, "flops": 2 * rows * V * H}
    # logits, the gradient of the states and the gradient of the vocabulary's rows: one product each
    return {"bytes": read + n * H * 4 + V * H * 4 + bias, "flops": 6 * rows * V * H}
