"""Node tokens around a BandedGGNN: first states from a token table, and the
tokens of chosen nodes predicted from the final states (hidden labels in
training, nodes that are asked for in serving).

`NodeTokens` owns the table, its gradient and optimizer state, and the token
lists; every arithmetic step runs in the library (ggnn_embed, ggnn_dropout,
ggnn_forward, ggnn_vocab_loss_grad, ggnn_vocab_distill_grad, ggnn_backward,
ggnn_embed_bwd, ggnn_sgd_momentum; ggnn_vocab_loss and ggnn_vocab_top in
serving, the latter under `TokenRules`).  The table serves both ends: a node's state is the scaled
mean (or sum) of its tokens' rows, and a token's logit is the product of a
node's final state with its row, plus a bias per token.
"""
from __future__ import annotations

import contextlib

import numpy as np

from . import capi
from .driver import BandedGGNN, torch_dtype


MAX_TOKENS = 1 << 30   # listed tokens that the library takes
MAX_LIST = 64          # tokens of one row's list of best ones


def _ids32(ids) -> np.ndarray:
    """Token ids as int32; those past 32 bits become -1, which names no token either."""
    ids = np.asarray(ids, np.int64)
    return np.where((ids < 0) | (ids >= 2**31), -1, ids).astype(np.int32)


def token_lists(lists, n_pad: int):
    """(tok_ptr [n_pad + 1], tok) of one list of token ids per node, in the
    final labels; nodes beyond the lists have none."""
    if len(lists) > n_pad:
        raise ValueError(f"{len(lists)} token lists for {n_pad} nodes")
    ends = np.cumsum([len(x) for x in lists], dtype=np.int64)
    total = int(ends[-1]) if len(lists) else 0
    if total > MAX_TOKENS:
        raise ValueError(f"{total} listed tokens, at most 2^30 are taken")
    ptr = np.zeros(n_pad + 1, np.int32)
    ptr[1:len(lists) + 1] = ends
    ptr[len(lists) + 1:] = total
    return ptr, np.concatenate([_ids32(x) for x in lists]) if total else np.zeros(1, np.int32)


def _csr(lists):
    """(offsets, ids) of one list of token ids per row, as token_lists() without padding nodes."""
    return token_lists(lists, len(lists))


class TokenRules:
    """Rules for the answers of n_rows chosen nodes over a vocabulary of V tokens
    (ggnn_token_rules), uploaded once and used by as many calls as they fit.

    allowed: bool array [masks, V], what each mask lets through; allowed_of: [n_rows]
    int, the mask of each row (any other number: all tokens), or None: row r has mask
    r.  seen: one list of token ids per row, repeated ones as often as they were seen,
    with repetition, presence and frequency as the penalties.  bias: per row a dict
    or list of (token, value), value -inf taking the token out; a token listed
    twice takes the sum."""

    def __init__(self, V: int, n_rows: int, allowed=None, allowed_of=None, seen=None, repetition: float = 1.0,
                 presence: float = 0.0, frequency: float = 0.0, bias=None, device="cuda"):
        import torch
        self.V, self.n_rows, self.tensors = V, n_rows, []
        kw = dict(repetition=repetition, presence=presence, frequency=frequency)

        def up(a):
            self.tensors.append(torch.from_numpy(np.ascontiguousarray(a)).to(device))
            return self.tensors[-1]

        def check(name, rows):
            if len(rows) != n_rows:
                raise ValueError(f"{len(rows)} {name} lists for {n_rows} rows")

        if not (np.isfinite(repetition) and repetition > 0 and np.isfinite(presence) and np.isfinite(frequency)):
            raise ValueError("penalties must be finite, and repetition positive")
        if allowed is not None:
            allowed = np.asarray(allowed)
            if allowed.ndim != 2 or allowed.shape[1] != V or allowed.dtype != np.bool_:
                raise ValueError(f"allowed must be a bool array [masks, {V}]")
            words = -(-V // 32)
            bits = np.zeros((len(allowed), 32 * words), np.uint8)
            bits[:, :V] = allowed
            if len(allowed):
                kw.update(mask=up(np.packbits(bits, axis=1, bitorder="little").view("<i4")), n_masks=len(allowed),
                          mask_words=words)
            if allowed_of is not None:
                of = np.asarray(allowed_of, np.int64)
                if of.shape != (n_rows,):
                    raise ValueError(f"allowed_of of shape {of.shape}, ({n_rows},) is needed")
                kw["mask_of"] = up(_ids32(of))
        elif allowed_of is not None:
            raise ValueError("allowed_of without allowed")
        if seen is not None:
            check("seen", seen)
            ptr, ids = _csr(seen)
            if ptr[-1]:
                kw.update(seen_ptr=up(ptr), seen=up(ids), n_seen=int(ptr[-1]))
        if bias is not None:
            check("bias", bias)
            pairs = [list(b.items()) if isinstance(b, dict) else list(b) for b in bias]
            ptr, ids = _csr([[v for v, _ in b] for b in pairs])
            if ptr[-1]:
                value = np.asarray([x for b in pairs for _, x in b], np.float32)
                kw.update(add_ptr=up(ptr), add=up(ids), value=up(value), n_add=int(ptr[-1]))
        self.n_listed = kw.get("n_seen", 0) + kw.get("n_add", 0)
        if self.n_listed > MAX_TOKENS:
            raise ValueError(f"{self.n_listed} listed tokens, at most 2^30 are taken")
        self.struct = capi.token_rules(**kw)

    def record_stream(self, stream):
        """The arrays are in use on `stream`, which need not be the one that they were uploaded on."""
        for x in self.tensors:
            x.record_stream(stream)


class NodeTokens:
    """Token table [V][H], per-token bias [V] and token lists of one workload.

    stream arguments: a torch stream or its handle, None for the current one; all
    of a call's work, fills and uploads among it, goes to that stream.  Work on
    other streams, the set-up's among it, is the caller's to order."""

    def __init__(self, model: BandedGGNN, table, tok_ptr, tok, bias=None, scale: float = 1.0, mean: bool = True,
                 p_in: float = 0.0, p_out: float = 0.0, seed: int = 0):
        """model: its X[0] is written from the tokens.  table: float array [V, H]
        (exact in the model's dtype, as the model's parameters are).  tok_ptr,
        tok: as ggnn_embed takes them (token_lists() makes them).  bias: -1e30 or
        less takes a token out of the answers, in training for good (it is kept
        as -inf, which the update leaves alone).  p_in, p_out: dropout of the
        first and of the final states while training."""
        import torch
        self.torch, self.model = torch, model
        table = np.asarray(table, np.float64)
        if table.ndim != 2 or table.shape[1] != model.H or table.shape[0] < 1:
            raise ValueError(f"table of shape {table.shape}, (V, {model.H}) is needed")
        self.V, n, H, dt, dev = table.shape[0], model.comp.n_pad, model.H, model.dt, model.device
        tok_ptr, tok = np.asarray(tok_ptr, np.int64), np.asarray(tok, np.int64)
        if len(tok_ptr) != n + 1 or tok_ptr[0] != 0 or np.any(np.diff(tok_ptr) < 0) or tok_ptr[-1] > len(tok):
            raise ValueError(f"tok_ptr must hold n_pad + 1 = {n + 1} offsets that start at 0, do not decrease and end "
                             "within the token list")
        if tok_ptr[-1] > MAX_TOKENS:
            raise ValueError(f"{tok_ptr[-1]} listed tokens, at most 2^30 are taken")
        self.n_tok = int(tok_ptr[-1])
        self.tok_ptr = torch.from_numpy(tok_ptr.astype(np.int32)).to(dev)
        self.tok = torch.from_numpy(_ids32(tok) if len(tok) else np.zeros(1, np.int32)).to(dev)
        self.scale, self.mean, self.p_in, self.p_out, self.seed = scale, mean, p_in, p_out, seed
        # table and bias in one buffer, so that one fill clears their gradients and one launch updates both
        nb = -(-self.V // 64) * 64
        self.master = torch.zeros((self.V * H + nb,), dtype=torch.float32, device=dev)
        self.master[:self.V * H].copy_(torch.from_numpy(table.astype(np.float32).reshape(-1)))
        self.bias = self.master[self.V * H:self.V * H + self.V]
        if bias is not None:
            bias = np.asarray(bias, np.float32)
            if bias.shape != (self.V,):
                raise ValueError(f"bias of shape {bias.shape}, ({self.V},) is needed")
            self.bias.copy_(torch.from_numpy(np.where(bias <= -1e30, np.float32(-np.inf), bias)))
        self.compute_copy = self.master.to(torch_dtype(dt)) if dt == "bf16" else None
        self.table = (self.master if self.compute_copy is None else self.compute_copy)[:self.V * H].view(self.V, H)
        self.grad = torch.zeros_like(self.master)
        self.dtable = self.grad[:self.V * H].view(self.V, H)
        self.dbias = self.grad[self.V * H:self.V * H + self.V]
        self.XT = torch.empty_like(model.X[0])   # the final states after dropout
        need = capi.ggnn_embed_bwd_workspace_bytes(n, H, self.V, self.n_tok)
        self.embed_ws = torch.empty((max(need, 16),), dtype=torch.uint8, device=dev)
        self.opt = None

    # ---------------------------------------------------------------- parts

    def _on(self, stream):
        """The context in which `stream` is the current one."""
        t = self.torch
        if stream is None:
            return contextlib.nullcontext()
        if isinstance(stream, int):
            stream = t.cuda.ExternalStream(stream) if stream else t.cuda.default_stream(self.model.device)
        return t.cuda.stream(stream)

    def embed(self, step: int = -1, stream=None):
        """X[0] from the tokens; step >= 0: with the dropout of that step."""
        m = self.model
        capi.ggnn_embed(m.dt, m.comp.n_pad, m.H, self.V, self.table, self.tok_ptr, self.tok, self.n_tok, self.scale,
                        self.mean, self.p_in if step >= 0 else 0.0, self.seed, 2 * max(step, 0), m.X[0], stream)

    def _rows(self, node, target):
        node = np.asarray(node, np.int64)
        if node.ndim != 1 or (len(node) and (node.min() < 0 or node.max() >= self.model.comp.n_pad)):
            raise ValueError(f"node ids must lie in [0, {self.model.comp.n_pad})")
        t = self.torch
        up = (lambda a: t.from_numpy(np.ascontiguousarray(a, np.int32)).to(self.model.device))
        if target is not None:
            target = np.asarray(target, np.int64)
            if target.shape != node.shape:
                raise ValueError("one target per chosen node is needed")
            if len(target) and target.max() >= self.V:
                raise ValueError(f"targets must lie below V={self.V} (negative: no loss)")
            target = np.maximum(target, -1)
        return up(node), None if target is None else up(target)

    def _space(self, name: str, nbytes: int):
        if not hasattr(self, name) or getattr(self, name).numel() < nbytes:
            setattr(self, name, self.torch.empty((max(nbytes, 16),), dtype=self.torch.uint8, device=self.model.device))
        ws = getattr(self, name)
        ws.record_stream(self.torch.cuda.current_stream())   # which need not be the one that it was allocated on
        return ws

    # ------------------------------------------------------------- serving

    def evaluate(self, node, target=None, stream=None):
        """Forward pass without dropout and, for the chosen nodes, the best
        token and log sum of the logits' exponentials (and, with targets, the
        losses): dict of device tensors."""
        with self._on(stream):
            node, target = self._rows(node, target)
            m, t = self.model, self.torch
            R = len(node)
            out = {"best": t.empty((R,), dtype=t.int32, device=m.device), "lse": t.empty((R,), device=m.device)}
            if target is not None:
                out["loss"] = t.empty((R,), device=m.device)
            self.embed()
            m.forward()
            ws = self._space("eval_ws", capi.ggnn_vocab_workspace_bytes(m.dt, m.H, R, self.V, False))
            capi.ggnn_vocab_loss(m.dt, m.comp.n_pad, m.H, R, self.V, m.X[m.T], self.table, self.bias, node, target,
                                 out.get("loss"), out["lse"], out["best"], ws, ws.numel())
            return out

    def rules(self, n_rows: int, **kw) -> TokenRules:
        """TokenRules over this vocabulary, on the model's device."""
        return TokenRules(self.V, n_rows, device=self.model.device, **kw)

    def top(self, node, k: int, rules: TokenRules | None = None, temperature: float = 1.0, stream=None):
        """Forward pass without dropout and, for the chosen nodes, the k best
        tokens under the rules: dict of device tensors token [R, k] (-1: no token
        is left), logit [R, k] in descending order, and lse [R], the log sum at the
        temperature; and that temperature, a number on the host.  It is what a
        student's setup_training() takes as `teacher`."""
        if not 1 <= k <= MAX_LIST:
            raise ValueError(f"k={k} must be in [1, {MAX_LIST}]")
        with self._on(stream):
            node, _ = self._rows(node, None)
            m, t, R = self.model, self.torch, len(node)
            if rules is not None:
                if rules.n_rows != R or rules.V != self.V:
                    raise ValueError(f"rules for {rules.n_rows} rows over {rules.V} tokens, {R} over {self.V} are needed")
                at = m.X[m.T].device
                if any(x.device != at for x in rules.tensors):   # the kernels follow the addresses as they are
                    raise ValueError(f"rules on {rules.tensors[0].device}, the model is on {at}")
                rules.record_stream(t.cuda.current_stream())
            out = {"token": t.empty((R, k), dtype=t.int32, device=m.device),
                   "logit": t.empty((R, k), device=m.device), "lse": t.empty((R,), device=m.device),
                   "temperature": t.tensor(float(temperature), dtype=t.float64)}
            self.embed()
            m.forward()
            listed = 0 if rules is None else rules.n_listed
            ws = self._space("top_ws", capi.ggnn_vocab_top_workspace_bytes(m.dt, m.H, R, self.V, k, listed))
            capi.ggnn_vocab_top(m.dt, m.comp.n_pad, m.H, R, self.V, m.X[m.T], self.table, self.bias, node,
                                None if rules is None else rules.struct, temperature, k, out["token"], out["logit"],
                                out["lse"], ws, ws.numel())
            return out

    # ------------------------------------------------------------ training

    def _teacher(self, teacher, R: int):
        """A teacher's lists for R chosen nodes on the device: (token, logit, lse or None, rows with a token)."""
        t = self.torch
        here = (lambda x, dt: t.as_tensor(x).to(device=self.model.device, dtype=dt).contiguous())
        token, logit = t.as_tensor(teacher["token"]), here(teacher["logit"], t.float32)
        if token.ndim != 2 or token.shape[0] != R or not 1 <= token.shape[1] <= MAX_LIST or logit.shape != token.shape:
            raise ValueError(f"teacher lists of shapes {tuple(token.shape)} and {tuple(logit.shape)}, ({R}, 1 .. "
                             f"{MAX_LIST}) are needed")
        if token.numel() and int(token.max()) >= self.V:
            raise ValueError(f"teacher tokens must lie below V={self.V} (negative: none)")
        lse = teacher.get("lse")
        if lse is not None:
            lse = here(lse, t.float32)
            if lse.shape != (R,):
                raise ValueError(f"teacher log sums of shape {tuple(lse.shape)}, ({R},) is needed")
        taught = int((token >= 0).any(1).sum())
        return here(token.clamp(min=-1), t.int32), logit, lse, taught

    def setup_training(self, node, target, lr: float = 0.01, momentum: float = 0.9, weight_decay: float = 0.0,
                       nesterov: bool = False, teacher=None, temperature: float | None = None, soft: float = 0.5):
        """The nodes whose tokens are predicted (each once) and their targets,
        and zero velocities.  (Their own tokens should not be in their lists.)

        teacher: a teacher's top() of the same nodes (token, logit, and lse where
        the log sums over its whole vocabulary at this temperature are to count;
        without, each list's probabilities add up to 1).  temperature: None is the
        one that the teacher's dict holds, 2 where it holds none; log sums at
        another one than this are refused.  The loss is then
        (1 - soft) times the mean cross entropy and soft * temperature^2 times the
        mean distillation loss of the nodes that have a list."""
        if len(np.unique(np.asarray(node))) != len(np.asarray(node)):
            raise ValueError("a node appears more than once among the chosen nodes")
        node, target = self._rows(node, target)
        m, t, R, soft_part = self.model, self.torch, len(node), None
        n_live = int((target >= 0).sum())
        if teacher is not None:
            told = None if teacher.get("temperature") is None else float(teacher["temperature"])
            if temperature is None:
                temperature = 2.0 if told is None else told
            elif told is not None and teacher.get("lse") is not None and np.float32(told) != np.float32(temperature):
                raise ValueError(f"the teacher's log sums are at temperature {told:g}, not {temperature:g}: its top() at this "
                                 "one is needed, or its lists without lse")
            if not 0.0 <= soft <= 1.0 or not 1e-3 <= temperature <= 1e3:
                raise ValueError(f"soft={soft} must be in [0, 1] and temperature={temperature} in [0.001, 1000]")
            token, logit, lse, taught = self._teacher(teacher, R)
            soft_part = dict(K=token.shape[1], token=token, logit=logit, lse=lse, temperature=temperature, soft=soft,
                             scale=soft * temperature ** 2 / max(taught, 1))
        # (from here on nothing is refused: a refused call leaves the set-up before it as it was)
        self.node, self.target, self.n_rows, self.teacher = node, target, R, soft_part
        self.n_live = n_live
        self.loss = t.empty((R,), device=m.device)
        self.lse = t.empty_like(self.loss)
        self.loss_ws = t.empty((max(capi.ggnn_vocab_workspace_bytes(m.dt, m.H, R, self.V, True), 16),),
                               dtype=t.uint8, device=m.device)
        if soft_part is not None:
            self.soft_loss, self.soft_lse = t.empty_like(self.loss), t.empty_like(self.loss)
            need = capi.ggnn_vocab_distill_workspace_bytes(m.dt, m.H, R, self.V, soft_part["K"], True)
            self.soft_ws = t.empty((max(need, 16),), dtype=t.uint8, device=m.device)
        self.opt = dict(lr=lr, momentum=momentum, weight_decay=weight_decay, nesterov=nesterov)
        self.velocity, self.model_velocity = t.zeros_like(self.master), t.zeros_like(m.master)
        self.step = 0

    def gradients(self, step: int, stream=None):
        """Forward pass with the dropout of `step`, the mean loss over the
        chosen nodes (with a teacher: both losses), and its gradients: in self.grad
        (table and bias) and the model's grad_buf.  self.loss holds the rows' cross
        entropies, self.soft_loss their distillation losses."""
        m = self.model
        n, H = m.comp.n_pad, m.H
        with self._on(stream):
            self.embed(step)
            m.forward()
            capi.ggnn_dropout(m.dt, n * H, m.X[m.T], self.p_out, self.seed, 2 * step + 1, self.XT)
            self.grad.zero_()
            m.grad_buf.zero_()
            s = self.teacher
            capi.ggnn_vocab_loss_grad(m.dt, n, H, self.n_rows, self.V, self.XT, self.table, self.bias, self.node,
                                      self.target, None, (1.0 if s is None else 1.0 - s["soft"]) / max(self.n_live, 1),
                                      self.loss, self.lse, m.dX, self.dtable, self.dbias, self.loss_ws,
                                      self.loss_ws.numel())
            if s is not None:
                capi.ggnn_vocab_distill_grad(m.dt, n, H, self.n_rows, self.V, self.XT, self.table, self.bias, self.node,
                                             s["K"], s["token"], s["logit"], s["lse"], s["temperature"], None, s["scale"],
                                             True, self.soft_loss, self.soft_lse, m.dX, self.dtable, self.dbias,
                                             self.soft_ws, self.soft_ws.numel())
            capi.ggnn_dropout("f32", n * H, m.dX, self.p_out, self.seed, 2 * step + 1, m.dX)
            capi.ggnn_backward(m.model, m.act, m.grads)
            capi.ggnn_embed_bwd(n, H, self.V, self.tok_ptr, self.tok, self.n_tok, self.scale, self.mean, self.p_in,
                                self.seed, 2 * step, m.dX, self.dtable, self.embed_ws, self.embed_ws.numel())

    def train_step(self, stream=None):
        """One training step: gradients(), then the Momentum update of the
        model's parameters and of the table and bias."""
        if self.opt is None:
            raise RuntimeError("setup_training() first")
        m, o = self.model, self.opt
        self.gradients(self.step, stream)
        for master, vel, g, copy in ((m.master, self.model_velocity, m.grad_buf, m.compute_copy),
                                     (self.master, self.velocity, self.grad, self.compute_copy)):
            capi.ggnn_sgd_momentum(master.numel(), master, vel, g, o["lr"], o["momentum"], o["weight_decay"],
                                   o["nesterov"], m.dt, copy, stream)
        m.refresh_weights(stream)
        self.step += 1
