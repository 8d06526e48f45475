"""Node tokens around a BandedGGNN: first states from a token table, and the
tokens of chosen nodes predicted from the final states (hidden labels in
training, nodes that are asked for in serving).

`NodeTokens` owns the table, its gradient and optimizer state, and the token
lists; every arithmetic step runs in the library (ggnn_embed, ggnn_dropout,
ggnn_forward, ggnn_vocab_loss_grad, ggnn_backward, ggnn_embed_bwd,
ggnn_sgd_momentum).  The table serves both ends: a node's state is the scaled
mean (or sum) of its tokens' rows, and a token's logit is the product of a
node's final state with its row, plus a bias per token.
"""
from __future__ import annotations

import contextlib

import numpy as np

from . import capi
from .driver import BandedGGNN, torch_dtype


MAX_TOKENS = 1 << 30   # listed tokens that the library takes


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

    # ------------------------------------------------------------ training

    def setup_training(self, node, target, lr: float = 0.01, momentum: float = 0.9, weight_decay: float = 0.0,
                       nesterov: bool = False):
        """The nodes whose tokens are predicted (each once) and their targets,
        and zero velocities.  (Their own tokens should not be in their lists.)"""
        if len(np.unique(np.asarray(node))) != len(np.asarray(node)):
            raise ValueError("a node appears more than once among the chosen nodes")
        self.node, self.target = self._rows(node, target)
        m, t = self.model, self.torch
        self.n_rows = len(self.node)
        self.n_live = int((self.target >= 0).sum())
        self.loss = t.empty((self.n_rows,), device=m.device)
        self.lse = t.empty_like(self.loss)
        self.loss_ws = t.empty((max(capi.ggnn_vocab_workspace_bytes(m.dt, m.H, self.n_rows, self.V, True), 16),),
                               dtype=t.uint8, device=m.device)
        self.opt = dict(lr=lr, momentum=momentum, weight_decay=weight_decay, nesterov=nesterov)
        self.velocity, self.model_velocity = t.zeros_like(self.master), t.zeros_like(m.master)
        self.step = 0

    def gradients(self, step: int, stream=None):
        """Forward pass with the dropout of `step`, the mean loss over the
        chosen nodes, and its gradients: in self.grad (table and bias) and the
        model's grad_buf.  self.loss holds the rows' losses."""
        m = self.model
        n, H = m.comp.n_pad, m.H
        with self._on(stream):
            self.embed(step)
            m.forward()
            capi.ggnn_dropout(m.dt, n * H, m.X[m.T], self.p_out, self.seed, 2 * step + 1, self.XT)
            self.grad.zero_()
            m.grad_buf.zero_()
            capi.ggnn_vocab_loss_grad(m.dt, n, H, self.n_rows, self.V, self.XT, self.table, self.bias, self.node,
                                      self.target, None, 1.0 / max(self.n_live, 1), self.loss, self.lse, m.dX,
                                      self.dtable, self.dbias, self.loss_ws, self.loss_ws.numel())
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
