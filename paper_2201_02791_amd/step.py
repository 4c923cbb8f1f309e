"""One training step of Algorithm 1 on one partition: buffer ownership and call order.

Holds the torch tensors (device memory only) and issues the library calls in order on one
stream: negatives -> [computational sub-graph of the batch] -> encoder forward -> score/loss ->
encoder backward.  No arithmetic of the method happens in Python or torch.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import numpy as np

from . import binding as kb


class FeatureBlock:
    """The encoder's input from fixed vertex features, learned: H0 = norm(act(X W + b) [+ X]).

    Owns X and Z = act(X W + b) [+ X] in the block's type (bf16 rows with bf16 messages, else fp32), the parameters W, b,
    gamma, beta in fp32 (with bf16 rows a bf16 copy of W, which AdamW keeps up) and their gradients.
    params: X [N][f], W [f][d], b [d], gamma [d], beta [d]; residual needs f == d."""

    def __init__(self, params: Dict[str, object], act: int = kb.ACT_RELU, residual: bool = False, eps: float = 1e-5,
                 bf16: bool = False, device: str = "cuda:0"):
        import torch
        dev = torch.device(device)
        t = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dev)
        self.dtype = torch.bfloat16 if bf16 else torch.float32
        self.X = t(params["X"]).to(self.dtype)
        self.W, self.b, self.gamma, self.beta = (t(params[k]) for k in ("W", "b", "gamma", "beta"))
        n, (f, d) = self.X.shape[0], self.W.shape
        assert self.X.shape[1] == f and (not residual or f == d)
        self.residual = residual
        self.W_rows = self.W.to(self.dtype) if bf16 else self.W
        self.layer = dict(W=self.W_rows, b=self.b, act=int(act))
        self.norm = dict(gamma=self.gamma, beta=self.beta, eps=float(eps))
        rows = lambda: torch.empty((n, d), dtype=self.dtype, device=dev)
        self.Z, self.pre, self.dZ = rows(), rows(), rows()
        self.mean = torch.empty(n, dtype=torch.float32, device=dev)
        self.rstd = torch.empty_like(self.mean)
        self.dW, self.db, self.dgamma, self.dbeta = (torch.empty_like(x) for x in (self.W, self.b, self.gamma, self.beta))
        need = max(kb.dense_workspace_bytes(self.layer, n), kb.layer_norm_workspace_bytes(d, n))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)

    def forward(self, H0, stream=None):
        kb.dense_forward(self.layer, self.X, R=self.X if self.residual else None, Y=self.Z, pre=self.pre, stream=stream)
        kb.layer_norm_forward(self.norm, self.Z, Y=H0, mean=self.mean, rstd=self.rstd, stream=stream)

    def backward(self, dH0, stream=None):
        kb.layer_norm_backward(self.norm, self.Z, self.mean, self.rstd, dH0, dX=self.dZ, dgamma=self.dgamma,
                               dbeta=self.dbeta, workspace=self.workspace, stream=stream)
        kb.dense_backward(self.layer, self.X, self.pre, self.dZ, need_dX=False, dW=self.dW, db=self.db,
                          workspace=self.workspace, stream=stream)


class TrainStep:
    def __init__(self, part: kb.Partition, params: Dict[str, object], acts: Sequence[int],
                 msg_dtype: int = kb.MSG_F32, need_dH0: bool = True, device: str = "cuda:0",
                 keep_scores: bool = True, cone: bool = False, order: int = kb.ORDER_PROJECT_FIRST,
                 dropout: float = 0.0, score_index: bool = True, block: Optional[dict] = None):
        """block: a FeatureBlock's settings (act, residual, eps) and params["block"] its parameters: the layer-1 input is then
        the block's output, its gradient goes through the block, and params["H0"] is not read."""
        import torch
        self.torch = torch
        self.part = part
        self.dev = torch.device(device)
        self.msg_dtype = msg_dtype
        t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(self.dev)
        self.layers: List[dict] = []
        for V, a, W0, act in zip(params["V"], params["a"], params["W0"], acts):
            self.layers.append(dict(V=t(V), a=t(a), W0=t(W0), act=int(act), order=int(order),
                                    dropout=float(dropout), drop_seed=0, drop_step=0))
        self.M = t(params["M"])
        N = part.n_vert
        self.block = None
        if block is not None:
            self.block = FeatureBlock(params["block"], bf16=msg_dtype == kb.MSG_BF16, device=device, **block)
            need_dH0 = True
            self.H0 = torch.empty((self.block.X.shape[0], self.block.W.shape[1]), dtype=torch.float32, device=self.dev)
            assert self.H0.shape[1] == self.layers[0]["V"].shape[1]
        else:
            self.H0 = t(params["H0"])
        assert self.H0.shape[0] == N
        d_out = self.layers[-1]["V"].shape[2]
        self.H_out = torch.empty((N, d_out), dtype=torch.float32, device=self.dev)
        self.dH_out = torch.empty_like(self.H_out)
        self.dM = torch.empty_like(self.M)
        self.loss = torch.zeros(1, dtype=torch.float32, device=self.dev)
        self.grads = [dict(dV=torch.empty_like(l["V"]), da=torch.empty_like(l["a"]),
                           dW0=torch.empty_like(l["W0"])) for l in self.layers]
        self.dH0 = torch.empty_like(self.H0) if need_dH0 else None
        self.ws_bytes = kb.workspace_bytes(part, self.layers, msg_dtype)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.dev)
        assert self.workspace.data_ptr() % 256 == 0
        self.keep_scores = keep_scores
        # cone: propagate only the batch's computational sub-graph (Algorithm 1, getComputeGraph)
        self.cg = kb.ComputeGraph(part, len(self.layers)) if cone else None
        self.pos = None
        self.neg_ent = self.neg_side = self.scores = None
        self.n_neg = 0
        # score_index: the atomic-free form of the scoring call (its scratch is allocated with the batch)
        self.want_index = score_index
        self.index = None

    def set_batch(self, pos_core_idx: np.ndarray, n_neg: int):
        torch = self.torch
        self.pos = torch.from_numpy(np.ascontiguousarray(pos_core_idx, np.int32)).to(self.dev)
        n_pos = self.pos.numel()
        self.n_neg = int(n_neg)
        self.neg_ent = torch.empty((n_pos, max(n_neg, 1)), dtype=torch.int32, device=self.dev)
        self.neg_side = torch.empty((n_pos, max(n_neg, 1)), dtype=torch.uint8, device=self.dev)
        self.scores = (torch.empty((n_pos, 1 + n_neg), dtype=torch.float32, device=self.dev)
                       if self.keep_scores else None)
        self.index = (kb.ScoreIndex(self.part, max(n_pos, 1), self.n_neg, self.H_out.shape[1])
                      if self.want_index else None)

    def set_candidates(self, n_cand: int):
        """Candidates per positive of run_hard, from which set_batch's n_neg negatives are drawn."""
        torch, n_pos = self.torch, self.pos.numel()
        if n_cand < 1:
            raise ValueError("one candidate at least is wanted")
        new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device=self.dev)  # noqa: E731
        self.cand_ent, self.cand_side = new(n_pos, n_cand, dtype=torch.int32), new(n_pos, n_cand, dtype=torch.uint8)
        self.cand_scores = new(n_pos, 1 + n_cand, dtype=torch.float32)
        self.choice = new(n_pos, self.n_neg, dtype=torch.int32)
        self.cand_index = (kb.ScoreIndex(self.part, max(n_pos, 1), n_cand, self.H_out.shape[1]) if self.want_index else None)
        self.cand_workspace, self.cand_workspaces = None, []

    def stage_batches(self, batches):
        """Copy several mini-batches (equal-length index arrays) to the device ahead of a loop; returns the
        tensor [n_batches, n_pos] whose rows `use_batch` takes."""
        torch = self.torch
        return torch.from_numpy(np.ascontiguousarray(np.stack(batches), np.int32)).to(self.dev)

    def use_batch(self, pos_dev):
        """Switch to another mini-batch of the size set_batch was given (a device tensor; nothing is allocated)."""
        assert pos_dev.numel() == self.pos.numel() and pos_dev.dtype == self.pos.dtype
        self.pos = pos_dev

    def view(self, which: int, layer: int):
        """Torch view [N, width] of one intermediate inside the workspace (see kge_workspace_slice)."""
        torch = self.torch
        off, nbytes = kb.workspace_slice(self.part, self.layers, which, layer, self.msg_dtype)
        raw = self.workspace[off:off + nbytes]
        bf = self.msg_dtype == kb.MSG_BF16 and which in (kb.WS_P, kb.WS_DP, kb.WS_Z, kb.WS_U)
        t = raw.view(torch.bfloat16 if bf else torch.float32)
        if which == kb.WS_U:          # flat: the caller reshapes to [S, d_out] (u) or [S, d_in] (dz)
            return t
        return t.view(self.part.n_seg if which == kb.WS_Z else self.part.n_vert, -1)

    # --- the four per-step calls, in Algorithm 1's order
    def compute_graph(self, stream=None):
        if self.cg is not None:
            kb.compute_graph(self.part, self.cg, self.pos, self.neg_ent if self.n_neg > 0 else None, stream)

    def forward(self, stream=None):
        if self.block is not None:
            self.block.forward(self.H0, stream)
        kb.rgcn_forward(self.part, self.layers, self.H0, self.workspace, self.H_out, self.msg_dtype, stream,
                        self.cg)

    def sample(self, mode: int, seed: int, step: int, stream=None):
        kb.sample_negatives(self.part, self.pos, self.n_neg, mode, seed, step, self.neg_ent, self.neg_side, stream)

    def score_loss(self, stream=None):
        kb.distmult_score_loss(self.part, self.H_out, self.M, self.pos, self.neg_ent, self.neg_side,
                               self.n_neg, self.scores, self.loss, self.dH_out, self.dM, stream, self.index)

    def backward(self, stream=None):
        kb.rgcn_backward(self.part, self.layers, self.H0, self.workspace, self.dH_out, self.grads,
                         self.dH0, self.msg_dtype, stream, self.cg)
        if self.block is not None:
            self.block.backward(self.dH0, stream)

    def set_dropout_state(self, seed: int, step: int):
        """Seed and step of the dropout masks (Sec. 4 training setting); forward and backward of one
        step must see the same pair."""
        for lay in self.layers:
            lay["drop_seed"], lay["drop_step"] = int(seed), int(step)

    def run(self, mode: int, seed: int, step: int, stream=None):
        self.set_dropout_state(seed, step)
        self.sample(mode, seed, step, stream)
        self.compute_graph(stream)
        self.forward(stream)
        self.score_loss(stream)
        self.backward(stream)

    def run_hard(self, mode: int, seed: int, step: int, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None):
        """run() with negatives that the model takes for true: of each positive's candidates (set_candidates; drawn as run()
        draws negatives) n_neg are drawn by their scores' softmax at `temperature`, of the top_k, top_p and min_p that are
        left, from the random numbers u ([n_pos][n_neg] in [0, 1)).  A candidate that is the positive itself is not drawn,
        unless a positive has no other."""
        cand = getattr(self, "cand_ent", None)
        if cand is None or cand.shape[0] != self.pos.numel() or self.choice.shape[1] != self.n_neg or self.n_neg == 0:
            raise ValueError("set_candidates comes after set_batch, and before a step that draws negatives from them")
        if tuple(u.shape) != tuple(self.choice.shape):
            raise ValueError("u: a number for each negative is wanted, %d x %d" % tuple(self.choice.shape))
        self.set_dropout_state(seed, step)
        n_cand = cand.shape[1]
        kb.sample_negatives(self.part, self.pos, n_cand, mode, seed, step, self.cand_ent, self.cand_side, stream)
        if self.cg is not None:
            kb.compute_graph(self.part, self.cg, self.pos, self.cand_ent, stream)
        self.forward(stream)
        kb.distmult_score_loss(self.part, self.H_out, self.M, self.pos, self.cand_ent, self.cand_side, n_cand, self.cand_scores,
                               self.loss, self.dH_out, self.dM, stream, self.cand_index)
        scores = self.cand_scores[:, 1:]
        kb.hide_positives(self.part, self.pos, self.cand_ent, self.cand_side, scores, stream)
        need = kb.sample_workspace_bytes(*scores.shape, temperature, top_k, top_p, min_p)
        if self.cand_workspace is None or self.cand_workspace.numel() < need:          # the first step of these settings
            self.cand_workspace = kb._workspace(None, need, scores, stream)
            self.cand_workspaces.append(self.cand_workspace)     # a graph may have been captured with the last one: it is kept
        kb.sample_scores(scores, u, temperature, top_k, top_p, min_p, choice=self.choice, workspace=self.cand_workspace, stream=stream)
        kb.pick_negatives(self.cand_ent, self.cand_side, self.choice, self.neg_ent, self.neg_side, stream)
        # from here on the step is that on the drawn negatives: its sub-graph lies in the one that was propagated, and its flags name
        # the rows that have gradients, which are those an update takes
        self.compute_graph(stream)
        self.score_loss(stream)
        self.backward(stream)

    # --- Algorithm 1, "optimizer.step()": every parameter the step has a gradient for
    def optimizer_step(self, kind: int = kb.OPT_ADAM, lr: float = 0.01, beta1: float = 0.9, beta2: float = 0.999,
                       eps: float = 1e-8, stream=None, max_norm: Optional[float] = None):
        """The state is that of init_optimizer, or of the first call's kind; plain gradient descent needs none.  A call that is
        refused is no step: the next one has its number.  max_norm: the gradients of all parameters together are scaled to this
        norm where theirs is larger; self.grad_norm (device) is theirs before.  OPT_ADAMW takes the factor along and leaves the
        gradients as they are; where they are not finite, it leaves the parameters and its state as they are, and the next step
        has this one's number."""
        self._check_kind(kind)
        if kind != kb.OPT_ADAMW and self.block is not None and self.block.W_rows is not self.block.W:
            raise ValueError("a feature block in bf16 takes OPT_ADAMW, which writes the bf16 copy of its weight")
        if not hasattr(self, "_opt_t"):
            self.init_optimizer(kind)
        if kind not in (kb.OPT_SGD, self.opt_kind):
            raise ValueError("the optimizer's state is of another kind: init_optimizer makes this one's")
        if kind == kb.OPT_ADAMW:
            self._adamw_step(lr, beta1, beta2, eps, stream, max_norm)
            return
        t = 1 if self._opt_t is None else self._opt_t + 1        # None: the state is AdamW's, and descent has no use for a number
        if max_norm is not None:
            kb.check_optimizer(kind, self.M, lr, beta1, beta2, eps, t)   # before the gradients are scaled
            self._clip(kb.clip_grads, max_norm, stream)
        # the entity table: only the rows the step read (flags of the sub-graph's input rows; without a
        # sub-graph the kernel skips rows whose gradient is all zero)
        mask = self.cg.input_rows_ptr() if self.cg is not None else None
        for name, p, g, rows in self._opt_pairs():
            m, v = self.opt_state.get(name, (None, None)) if kind == kb.OPT_ADAM else (None, None)
            kb.optimizer_step(kind, p, g, m, v, lr, beta1, beta2, eps, t, rows=rows,
                              row_mask=mask if rows else None, stream=stream)
        self._count(stream)

    def _adamw_step(self, lr, beta1, beta2, eps, stream, max_norm):
        if max_norm is None and self._opt_t is not None:
            kb.adamw_step(self.opt_plan, lr, beta1, beta2, eps, self._opt_t + 1, stream=stream)
            self._count(stream)
            return
        kb.check_adamw(lr, beta1, beta2, eps, 1 if self._opt_t is None else self._opt_t + 1)       # before the number grows
        if max_norm is None:
            self._count(stream)
            kb.adamw_step(self.opt_plan, lr, beta1, beta2, eps, t_dev=self.opt_t_dev, stream=stream)
            return
        # whether the gradients are finite only the device knows: from here on the number is there.  A call that is captured while it is not makes
        # nothing yet: its replays have the number that it has now, as those of a call without max_norm do
        number, captured = self.opt_t_dev, False
        if self._opt_t is not None:
            with self._on(stream):
                captured = self.torch.cuda.is_current_stream_capturing()
                if captured:
                    number = self.torch.empty_like(number)
                number.fill_(self._opt_t)
            if not captured:
                self._opt_t = None
        self._clip(kb.grad_norm, max_norm, stream, t_dev=number)
        kb.adamw_step(self.opt_plan, lr, beta1, beta2, eps, t_dev=number, stream=stream, factor=self.grad_factor)
        if captured:
            self._opt_t += 1

    @property
    def opt_t(self) -> int:
        """Steps so far.  Once AdamW has made a step with a largest norm, their number is on the device, which reading it waits for; a step
        captured from then on counts at each replay."""
        if self._opt_t is not None:
            return self._opt_t
        self.torch.cuda.synchronize(self.M.device)
        return int(self.opt_t_dev)

    @opt_t.setter
    def opt_t(self, steps: int):
        self._opt_t = int(steps)

    def _count(self, stream):
        if self._opt_t is not None:
            self._opt_t += 1
            return
        with self._on(stream):
            self.opt_t_dev.add_(1)

    def _on(self, stream):
        """torch's own calls on the stream of a library call"""
        torch = self.torch
        if stream is not None and not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(stream, self.M.device) if stream else torch.cuda.default_stream(self.M.device)
        return torch.cuda.stream(stream)

    def _clip(self, call, max_norm: float, stream, **more):
        if not hasattr(self, "grad_plan"):
            mask = self.cg.input_rows_ptr() if self.cg is not None else None
            self.grad_plan = kb.GradTensors([dict(grad=g, row_mask=mask if rows else None) for _, _, g, rows in self._opt_pairs()])
            self.grad_norm, self.grad_factor = (kb._new(self.M, (), self.torch.float32, stream) for _ in range(2))
            self.grad_workspace = kb._workspace(None, self.grad_plan.workspace_bytes, self.M, stream)
        call(self.grad_plan, max_norm, self.grad_norm, self.grad_factor, self.grad_workspace, stream, **more)

    @staticmethod
    def _check_kind(kind):
        if kind not in (kb.OPT_SGD, kb.OPT_ADAM, kb.OPT_ADAMW):
            raise ValueError("OPT_SGD, OPT_ADAM or OPT_ADAMW is wanted, not %r" % (kind,))

    def _opt_pairs(self):
        pairs = [("M", self.M, self.dM, False)]
        for l, (lay, g) in enumerate(zip(self.layers, self.grads)):
            pairs += [("V%d" % l, lay["V"], g["dV"], False), ("a%d" % l, lay["a"], g["da"], False),
                      ("W0%d" % l, lay["W0"], g["dW0"], False)]
        if self.block is not None:
            f = self.block
            pairs += [("W", f.W, f.dW, False), ("b", f.b, f.db, False), ("gamma", f.gamma, f.dgamma, False),
                      ("beta", f.beta, f.dbeta, False)]
        elif self.dH0 is not None:
            pairs.append(("H0", self.H0, self.dH0, True))      # entity embeddings: only rows the step reached
        return pairs

    def init_optimizer(self, kind: int = kb.OPT_ADAM, state_bits: int = 32, weight_decay: float = 0.01):
        """Allocate (zeroed) moments for every parameter, so that no step allocates.  OPT_ADAMW: all parameters in one launch;
        moments of 32 or 8 bits (tensors of fewer than 4096 elements keep 32); weight_decay for every matrix but the entity
        table, whose rows the batches reach unevenly."""
        self._check_kind(kind)
        self.opt_t, self.opt_kind = 0, kind
        self.opt_state = {}
        if kind == kb.OPT_ADAM:
            for name, p, _, _ in self._opt_pairs():
                self.opt_state[name] = (self.torch.zeros_like(p), self.torch.zeros_like(p))
        elif kind == kb.OPT_ADAMW:
            tensors = []
            for name, p, g, rows in self._opt_pairs():
                state = kb.adamw_state(p, state_bits if p.numel() >= 4096 else 32)
                self.opt_state[name] = state
                t = dict(param=p, grad=g, weight_decay=weight_decay if p.dim() > 1 and not rows else 0.0, **state)
                if rows and self.cg is not None:
                    t.update(rows="mask", row_mask=self.cg.input_rows_ptr())
                elif rows:
                    t.update(rows="nonzero")
                if self.block is not None and p is self.block.W and self.block.W_rows is not p:
                    t["copy"] = self.block.W_rows
                tensors.append(t)
            self.opt_plan = kb.AdamWTensors(tensors)
            self.opt_t_dev = self.torch.empty((), dtype=self.torch.int64, device=self.M.device)      # filled when the number moves there
