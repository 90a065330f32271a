"""Marshal a generated workload onto the GPU and drive the library through the binding.

Used by the tests, ``bench.py`` and the smoke check: it only moves arrays
between host and device and calls the C ABI; all arithmetic happens in the
HIP kernels."""
from __future__ import annotations

import numpy as np
import torch

from . import fold as F
from . import gen


def bf16_tensor(x: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(gen.to_bf16_bits(np.ascontiguousarray(x, np.float32)).view(np.int16)).view(torch.bfloat16)


def pad_cols(x: np.ndarray, ld: int) -> np.ndarray:
    x = np.asarray(x, np.float32)
    if x.shape[1] == ld:
        return np.ascontiguousarray(x)
    out = np.zeros((x.shape[0], ld), np.float32)
    out[:, :x.shape[1]] = x
    return out


class DeviceRun:
    def __init__(self, w: gen.Workload, device: str = "cuda", stream=None, with_backward=None):
        self.w = w
        self.device = device
        self.stream = stream
        H = w.hidden
        self.H = H
        self.ld = F.fold_row_ld(H)
        self.bf16 = w.dtype == "bf16"
        self.fdtype = F.FOLD_BF16 if self.bf16 else F.FOLD_F32
        self.tdtype = torch.bfloat16 if self.bf16 else torch.float32
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(device)
        self.graph_ptr, self.node_op = i32(w.graph_ptr), i32(w.node_op)
        self.child_ptr, self.child_idx, self.node_input = i32(w.child_ptr), i32(w.child_idx), i32(w.node_input)
        self.ops = [(o.kind, o.arity, o.has_input, o.param_set) for o in w.ops]
        self.leaf_rows = int(w.leaf_table.shape[0])
        self.sched = F.Schedule(self.graph_ptr, self.node_op, self.child_ptr, self.child_idx, self.node_input,
                                self.ops, self.leaf_rows, stream)
        self.set_tensors = []
        for p in w.params:
            self.set_tensors.append(dict(
                kind=p.kind, in_dim=p.in_dim, arity=p.arity,
                W_in=None if p.W_in is None else self._wt(p.W_in),
                W_rec=None if p.W_rec is None else self._wt(p.W_rec),
                bias=(None if p.kind == gen.KIND_EMBED or p.bias is None or p.bias.size == 0
                      else torch.from_numpy(p.bias.astype(np.float32)).to(device))))
        self.packed = F.Packed(self.fdtype, H, self.set_tensors, stream)
        in_dim = int(w.leaf_table.shape[1])
        self.tld = F.fold_row_ld(in_dim)
        tab = pad_cols(w.leaf_table, self.tld)
        self.table = (bf16_tensor(tab) if self.bf16 else torch.from_numpy(tab)).to(device)
        N, R = w.num_nodes, self.sched.info.num_roots
        self.N, self.R = N, R
        self.h_pool = torch.zeros((max(N, 1), self.ld), dtype=self.tdtype, device=device)
        self.c_pool = torch.zeros((max(N, 1), self.ld), dtype=torch.float32, device=device)
        self.roots = torch.zeros((max(R, 1), self.ld), dtype=self.tdtype, device=device)
        self.fwd_bytes, self.bwd_bytes = F.fold_workspace_size(self.sched.handle, self.packed.handle)
        backward = w.backward if with_backward is None else with_backward
        self.ws_bytes = self.bwd_bytes if backward else self.fwd_bytes
        self.ws = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=device)
        self.grads = None
        self.dh_roots = None
        self.dh_nodes = None

    def _wt(self, a):
        a = np.ascontiguousarray(a, np.float32)
        return (bf16_tensor(a) if self.bf16 else torch.from_numpy(a)).to(self.device)

    # ------------------------------------------------------------------ calls
    def forward(self, u_mask=None):
        """u_mask: recurrent-dropout mask [N, ld] fp32 in pool order (fold_forward_dropout), or None."""
        if u_mask is not None:
            F.fold_forward_dropout(self.sched.handle, self.packed.handle, self.table, self.leaf_rows, self.h_pool,
                                   self.c_pool, self.roots, u_mask, self.ws, self.ws_bytes, self.stream)
            return
        F.fold_forward(self.sched.handle, self.packed.handle, self.table, self.leaf_rows, self.h_pool,
                       self.c_pool, self.roots, self.ws, self.ws_bytes, self.stream)

    def alloc_grads(self, table_grad=True):
        sets = []
        for p in self.w.params:
            g = gen.NUM_GATES[p.kind] * self.H
            z = lambda *s: torch.zeros(s, dtype=torch.float32, device=self.device)
            if p.kind == gen.KIND_ATTN_SCORE:  # dw as [H, 1], db [1]
                sets.append((None, z(self.H, 1), z(1)))
                continue
            if p.kind == gen.KIND_EMBED or p.kind in gen.ATTN_KINDS:
                sets.append((None, None, None))
                continue
            sets.append((z(p.in_dim, g) if p.W_in is not None else None,
                         z(p.arity * self.H, g) if p.W_rec is not None else None, z(g)))
        self.grad_tensors = sets
        self.d_table = (torch.zeros((self.leaf_rows, self.tld), dtype=torch.float32, device=self.device)
                        if table_grad else None)
        self.grads = F.make_grads(sets, self.d_table)
        return sets

    def set_upstream(self, dh_roots: np.ndarray, dh_nodes_node_order: np.ndarray | None = None):
        self.dh_roots = torch.from_numpy(pad_cols(dh_roots, self.ld)).to(self.device) if self.R else None
        if dh_nodes_node_order is not None:
            node_pos = self.sched_arrays()["node_pos"]
            pool = np.zeros((self.N, self.ld), np.float32)
            pool[node_pos, :self.H] = dh_nodes_node_order
            self.dh_nodes = torch.from_numpy(pool).to(self.device)
        else:
            self.dh_nodes = None

    def zero_grads(self):
        for t in self.grad_tensors:
            for x in t:
                if x is not None:
                    x.zero_()
        if self.d_table is not None:
            self.d_table.zero_()

    def backward(self, dh_out=None, dc_out=None, u_mask=None):
        if u_mask is not None:
            F.fold_backward_dropout(self.sched.handle, self.packed.handle, self.table, self.leaf_rows, self.h_pool,
                                    self.c_pool, u_mask, self.dh_roots, self.dh_nodes, self.grads, dh_out, dc_out,
                                    self.ws, self.ws_bytes, self.stream)
            return
        F.fold_backward(self.sched.handle, self.packed.handle, self.table, self.leaf_rows, self.h_pool,
                        self.c_pool, self.dh_roots, self.dh_nodes, self.grads, dh_out, dc_out, self.ws,
                        self.ws_bytes, self.stream)

    def make_graph(self, backward=None, zero_grads=True, dh_out=None, dc_out=None):
        """Record one step (forward, then backward with the gradients zeroed first) as a HIP graph."""
        backward = self.w.backward if backward is None else backward
        return F.StepGraph(self.sched, self.packed, self.table, self.leaf_rows, self.h_pool, self.c_pool,
                           self.roots, self.ws, self.ws_bytes, backward=backward, dh_roots=self.dh_roots,
                           dh_nodes=self.dh_nodes, grads=self.grads if backward else None, dh_out=dh_out,
                           dc_out=dc_out, zero_grads=zero_grads and backward)

    # ------------------------------------------------------------------ results
    def sched_arrays(self):
        if not hasattr(self, "_sa"):
            self._sa = self.sched.arrays()
        return self._sa

    def node_states(self):
        """h, c in node order as float64 [N, H]."""
        torch.cuda.synchronize()
        node_pos = self.sched_arrays()["node_pos"]
        h = self.h_pool.float().cpu().numpy()[:self.N, :self.H].astype(np.float64)
        c = self.c_pool.cpu().numpy()[:self.N, :self.H].astype(np.float64)
        return h[node_pos], c[node_pos]

    def weight_grads(self):
        torch.cuda.synchronize()
        out = []
        for t in self.grad_tensors:
            out.append({k: (None if x is None else x.cpu().numpy().astype(np.float64))
                        for k, x in zip(("W_in", "W_rec", "bias"), t)})
        dt = None if self.d_table is None else self.d_table.cpu().numpy()[:, :self.w.leaf_table.shape[1]].astype(np.float64)
        return out, dt


def trained_tensors(dev: DeviceRun, train_table: bool):
    """(fp32 master, bf16 copy or None, gradient) of every trained tensor of a workload's own parameters."""
    out = []
    for p, st, gt in zip(dev.w.params, dev.set_tensors, dev.grad_tensors):
        if p.kind == gen.KIND_EMBED:
            continue
        for name, g in zip(("W_in", "W_rec", "bias"), gt):
            if g is None:
                continue
            cur = st[name]
            out.append((cur, None, g) if cur.dtype == torch.float32 else (cur.float(), cur, g))
    if train_table:
        out.append((dev.table.float(), dev.table, dev.d_table) if dev.bf16 else (dev.table, None, dev.d_table))
    return out


class TrainStep:
    """One training step of a workload through the C ABI (Section 3.5's setting: a class label on every node,
    softmax cross entropy on every node's state, Adam): zero the gradients, fold_forward,
    fold_loss_softmax_ce, fold_backward from the head's dh alone, fold_adam_step on every parameter tensor
    (the weights of every set, the biases, the leaf table if trained, the classifier), fold_pack_update.

    fp32 master copies of the weights are kept here; for bf16 workloads Adam also writes the bf16 weights
    that fold_pack_update packs.  The loss is the mean over the labelled nodes (scale = 1 / their count).

    dropout > 0 trains with recurrent dropout (Section 3.5): every step first draws a fresh mask on the GPU
    (fold_dropout_mask with counter = (node, unit block, step number), key = dropout_seed) and runs
    fold_forward_dropout / fold_backward_dropout with it."""

    def __init__(self, w: gen.Workload, labels: np.ndarray, num_classes: int, train_table: bool, seed: int = 0,
                 lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 dropout: float = 0.0, dropout_seed: int = 0):
        self.dev = dev = DeviceRun(w)
        self.dropout = float(dropout)
        self.dropout_seed = int(dropout_seed)
        self.u_mask = (torch.zeros((max(dev.N, 1), dev.ld), dtype=torch.float32, device=dev.device)
                       if self.dropout > 0 else None)
        self.C = num_classes
        self.hyper = (lr, beta1, beta2, eps)
        self.t = 0
        rng = np.random.default_rng(seed)
        cuda = lambda a, dt=torch.float32: torch.from_numpy(np.ascontiguousarray(a)).to(dtype=dt, device=dev.device)
        self.labels = cuda(labels, torch.int32)
        self.scale = 1.0 / max(1, int((labels >= 0).sum()))
        self.W_cls = cuda((0.1 * rng.standard_normal((w.hidden, num_classes))).astype(np.float32))
        self.b_cls = torch.zeros(num_classes, dtype=torch.float32, device=dev.device)
        self.dW_cls = torch.zeros_like(self.W_cls)
        self.db_cls = torch.zeros_like(self.b_cls)
        self.node_loss = torch.zeros(max(dev.N, 1), dtype=torch.float32, device=dev.device)
        self.dh_nodes = torch.zeros((max(dev.N, 1), dev.ld), dtype=torch.float32, device=dev.device)
        self.loss_ws_bytes = F.fold_loss_workspace_size(dev.packed.handle, num_classes)
        self.loss_ws = torch.empty(self.loss_ws_bytes, dtype=torch.uint8, device=dev.device)
        dev.alloc_grads(train_table)
        dev.set_upstream(np.zeros_like(w.dh_roots))
        dev.dh_nodes = self.dh_nodes
        self.tensors = trained_tensors(dev, train_table)
        self.tensors += [(self.W_cls, None, self.dW_cls), (self.b_cls, None, self.db_cls)]
        self.moments = [(torch.zeros_like(m), torch.zeros_like(m)) for m, _, _ in self.tensors]

    def draw_mask(self):
        """The recurrent-dropout mask of step self.t into self.u_mask (pool order)."""
        F.fold_dropout_mask(self.dev.sched.handle, self.dev.H, self.dropout, self.dropout_seed, self.t, self.u_mask,
                            self.dev.stream)

    def gradients(self):
        """Zero the gradients, forward, head, backward (kernel launches only: capturable as a graph).  With
        dropout they read the mask that step() draws first."""
        dev = self.dev
        dev.zero_grads()
        self.dW_cls.zero_()
        self.db_cls.zero_()
        dev.forward(self.u_mask)
        F.fold_loss_softmax_ce(dev.sched.handle, dev.packed.handle, dev.h_pool, self.labels, self.C, self.W_cls,
                               self.b_cls, self.scale, self.node_loss, self.dh_nodes, self.dW_cls, self.db_cls,
                               self.loss_ws, self.loss_ws_bytes, dev.stream)
        dev.backward(u_mask=self.u_mask)

    def capture_gradients(self):
        """Record gradients() once as a graph (torch.cuda.CUDAGraph over the library's launches on the capture
        stream); step(graph=True) then replays it.  Adam, the re-pack and the mask draw stay outside: the step
        count enters each of them."""
        self.graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(self.graph):
            self.gradients()
        torch.cuda.synchronize()

    def step(self, graph: bool = False):
        dev = self.dev
        self.t += 1
        if self.u_mask is not None:
            self.draw_mask()
        if graph:
            self.graph.replay()
        else:
            self.gradients()
        lr, b1, b2, eps = self.hyper
        for (master, low, grad), (m, v) in zip(self.tensors, self.moments):
            F.fold_adam_step(master.numel(), master, low, grad, m, v, lr, b1, b2, eps, self.t, dev.stream)
        dev.packed.update(dev.set_tensors, dev.stream)


def nodes_with_target(num_nodes: int, vocab: int, labels=None, teacher_token=None, teacher_logit=None):
    """[N] bool: the nodes whose loss fold_loss_distill computes, with a label in [0, vocab) or a teacher's entry that
    counts (its token in [0, vocab), its logit not -inf)."""
    have = torch.zeros(num_nodes, dtype=torch.bool)
    if labels is not None:
        have |= ((labels >= 0) & (labels < vocab)).cpu()
    if teacher_token is not None and teacher_logit is not None:
        counts = (teacher_token >= 0) & (teacher_token < vocab) & (teacher_logit != -float("inf"))
        have |= counts.any(1).cpu()
    return have


class VocabStep:
    """One training step of a workload whose nodes each name a token of a vocabulary, through the C ABI: zero the
    gradients, fold_forward, fold_vocab_logits on the whole pool, fold_loss_distill (a teacher's top logits, labels, or
    both; the gradient over the logits, in place), fold_vocab_backward (its d_states are fold_backward's dh_nodes),
    fold_backward, fold_adam_step on every parameter tensor and the head, fold_pack_update.

    labels [N], teacher_token and teacher_logit [N, num_teacher] are in node order; the loss is the mean over the nodes
    that have a target.  tied: the leaf table is the head's W (a table of `hidden` columns; the vocabulary is its rows)
    and the head's dW is added to the table's gradient.  score() gives the log probabilities of tokens under the current
    weights."""

    def __init__(self, w: gen.Workload, vocab: int, labels=None, teacher_token=None, teacher_logit=None,
                 temperature: float = 1.0, soft_weight: float = 1.0, hard_weight: float = 0.0, train_table: bool = True,
                 tied: bool = False, seed: int = 0, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8):
        self.dev = dev = DeviceRun(w)
        if tied and (not train_table or w.leaf_table.shape != (vocab, w.hidden)):
            raise ValueError("a tied head needs a trained leaf table [vocab, hidden]")
        self.vocab, self.tied, self.hyper, self.t = vocab, tied, (lr, beta1, beta2, eps), 0
        cuda = lambda a, dt: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dt).to(dev.device)
        self.labels = cuda(labels, torch.int32)
        self.teacher_token, self.teacher_logit = cuda(teacher_token, torch.int32), cuda(teacher_logit, torch.float32)
        self.loss_args = dict(temperature=temperature, soft_weight=soft_weight, hard_weight=hard_weight)
        have = nodes_with_target(dev.N, vocab, self.labels, self.teacher_token, self.teacher_logit)
        self.scale = 1.0 / max(1, int(have.sum()))
        dev.alloc_grads(train_table)
        dev.set_upstream(np.zeros_like(w.dh_roots))
        self.dh_nodes = dev.dh_nodes = torch.zeros((dev.N, dev.ld), dtype=torch.float32, device=dev.device)
        self.tensors = trained_tensors(dev, train_table)
        self.bias = torch.zeros(vocab, dtype=torch.float32, device=dev.device)
        self.db = torch.zeros_like(self.bias)
        if tied:
            self.W, self.dW = dev.table, dev.d_table
        else:
            rng = np.random.default_rng(seed)
            W = torch.from_numpy(pad_cols(0.1 * rng.standard_normal((vocab, w.hidden)), dev.ld)).to(dev.device)
            self.W, self.dW = W.to(dev.tdtype), torch.zeros_like(W)
            self.tensors.append((self.W.float(), self.W, self.dW) if dev.bf16 else (self.W, None, self.dW))
        self.tensors.append((self.bias, None, self.db))
        self.head = F.VocabHead(self.W, self.bias, w.hidden)
        self.states = dev.h_pool[:dev.N]  # the pool has a row also for a batch without nodes
        self.logits = torch.zeros((dev.N, F.fold_row_ld(vocab)), dtype=dev.tdtype, device=dev.device)
        self.node_loss = None
        self.moments = [(torch.zeros_like(m), torch.zeros_like(m)) for m, _, _ in self.tensors]

    def gradients(self):
        """Zero the gradients, forward, head, loss, both backward passes (kernel launches only)."""
        dev, st = self.dev, self.dev.stream
        dev.zero_grads()
        dev.forward()
        self.head.logits(self.states, out=self.logits, stream=st)
        self.node_loss, _ = F.distill_loss(self.logits, self.vocab, self.teacher_token, self.teacher_logit, self.labels,
                                           scale=self.scale, dlogits=self.logits, sched=dev.sched, stream=st,
                                           **self.loss_args)
        self.db.zero_()
        self.head.backward(self.states, self.logits, self.dh_nodes, self.dW, self.db, accumulate=self.tied, stream=st)
        dev.backward()

    def step(self):
        dev = self.dev
        self.t += 1
        self.gradients()
        lr, b1, b2, eps = self.hyper
        for (master, low, grad), (m, v) in zip(self.tensors, self.moments):
            F.fold_adam_step(master.numel(), master, low, grad, m, v, lr, b1, b2, eps, self.t, dev.stream)
        dev.packed.update(dev.set_tensors, dev.stream)

    def score(self, tokens, top_k: int = 0):
        """F.TokenLogprobs of `tokens` [N, num_tokens] (node order) under the current weights."""
        dev = self.dev
        dev.forward()
        self.head.logits(self.states, out=self.logits, stream=dev.stream)
        return F.token_logprobs(self.logits, self.vocab, tokens, top_k, sched=dev.sched, stream=dev.stream)
