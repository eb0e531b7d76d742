"""Device-side driver for one batch: uploads a workload, schedules it and runs
forward + backward through the C ABI.  Used by the tests, the smoke check and
the benchmark; it only allocates tensors and calls the binding."""
from __future__ import annotations

from typing import Optional

import numpy as np
import torch

from . import binding as B
from .workloads import Workload


class Batch:
    def __init__(self, wl: Workload, ctx: Optional[B.Context] = None, device: int = 0):
        self.wl = wl
        self.ctx = ctx if ctx is not None else B.Context(device)
        dev = self.ctx.torch_device
        self.dev = dev

        def i32(a):
            return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)

        def f32(a):
            if a is None or a.size == 0:
                return None
            return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev)

        self.child = i32(wl.child.reshape(wl.V, wl.N))
        # graph inputs pass no parent array
        self.parent = None if getattr(wl, "dag", False) else i32(wl.parent)
        self.pull_idx = i32(wl.pull_idx)
        self.push_idx = i32(wl.push_idx)
        self.X = f32(wl.X)
        self.Y = f32(wl.Y) if wl.loss == B.LOSS_L2 else None
        self.params = B.Params(cell=wl.cell, prec=wl.prec, loss=wl.loss, D=wl.D, H=wl.H, N=wl.N,
                               C=wl.C if wl.loss == B.LOSS_CE else 0,
                               Wx=f32(wl.Wx) if wl.cell == B.TREE_LSTM else None,
                               U=f32(wl.U), b=f32(wl.b),
                               Ws=f32(wl.Ws) if wl.loss == B.LOSS_CE else None,
                               bs=f32(wl.bs) if wl.loss == B.LOSS_CE else None)
        self.dH_ext: Optional[torch.Tensor] = None   # [V, H] external gradient of h_out
        self.sched: Optional[B.Schedule] = None
        self.ws = None
        self.ws_infer = None

    def schedule(self) -> B.Schedule:
        """cavs_schedule; reuses the schedule buffers from an earlier call."""
        wl = self.wl
        if self.sched is None:
            self.sched = B.alloc_schedule(self.ctx, wl.V, wl.N, wl.n_x)
        B.run_schedule(self.ctx, self.sched, self.child, self.parent, self.pull_idx,
                       self.push_idx, n_x=wl.n_x, n_push=wl.n_push)
        return self.sched

    def alloc(self):
        wl, dev = self.wl, self.dev
        nbytes = B.workspace_bytes(self.params, self.sched)
        self.ws = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
        f = dict(dtype=torch.float32, device=dev)
        self.h = torch.empty(wl.V, wl.H, **f)
        self.c = torch.empty(wl.V, wl.H, **f) if wl.cell == B.TREE_LSTM else None
        self.loss = torch.empty(1, **f)
        H, D, C = wl.H, wl.D, wl.C
        g = {}
        if wl.cell == B.TREE_LSTM:
            g["dWx"] = torch.empty(D, 4 * H, **f)
            g["dU"] = torch.empty(H, 4 * H, **f)
            g["db"] = torch.empty(4 * H, **f)
        else:
            g["dU"] = torch.empty(wl.N * H, H, **f)
            g["db"] = torch.empty(H, **f)
        if wl.loss == B.LOSS_CE:
            g["dWs"] = torch.empty(H, C, **f)
            g["dbs"] = torch.empty(C, **f)
        g["dX"] = torch.empty(max(wl.n_x, 0), D, **f)
        self.grads = g

    def forward(self):
        B.forward(self.ctx, self.params, self.sched, self.X, self.Y, self.ws, self.h, self.c,
                  self.loss)

    def backward(self):
        B.backward(self.ctx, self.params, self.sched, self.X, self.Y, self.ws, self.grads,
                   self.dH_ext)

    def infer(self):
        """cavs_infer into the same h / c / loss outputs, with its own smaller workspace."""
        if self.ws_infer is None:
            nbytes = B.infer_workspace_bytes(self.params, self.sched)
            self.ws_infer = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=self.dev)
        B.infer(self.ctx, self.params, self.sched, self.X, self.Y, self.ws_infer, self.h,
                self.c, self.loss)

    def run_infer(self) -> dict:
        """Schedule (if needed), cavs_infer, and the outputs as float64 numpy arrays."""
        if self.sched is None:
            self.schedule()
        if self.ws is None:
            self.alloc()
        self.infer()
        self.ctx.sync()
        return self.results(backward=False)

    def step(self):
        """One pass of the whole path: schedule, forward, backward (async tail)."""
        self.schedule()
        self.forward()
        self.backward()

    def run(self, backward: bool = True) -> dict:
        if self.sched is None:
            self.schedule()
        if self.ws is None:
            self.alloc()
        self.forward()
        if backward:
            self.backward()
        self.ctx.sync()
        return self.results(backward)

    def results(self, backward: bool = True) -> dict:
        r = dict(h=self.h.double().cpu().numpy(), loss=float(self.loss.item()))
        if self.c is not None:
            r["c"] = self.c.double().cpu().numpy()
        if backward:
            for k, v in self.grads.items():
                r[k] = v.double().cpu().numpy()
        return r


class LmBatch(Batch):
    """A language model over one batch: the words that vertices pull come from a
    table (``words[r]`` is the word of input row r), and every labelled vertex's
    state is scored over the vocabulary by cavs_vocab_grad, which keeps no
    logits.  The workload's X is not used; its Ws, bs and push_idx are the head
    and the labels.  ``teacher``: (words [V, K], logits [V, K], alpha, temp) of a
    model to learn from; ``head_dtype``: the type of the head's weights."""

    def __init__(self, wl: Workload, table: torch.Tensor, words, ctx: Optional[B.Context] = None,
                 device: int = 0, scale: float = 1.0, teacher=None,
                 head_dtype: torch.dtype = torch.float32):
        super().__init__(wl, ctx, device)
        p, dev = self.params, self.dev
        self.emb = B.Embedding(table, scale)
        self.words = torch.as_tensor(np.ascontiguousarray(words, dtype=np.int32)).to(dev)
        self.X = torch.empty(wl.n_x, wl.D, dtype=torch.float32, device=dev)
        # rounded on the host: a kernel on torch's stream is one that ctx's does not wait for
        self.Ws = (p.Ws if head_dtype == torch.float32 else
                   torch.from_numpy(np.ascontiguousarray(wl.Ws, dtype=np.float32)).to(head_dtype).to(dev))
        self.bs = p.bs
        self.params = B.Params(p.cell, p.prec, B.LOSS_NONE, p.D, p.H, p.N, 0, p.Wx, p.U, p.b,
                               None, None)
        self.teacher = teacher
        self.head: Optional[B.VocabHead] = None

    def alloc(self):
        super().alloc()
        wl, dev = self.wl, self.dev
        t = {}
        if self.teacher is not None:
            word, logit, alpha, temp = self.teacher
            t = dict(top_word=torch.as_tensor(word, dtype=torch.int32).to(dev),
                     top_logit=torch.as_tensor(logit, dtype=torch.float32).to(dev),
                     alpha=alpha, temp=temp)
        self.head = B.VocabHead(h=self.h, Ws=self.Ws, bs=self.bs, label=self.push_idx, **t)
        self.dH_ext = torch.empty_like(self.h)
        self.grads["dWs"] = torch.empty_like(self.Ws)
        self.grads["dbs"] = torch.empty_like(self.bs)
        self.grads["dE"] = torch.empty_like(self.emb.E)
        self.row_loss = torch.empty(wl.V, dtype=torch.float32, device=dev)
        # CAVS_LOSS_NONE's 0; kept, as the context's stream may write it after the call
        self.no_loss = torch.empty_like(self.loss)
        u8 = dict(dtype=torch.uint8, device=dev)
        self.ws_head = torch.empty(max(1, B.vocab_workspace_bytes(self.head, True)), **u8)
        self.ws_emb = torch.empty(max(1, B.embed_grad_workspace_bytes(self.emb, wl.n_x)), **u8)

    def forward(self):
        B.embed(self.ctx, self.emb, self.words, self.X)
        B.forward(self.ctx, self.params, self.sched, self.X, None, self.ws, self.h, self.c,
                  self.no_loss)
        g = self.grads
        B.vocab_grad(self.ctx, self.head, self.loss, self.row_loss, self.dH_ext, g["dWs"], g["dbs"],
                     self.ws_head)

    def backward(self):
        super().backward()
        B.embed_grad(self.ctx, self.emb, self.words, self.grads["dX"], self.grads["dE"], self.ws_emb)

    def infer(self):
        """The states and the loss alone (cavs_infer, cavs_vocab_loss)."""
        B.embed(self.ctx, self.emb, self.words, self.X)
        if self.ws_infer is None:
            n = B.infer_workspace_bytes(self.params, self.sched)
            self.ws_infer = torch.empty(max(n, 1), dtype=torch.uint8, device=self.dev)
        B.infer(self.ctx, self.params, self.sched, self.X, None, self.ws_infer, self.h, self.c,
                self.no_loss)
        B.vocab_loss(self.ctx, self.head, self.loss, self.row_loss, self.ws_head)
