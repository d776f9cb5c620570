"""A bias-free ReLU network of any width whose rows choose their matrices (Definition 1 of the paper, with a set of
matrices for each frame, view or block of space instead of one for the whole batch), trained with first-order gradients.

Every layer has one matrix per group of consecutive rows, or one matrix for all rows and a low-rank adapter per group.  For the
backward pass it keeps its input as it is, or in 8 bits where the caller wants that, and the ReLU masks in single bits (9.25 bits a
feature instead of 33); activations that are kept in 8 bits, and gradients, pass from layer to layer through two buffers.
This module orders calls of the library and owns the buffers; all arithmetic is in the library.
"""
from __future__ import annotations

from typing import Optional, Sequence

from . import binding as nb


class RowNetwork:
    def __init__(self, dims: Sequence[int], n: int, groups: int, matrices, dtype: str = "f32", adapters=None, slots=None,
                 keep8: bool = False, train_matrices: bool = True, device="cuda"):
        """`n` rows in every batch, all of them in some group.  `dims`: widths, input first.  `matrices[l]`: [groups, dims[l+1], dims[l]], or with adapters [dims[l+1], dims[l]].
        `adapters[l]`: (A [bank, rank, dims[l]], B [bank, dims[l+1], rank], scales [bank]); `slots` [groups] the adapter of
        each group (None: its own number).  `keep8`: layer inputs are kept in 8 bits, and matrix gradients are those of the
        rounded inputs (each off by at most 1/127 of the largest of its 32).  `train_matrices`: False leaves shared matrices as
        they are (adapters only)."""
        import torch
        self.torch, self.dims, self.n, self.groups, self.dtype = torch, list(dims), n, groups, dtype
        self.layers_count = len(dims) - 1
        if len(matrices) != self.layers_count or adapters is not None and len(adapters) != self.layers_count:
            raise ValueError(f"{self.layers_count} layers need as many matrices and adapters")
        self.keep8, self.train_matrices, self.device = keep8, train_matrices or adapters is None, device
        self.tdt = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        # copies: training changes the network's matrices, not the caller's
        own = lambda t, dtype: torch.as_tensor(t).detach().to(device=device, dtype=dtype, copy=True).contiguous()
        move = lambda t: own(t, self.tdt)
        f32 = dict(dtype=torch.float32, device=device)
        self.W = [move(m) for m in matrices]
        self.dW = [torch.zeros(w.shape, **f32) if self.train_matrices else None for w in self.W]
        self.slots = None if slots is None else own(slots, torch.int32)
        self.adapters = None
        if adapters is not None:
            self.adapters = [(move(A), move(B), own(s, torch.float32)) for A, B, s in adapters]
            self.dA = [torch.zeros(A.shape, **f32) for A, _, _ in self.adapters]
            self.dB = [torch.zeros(B.shape, **f32) for _, B, _ in self.adapters]
        self.layer, self.dense = [], []
        for l in range(self.layers_count):
            last = l + 1 == self.layers_count
            rank, bank = (self.adapters[l][0].shape[1], self.adapters[l][0].shape[0]) if self.adapters else (0, 0)
            self.layer.append(nb.make_layer(dtype, groups, dims[l], dims[l + 1], rank=rank, adapters=bank, relu=not last))
            self.dense.append(nb.make_layer(dtype, 1, dims[l], dims[l + 1]))
        rows = lambda width: torch.zeros(n, width, dtype=self.tdt, device=device)
        # what one layer hands to the next and nobody needs afterwards: two buffers in turn
        turns = [torch.zeros(n * max(dims[1:-1], default=0), dtype=self.tdt, device=device) for _ in range(4 if keep8 else 2)]
        in_turn = lambda l, at: turns[at + l % 2][:n * dims[l]].view(n, dims[l])
        # activations (the input of layer l is rows[l]) and the gradients with respect to them
        self.rows = [None] + [in_turn(l, 2) if keep8 else rows(dims[l]) for l in range(1, len(dims) - 1)] + [rows(dims[-1])]
        self.grad = [rows(dims[0])] + [in_turn(l, 0) for l in range(1, len(dims) - 1)] + [None]
        packed = lambda d: (torch.zeros(n, (d + 31) // 32 * 32, dtype=torch.int8, device=device),
                            torch.zeros(n, (d + 31) // 32, dtype=torch.uint8, device=device))
        self.kept = [packed(d) for d in dims[:-1]] if keep8 else None
        self.masks = [None] + [torch.zeros(n, (d + 31) // 32, dtype=torch.int32, device=device) for d in dims[1:-1]]
        self.u = [torch.zeros(n, a[0].shape[1], **f32) for a in self.adapters] if self.adapters else None
        need = [nb.grouped_workspace_bytes(self.dense[l] if self.adapters else self.layer[l], n) for l in range(self.layers_count)]
        if self.adapters:
            need += [nb.adapter_workspace_bytes(layer, n) for layer in self.layer]
        self.workspace = torch.zeros(max(max(need) // 4, 4), dtype=torch.int32, device=device)
        self.opt = None

    def forward(self, x, offsets):
        """x [n, dims[0]], offsets [groups + 1]: the network's outputs [n, dims[-1]] (a buffer of this object)."""
        self.offsets = offsets
        self.rows[0] = x
        for l in range(self.layers_count):
            if self.keep8 or l > 0:
                nb.pack8(self.rows[l], *(self.kept[l] if self.keep8 else (None, None)), self.masks[l] if l > 0 else None)
            if self.adapters:
                nb.adapter_fwd(self.layer[l], self.rows[l], self.W[l], *self.adapters[l], self.slots, offsets, self.u[l], self.rows[l + 1])
            else:
                nb.grouped_fwd(self.layer[l], self.rows[l], self.W[l], offsets, self.rows[l + 1])
        return self.rows[-1]

    def backward(self, dy, want_dx: bool = False):
        """dy [n, dims[-1]]: fills dW (and dA, dB); returns the gradient with respect to x, or None.  Goes with the last forward
        call, whose x (with `keep8` false) must still be what it was."""
        for l in reversed(range(self.layers_count)):
            x = self.kept[l] if self.keep8 else self.rows[l]
            dx = self.grad[l] if l > 0 or want_dx else None
            if self.adapters:
                A, B, scales = self.adapters[l]
                nb.adapter_bwd(self.layer[l], x, self.W[l], A, B, scales, self.slots, self.offsets, self.u[l], dy, dx, self.dA[l],
                               self.dB[l], self.workspace, masks=self.masks[l])
                if self.train_matrices:
                    nb.grouped_bwd(self.dense[l], x, None, None, dy, None, self.dW[l].unsqueeze(0), self.workspace)
            else:
                nb.grouped_bwd(self.layer[l], x, self.W[l], self.offsets, dy, dx, self.dW[l], self.workspace, masks=self.masks[l])
            dy = dx
        return dy

    def init_optimizer(self, lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-15) -> None:
        """Adam state of everything that is trained; fp16 matrices keep an fp32 master copy (bf16 ones cannot be trained here)."""
        if self.dtype == "bf16":
            raise ValueError("bf16 matrices: the library's Adam step updates fp32 and fp16 parameters")
        pairs = [(w, g) for w, g in zip(self.W, self.dW) if g is not None]
        if self.adapters:
            pairs += [(a[0], g) for a, g in zip(self.adapters, self.dA)] + [(a[1], g) for a, g in zip(self.adapters, self.dB)]
        zeros = self.torch.zeros_like
        self.opt = {"lr": lr, "b1": beta1, "b2": beta2, "eps": eps, "t": 0,
                    "params": [(p, p.float() if self.dtype == "f16" else None, g, zeros(g), zeros(g)) for p, g in pairs]}

    def adam(self) -> None:
        """One Adam step on the gradients of the last backward call."""
        o = self.opt
        o["t"] += 1
        for param, master, grad, m, v in o["params"]:
            nb.adam_step(param, master, grad, m, v, 1 if self.dtype == "f16" else 0, o["lr"], o["b1"], o["b2"], o["eps"], o["t"],
                         zero_grad=False)
