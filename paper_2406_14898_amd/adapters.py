"""Low-rank adapters of many clients beside a projection that they share
(device memory via torch; the arithmetic is the library's fl_adapter_forward /
fl_adapter_backward, and the fl_server_stack_*_adapters calls of ServerStack)."""

from __future__ import annotations

from typing import Dict, Optional, Sequence

from . import flglm as F


class ClientAdapters:
    """n slots of pairs A [rank, in_features], B [out_features, rank]: for the
    rows of a client with slot s, v = x A_s^T and y = base + scale v B_s^T.
    A client without a slot (-1) has y = base; clients may share slots."""

    def __init__(self, num_adapters: int, rank: int, in_features: int, out_features: int, dtype: str = "bf16",
                 scale: float = 1.0):
        import torch
        self.desc = F.fl_adapter_desc(num_adapters, rank, in_features, out_features, scale,
                                      F.FL_BF16 if dtype == "bf16" else F.FL_F32)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.f32 = torch.float32
        self.shape_a = (num_adapters, rank, in_features)
        self.shape_b = (num_adapters, out_features, rank)

    def workspace(self, batch: F.BatchDesc, device="cuda"):
        """Scratch of one call, forward or backward, on this batch."""
        import torch
        return torch.empty(F.fl_adapter_workspace_bytes(self.desc, batch), dtype=torch.uint8, device=device)

    def forward(self, batch: F.BatchDesc, client_adapter, x, a, b, base, y, v, workspace, stream=None) -> None:
        """client_adapter: each client's slot or -1 (host).  x [T, in], base [T,
        out] (None: 0; may be y) and y [T, out] may have rows apart in memory; v
        fp32 [T, rank] is what backward() reads."""
        T, (_, r, inn), out, dt = batch.total_tokens, self.shape_a, self.shape_b[1], self.dtype
        dev = F.current_device()
        x, ldx = F.matrix("x", x, dev, (T, inn), dt)
        base, ld_base = F.matrix("base", base, dev, (T, out), dt)
        y, ldy = F.matrix("y", y, dev, (T, out), dt)
        a, b = F.address("a", a, dev, self.shape_a, dt), F.address("b", b, dev, self.shape_b, dt)
        v = F.address("v", v, dev, (T, r), self.f32)
        F.fl_adapter_forward(self.desc, batch, client_adapter, x, ldx, a, b, base, ld_base, y, ldy, v, workspace,
                             workspace.numel(), stream)

    def backward(self, batch: F.BatchDesc, client_adapter, dy, x, a, b, v, dres, dx, da, db, workspace,
                 stream=None) -> None:
        """dx = dres + dv A (dres None: 0, may be dx; dx None: not formed); da, db
        fp32, accumulated (+=)."""
        T, (_, r, inn), out, dt = batch.total_tokens, self.shape_a, self.shape_b[1], self.dtype
        dev = F.current_device()
        dy, ld_dy = F.matrix("dy", dy, dev, (T, out), dt)
        x, ldx = F.matrix("x", x, dev, (T, inn), dt)
        dres, ld_dres = F.matrix("dres", dres, dev, (T, inn), dt)
        dx, ld_dx = F.matrix("dx", dx, dev, (T, inn), dt)
        a, b = F.address("a", a, dev, self.shape_a, dt), F.address("b", b, dev, self.shape_b, dt)
        v = F.address("v", v, dev, (T, r), self.f32)
        da, db = F.address("da", da, dev, self.shape_a, self.f32), F.address("db", db, dev, self.shape_b, self.f32)
        F.fl_adapter_backward(self.desc, batch, client_adapter, dy, ld_dy, x, ldx, a, b, v, dres, ld_dres, dx, ld_dx, da,
                              db, workspace, workspace.numel(), stream)


class StackAdapters:
    """Adapters on the fused query / key / value projection of every block of a
    ServerStack, for batches of one shape: what its forward() and backward()
    take as `adapters`.  layers / grads: one dict "a" [n, rank, H], "b" [n, 3H,
    rank] a block (gradients fp32, accumulated; None: forward only).  Owns the
    workspace, in which a forward leaves what its backward reads: calls on
    different streams, or graphs captured with it, must not overlap, and it lives
    as long as such a graph.  (Calls on any stream may outlive it.)"""

    def __init__(self, stack, batch: F.BatchDesc, client_adapter, layers: Sequence[Dict],
                 grads: Optional[Sequence[Dict]] = None, scale: float = 1.0, device="cuda"):
        import torch
        dt = torch.bfloat16 if stack.dtype == F.FL_BF16 else torch.float32
        if len(layers) != stack.num_layers or (grads is not None and len(grads) != stack.num_layers):
            raise F.FlglmError(F.FL_ERR_ARG, f"adapters of {len(layers)} blocks for a stack of {stack.num_layers}")
        n, r, _ = layers[0]["a"].shape
        dev = F.current_device()
        for what, rows, t in (("adapter", layers, dt), ("adapter gradient", grads or (), torch.float32)):
            for l, d in enumerate(rows):
                F.address(f"{what} a of block {l}", d["a"], dev, (n, r, stack.hidden), t)
                F.address(f"{what} b of block {l}", d["b"], dev, (n, 3 * stack.hidden, r), t)
        # the record holds addresses: the tensors themselves, not only their dicts, live as long
        self.tensors = [d[k] for rows in (layers, grads or ()) for d in rows for k in ("a", "b")]
        self.stack, self.device, self.has_grads = stack, dev, grads is not None
        self.clients, self.tokens = batch.desc.num_clients, batch.total_tokens
        self.record = F.stack_adapters(n, r, scale, batch, client_adapter, layers, grads)
        self.workspace = torch.empty(F.fl_stack_adapter_bytes(stack.handle, batch, self.record), dtype=torch.uint8,
                                     device=device)
        self.memory = F.Memory(self.workspace, *self.tensors)

    def check(self, stack, batch: F.BatchDesc, backward: bool = False) -> None:
        """Refuses a call that the record and the workspace were not made for."""
        if stack is not self.stack:
            raise F.FlglmError(F.FL_ERR_ARG, "the adapters are another stack's")
        if batch.desc.num_clients != self.clients or batch.total_tokens != self.tokens:
            raise F.FlglmError(F.FL_ERR_ARG, f"adapters for {self.clients} clients and {self.tokens} tokens, a batch of "
                                             f"{batch.desc.num_clients} and {batch.total_tokens}")
        if F.current_device() != self.device:
            raise F.FlglmError(F.FL_ERR_ARG, f"the adapters are on device {self.device}, not on the current one")
        if backward and not self.has_grads:
            raise F.FlglmError(F.FL_ERR_ARG, "the adapters have no gradients")
