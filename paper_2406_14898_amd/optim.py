"""Flat parameter arenas for the server update (device memory via torch; the
arithmetic is the library's fl_adam_step / fl_average_replicas).

An arena holds a set of named tensors back to back in one fp32 master
buffer, with fp32 gradient and Adam moment buffers of the same layout and,
optionally, a bf16 compute copy.  The per-tensor views are what the stack
reads (the bf16 views, or the fp32 masters for the fp32 stack) and
accumulates into (the gradient views), so one launch updates every tensor.
"""

from __future__ import annotations

import ctypes
from typing import Dict, Iterable, List, Optional, Sequence, Tuple

from . import flglm as F

_ALIGN = 8  # elements: every view starts 16-byte aligned in fp32 and bf16


class ParamArena:
    def __init__(self, shapes: Iterable[Tuple[str, Tuple[int, ...]]], bf16_copy: bool, device="cuda"):
        import torch
        self.names: List[str] = []
        self.offsets: Dict[str, Tuple[int, Tuple[int, ...]]] = {}
        n = 0
        for name, shape in shapes:
            size = 1
            for s in shape:
                size *= int(s)
            self.names.append(name)
            self.offsets[name] = (n, tuple(shape))
            n += (size + _ALIGN - 1) // _ALIGN * _ALIGN
        self.n = n
        z = dict(dtype=torch.float32, device=device)
        self.master = torch.zeros(max(n, _ALIGN), **z)
        self.grad = torch.zeros(max(n, _ALIGN), **z)
        self.exp_avg = torch.zeros(max(n, _ALIGN), **z)
        self.exp_avg_sq = torch.zeros(max(n, _ALIGN), **z)
        self.compute = torch.zeros(max(n, _ALIGN), dtype=torch.bfloat16, device=device) if bf16_copy else None
        self.step_count = 0
        self._norm: Optional[GradNorm] = None
        self._clipped: List = []

    def _view(self, buf, name):
        off, shape = self.offsets[name]
        size = 1
        for s in shape:
            size *= s
        return buf[off:off + size].view(shape)

    def master_views(self) -> Dict[str, "object"]:
        return {k: self._view(self.master, k) for k in self.names}

    def grad_views(self) -> Dict[str, "object"]:
        return {k: self._view(self.grad, k) for k in self.names}

    def compute_views(self) -> Dict[str, "object"]:
        """The tensors the stack reads: the bf16 copy, else the fp32 masters."""
        buf = self.compute if self.compute is not None else self.master
        return {k: self._view(buf, k) for k in self.names}

    def load(self, values: Dict[str, "object"]) -> None:
        """Sets the masters (and the bf16 copy, rounded) from tensors."""
        for k, v in values.items():
            self._view(self.master, k).copy_(v)
        self.refresh_compute()

    def refresh_compute(self) -> None:
        """bf16 copy := the masters rounded to nearest even (after the
        masters were written directly through master_views())."""
        if self.compute is not None:
            self.compute.copy_(self.master)

    def _runs(self) -> List[Tuple[int, int]]:
        """(first element, elements) of the tensors' values, neighbours without
        padding between them as one."""
        runs: List[Tuple[int, int]] = []
        for off, shape in self.offsets.values():
            n = 1
            for s in shape:
                n *= int(s)
            if n and runs and sum(runs[-1]) == off:
                runs[-1] = (runs[-1][0], runs[-1][1] + n)
            elif n:
                runs.append((off, n))
        return runs

    def clip_grad_norm(self, max_norm: float, stream=None):
        """Scales the gradients in place so that their global norm is at most
        max_norm; returns the norm before (device fp32 [1], which the next call
        overwrites: clone it to keep it).  The padding between tensors, which
        nothing clears but a whole step, keeps its zeros: a NaN coefficient would
        stay in it for every later norm."""
        if self._norm is None or self._norm.grads[0] is not self.grad:
            self._norm = GradNorm([self.grad])
            self._clipped = [self.grad[a:a + n] for a, n in self._runs()]
        norm = self._norm.norm(max_norm, stream)
        if self._clipped:
            at = F.pointers(self._clipped)
            F.fl_clip_grads(F.FL_F32, at, at, [t.numel() for t in self._clipped], self._norm.result, stream)
        return norm

    def adam_step(self, lr: float = 2e-2, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                  zero_grad: bool = True, stream=None) -> None:
        """One Adam step over every tensor of the arena (time step advances)."""
        self.step_count += 1
        F.fl_adam_step(self.master, self.grad, self.exp_avg, self.exp_avg_sq, self.compute, self.n, self.step_count,
                       lr, beta1, beta2, eps, zero_grad, stream)


class GradNorm:
    """Global norm of a list of gradients (fp32 or bf16, all of one type) and
    their clipping.  Owns the workspace and the result: calls of one GradNorm
    on different streams, or graphs captured from it, must not overlap, and it
    lives as long as such a graph.  (Calls on any stream may outlive it.)  The
    norm that a call returns is a view of the result, which the next call
    overwrites: clone it to keep it."""

    def __init__(self, grads: Sequence):
        import torch
        if not grads:
            raise F.FlglmError(F.FL_ERR_ARG, "no gradients")
        self.grads = list(grads)
        self.dtype = self.grads[0].dtype
        if self.dtype not in (torch.float32, torch.bfloat16):
            raise F.FlglmError(F.FL_ERR_ARG, f"gradients are fp32 or bf16, not {self.dtype}")
        dev = F.current_device()
        for i, g in enumerate(self.grads):
            F.address(f"gradient {i}", g, dev, g.shape, self.dtype)
        self.kind = F.FL_F32 if self.dtype == torch.float32 else F.FL_BF16
        self.numel = [g.numel() for g in self.grads]
        self.sizes = F._sizes(self.numel)
        self.array = ctypes.c_void_p * len(self.grads)
        self.workspace = torch.empty(F.fl_grad_norm_workspace_bytes(self.sizes), dtype=torch.uint8, device=dev)
        self.result = torch.empty(2, dtype=torch.float32, device=dev)  # norm, coefficient
        self.memory = F.Memory(self.workspace, self.result)
        self.device = dev

    def norm(self, max_norm: float = float("inf"), stream=None):
        """Device fp32 [1]: the norm of the gradients' present values.  The
        coefficient min(1, max_norm / (norm + 1e-6)) is left in result[1]."""
        self._norm(self._addresses(self.grads), max_norm, stream)
        return self.result[:1]

    def clip(self, max_norm: float, out: Optional[Sequence] = None, stream=None):
        """Gradients times the coefficient, into `out` (tensors like the
        gradients; None: in place); returns the norm before."""
        grads = to = self._addresses(self.grads)
        if out is not None:
            if len(out) != len(self.numel):
                raise F.FlglmError(F.FL_ERR_ARG, f"{len(out)} outputs for {len(self.numel)} gradients")
            t = type(self.result)  # the checks one by one over all tensors: 52 of them 8 us, tensor by tensor 22
            if not (list(map(t.numel, out)) == self.numel and {o.dtype for o in out} == {self.dtype} and
                    set(map(t.get_device, out)) == {self.device} and all(map(t.is_contiguous, out))):
                raise F.FlglmError(F.FL_ERR_ARG, f"an output is not as many contiguous elements as its gradient, in "
                                                 f"{self.dtype} on device {self.device}")
            to = self._addresses(out)
        stream = self._norm(grads, max_norm, stream)
        F.fl_clip_grads(self.kind, grads, to, self.sizes, self.result, stream)
        return self.result[:1]

    def _addresses(self, tensors):
        return self.array(*map(type(self.result).data_ptr, tensors))

    def _norm(self, grads, max_norm, stream):
        if F.current_device() != self.device:
            raise F.FlglmError(F.FL_ERR_ARG, f"the gradients are on device {self.device}, not on the current one")
        stream = self.memory.on(stream)
        F.fl_grad_norm(self.kind, grads, self.sizes, max_norm, self.result, self.workspace, self.workspace.numel(),
                       stream)
        return stream


def average(arenas: Sequence[ParamArena], stream=None) -> None:
    """Server-hierarchical aggregation: every arena's masters (and bf16
    copies) become the elementwise mean over the arenas."""
    n = arenas[0].n
    if any(a.n != n for a in arenas):
        raise ValueError("arenas differ in layout")
    c16: Optional[list] = [a.compute for a in arenas] if arenas[0].compute is not None else None
    F.fl_average_replicas([a.master for a in arenas], c16, n, stream)
