"""Preference loss on pairs of packed sequences (device memory via torch; the
arithmetic is the library's fl_preference_forward / fl_preference_backward)."""

from __future__ import annotations

from . import flglm as F


class PreferenceLoss:
    """Sequences 2p (preferred) and 2p + 1 (rejected) of the batch:
    L_p = (1 - label_smoothing) softplus(-z) + label_smoothing softplus(z) with
    z = beta ((l_2p - ref_2p) - (l_2p+1 - ref_2p+1)), l_s the log-probability of
    sequence s's labelled tokens."""

    def __init__(self, vocab: int, dtype: str = "bf16", beta: float = 0.1, label_smoothing: float = 0.0):
        import torch
        self.vocab = vocab
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.f32, self.i32 = torch.float32, torch.int32
        self.desc = F.fl_preference_desc(vocab, F.FL_BF16 if dtype == "bf16" else F.FL_F32, beta, label_smoothing)

    def workspace(self, batch: F.BatchDesc, device="cuda"):
        """Holds what backward() needs of forward()."""
        import torch
        return torch.empty(F.fl_preference_workspace_bytes(self.desc, batch), dtype=torch.uint8, device=device)

    def outputs(self, batch: F.BatchDesc, device="cuda"):
        """Empty (logp [S], loss [S / 2], loss_sum [1])."""
        import torch
        S = batch.desc.num_seqs
        return tuple(torch.empty(n, dtype=torch.float32, device=device) for n in (S, S // 2, 1))

    def check_outputs(self, batch: F.BatchDesc, device: int, ref_logp, logp, loss, loss_sum):
        """Addresses of ref_logp [S] (or None), logp [S], loss [S / 2], loss_sum [1]."""
        S, f = batch.desc.num_seqs, self.f32
        return (F.address("ref_logp", ref_logp, device, (S,), f), F.address("logp", logp, device, (S,), f),
                F.address("loss", loss, device, (S // 2,), f), F.address("loss_sum", loss_sum, device, (1,), f))

    def _logits(self, batch, device, t, name):
        width = t.shape[1] if t.dim() == 2 else 0
        if width < self.vocab:
            raise F.FlglmError(F.FL_ERR_ARG, f"{name} is {tuple(t.shape)}, expected rows of at least {self.vocab}")
        return F.matrix(name, t, device, (batch.total_tokens, width), self.dtype)

    def forward(self, batch: F.BatchDesc, logits, labels, ref_logp, logp, loss, loss_sum, workspace,
                stream=None) -> None:
        """logits [T, >= vocab]; labels int32 [T] on the device (outside [0, vocab):
        none); ref_logp [S] or None (a reference model's pass itself: its logp)."""
        dev = F.current_device()
        logits, ld = self._logits(batch, dev, logits, "logits")
        labels = F.address("labels", labels, dev, (batch.total_tokens,), self.i32)
        ref_logp, logp, loss, loss_sum = self.check_outputs(batch, dev, ref_logp, logp, loss, loss_sum)
        F.fl_preference_forward(self.desc, batch, logits, ld, labels, ref_logp, logp, loss, loss_sum, workspace,
                                workspace.numel(), stream)

    def backward(self, batch: F.BatchDesc, logits, labels, grad_scale: float, dlogits, workspace, stream=None) -> None:
        """dlogits [T, >= vocab] = gradient of grad_scale * loss_sum, 0 past vocab;
        may be the logits."""
        dev = F.current_device()
        logits, ld = self._logits(batch, dev, logits, "logits")
        width = dlogits.shape[-1]
        dlogits, ld_d = self._logits(batch, dev, dlogits, "dlogits")
        labels = F.address("labels", labels, dev, (batch.total_tokens,), self.i32)
        F.fl_preference_backward(self.desc, batch, logits, ld, labels, grad_scale, dlogits, ld_d, width, workspace,
                                 workspace.numel(), stream)
