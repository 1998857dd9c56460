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

    def _outputs(self, batch, ref_logp, logp, loss, loss_sum):
        import torch
        S, f = batch.desc.num_seqs, torch.float32
        F.tensors(("ref_logp", ref_logp, (S,), f), ("logp", logp, (S,), f), ("loss", loss, (S // 2,), f),
                  ("loss_sum", loss_sum, (1,), f))

    def _logits(self, batch, t, name):
        if t.dim() != 2 or t.shape[1] < self.vocab:
            raise F.FlglmError(F.FL_ERR_ARG, f"{name} is {tuple(t.shape)}, expected rows of at least {self.vocab}")
        return F.matrix(t, batch.total_tokens, t.shape[1], self.dtype, name)

    def forward(self, batch: F.BatchDesc, logits, labels, ref_logp, logp, loss, loss_sum, workspace,
                stream=None) -> None:
        """logits [T, >= vocab]; labels int32 [T] on the device (outside [0, vocab):
        none); ref_logp [S] or None (a reference model's pass itself: its logp)."""
        import torch
        logits, ld = self._logits(batch, logits, "logits")
        F.tensors(("labels", labels, (batch.total_tokens,), torch.int32))
        self._outputs(batch, ref_logp, logp, loss, loss_sum)
        F.fl_preference_forward(self.desc, batch, logits, ld, labels, ref_logp, logp, loss, loss_sum, workspace,
                                workspace.numel(), stream)

    def backward(self, batch: F.BatchDesc, logits, labels, grad_scale: float, dlogits, workspace, stream=None) -> None:
        """dlogits [T, >= vocab] = gradient of grad_scale * loss_sum, 0 past vocab;
        may be the logits."""
        import torch
        logits, ld = self._logits(batch, logits, "logits")
        dlogits, ld_d = self._logits(batch, dlogits, "dlogits")
        F.tensors(("labels", labels, (batch.total_tokens,), torch.int32))
        F.fl_preference_backward(self.desc, batch, logits, ld, labels, grad_scale, dlogits, ld_d, dlogits.shape[1],
                                 workspace, workspace.numel(), stream)
