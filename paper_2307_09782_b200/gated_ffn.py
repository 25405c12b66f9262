"""The gated feed-forward block on the FP8 operators with block scales: y = (act(x Wg^T) * (x Wu^T)) Wd^T, for serving and
for training with 8-bit activation checkpoints.  It keeps the weights and
the workspaces; the work is done by the calls of :mod:`binding`.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding
from .binding import Fp8Weight


class GatedFfnFp8:
    """``gate_up``: stacked gate and up weights (parts = 2, [F, K]); ``down``: [K_out, F].

    ``mode``: how activations are scaled, "none" (FP32 scales) or "M1" (powers of two, which the 8-bit checkpoints
    turn back into bf16 without rounding: the one to train with).  ``training`` lays the transposed weights out as well.
    A block is used on the device of its weights, which has to be the current one.  It keeps one workspace per thread and stream,
    grown on demand; a call that is captured into a CUDA graph gets one of its own, in the graph's memory.
    """

    def __init__(self, gate_up: Fp8Weight, down: Fp8Weight, act: str = "silu", mode: str = "none", training: bool = False):
        if gate_up.parts != 2 or down.parts != 1 or down.K != gate_up.N:
            raise ValueError(f"gate_up is 2 x [F, K] and down [K_out, F]: got {gate_up.parts} x [{gate_up.N}, {gate_up.K}] "
                             f"and [{down.N}, {down.K}]")
        self.gate_up, self.down, self.act, self.mode = gate_up, down, act, mode
        self.gate_up_t: Optional[Fp8Weight] = None
        self.down_t: Optional[Fp8Weight] = None
        self._workspaces = binding.KeptWorkspaces()
        if training:
            self.gate_up_t = binding.transpose_fp8_weight(gate_up)
            self.down_t = binding.transpose_fp8_weight(down)

    @classmethod
    def from_weights(cls, gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor, **kw) -> "GatedFfnFp8":
        """From float32 weights [F, K], [F, K], [K_out, F] (their blocks are scaled with the rule ``mode`` names)."""
        mode = kw.get("mode", "none")
        return cls(binding.quantize_weight_fp8_block(torch.stack([gate, up]), mode),
                   binding.quantize_weight_fp8_block(down.contiguous(), mode), **kw)

    def _new_workspace(self, M: int) -> torch.Tensor:
        return binding.make_workspace(binding.fp8_gated_ffn_workspace_bytes(M, self.gate_up.K, self.gate_up.N, self.down.N,
                                                                            self.down_t is not None), self.down.codes.device)

    def workspace(self, M: int) -> torch.Tensor:
        if binding._capturing():
            return self._new_workspace(M)
        key = self.down.codes.device.index, binding._stream()
        kept = self._workspaces.of
        ws, rows = kept.get(key, (None, -1))
        if rows < M:
            ws = self._new_workspace(M)
            kept[key] = (ws, M)
        return ws

    def forward(self, x: torch.Tensor, out_dtype=torch.bfloat16) -> torch.Tensor:
        """x bf16 [M, K] -> y [M, K_out]; h goes from one kernel to the next in its quantized form."""
        return binding.fp8_gated_ffn(self.gate_up, self.down, x, act=self.act, mode=self.mode, out_dtype=out_dtype,
                                     workspace=self.workspace(x.shape[0]))

    def forward_train(self, x: torch.Tensor, out_dtype=torch.bfloat16):
        """(y, what :meth:`backward` needs: x, gate, up and h as 8-bit checkpoints in one buffer)."""
        return binding.fp8_gated_ffn(self.gate_up, self.down, x, act=self.act, mode=self.mode, out_dtype=out_dtype,
                                     save=True, workspace=self.workspace(x.shape[0]))

    def backward(self, dy: torch.Tensor, saved: torch.Tensor, out_dtype=torch.bfloat16):
        """dy bf16 [M, K_out] -> (dx [M, K], dW of (gate, up) [2, F, K], dW of down [K_out, F])."""
        if self.down_t is None or self.gate_up_t is None:
            raise ValueError("the backward pass needs the transposed weights: construct the block with training=True")
        return binding.fp8_gated_ffn_backward(self.gate_up_t, self.down_t, dy, saved, act=self.act, mode=self.mode,
                                              out_dtype=out_dtype, workspace=self.workspace(dy.shape[0]))
