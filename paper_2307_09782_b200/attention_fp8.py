"""The attention block of a decoder layer on the FP8 operators, for serving: x -> queries, keys and values (FP8 linear layer), norms of
queries and keys and their rotation, the new tokens into the 8-bit cache, attention over it, output projection (FP8 linear
layer).  It keeps the weights and the workspaces; the work is done by the calls of :mod:`binding`.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding
from .binding import Fp8KvCache, Fp8Weight


class AttentionFp8:
    """``qkv``: stacked projections [(Hq + 2 H) D, K] to Hq heads of queries and H of keys and values; ``out``: [K_out, Hq D].

    ``table``: cosines and sines of the positions (:func:`binding.rotary_table`); ``q_norm``, ``k_norm``: weights of the norms,
    float32 [D], or neither; ``mode``: how activations are scaled, "none" or "M1"; ``cache_mode``: the same for the cache's blocks.
    A block is used on the device of its weights, which has to be the current one.  Workspaces are kept per thread and stream, and a
    captured call has its own, as for the calls of :mod:`binding`.
    """

    def __init__(self, qkv: Fp8Weight, out: Fp8Weight, Hq: int, H: int, table: torch.Tensor, *, q_norm: Optional[torch.Tensor] = None,
                 k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, pairs="halves", window: int = 0,
                 sm_scale: Optional[float] = None, mode: str = "none", cache_mode: str = "none"):
        if H < 1 or Hq % H or qkv.parts != 1 or out.parts != 1 or qkv.N % (Hq + 2 * H) or out.K * (Hq + 2 * H) != qkv.N * Hq:
            raise ValueError(f"qkv is [(Hq + 2 H) D, K] and out [K_out, Hq D] with Hq a multiple of H: got {qkv.parts} x "
                             f"[{qkv.N}, {qkv.K}] and {out.parts} x [{out.N}, {out.K}] for {Hq} and {H} heads")
        self.qkv, self.out, self.Hq, self.H, self.D = qkv, out, Hq, H, qkv.N // (Hq + 2 * H)
        self.table, self.q_norm, self.k_norm, self.eps, self.pairs = table, q_norm, k_norm, eps, pairs
        self.window, self.sm_scale, self.mode, self.cache_mode = window, sm_scale, mode, cache_mode

    @classmethod
    def from_weights(cls, qkv: torch.Tensor, out: torch.Tensor, Hq: int, H: int, table: torch.Tensor, **kw) -> "AttentionFp8":
        """From float32 weights [(Hq + 2 H) D, K] and [K_out, Hq D] (their blocks are scaled with the rule ``mode`` names)."""
        mode = kw.get("mode", "none")
        return cls(binding.quantize_weight_fp8_block(qkv, mode), binding.quantize_weight_fp8_block(out, mode), Hq, H, table, **kw)

    def new_cache(self, pages: int, page: int = 64) -> Fp8KvCache:
        return binding.make_kv_cache(pages, self.H, self.D, page, self.out.codes.device)

    def forward(self, x: torch.Tensor, cache: Fp8KvCache, pages: torch.Tensor, lens: torch.Tensor, positions: torch.Tensor, *,
                cu: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16) -> torch.Tensor:
        """x bf16 [T, K], the new tokens of B sequences -> [T, K_out].  ``pages`` int32 [B, pages of a sequence], ``lens`` int32 [B]: tokens
        with the new ones, ``cu`` int32 [B + 1]: the sequences' rows (without it one new token each, which is faster), ``positions``
        int32 [T].  Rows from cu[B] on are padding: only the projections work on them, and what comes out for them means nothing."""
        T, Hq, H = x.shape[0], self.Hq, self.H
        qkv = binding.fp8_block_linear(self.qkv, x=x, mode=self.mode, out_dtype=torch.bfloat16).view(T, Hq + 2 * H, self.D)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        binding.qk_norm_rope(q, k, self.table, positions, wq=self.q_norm, wk=self.k_norm, eps=self.eps, pairs=self.pairs, out=(q, k))
        binding.kv_cache_write(cache, k, v, pages, lens, cu=cu, mode=self.cache_mode)
        o = binding.kv_attention(cache, q, pages, lens, cu=cu, window=self.window, sm_scale=self.sm_scale)
        return binding.fp8_block_linear(self.out, x=o.view(T, Hq * self.D), mode=self.mode, out_dtype=out_dtype)
