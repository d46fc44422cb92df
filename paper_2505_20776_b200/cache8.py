"""The target's prefix cache in 8 bits (allocation and marshalling only).

`KvCache8` owns the codes (e4m3) and scales (e8m0, one per block of tokens and KV head) of one layer's keys and values and
counts the tokens in them; `append` puts tokens behind the last one (or at `start`, which drops what lay behind it), and
`HotPath.verify_attn_q8` attends to it.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import api


class KvCache8:
    def __init__(self, n_kv_heads: int, head_dim: int, capacity: int, block_tokens: int = 32, device="cuda:0"):
        if block_tokens not in (32, 64, 128):
            raise ValueError("block_tokens must be 32, 64 or 128")
        self.Hkv, self.D, self.capacity, self.block_tokens = n_kv_heads, head_dim, capacity, block_tokens
        self.device = torch.device(device)
        blocks = -(-capacity // block_tokens)
        self.K, self.V = (self._alloc((capacity, n_kv_heads, head_dim), torch.float8_e4m3fn) for _ in range(2))
        self.K_scale, self.V_scale = (self._alloc((blocks, n_kv_heads), torch.float8_e8m0fnu) for _ in range(2))
        self.status = self._alloc((1,), torch.int32).zero_()
        self.length = 0

    def _alloc(self, shape, dtype) -> torch.Tensor:
        """Every device buffer of the cache comes from here (a subclass may place them differently)."""
        return torch.empty(shape, dtype=dtype, device=self.device)

    def append(self, K: torch.Tensor, V: torch.Tensor, rows: Optional[torch.Tensor] = None,
               start: Optional[int] = None) -> None:
        """Appends K and V [n][Hkv][D] (bf16), or the rows of them that the int32 vector `rows` names, behind the last token;
        `start` <= length begins there instead (tokens behind it are given up)."""
        at = self.length if start is None else start
        n = K.shape[0] if rows is None else rows.shape[0]
        if not 0 <= at <= self.length or at + n > self.capacity:
            raise ValueError("tokens can begin inside or right behind those that are there, and must fit the capacity")
        api.specext_quantize_kv(K, V, at, self.K, self.V, self.K_scale, self.V_scale, self.block_tokens, self.status, rows)
        self.length = at + n

    def read_status(self) -> int:
        return api.specext_read_status(self.status)
