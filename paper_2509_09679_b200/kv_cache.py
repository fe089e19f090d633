"""The paged low-bit cache of rotated keys and values that Plan.append_kv, read_kv and attend_kv work on: four tensors and their format.

A page holds `page_size` places for every head.  For keys and for values there are codes, uint8 [pages][heads][page_size][head_dim * bits / 8]
(packed two's complement, as Plan.forward_quant writes them), and scales, fp16 [pages][heads][page_size], one for each row of head_dim elements.
Slot s is place s % page_size of page s // page_size.  Which pages a sequence has is the caller's to keep (a block table).
"""
from __future__ import annotations

import torch


class KVCache:
    """A cache made of the caller's tensors; pages may lie apart (any stride of the first dimension that is a multiple of 16 bytes), what is
    in a page is contiguous."""

    def __init__(self, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor, bits: int):
        if bits not in (4, 8):
            raise ValueError(f"bits must be 4 or 8, got {bits}")
        shape = tuple(k_codes.shape)
        if len(shape) != 4:
            raise ValueError(f"k_codes: expected [pages][heads][page_size][bytes], got {shape}")
        pages, heads, page_size, width = shape
        for t, dtype, expected, what in ((k_codes, torch.uint8, shape, "k_codes"), (v_codes, torch.uint8, shape, "v_codes"),
                                         (k_scales, torch.float16, shape[:3], "k_scales"), (v_scales, torch.float16, shape[:3], "v_scales")):
            if t.dtype != dtype or tuple(t.shape) != expected:
                raise ValueError(f"{what}: expected {dtype} of shape {expected}, got {t.dtype}, {tuple(t.shape)}")
            if t.device != k_codes.device:
                raise ValueError(f"{what}: tensor is on {t.device}, the keys' codes are on {k_codes.device}")
            if pages and not t[0].is_contiguous():
                raise ValueError(f"{what}: a page must be contiguous")
            if pages > 1 and (t.stride(0) < t[0].numel() or t.stride(0) * t.element_size() % 16):
                raise ValueError(f"{what}: pages overlap, or are not a multiple of 16 bytes apart")
        if page_size not in (16, 32, 64, 128, 256):
            raise ValueError(f"page_size must be a power of two from 16 to 256, got {page_size}")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales, self.bits = k_codes, k_scales, v_codes, v_scales, int(bits)
        self.pages, self.heads, self.page_size, self.head_dim = pages, heads, page_size, width * 8 // self.bits
        self.device = k_codes.device

    @classmethod
    def empty(cls, pages: int, heads: int, head_dim: int, page_size: int = 64, bits: int = 4, device=None) -> "KVCache":
        """New pages, all codes and scales zero."""
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        codes, scales = (pages, heads, page_size, head_dim * bits // 8), (pages, heads, page_size)
        k, v = (torch.zeros(codes, dtype=torch.uint8, device=device) for _ in range(2))
        ks, vs = (torch.zeros(scales, dtype=torch.float16, device=device) for _ in range(2))
        return cls(k, ks, v, vs, bits)
