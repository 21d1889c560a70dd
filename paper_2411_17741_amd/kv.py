"""PyTorch plumbing around the paged key-value cache (include/lora_kv.h): device memory for its pages, stream handles,
shapes and strides of the tensors it is given.  No arithmetic of the method happens here."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


def _dtype(dtype: int) -> torch.dtype:
    return torch.bfloat16 if dtype == B.LORA_BF16 else torch.float32


class KvCache:
    """Owns the cache handle and, unless the caller brings them, the pages' memory: a tensor
    [n_pages][n_layers][2][n_kv_heads][page_tokens * head_dim] (see the header for what lies where in it).

    max_batch_pages: pages that the sequences of a batch may have together, one that they share counted for each; a batch with more is refused.  By default
    whatever max_batch_seqs sequences can have, up to 4 million or 4 times the pages there are."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, page_tokens: int = 64, max_seqs: int = 512,
                 max_batch_tokens: int = 4096, max_batch_seqs: int = 512, max_batch_pages: int = 0, n_batches: int = 2,
                 dtype: int = B.LORA_BF16, device: str = "cuda:0", pages: Optional[torch.Tensor] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("KvCache needs a GPU: the library has no CPU path")
        index = torch.device(device).index
        self._index = index if index is not None else torch.cuda.current_device()
        self.device = torch.device("cuda", self._index)
        self.n_heads, self.n_kv_heads, self.head_dim, self.dtype = n_heads, n_kv_heads, head_dim, _dtype(dtype)
        # Forks share pages: the sequences of a batch may name more pages than there are.  Every sequence may name all of them, up to a list of 16 MB for each batch
        max_batch_pages = max_batch_pages or min(max_batch_seqs * n_pages, max(4 * n_pages, 1 << 22))
        self.cfg = B.make_kv_config(n_layers, n_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs, max_batch_seqs, max_batch_tokens,
                                    max_batch_pages, n_batches, dtype)
        n_bytes, work = B.lora_kv_pages_bytes(self.cfg), B.lora_kv_work_bytes(self.cfg)
        if n_bytes == 0:
            raise B.LoraError(B.LORA_E_INVAL, "lora_kv_pages_bytes")
        shape = (n_pages, n_layers, 2, n_kv_heads, page_tokens * head_dim)
        if pages is None:
            pages = torch.empty(shape, dtype=self.dtype, device=self.device)
        if tuple(pages.shape) != shape or pages.dtype != self.dtype or pages.get_device() != self._index or not pages.is_contiguous():
            raise ValueError(f"pages: a contiguous {self.dtype} tensor of shape {shape} on {self.device} is wanted")
        self.pages = pages
        self.work = torch.empty(work + 256, dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self._index):  # the cache belongs to the device that is current now
            rc, self.handle = B.lora_kv_create(self.cfg, pages.data_ptr(), n_bytes, (self.work.data_ptr() + 255) // 256 * 256, work)
        B.check(rc, "lora_kv_create")

    def close(self) -> None:
        if getattr(self, "handle", None) is not None:
            torch.cuda.synchronize(self.device)
            B.lora_kv_destroy(self.handle)
            self.handle = None
            self.pages = self.work = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self, stream) -> int:
        return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(self._index)

    # -- sequences (ids: a number or an array of them) --------------------------------
    def add(self, ids) -> None:
        B.check(B.lora_kv_seq_add(self.handle, ids), "lora_kv_seq_add")

    def fork(self, parent: int, ids, n_tokens: int = -1) -> None:
        B.check(B.lora_kv_seq_fork(self.handle, parent, ids, n_tokens), "lora_kv_seq_fork")

    def extend(self, ids, n_tokens, stream: Optional[torch.cuda.Stream] = None) -> None:
        B.check(B.lora_kv_seq_extend(self.handle, ids, n_tokens, self._stream(stream)), "lora_kv_seq_extend")

    def truncate(self, ids, n_tokens) -> None:
        B.check(B.lora_kv_seq_truncate(self.handle, ids, n_tokens), "lora_kv_seq_truncate")

    def free(self, ids) -> None:
        B.check(B.lora_kv_seq_free(self.handle, ids), "lora_kv_seq_free")

    def length(self, seq: int) -> int:
        rc, info = B.lora_kv_seq_info(self.handle, seq)
        B.check(rc, "lora_kv_seq_info")
        return info.n_tokens

    def pages_of(self, seq: int):
        rc, pages = B.lora_kv_seq_pages(self.handle, seq)
        B.check(rc, "lora_kv_seq_pages")
        return pages

    # -- pages ----------------------------------------------------------------------------
    def compact(self, stream: Optional[torch.cuda.Stream] = None) -> int:
        rc, moved = B.lora_kv_compact(self.handle, self._stream(stream))
        B.check(rc, "lora_kv_compact")
        return moved

    def set_limit(self, limit: int) -> None:
        B.check(B.lora_kv_set_limit(self.handle, limit), "lora_kv_set_limit")

    def stats(self):
        rc, st = B.lora_kv_stats(self.handle)
        B.check(rc, "lora_kv_stats")
        return st

    # -- batches --------------------------------------------------------------------------
    def batch(self, seg_seq, seg_offsets, stream: Optional[torch.cuda.Stream] = None):
        rc, b = B.lora_kv_batch_create(self.handle, seg_seq, seg_offsets, self._stream(stream))
        B.check(rc, "lora_kv_batch_create")
        b.n_tokens = int(seg_offsets[-1])
        return b

    def batch_destroy(self, batch) -> None:
        B.check(B.lora_kv_batch_destroy(self.handle, batch), "lora_kv_batch_destroy")

    def _rows(self, t: torch.Tensor, name: str, batch, heads: int):
        """(address, values between tokens) of [T][heads][head_dim] or [T][heads * head_dim], the heads of a token one after the other"""
        d, n, shape, stride = self.head_dim, batch.n_tokens, t.shape, t.stride()
        flat = len(shape) == 2 and shape[1] == heads * d and stride[1] == 1
        if not (flat or (len(shape) == 3 and shape[1] == heads and shape[2] == d and stride[2] == 1 and (stride[1] == d or heads == 1))):
            raise ValueError(f"{name}: [{n}][{heads}][{d}] with the heads of a token in a row is wanted, got {tuple(shape)}, strides {stride}")
        if shape[0] != n or t.dtype is not self.dtype or t.get_device() != self._index:
            raise ValueError(f"{name}: {n} tokens of {self.dtype} on {self.device} are wanted, got {tuple(shape)} of {t.dtype} on {t.device}")
        return t.data_ptr(), stride[0] if n > 1 else heads * d

    def append(self, batch, layer: int, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               rope: Optional[torch.Tensor] = None, neighbours: bool = False, stream: Optional[torch.cuda.Stream] = None) -> None:
        """rope: [positions][rope_dim] fp32, the cosines of a position and then its sines.  q_out: q itself if not given."""
        rows = self._rows
        kp, ks = rows(k, "k", batch, self.n_kv_heads)
        vp, vs = rows(v, "v", batch, self.n_kv_heads)
        qp = qs = op = os_ = 0
        if q is not None:
            qp, qs = rows(q, "q", batch, self.n_heads)
            op, os_ = (qp, qs) if q_out is None else rows(q_out, "q_out", batch, self.n_heads)
        elif q_out is not None:
            raise ValueError("q_out without q")
        rp = rn = rd = 0
        if rope is not None:
            if rope.dim() != 2 or rope.dtype != torch.float32 or rope.get_device() != self._index or not rope.is_contiguous():
                raise ValueError(f"rope: a contiguous fp32 tensor [positions][rope_dim] on {self.device} is wanted")
            rp, (rn, rd) = rope.data_ptr(), rope.shape
        B.check(B.lora_kv_append(self.handle, batch, layer, kp, vp, ks, vs, qp, op, qs, os_, rp, min(rn, 2**31 - 1), rd,
                                 B.LORA_ROPE_NEIGHBOURS if neighbours else B.LORA_ROPE_HALVES, self._stream(stream)), "lora_kv_append")

    def attend(self, batch, layer: int, q: torch.Tensor, out: torch.Tensor, scale: float, stream: Optional[torch.cuda.Stream] = None) -> None:
        qp, qs = self._rows(q, "q", batch, self.n_heads)
        op, os_ = self._rows(out, "out", batch, self.n_heads)
        B.check(B.lora_kv_attend(self.handle, batch, layer, qp, qs, op, os_, scale, self._stream(stream)), "lora_kv_attend")
