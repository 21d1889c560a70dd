"""PyTorch plumbing around the paged key-value cache (include/lora_kv.h): device memory for its pages, stream handles,
shapes and strides of the tensors it is given.  No arithmetic of the method happens here."""
from __future__ import annotations

from typing import Optional, Union

import numpy as np
import torch

from . import binding as B


def _dtype(dtype: int) -> torch.dtype:
    return torch.bfloat16 if dtype == B.LORA_BF16 else torch.float32


class KvCache:
    """Owns the cache handle and, unless the caller brings them, the pages' memory: a tensor
    [n_pages][n_layers][2][n_kv_heads][page_tokens * head_dim] (see the header for what lies where in it).

    e4m3: keys and values are held in 8 bits, with an exponent for each token and head.  The pages are bytes then, a tensor
    [n_pages][n_layers][2 * n_kv_heads * page_tokens * (head_dim + 1)]; queries, keys, values and outputs of the calls are bf16 as before.

    max_batch_pages: pages that the sequences of a batch may have together, one that they share counted for each; a batch with more is refused.  By default
    whatever max_batch_seqs sequences can have, up to 4 million or 4 times the pages there are."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, page_tokens: int = 64, max_seqs: int = 512,
                 max_batch_tokens: int = 4096, max_batch_seqs: int = 512, max_batch_pages: int = 0, n_batches: int = 2,
                 dtype: int = B.LORA_BF16, device: str = "cuda:0", pages: Optional[torch.Tensor] = None,
                 e4m3: bool = False):
        if not torch.cuda.is_available():
            raise RuntimeError("KvCache needs a GPU: the library has no CPU path")
        index = torch.device(device).index
        self._index = index if index is not None else torch.cuda.current_device()
        self.device = torch.device("cuda", self._index)
        self.n_heads, self.n_kv_heads, self.head_dim, self.dtype = n_heads, n_kv_heads, head_dim, _dtype(dtype)
        # Forks share pages: the sequences of a batch may name more pages than there are.  Every sequence may name all of them, up to a list of 16 MB for each batch
        max_batch_pages = max_batch_pages or min(max_batch_seqs * n_pages, max(4 * n_pages, 1 << 22))
        self.cfg = B.make_kv_config(n_layers, n_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs, max_batch_seqs, max_batch_tokens,
                                    max_batch_pages, n_batches, dtype, B.LORA_KV_PAGES_E4M3 if e4m3 else 0)
        n_bytes, work = B.lora_kv_pages_bytes(self.cfg), B.lora_kv_work_bytes(self.cfg)
        if n_bytes == 0:
            raise B.LoraError(B.LORA_E_INVAL, "lora_kv_pages_bytes")
        if e4m3:
            shape, held = (n_pages, n_layers, 2 * n_kv_heads * page_tokens * (head_dim + 1)), torch.uint8
        else:
            shape, held = (n_pages, n_layers, 2, n_kv_heads, page_tokens * head_dim), self.dtype
        if pages is None:
            pages = torch.empty(shape, dtype=held, device=self.device)
        if tuple(pages.shape) != shape or pages.dtype != held or pages.get_device() != self._index or not pages.is_contiguous():
            raise ValueError(f"pages: a contiguous {held} tensor of shape {shape} on {self.device} is wanted")
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

    def read(self, ids, layer: int, k: torch.Tensor, v: torch.Tensor, first=None, n_tokens=None, stream: Optional[torch.cuda.Stream] = None) -> None:
        """Keys and values of tokens [first[i], first[i] + n_tokens[i]) of each sequence -- from the first one on, up to the last, if not given -- out of the pages: k and v
        [tokens of all of them][n_kv_heads][head_dim], one sequence's behind the other's."""
        n = k.shape[0]
        kp, ks = self._rows(k, "k", n, self.n_kv_heads)
        vp, vs = self._rows(v, "v", n, self.n_kv_heads)
        B.check(B.lora_kv_seq_read(self.handle, ids, first, n_tokens, layer, kp, ks, vp, vs, n, self._stream(stream)), "lora_kv_seq_read")

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
    def batch(self, seg_seq, seg_offsets, stream: Optional[torch.cuda.Stream] = None, shared: Union[bool, int] = False):
        """shared: attention reads pages that sequences of the batch share once for all of them, where that is worth it (True, 0), or from so many shared tokens on (a number)."""
        if not shared and isinstance(shared, (bool, np.bool_)):
            rc, b = B.lora_kv_batch_create(self.handle, seg_seq, seg_offsets, self._stream(stream))
            B.check(rc, "lora_kv_batch_create")
        else:
            rc, b = B.lora_kv_batch_create_shared(self.handle, seg_seq, seg_offsets, 0 if isinstance(shared, (bool, np.bool_)) else max(-1, min(int(shared), 2**31 - 1)), self._stream(stream))
            B.check(rc, "lora_kv_batch_create_shared")
        b.n_tokens = int(seg_offsets[-1])
        return b

    def batch_destroy(self, batch) -> None:
        B.check(B.lora_kv_batch_destroy(self.handle, batch), "lora_kv_batch_destroy")

    def _rows(self, t: torch.Tensor, name: str, n: int, heads: int):
        """(address, values between tokens) of [n][heads][head_dim] or [n][heads * head_dim], the heads of a token one after the other"""
        d, shape, stride = self.head_dim, t.shape, t.stride()
        if len(shape) == 3:
            fits = shape[1] == heads and shape[2] == d and stride[2] == 1 and (stride[1] == d or heads == 1)
        else:
            fits = len(shape) == 2 and shape[1] == heads * d and stride[1] == 1
        if not fits:
            raise ValueError(f"{name}: [{n}][{heads}][{d}] with the heads of a token in a row is wanted, got {tuple(shape)}, strides {stride}")
        if shape[0] != n or t.dtype is not self.dtype or t.get_device() != self._index:
            raise ValueError(f"{name}: {n} tokens of {self.dtype} on {self.device} are wanted, got {tuple(shape)} of {t.dtype} on {t.device}")
        return t.data_ptr(), stride[0] if n > 1 else heads * d

    def append(self, batch, layer: int, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               rope: Optional[torch.Tensor] = None, neighbours: bool = False, stream: Optional[torch.cuda.Stream] = None,
               q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6) -> None:
        """rope: [positions][rope_dim] fp32, the cosines of a position and then its sines.  q_out: q itself if not given.  q_norm, k_norm: the weights, fp32, of norms
        of every head of the queries and keys before they turn: [head_dim], or [heads][head_dim] with weights of each head's own."""
        rows, n, heads, kv_heads = self._rows, batch.n_tokens, self.n_heads, self.n_kv_heads
        kp, ks = rows(k, "k", n, kv_heads)
        vp, vs = rows(v, "v", n, kv_heads)
        qp = qs = op = os_ = 0
        if q is not None:
            qp, qs = rows(q, "q", n, heads)
            op, os_ = (qp, qs) if q_out is None else rows(q_out, "q_out", n, heads)
        elif q_out is not None:
            raise ValueError("q_out without q")
        rp = rn = rd = 0
        if rope is not None:
            if rope.dim() != 2 or rope.dtype != torch.float32 or rope.get_device() != self._index or not rope.is_contiguous():
                raise ValueError(f"rope: a contiguous fp32 tensor [positions][rope_dim] on {self.device} is wanted")
            rp, (rn, rd) = rope.data_ptr(), rope.shape
            rn = min(rn, 2**31 - 1)
        pairs = B.LORA_ROPE_NEIGHBOURS if neighbours else B.LORA_ROPE_HALVES
        if q_norm is None and k_norm is None:
            B.check(B.lora_kv_append(self.handle, batch, layer, kp, vp, ks, vs, qp, op, qs, os_, rp, rn, rd, pairs, self._stream(stream)), "lora_kv_append")
            return
        if q_norm is not None and q is None:
            raise ValueError("q_norm without q")
        qw, qws = self._weights(q_norm, "q_norm", heads)
        kw, kws = self._weights(k_norm, "k_norm", kv_heads)
        B.check(B.lora_kv_append_norm(self.handle, batch, layer, kp, vp, ks, vs, qp, op, qs, os_, rp, rn, rd, pairs, qw, kw, qws, kws, eps, self._stream(stream)), "lora_kv_append_norm")

    def _weights(self, w: Optional[torch.Tensor], name: str, heads: int):
        """(address, values between heads) of a norm's weights [head_dim] or [heads][head_dim]"""
        if w is None:
            return 0, 0
        shape, stride = w.shape, w.stride()
        if w.dtype is torch.float32 and w.get_device() == self._index and shape[-1:] == (self.head_dim,) and stride[-1] == 1:
            if len(shape) == 1:
                return w.data_ptr(), 0
            if len(shape) == 2 and shape[0] == heads:
                return w.data_ptr(), stride[0] if heads > 1 else 0
        raise ValueError(f"{name}: fp32 weights [{self.head_dim}] or [{heads}][{self.head_dim}] on {self.device} are wanted, got {tuple(shape)} of {w.dtype} on {w.device}")

    def attend(self, batch, layer: int, q: torch.Tensor, out: torch.Tensor, scale: float, stream: Optional[torch.cuda.Stream] = None) -> None:
        qp, qs = self._rows(q, "q", batch.n_tokens, self.n_heads)
        op, os_ = self._rows(out, "out", batch.n_tokens, self.n_heads)
        B.check(B.lora_kv_attend(self.handle, batch, layer, qp, qs, op, os_, scale, self._stream(stream)), "lora_kv_attend")
