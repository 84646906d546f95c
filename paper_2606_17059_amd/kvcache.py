"""Python binding of the pr_kv calls: a node's paged KV cache in torch tensors.

Method names follow the C ABI in include/prefix_router.h, which states what each
call does and skips.  As in router.py, every step runs in the library's HIP
kernels; this module checks shapes, dtypes and devices, passes raw pointers and
the current HIP stream, and allocates outputs and workspaces from torch's
allocator (so calls may be captured into a graph, each with scratch of its own).
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

from .router import PR_OK, KvDescription, _check, _dev, _load_torch, _stream_ptr, lib

PR_KV_BF16, PR_KV_F16, PR_KV_E4M3 = 0, 1, 2
PR_KV_WORK_EXTEND, PR_KV_WORK_ATTEND, PR_KV_WORK_COMPACT, PR_KV_WORK_CHANGE = 0, 1, 2, 3


class KVCache:
    """A paged KV cache: keys and values, and who holds which page.

    k        [layers, pages, kv_heads, head_dim / 8, page_tokens, 8]
    v        [layers, pages, kv_heads, page_tokens / 4, head_dim, 4]
             bfloat16, float16 or float8_e4m3fn (value = stored * scale); the
             first two dimensions may have any strides without overlap
    table    int32 [slots, pages a slot]: a sequence's pages, -1 past its last
    lengths  int32 [slots]: a sequence's tokens
    refs     int32 [pages]: sequences that hold the page
    free     int64 [ceil(pages / 64)]: bit p % 64 of word p / 64 set where refs[p] is 0
    skipped  int64 [1]: batch entries that calls left out since the last check

    The tensors are the caller's and stay as they are; `create` makes an empty
    cache.  Calls run on the current stream of the cache's device, or on `stream`.
    They have no derivatives: floating-point tensors that require gradients (but
    under torch.no_grad()) or carry a forward-mode tangent are refused.
    """

    def __init__(self, k, v, table, lengths, refs, free, k_scale: float = 1.0, v_scale: float = 1.0, skipped=None):
        torch = _load_torch()
        codes = {torch.bfloat16: PR_KV_BF16, torch.float16: PR_KV_F16, torch.float8_e4m3fn: PR_KV_E4M3}
        for name, t in (("k", k), ("v", v)):
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
            if t.dtype not in codes or t.dtype != k.dtype:
                raise TypeError("k and v must both be bfloat16, float16 or float8_e4m3fn")
            if t.dim() != 6 or t.numel() == 0 or not t[0, 0].is_contiguous():
                raise ValueError(f"{name} must have 6 dimensions, none empty, the last four contiguous")
            if t.requires_grad:
                raise ValueError(f"{name} must not require gradients: the calls have none")
        layers, pages, heads, eights, tokens, eight = k.shape
        dim = 8 * eights
        if eight != 8 or tuple(v.shape) != (layers, pages, heads, tokens // 4, dim, 4) or tokens % 4:
            raise ValueError("k must be [layers, pages, kv_heads, head_dim / 8, page_tokens, 8] and v [layers, pages, "
                             "kv_heads, page_tokens / 4, head_dim, 4]")
        if skipped is None:
            skipped = torch.zeros(1, dtype=torch.int64, device=k.device)
        for name, t, dtype in (("table", table, torch.int32), ("lengths", lengths, torch.int32),
                               ("refs", refs, torch.int32), ("free", free, torch.int64),
                               ("skipped", skipped, torch.int64)):
            _dev(t, dtype, name)
        if table.dim() != 2 or tuple(lengths.shape) != (table.shape[0],):
            raise ValueError("table must be [slots, pages a slot] and lengths [slots]")
        if tuple(refs.shape) != (pages,) or tuple(free.shape) != ((pages + 63) // 64,) or skipped.numel() != 1:
            raise ValueError("refs must hold [pages], free ceil(pages / 64) words and skipped one")
        self.device = k.device
        if any(t.device != k.device for t in (v, table, lengths, refs, free, skipped)):
            raise ValueError("all tensors of a cache must be on one device")
        self.k, self.v, self.table, self.lengths, self.refs, self.free = k, v, table, lengths, refs, free
        self.skipped, self.dtype = skipped, k.dtype
        self.layers, self.pages, self.kv_heads, self.page_tokens, self.head_dim = layers, pages, heads, tokens, dim
        self.k_scale, self.v_scale = float(k_scale), float(v_scale)
        # the stride of a dimension of one is never used, and may be anything
        strides = [t.stride(d) if t.shape[d] > 1 else 0 for t in (k, v) for d in (0, 1)]
        self._desc = KvDescription(
            k.device.index, codes[k.dtype], layers, heads, dim, tokens, pages, table.shape[0], table.shape[1],
            self.k_scale, self.v_scale, k.data_ptr() or None, v.data_ptr() or None, *strides, table.data_ptr() or None, lengths.data_ptr() or None, refs.data_ptr() or None,
            free.data_ptr() or None, skipped.data_ptr())
        self._ref = ctypes.byref(self._desc)
        self._torch, self._index, self._int32, self._int64 = torch, k.device.index, torch.int32, torch.int64
        self._forward_ad = torch.autograd.forward_ad
        # types that rows of new tokens and queries may have
        self._io = {torch.bfloat16: PR_KV_BF16, torch.float16: PR_KV_F16} if k.dtype.itemsize == 1 else \
            {k.dtype: codes[k.dtype]}
        self._scale = 1.0 / math.sqrt(dim)
        self._bytes = {}
        self._lib = lib()
        self._work_bytes(PR_KV_WORK_COMPACT, 0, 0)  # refuses what is no cache

    @classmethod
    def create(cls, layers: int, kv_heads: int, head_dim: int, page_tokens: int, num_pages: int, num_slots: int,
               slot_pages: int, dtype=None, device=None, k_scale: float = 1.0, v_scale: float = 1.0) -> "KVCache":
        """An empty cache (bfloat16 unless dtype says otherwise) on `device`."""
        torch = _load_torch()
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        dtype = torch.bfloat16 if dtype is None else dtype
        if head_dim % 8 or page_tokens % 4 or min(layers, kv_heads, head_dim, page_tokens, num_pages, num_slots,
                                                  slot_pages) < 1:
            raise ValueError("sizes must be positive, head_dim a multiple of 8 and page_tokens of 4")
        k = torch.empty((layers, num_pages, kv_heads, head_dim // 8, page_tokens, 8), dtype=dtype, device=dev)
        v = torch.empty((layers, num_pages, kv_heads, page_tokens // 4, head_dim, 4), dtype=dtype, device=dev)
        ints = [torch.empty(s, dtype=t, device=dev)
                for s, t in (((num_slots, slot_pages), torch.int32), ((num_slots,), torch.int32),
                             ((num_pages,), torch.int32), (((num_pages + 63) // 64,), torch.int64))]
        c = cls(k, v, *ints, k_scale=k_scale, v_scale=v_scale)
        c.init()
        return c

    # ---- helpers ----------------------------------------------------------------
    def _work_bytes(self, call: int, n: int, m: int) -> int:
        key = (call, n, m)
        b = self._bytes.get(key)
        if b is None:
            out = ctypes.c_int64(0)
            _check(self._lib.pr_kv_workspace(self._ref, call, n, m, ctypes.byref(out)))
            if len(self._bytes) >= 256:
                self._bytes.clear()
            b = self._bytes[key] = out.value
        return b

    def _empty(self, like, shape, stream):
        """A tensor of `like`'s type, of the allocator's pool for the call's stream."""
        if stream is None:
            return like.new_empty(shape)
        with self._torch.cuda.stream(stream):
            return like.new_empty(shape)

    def _work(self, call: int, n: int, m: int, stream):
        """(a workspace or None, its address, its size)."""
        size = self._work_bytes(call, n, m)
        if not size:
            return None, None, 0
        work = self._empty(self.lengths, (size + 3) // 4, stream)
        return work, work.data_ptr(), size

    def _st(self, stream) -> int:
        if stream is not None and stream.device != self.device:
            raise ValueError("stream must be of the cache's device")
        return _stream_ptr(stream, self.device)

    def _ints(self, t, dtype, name, count=None) -> int:
        """Checks a vector of integers; its length."""
        _dev(t, dtype, name)
        if t.get_device() != self._index:
            raise ValueError(f"{name} must be on the cache's device")
        shape = t.shape
        if len(shape) != 1 or (count is not None and shape[0] != count):
            raise ValueError(f"{name} must have one dimension" + (f" of {count}" if count is not None else ""))
        return shape[0]

    def _rows(self, t, name, count, heads):
        """Checks rows of heads x head_dim numbers, contiguous but for a row stride: (heads, row stride, type)."""
        try:
            index = t.get_device()
            shape, stride, io = t.shape, t.stride(), self._io.get(t.dtype, -1)
        except (AttributeError, RuntimeError):
            index = -1
        if index < 0:
            raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
        if index != self._index:
            raise ValueError(f"{name} must be on the cache's device")
        if len(shape) != 3 or shape[0] != count or shape[2] != self.head_dim or (heads and shape[1] != heads):
            raise ValueError(f"{name} must be [{count}, {heads or 'heads'}, {self.head_dim}]")
        if count and (stride[2] != 1 or (stride[1] != self.head_dim and shape[1] > 1)):
            raise ValueError(f"rows of {name} must be contiguous")
        if io < 0:
            raise TypeError(f"{name} must be of the cache's type, or bfloat16 or float16 for a float8 cache")
        if t.requires_grad or self._forward_ad._current_level >= 0:  # no tensor has a tangent outside a level
            self._no_derivative(t, name)
        return shape[1], stride[0], io

    def _no_derivative(self, t, name) -> None:
        if t.requires_grad and self._torch.is_grad_enabled():
            raise ValueError(f"{name} requires gradients, which this call does not give: detach it, or call under "
                             "torch.no_grad()")
        if self._forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError(f"{name} carries a tangent, which this call does not follow")

    # ---- calls --------------------------------------------------------------------
    def init(self, stream=None) -> None:
        """Empty the cache (pr_kv_init)."""
        _check(self._lib.pr_kv_init(self._ref, self._st(stream)))

    def extend(self, slots, offsets, rows: int, place=None, stream=None):
        """Room for offsets[i + 1] - offsets[i] new tokens of each slots[i]: returns place, int32 [rows]
        (pr_kv_extend).  offsets is a device tensor, so `rows`, its last entry, is given beside it."""
        n = self._ints(slots, self._int32, "slots")
        self._ints(offsets, self._int64, "offsets", n + 1)
        if rows < 0:
            raise ValueError("rows must not be negative")
        st = self._st(stream)
        if place is None:
            place = self._empty(slots, rows, stream)
        else:
            self._ints(place, self._int32, "place", rows)
        work, at, size = self._work(PR_KV_WORK_EXTEND, n, rows, stream)
        s = self._lib.pr_kv_extend(self._ref, slots.data_ptr() or None, offsets.data_ptr(), n, rows,
                                   place.data_ptr() or None, at, size, st)
        if s != PR_OK:
            _check(s)
        return place

    def write(self, layer: int, place, k, v, stream=None) -> None:
        """Rows [rows, kv_heads, head_dim] of new tokens into their places in one layer (pr_kv_write)."""
        rows = self._ints(place, self._int32, "place")
        _, k_stride, io = self._rows(k, "k", rows, self.kv_heads)
        _, v_stride, v_io = self._rows(v, "v", rows, self.kv_heads)
        if io != v_io:
            raise TypeError("k and v must have one dtype")
        layer = layer if 0 <= layer < self.layers else -1  # ctypes would cut it to 32 bits
        s = self._lib.pr_kv_write(self._ref, layer, place.data_ptr() or None, k.data_ptr() or None, k_stride,
                                  v.data_ptr() or None, v_stride, rows, io, self._st(stream))
        if s != PR_OK:
            _check(s)

    def attend(self, layer: int, slots, q, scale: Optional[float] = None, window: int = 0, out=None, lse=None,
               stream=None):
        """Attention of one new token a sequence, q [n, heads, head_dim], over its cached tokens in one layer, or
        the last `window` of them (pr_kv_attend).  scale: 1 / sqrt(head_dim) unless given.  lse: a float32
        tensor [n, heads] that gets the logarithm of the sum of exponentials."""
        n = self._ints(slots, self._int32, "slots")
        heads, stride, io = self._rows(q, "q", n, 0)
        st = self._st(stream)
        if out is None:
            dense = stream is None and stride == heads * self.head_dim
            out = self._torch.empty_like(q) if dense else self._empty(q, q.shape, stream)
        elif out.dtype != q.dtype or tuple(out.shape) != tuple(q.shape) or not out.is_contiguous():
            raise ValueError("out must be a contiguous tensor of q's dtype and shape")
        elif out.device != self.device:
            raise ValueError("out must be on the cache's device")
        else:
            self._no_derivative(out, "out")
        if lse is not None:
            _dev(lse, self._torch.float32, "lse")
            if tuple(lse.shape) != (n, heads) or lse.device != self.device:
                raise ValueError("lse must be [n, heads] on the cache's device")
            self._no_derivative(lse, "lse")
        work, at, size = self._work(PR_KV_WORK_ATTEND, n, heads, stream)
        layer, window = layer if 0 <= layer < self.layers else -1, min(max(window, -1), 0x7fffffff)
        s = self._lib.pr_kv_attend(self._ref, layer, slots.data_ptr() or None, n, q.data_ptr() or None, stride,
                                   heads, io, self._scale if scale is None else scale, window,
                                   out.data_ptr() or None, lse.data_ptr() or None if lse is not None else None,
                                   at, size, st)
        if s != PR_OK:
            _check(s)
        return out

    def fork(self, src, dst, tokens, stream=None) -> None:
        """Empty slots dst[i] become the first tokens[i] tokens of src[i], sharing their pages (pr_kv_fork)."""
        n = self._ints(src, self._int32, "src")
        self._ints(dst, self._int32, "dst", n)
        self._ints(tokens, self._int32, "tokens", n)
        st = self._st(stream)
        work, at, size = self._work(PR_KV_WORK_CHANGE, n, 0, stream)
        s = self._lib.pr_kv_fork(self._ref, src.data_ptr() or None, dst.data_ptr() or None,
                                 tokens.data_ptr() or None, n, at, size, st)
        if s != PR_OK:
            _check(s)

    def trim(self, slots, keep=None, stream=None) -> None:
        """Each slots[i] keeps its first keep[i] tokens, none without `keep` (pr_kv_trim).  keep may be a column of
        a route's match_len: a strided int32 vector."""
        torch = self._torch
        n = self._ints(slots, self._int32, "slots")
        stride = 1
        if keep is not None:
            if not isinstance(keep, torch.Tensor) or not keep.is_cuda or keep.dtype != torch.int32:
                raise TypeError("keep must be a CUDA (HIP) int32 torch tensor")
            if keep.device != self.device or tuple(keep.shape) != (n,):
                raise ValueError(f"keep must be [{n}] on the cache's device")
            stride = keep.stride(0)
        st = self._st(stream)
        work, at, size = self._work(PR_KV_WORK_CHANGE, n, 0, stream)
        s = self._lib.pr_kv_trim(self._ref, slots.data_ptr() or None,
                                 (keep.data_ptr() or None) if keep is not None else None, stride, n, at, size, st)
        if s != PR_OK:
            _check(s)

    def compact(self, stream=None):
        """Move the held pages to the lowest ids; returns int32 [2] on the device: pages moved, pages held
        (pr_kv_compact)."""
        st = self._st(stream)
        moved = self._empty(self.lengths, 2, stream)
        work, at, size = self._work(PR_KV_WORK_COMPACT, 0, 0, stream)
        s = self._lib.pr_kv_compact(self._ref, moved.data_ptr(), at, size, st)
        if s != PR_OK:
            _check(s)
        return moved

    def check(self, stream=None) -> None:
        """Wait for the stream; raise RouterError if calls skipped batch entries since the last check
        (pr_kv_check)."""
        _check(self._lib.pr_kv_check(self._ref, self._st(stream)))
