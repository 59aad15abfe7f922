"""AnswerSession: a target model's reads and writes of a repaired, paged cache.

RepairSession.apply_paged writes the repaired document caches into a paged,
layer-major cache.  An AnswerSession then takes a question's tokens and the
answer's tokens through it, layer by layer: ``append`` rotates and places their
K and V (and rotates Q), ``attend`` computes their attention, over each
request's own pages and, for requests in groups, over the prefix (document set)
that a group shares.  Everything computed runs in the library's kernels through
the C ABI; this class owns argument structs and workspaces only.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import numpy as np
import torch

from . import cr


def _stream_of(handle: int, device) -> torch.cuda.Stream:
    """The stream of a raw handle (0: the default one, for which ExternalStream would make another)."""
    return torch.cuda.ExternalStream(handle, device) if handle else torch.cuda.default_stream(device)


class AnswerBatch:
    """The plan of a batch: request r's new tokens are rows cu_q[r] .. cu_q[r + 1], and requests
    cu_group[g] .. cu_group[g + 1] share prefix g.  One plan serves all layers and steps of the
    batch; it holds the workspace of its calls, so it is used on one stream at a time (as with a
    tensor, the caller orders a stream behind the one before).  The workspace returns to the
    allocator when the batch is dropped and the streams that have used it are done; a captured
    graph needs the batch kept."""

    def __init__(self, plan: cr.cr_attention_batch, workspace: torch.Tensor, stream: Optional[int] = None):
        self.plan, self.workspace = plan, workspace
        self.streams = {stream}            # raw handles that the allocator knows of
        self.n_req, self.n_groups, self.n_tokens = plan.n_req, plan.n_groups, plan.n_tokens
        self.n_q_heads = plan.n_q_heads
        self.ref = ctypes.byref(plan)

    def used_on(self, stream: int):
        self.streams.add(stream)
        self.workspace.record_stream(_stream_of(stream, self.workspace.device))


def _refuse(name: str, t: torch.Tensor, device: int, expected: str):
    if t.get_device() != device:        # a kernel would follow its pointer
        raise ValueError(f"{name}: expected on cuda:{device} as the cache, got {t.device}")
    raise ValueError(f"{name}: {expected} expected, got {tuple(t.shape)} {t.dtype} with strides {t.stride()}")


def _rows(name: str, t: torch.Tensor, n: int, width: int, dtype, device: int) -> int:
    """The row stride of t, checked to be n rows of `width` contiguous values on the device."""
    if t.get_device() == device and t.dtype is dtype and t.shape == (n, width):
        ld, one = t.stride()
        if one == 1:
            return ld if n > 1 else width        # (one row's stride may be anything)
    _refuse(name, t, device, f"{n} rows of {width} contiguous values of {dtype}")


def _whole(name: str, t: torch.Tensor, shape, device: int, dtype=torch.int32):
    """Check t to be contiguous and of this shape on the device."""
    if t.get_device() != device or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _refuse(name, t, device, f"contiguous {dtype} of {shape}")


def _table(name: str, t: torch.Tensor, n: int, device: int) -> int:
    """The width of a block table of n rows."""
    if t.dim() != 2:
        raise ValueError(f"{name}: {n} rows of blocks expected, got {tuple(t.shape)}")
    width = t.shape[1]
    _whole(name, t, (n, width), device)
    return width


_BF16, _F32 = torch.bfloat16, torch.float32


class AnswerSession:
    """target: the cache's shape (bf16); n_q_heads: query heads (a multiple of its KV heads);
    paged_cache [2 L, num_slots, H_kv d_h] bf16, as RepairSession.apply_paged writes it, in
    blocks of block_size slots; inv_freq_target: R_M's frequencies (None: a cache of
    canonical K, nothing is rotated); scale: of the scores, above 0 (default 1 / sqrt(d_h))."""

    def __init__(self, target: cr.cr_target_dims, n_q_heads: int, paged_cache: torch.Tensor, *,
                 block_size: int = 16, max_tokens: int, max_requests: int = 256, inv_freq_target=None,
                 scale: Optional[float] = None):
        width = target.n_kv_heads * target.head_dim
        if (target.cache_dtype != cr.CR_BF16 or paged_cache.dtype != torch.bfloat16 or paged_cache.dim() != 3
                or paged_cache.shape[0] != 2 * target.n_layers or paged_cache.shape[2] != width
                or not paged_cache.is_contiguous()):
            raise ValueError(f"paged_cache: contiguous bf16 [{2 * target.n_layers}, num_slots, {width}] expected, "
                             f"got {tuple(paged_cache.shape)} {paged_cache.dtype}")
        self.target, self.n_q_heads, self.paged_cache = target, int(n_q_heads), paged_cache
        self.width, self.q_width = width, self.n_q_heads * target.head_dim
        self.max_tokens, self.max_requests = int(max_tokens), int(max_requests)
        self.scale = float(scale) if scale is not None else 1.0 / math.sqrt(target.head_dim)
        self.device = paged_cache.device
        self._layers = [cr.paged_layer(paged_cache, i, target.n_kv_heads, target.head_dim, block_size)
                        for i in range(target.n_layers)]
        self._refs = [ctypes.byref(x) for x in self._layers]
        self.rope_mode = cr.CR_ROPE_NONE if inv_freq_target is None else cr.CR_ROPE_GLOBAL
        self._freq = None if inv_freq_target is None else np.ascontiguousarray(inv_freq_target, np.float32)
        if self._freq is not None and self._freq.shape != (target.head_dim // 2,):
            raise ValueError(f"inv_freq_target: {target.head_dim // 2} frequencies expected")
        self._freq_ptr = None if self._freq is None else self._freq.ctypes.data
        lib = cr.lib()
        self._append, self._paged, self._prefix = lib.cr_paged_append, lib.cr_paged_attention, lib.cr_prefix_attention
        self._device_index = paged_cache.get_device()       # (-1: not a GPU's)

    def _stream(self, stream):
        """The raw handle of the given stream, or of the device's current one (a decode step has
        little time for building Stream objects); the device has to be the current one, on which
        the library launches."""
        if self._device_index < 0 or torch._C._cuda_getDevice() != self._device_index:
            raise ValueError(f"paged_cache on {self.device}: not the current CUDA device")
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self._device_index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream

    def _empty(self, shape, dtype, stream) -> torch.Tensor:
        """Memory of the given stream (the allocator gives a block on at once to the stream it
        belongs to, and only in that stream's order)."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        if not hasattr(stream, "cuda_stream"):
            stream = _stream_of(stream, self.device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _use(self, batch: AnswerBatch, stream) -> int:
        """The raw handle of the stream, which the batch's workspace is used on."""
        st = self._stream(stream)
        if st not in batch.streams:
            batch.used_on(st)
        return st

    def batch(self, cu_q, cu_group=None, stream=None) -> AnswerBatch:
        """Plan the batch of the given offsets (host) on the stream; the plan owns its workspace,
        which belongs to that stream."""
        cu = np.ascontiguousarray(cu_q, np.int32)
        cg = None if cu_group is None else np.ascontiguousarray(cu_group, np.int32)
        if len(cu) - 1 > self.max_requests or (len(cu) and int(cu[-1]) > self.max_tokens):
            raise ValueError(f"batch of {len(cu) - 1} requests, {int(cu[-1])} tokens: the session holds "
                             f"{self.max_requests} and {self.max_tokens}")
        heads = (self.n_q_heads, self.target.n_kv_heads, self.target.head_dim)
        need = cr.cr_attention_workspace_bytes(*heads, cu, cg)
        if need == 0:
            raise cr.CrError("cr_attention_workspace_bytes", cr.CR_ERR_INVALID_ARG, "invalid batch")
        workspace, st = self._empty((need,), torch.uint8, stream), self._stream(stream)
        return AnswerBatch(cr.cr_attention_plan(*heads, cu, workspace, cg, st), workspace, st)

    def append(self, layer: int, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, pos: torch.Tensor,
               slot_mapping: torch.Tensor, q_out: Optional[torch.Tensor] = None, stream=None):
        """Rotate and place K and V [n, H_kv d_h] (bf16 or fp32) at slot_mapping (int64, < 0 = skip);
        with q, write its rotation to q_out (allocated, on the stream, when None) and return that."""
        n, dtype = k.shape[0], k.dtype
        if dtype is not _BF16 and dtype is not _F32:
            raise ValueError(f"k: bf16 or fp32 expected, got {dtype}")
        dev = self._device_index
        ldk, ldv = _rows("k", k, n, self.width, dtype, dev), _rows("v", v, n, self.width, dtype, dev)
        _whole("pos", pos, (n,), dev)
        _whole("slot_mapping", slot_mapping, (n,), dev, torch.int64)
        if q is None:
            qp = op = None
            ldq = ldo = heads = 0
        else:
            ldq, heads, qp = _rows("q", q, n, self.q_width, dtype, dev), self.n_q_heads, q.data_ptr()
            if q_out is None:
                q_out = self._empty((n, self.q_width), _BF16, stream)
            ldo, op = _rows("q_out", q_out, n, self.q_width, _BF16, dev), q_out.data_ptr()
        st = self._append(self._refs[layer], k.data_ptr(), ldk, v.data_ptr(), ldv, qp, ldq, heads,
                          cr.CR_F32 if dtype is _F32 else cr.CR_BF16, n, pos.data_ptr(), self._freq_ptr,
                          self.rope_mode, slot_mapping.data_ptr(), op, ldo, self._stream(stream))
        if st:
            cr._check("cr_paged_append", st)
        return q_out

    def attend(self, layer: int, batch: AnswerBatch, q: torch.Tensor, block_table: torch.Tensor,
               kv_len: torch.Tensor, out: Optional[torch.Tensor] = None, *,
               prefix_table: Optional[torch.Tensor] = None, prefix_len: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of the batch's rows q (rotated, as append returns them) over their requests'
        tokens (block_table [n_req, max_blocks] int32, kv_len [n_req] int32, the new tokens
        included) and, for a batch with groups, over their group's prefix (prefix_table
        [n_groups, max_prefix_blocks], prefix_len [n_groups]).  Returns out (allocated, on the
        stream, when None)."""
        n = batch.n_tokens
        if batch.n_q_heads != self.n_q_heads:
            raise ValueError(f"batch: planned for {batch.n_q_heads} query heads, the session has {self.n_q_heads}")
        dev = self._device_index
        ldq = _rows("q", q, n, self.q_width, _BF16, dev)
        if out is None:
            out = self._empty((n, self.q_width), _BF16, stream)
        ldo = _rows("out", out, n, self.q_width, _BF16, dev)
        blocks = _table("block_table", block_table, batch.n_req, dev)
        _whole("kv_len", kv_len, (batch.n_req,), dev)
        if lse is None:
            lse_ptr = None
        else:
            _whole("lse", lse, (n, self.n_q_heads), dev, _F32)
            lse_ptr = lse.data_ptr()
        if batch.n_groups == 0:
            if prefix_table is not None or prefix_len is not None:
                raise ValueError("a prefix needs a batch with groups")
            st = self._paged(self._refs[layer], batch.ref, q.data_ptr(), ldq, block_table.data_ptr(), blocks,
                             kv_len.data_ptr(), self.scale, out.data_ptr(), ldo, lse_ptr, self._use(batch, stream))
            if st:
                cr._check("cr_paged_attention", st)
            return out
        if prefix_table is None or prefix_len is None:
            raise ValueError("a batch with groups needs prefix_table and prefix_len")
        prefix_blocks = _table("prefix_table", prefix_table, batch.n_groups, dev)
        _whole("prefix_len", prefix_len, (batch.n_groups,), dev)
        st = self._prefix(self._refs[layer], batch.ref, q.data_ptr(), ldq, block_table.data_ptr(), blocks,
                          kv_len.data_ptr(), prefix_table.data_ptr(), prefix_blocks, prefix_len.data_ptr(),
                          self.scale, out.data_ptr(), ldo, lse_ptr, self._use(batch, stream))
        if st:
            cr._check("cr_prefix_attention", st)
        return out
