"""Device-side plumbing for one mixed iteration: torch tensors for memory and streams,
every computation through the C ABI (binding.py).  No oracle, no fallback.

The hot path of one iteration (Cronus section 4.2 and 4.4) is, in order:
  1. ingest_prefix  - cronus_kv_append of the transferred prefix KV of the continuation
                      chunks (start_pos = 0)
  2. append_new     - cronus_kv_append of this iteration's K/V rows (start_pos = prefix); place_rows does
                      1 and 2 in one launch (cronus_kv_append_pair)
  3. attention      - cronus_attn_mixed over chunks and decodes; a step is one call for all three
                      (cronus_iteration)
DraftLoop holds the state of a loop whose lengths live on the device (drafted tokens verified as a tree).
The contexts of the decode requests were cached by earlier iterations; here they are
placed by setup_decode_context(), which is set-up, not part of the iteration.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B
from .workloads import Batch


def bf16_tensor_from_bits(bits: np.ndarray, device) -> torch.Tensor:
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)


def bits_from_bf16_tensor(t: torch.Tensor) -> np.ndarray:
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class DeviceIteration:
    """Device buffers of one batch and the three calls of the hot path."""

    def __init__(self, batch: Batch, device="cuda:0", pool_fill: int | None = None):
        self.batch = batch
        self.device = torch.device(device)
        sh = batch.shape
        self.fp8 = sh.kv_dtype == "fp8"
        self.elems_per_block = sh.n_kv_heads * 16 * sh.head_dim
        pool_dtype = torch.uint8 if self.fp8 else torch.int16
        n = batch.num_blocks * self.elems_per_block
        if pool_fill is None:
            self.k_pool = torch.empty(n, dtype=pool_dtype, device=self.device)
            self.v_pool = torch.empty(n, dtype=pool_dtype, device=self.device)
        else:
            self.k_pool = torch.full((n,), pool_fill, dtype=pool_dtype, device=self.device)
            self.v_pool = torch.full((n,), pool_fill, dtype=pool_dtype, device=self.device)
        self.block_tables = torch.from_numpy(np.ascontiguousarray(batch.block_tables)).to(self.device)
        self.k_scale = self.v_scale = None
        self.q = self.out = None
        self.prefix_k = self.prefix_v = self.new_k = self.new_v = None
        P, C = batch.prefix_lens.astype(np.int64), batch.chunk_lens.astype(np.int64)
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(self.device)
        is_dec = C == 1
        self.cu_prefix = i32(np.concatenate([[0], np.cumsum(np.where(is_dec, 0, P))]))  # chunk sequences only
        self.cu_ctx = i32(np.concatenate([[0], np.cumsum(np.where(is_dec, P, 0))]))     # decode sequences only
        self.n_ctx_tokens = int(P[is_dec].sum())
        self.ctx_k = self.ctx_v = None
        self.cu_new = i32(np.concatenate([[0], np.cumsum(C)]))
        self.zero_pos = i32(np.zeros(batch.n_seqs))
        self.prefix_pos = i32(P)
        self.n_prefix_tokens = int(P[~is_dec].sum())
        self.n_new_tokens = int(C.sum())
        self.sm_scale = 1.0 / float(np.sqrt(sh.head_dim))
        self._cache = None
        self.workspace = None
        self.workspace_bytes = 0

    # ---- inputs
    def load_host_inputs(self, kv=None):
        """Tensors drawn on the host by the seeded generators (bit-identical to what the
        oracle side sees).  Returns the per-sequence (k_bits, v_bits) for the caller, who
        may also pass them in (drawn already, e.g. by several threads)."""
        b = self.batch
        if kv is None:
            kv = [b.gen_kv(s) for s in range(b.n_seqs)]
        P = b.prefix_lens
        sh = b.shape
        empty = np.zeros((0, sh.n_kv_heads, sh.head_dim), dtype=np.uint16)
        cat = lambda xs: np.concatenate(xs) if xs else empty
        dec = b.chunk_lens == 1
        self.prefix_k = bf16_tensor_from_bits(cat([k[:P[s]] for s, (k, v) in enumerate(kv) if not dec[s]]), self.device)
        self.prefix_v = bf16_tensor_from_bits(cat([v[:P[s]] for s, (k, v) in enumerate(kv) if not dec[s]]), self.device)
        self.ctx_k = bf16_tensor_from_bits(cat([k[:P[s]] for s, (k, v) in enumerate(kv) if dec[s]]), self.device)
        self.ctx_v = bf16_tensor_from_bits(cat([v[:P[s]] for s, (k, v) in enumerate(kv) if dec[s]]), self.device)
        self.new_k = bf16_tensor_from_bits(cat([k[P[s]:] for s, (k, v) in enumerate(kv)]), self.device)
        self.new_v = bf16_tensor_from_bits(cat([v[P[s]:] for s, (k, v) in enumerate(kv)]), self.device)
        self.q = bf16_tensor_from_bits(b.gen_q(), self.device)
        self.out = torch.zeros_like(self.q)
        return kv

    def load_device_inputs(self, seed=0):
        """Same distribution drawn on the device (benchmarks of the full-size batches)."""
        sh = self.batch.shape
        g = torch.Generator(device=self.device)
        g.manual_seed(int(self.batch.seed) * 7919 + seed)
        mk = lambda n: (torch.randn((n, sh.n_kv_heads, sh.head_dim), generator=g, device=self.device,
                                    dtype=torch.float32) * 0.125).to(torch.bfloat16)
        self.prefix_k, self.prefix_v = mk(self.n_prefix_tokens), mk(self.n_prefix_tokens)
        self.ctx_k, self.ctx_v = mk(self.n_ctx_tokens), mk(self.n_ctx_tokens)
        self.new_k, self.new_v = mk(self.n_new_tokens), mk(self.n_new_tokens)
        self.q = (torch.randn((self.n_new_tokens, sh.n_q_heads, sh.head_dim), generator=g, device=self.device,
                              dtype=torch.float32) * 0.125).to(torch.bfloat16)
        self.out = torch.zeros_like(self.q)

    def set_fp8_scales(self, k_scale: np.ndarray, v_scale: np.ndarray):
        self.k_scale = torch.from_numpy(np.ascontiguousarray(k_scale, dtype=np.float32)).to(self.device)
        self.v_scale = torch.from_numpy(np.ascontiguousarray(v_scale, dtype=np.float32)).to(self.device)
        self._cache = None

    def amax_scales(self):
        """Per-KV-head scale = amax / 448 in fp32 over the tensors about to be cached."""
        def amax(a, b, c):
            x = torch.cat([t.abs().amax(dim=(0, 2))[None] for t in (a, b, c) if t.shape[0]]).amax(dim=0)
            return (x.to(torch.float32) / 448.0).cpu().numpy().astype(np.float32)
        return amax(self.prefix_k, self.new_k, self.ctx_k), amax(self.prefix_v, self.new_v, self.ctx_v)

    # ---- the C ABI calls
    @property
    def cache(self) -> B.cronus_kv_cache:
        if self._cache is None:
            sh = self.batch.shape
            self._cache = B.make_cache(self.k_pool, self.v_pool, self.batch.num_blocks, sh.n_q_heads, sh.n_kv_heads,
                                       sh.head_dim, B.CRONUS_KV_FP8_E4M3 if self.fp8 else B.CRONUS_KV_BF16,
                                       self.k_scale, self.v_scale)
        return self._cache

    def _stream(self):
        # what torch.cuda.current_stream(device).cuda_stream gives, without the Stream object around it (1.9 us): a step looks it up
        # before its first launch
        index = self.device.index
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if index is None else index)

    def setup_decode_context(self):
        """Set-up: the KV that earlier iterations of the decode requests left in the cache."""
        b = self.batch
        return B.cronus_kv_append(self.cache, self.ctx_k, self.ctx_v, self.cu_ctx, self.zero_pos,
                                  self.block_tables, b.max_blocks, b.n_seqs, self.n_ctx_tokens, self._stream())

    def ingest_prefix(self):
        """Hot path: the transferred prefix of every continuation chunk."""
        b = self.batch
        return B.cronus_kv_append(self.cache, self.prefix_k, self.prefix_v, self.cu_prefix, self.zero_pos,
                                  self.block_tables, b.max_blocks, b.n_seqs, self.n_prefix_tokens, self._stream())

    def append_new(self):
        b = self.batch
        return B.cronus_kv_append(self.cache, self.new_k, self.new_v, self.cu_new, self.prefix_pos,
                                  self.block_tables, b.max_blocks, b.n_seqs, self.n_new_tokens, self._stream())

    def _rows(self):
        return ((self.prefix_k, self.prefix_v, self.cu_prefix, self.zero_pos, self.n_prefix_tokens),
                (self.new_k, self.new_v, self.cu_new, self.prefix_pos, self.n_new_tokens))

    def place_rows(self, stream=None):
        """ingest_prefix and append_new in one launch (the rows go to different slots)."""
        b = self.batch
        return B.cronus_kv_append_pair(self.cache, *self._rows(), self.block_tables, b.max_blocks, b.n_seqs,
                                       self._stream() if stream is None else stream)

    def ensure_workspace(self):
        """Workspace for this batch's lengths (sized once: the lengths of a batch do not change)."""
        if self.workspace is None:
            need = B.cronus_attn_mixed_workspace_bytes(self.cache, self.batch.prefix_lens, self.batch.chunk_lens)
            if need == 0:
                raise RuntimeError("cronus_attn_mixed_workspace_bytes rejected the batch")
            self.workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
            self.workspace_bytes = need
        return self.workspace_bytes

    def attention(self, stream=None):
        b = self.batch
        self.ensure_workspace()
        return B.cronus_attn_mixed(self.cache, self.q, self.out, b.prefix_lens, b.chunk_lens, self.block_tables,
                                   b.max_blocks, self.sm_scale, self.workspace, self.workspace_bytes,
                                   self._stream() if stream is None else stream)

    def step(self):
        """One pass of the whole hot path (after setup_decode_context()): place_rows and attention in one call."""
        b = self.batch
        self.ensure_workspace()
        B.cronus_iteration(self.cache, *self._rows(), self.q, self.out, b.prefix_lens, b.chunk_lens, self.block_tables,
                           b.max_blocks, self.sm_scale, self.workspace, self.workspace_bytes, self._stream())


class DraftLoop:
    """Device state of a loop that drafts tokens and keeps the accepted ones: every layer's cache, the tables, the free list and
    the lengths, none of which the host reads.  An iteration is
      1. begin    - cronus_build_tables: blocks for the new rows of every sequence (-1: the sequence has ended)
      2. per layer  append (cronus_kv_append) and attend (cronus_attn_tree)
      3. commit   - cronus_kv_commit: the accepted path's rows stay, the lengths grow by them
    all on the current stream.  Nothing is allocated after construction, so an iteration can be captured into a graph (not across a
    change of the tensors that are passed in).  `report` says whether the blocks sufficed; where they did not, the iteration leaves
    everything as it was."""

    def __init__(self, shape, n_layers: int, n_seqs: int, num_blocks: int, max_blocks: int, max_rows: int, max_path: int,
                 device="cuda:0", scales=None, pool_fill=0):
        self.shape, self.n_seqs, self.max_blocks, self.max_rows, self.max_path = shape, n_seqs, max_blocks, max_rows, max_path
        self.num_blocks, self.max_tokens = num_blocks, n_seqs * max_rows
        self.device = torch.device(device)
        fp8 = shape.kv_dtype == "fp8"
        size = num_blocks * shape.n_kv_heads * 16 * shape.head_dim
        pool = lambda: [torch.full((size,), pool_fill, dtype=torch.uint8 if fp8 else torch.int16, device=self.device) for _ in range(n_layers)]
        self.k_pools, self.v_pools = pool(), pool()
        self.scales = [None if s is None else torch.as_tensor(s, dtype=torch.float32, device=self.device) for s in scales or (None, None)]
        caches = [B.make_cache(k, v, num_blocks, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                               B.CRONUS_KV_FP8_E4M3 if fp8 else B.CRONUS_KV_BF16, *self.scales) for k, v in zip(self.k_pools, self.v_pools)]
        self.caches = B.cache_array(caches)
        i32 = lambda *n, fill=0: torch.full(n, fill, dtype=torch.int32, device=self.device)
        self.block_tables, self.held, self.kv_lens = i32(n_seqs, max_blocks, fill=-1), i32(n_seqs), i32(n_seqs)
        self.free_blocks, self.free_count = torch.arange(num_blocks, dtype=torch.int32, device=self.device), i32(1, fill=num_blocks)
        self.cu_rows, self.start_pos, self.cu_blocks, self.report = i32(n_seqs + 1), i32(n_seqs), i32(n_seqs + 1), i32(4)
        self.slot_map = torch.full((self.max_tokens,), -1, dtype=torch.int64, device=self.device)
        self.sm_scale = 1.0 / float(np.sqrt(shape.head_dim))
        self.workspace_bytes = B.cronus_attn_tree_workspace_bytes(self.caches[0], max_rows)
        if self.workspace_bytes == 0:
            raise RuntimeError("cronus_attn_tree_workspace_bytes rejected the shape")
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)

    def _stream(self):
        return torch.cuda.current_stream(self.device).cuda_stream

    def begin(self, new_lens):
        """new_lens: device int32 [n_seqs]."""
        return B.cronus_build_tables((self.block_tables, self.max_blocks, self.held, self.held, self.free_blocks, self.num_blocks,
                                      self.free_count, self.free_count), self.kv_lens, new_lens, self.n_seqs, self.cu_rows,
                                     self.start_pos, self.cu_blocks, self.slot_map, self.max_tokens, self.report, self._stream())

    def append(self, layer: int, k, v):
        """k, v: the new rows of all sequences, back to back (bf16 [rows][Hkv][D]; rows behind the last sequence's are not read)."""
        return B.cronus_kv_append(self.caches[layer], k, v, self.cu_rows, self.start_pos, self.block_tables, self.max_blocks,
                                  self.n_seqs, k.shape[0], self._stream())

    def attend(self, layer: int, q, out, mask=None):
        """mask: int64 [rows][words], None for a chain."""
        return B.cronus_attn_tree(self.caches[layer], q, out, self.start_pos, self.cu_rows, mask, 0 if mask is None else mask.shape[1],
                                  self.block_tables, self.max_blocks, self.n_seqs, self.max_rows, self.sm_scale, self.workspace,
                                  self.workspace_bytes, self._stream())

    def commit(self, paths, path_lens):
        """paths: device int32 [n_seqs][max_path]; path_lens: device int32 [n_seqs]."""
        return B.cronus_kv_commit(self.caches, self.start_pos, self.cu_rows, paths, self.max_path, path_lens, self.block_tables,
                                  self.max_blocks, self.n_seqs, self.kv_lens, self._stream())
