"""Convenience wrapper over the C ABI: owns a pool handle, hands out zero-copy torch views of the
mapped part of a layer's range and keeps a decode workspace.  No arithmetic happens here."""
from __future__ import annotations

import torch

from . import _binding as B


class _RawCuda:
    """Minimal __cuda_array_interface__ carrier for a raw device range (int16 elements unless told otherwise).  A tensor
    made of it keeps it, and so the pool whose memory it views: a view that outlives the caller's last name for the pool
    stays readable until the view goes too (an explicit close() still ends it)."""

    def __init__(self, ptr: int, nelem: int, typestr: str = "<i2", owner=None):
        self.owner = owner
        self.__cuda_array_interface__ = {"shape": (nelem,), "typestr": typestr, "data": (ptr, False), "version": 3,
                                         "strides": None}


class Pool:
    def __init__(self, *, num_q_heads, num_kv_heads, head_dim, base_blocks, elastic_blocks=0, num_layers=1,
                 block_size=16, device=0, start_grown=False, fused_range=False, prefill_warp_mma=False,
                 prefill_one_head=False, prefill_two_head=False, dtype=B.EKV_BF16):
        self.device = torch.device("cuda", device)
        torch.cuda.set_device(self.device)
        self.handle = B.ekv_pool_create(device=device, num_layers=num_layers, num_q_heads=num_q_heads,
                                        num_kv_heads=num_kv_heads, head_dim=head_dim, block_size=block_size,
                                        base_blocks=base_blocks, elastic_blocks=elastic_blocks, dtype=dtype,
                                        flags=(B.EKV_START_GROWN if start_grown else 0) | (B.EKV_FUSED_RANGE if fused_range else 0) |
                                        (B.EKV_PREFILL_WARP_MMA if prefill_warp_mma else 0) |
                                        (B.EKV_PREFILL_ONE_HEAD if prefill_one_head else 0) |
                                        (B.EKV_PREFILL_TWO_HEAD if prefill_two_head else 0))
        self.num_q_heads, self.num_kv_heads, self.head_dim, self.block_size = num_q_heads, num_kv_heads, head_dim, block_size
        self.num_layers = num_layers
        self.dtype = dtype
        self._ws = None

    # -- lifetime
    def close(self):
        if self.handle:
            torch.cuda.synchronize(self.device)
            B.ekv_pool_destroy(self.handle)
            self.handle = None
            self._ws = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- state
    @property
    def info(self) -> B.PoolInfo:
        return B.ekv_pool_info(self.handle)

    def layer_ptr(self, layer: int) -> int:
        return B.ekv_layer_ptr(self.handle, layer)

    def layer_tensor(self, layer: int, first_block: int = 0, num_blocks: int | None = None) -> torch.Tensor:
        """View [blocks, 2, Hkv, block_size, head_dim] of blocks first_block.. of a layer: bf16, or the e4m3 codes of an
        EKV_E4M3 pool (layer_scales has their scales).
        Only LIVE blocks may be viewed: unmapped elastic addresses fault when touched."""
        info = self.info
        if num_blocks is None:
            num_blocks = info.live_blocks - first_block
        if first_block < 0 or first_block + num_blocks > info.live_blocks:
            raise ValueError("view would reach past the live (mapped) blocks")
        size = 1 if self.dtype == B.EKV_E4M3 else 2
        elems = info.block_bytes // size
        stride = info.block_stride_bytes // size   # elements between consecutive block ids of this layer
        span = (num_blocks - 1) * stride + elems if num_blocks > 0 else 0
        raw = _RawCuda(self.layer_ptr(layer) + first_block * info.block_stride_bytes, max(span, 1),
                       "|u1" if size == 1 else "<i2", self)
        flat = torch.as_tensor(raw, device=self.device).view(torch.float8_e4m3fn if size == 1 else torch.bfloat16)
        d, bs, hk = self.head_dim, self.block_size, self.num_kv_heads
        # dense when stride == elems (one range per layer); a strided view over the fused range otherwise
        return torch.as_strided(flat, (num_blocks, 2, hk, bs, d), (stride, hk * bs * d, bs * d, d, 1))

    def layer_scales(self, layer: int, first_block: int = 0, num_blocks: int | None = None) -> torch.Tensor:
        """float32 view [blocks, 2, Hkv] of an EKV_E4M3 pool's scales (elastic ids included, mapped or not)."""
        info = self.info
        total = info.base_blocks + info.elastic_blocks
        if num_blocks is None:
            num_blocks = total - first_block
        if first_block < 0 or num_blocks < 0 or first_block + num_blocks > total:
            raise ValueError("view would reach past the pool's blocks")
        raw = _RawCuda(B.ekv_layer_scales(self.handle, layer), total * 2 * self.num_kv_heads, "<f4", self)
        return torch.as_tensor(raw, device=self.device).view(total, 2, self.num_kv_heads)[first_block:first_block + num_blocks]

    def grow(self, stream=None):
        return B.ekv_grow(self.handle, stream)

    def shrink(self, keep_physical: bool = False, stream=None):
        return B.ekv_shrink(self.handle, stream, B.EKV_KEEP_PHYSICAL if keep_physical else 0)

    def poll_status(self) -> B.Status:
        return B.ekv_poll_status(self.handle)

    # -- compute (argument marshalling only)
    def write_kv(self, layer, k, v, slot_mapping, stream=None):
        B.ekv_write_kv(self.handle, layer, k, v, slot_mapping, stream)

    def read_kv(self, layer, slot_mapping, k_out=None, v_out=None, stream=None):
        """Values stored in the slots as bf16 rows (k, v), each [T, Hkv, head_dim].  Rows of negative slots are left as they
        were: hand in tensors of your own if the mapping has any."""
        T, = slot_mapping.shape
        if slot_mapping.dtype is not torch.int64 or slot_mapping.get_device() != self.device.index or not slot_mapping.is_contiguous():
            B._refuse("read_kv", "slot_mapping", slot_mapping, f"contiguous int64 on {self.device}")
        shape = (T, self.num_kv_heads, self.head_dim)
        if k_out is None:
            k_out = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        else:
            self._check_rows("k_out", k_out, shape)
        if v_out is None:
            v_out = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        else:
            self._check_rows("v_out", v_out, shape)
        B._check(B.load_library().ekv_read_kv(self.handle, layer, k_out.data_ptr(), v_out.data_ptr(), slot_mapping.data_ptr(), T, B._stream(stream)))
        return k_out, v_out

    def _check_rows(self, name, t, shape):
        if t.dtype is not torch.bfloat16 or t.shape[:1] != shape[:1] or t.numel() != shape[0] * shape[1] * shape[2] or t.get_device() != self.device.index or not t.is_contiguous():
            B._refuse("read_kv", name, t, f"contiguous bfloat16 {shape} on {self.device}")

    def _on_device(self, t):
        if t.get_device() != self.device.index:
            raise ValueError(f"a tensor on {t.device} for a pool on {self.device}")

    def extend_tables(self, new_tokens, seq_lens, block_tables, free_ids, free_cursor, slot_mapping, cu_q_lens,
                      seq_lens_out=None, free_cursor_out=None, stream=None):
        self._on_device(block_tables)
        B.ekv_extend_tables(self.handle, new_tokens, seq_lens, block_tables, free_ids, free_cursor, slot_mapping, cu_q_lens,
                            seq_lens_out, free_cursor_out, stream)

    def workspace(self, batch: int, max_seq_len: int) -> torch.Tensor:
        need = B.ekv_attn_workspace_bytes(self.handle, batch, max_seq_len)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    def attn_decode(self, layer, q, block_tables, seq_lens, scale, out=None, workspace=None, stream=None):
        if out is None:
            out = torch.empty_like(q)
        if workspace is None:
            workspace = self.workspace(int(seq_lens.shape[0]), int(block_tables.shape[1]) * self.block_size)
        B.ekv_attn_decode(self.handle, layer, q, out, block_tables, seq_lens, scale, workspace, stream)
        return out

    def attn_prefill_chunk(self, layer, q, block_tables, cu_q_lens, cu_q_lens_host, seq_lens, scale, out=None,
                           stream=None):
        if out is None:
            out = torch.empty_like(q)
        B.ekv_attn_prefill_chunk(self.handle, layer, q, out, block_tables, cu_q_lens, cu_q_lens_host, seq_lens,
                                 scale, stream)
        return out


class HostStep:
    """Decode steps driven from pinned host tensors (ekv_hoststep_*): copies in, write_kv + decode, copy out,
    double-buffered on the library's own copy streams.  Close it before its pool."""

    def __init__(self, pool: Pool, max_batch: int, max_blocks_per_seq: int, depth: int = 2):
        self.pool = pool
        self.handle = B.ekv_hoststep_create(pool.handle, max_batch, max_blocks_per_seq, depth)

    def decode(self, layer, h_q, h_block_tables, h_seq_lens, scale, h_out, h_k=None, h_v=None, h_slot_mapping=None,
               stream=None):
        B.ekv_hoststep_decode(self.handle, layer, h_q, h_k, h_v, h_slot_mapping, h_block_tables, h_seq_lens, scale, h_out,
                              stream)

    def flush(self, stream=None):
        B.ekv_hoststep_flush(self.handle, stream)

    def close(self):
        if self.handle:
            B.ekv_hoststep_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
