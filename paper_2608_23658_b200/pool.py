"""Convenience wrapper over the C ABI: owns a pool handle, hands out zero-copy torch views of the
mapped part of a layer's range and keeps a decode workspace.  No arithmetic happens here."""
from __future__ import annotations

import contextlib
import threading

import torch

from . import _binding as B


def _raw_stream(device: int) -> int:
    """Address of torch's current stream on a device (by the raw call where torch has it: building the Stream object costs more than the
    rest of a small call)."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device) if raw else torch.cuda.current_stream(device).cuda_stream


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
        self._parts = {}  # workspaces of scored and shared attention, by stream
        self._lock = threading.Lock()  # held while a call that uses one makes its launches: another thread's must not fall between them

    # -- lifetime
    def close(self):
        if self.handle:
            torch.cuda.synchronize(self.device)
            B.ekv_pool_destroy(self.handle)
            self.handle = None
            self._ws = None
            self._parts = {}

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
            k_out = self._made(shape, stream)
        else:
            self._check_rows("k_out", k_out, shape)
        if v_out is None:
            v_out = self._made(shape, stream)
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

    def _current(self, stream):
        """Address of the given stream, or of the current one on the pool's own device."""
        if stream is None:
            return _raw_stream(self.device.index)
        return stream if isinstance(stream, int) else stream.cuda_stream

    def _on(self, stream):
        """Where memory that a call makes is made, if a stream was given: on that stream, so that no kernel under way elsewhere may still use it, what
        becomes of it later is in the stream's order, and it belongs to the stream's graph while one is captured."""
        return torch.cuda.stream(torch.cuda.ExternalStream(self._current(stream), device=self.device))

    def _made(self, shape, stream):
        """A bf16 tensor that the call on that stream writes."""
        if stream is None:
            return torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        with self._on(stream):
            return torch.empty(shape, dtype=torch.bfloat16, device=self.device)

    def _want(self, call, name, t, dtype, shape):
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self.device.index or not t.is_contiguous():
            B._refuse(call, name, t, f"contiguous {dtype} {shape} on {self.device}")

    def _heads(self, call, name, t, T, heads):
        """bf16 [T, heads, head_dim] whose tokens may stand apart (a part of a wider row; the library looks at the distance)."""
        stride = t.stride()
        if (t.dtype is not torch.bfloat16 or t.shape != (T, heads, self.head_dim) or t.get_device() != self.device.index
                or stride[2] != 1 or (stride[1] != self.head_dim and heads > 1)):
            B._refuse(call, name, t, f"bfloat16 {(T, heads, self.head_dim)} on {self.device}, a token's heads side by side")
        return stride[0]

    def rope_write_kv(self, layer, q, k, v, positions, inv_freq, slot_mapping, q_weight=None, k_weight=None, eps=1e-6, weight_offset=0.0,
                      factor=1.0, interleaved=False, axes=None, q_out=None, k_out=None, stream=None):
        """Norms (where a weight is given) and turns queries [T, Hq, D] and keys [T, Hkv, D] by their positions, writes keys and values
        into the slots, returns the queries.  q, k, v may be parts of one projection's rows.  positions: int32 [T], or [axes, T] with
        `axes` naming the axis of each pair of channels; inv_freq: float32 [rotary_dim / 2]; interleaved: pairs are neighbours.  q_out may be q.  8-bit pools: k_out
        receives the finished keys as bf16 before they are quantised (one is made if none is given)."""
        call, i32, f32, bf16, dev, D = "rope_write_kv", torch.int32, torch.float32, torch.bfloat16, self.device.index, self.head_dim
        T, pairs, where = slot_mapping.shape[0], inv_freq.shape[0], positions.shape
        num_axes = where[0] if len(where) == 2 else 1
        heads, kv_heads = self.num_q_heads, self.num_kv_heads
        rows, row, qs, ks, vs = (T, kv_heads, D), (D,), q.stride(), k.stride(), v.stride()
        # (one look at everything; what is wrong is found out after that)
        if not (q.dtype is bf16 and k.dtype is bf16 and v.dtype is bf16 and q.shape == (T, heads, D) and k.shape == rows and v.shape == rows
                and qs[2] == 1 and ks[2] == 1 and vs[2] == 1 and qs[1] == D and ks[1] == D and vs[1] == D
                and q.get_device() == dev and k.get_device() == dev and v.get_device() == dev):
            for name, t, n in (("q", q, heads), ("k", k, kv_heads), ("v", v, kv_heads)):
                self._heads(call, name, t, T, n)
        if not (slot_mapping.dtype is torch.int64 and inv_freq.dtype is f32 and positions.dtype is i32 and 1 <= len(where) <= 2 and where[-1] == T
                and slot_mapping.dim() == 1 and inv_freq.dim() == 1 and slot_mapping.is_contiguous() and inv_freq.is_contiguous() and positions.is_contiguous()
                and slot_mapping.get_device() == dev and inv_freq.get_device() == dev and positions.get_device() == dev):
            self._want(call, "slot_mapping", slot_mapping, torch.int64, (T,))
            self._want(call, "inv_freq", inv_freq, f32, (pairs,))
            self._want(call, "positions", positions, i32, (num_axes, T) if num_axes > 1 else (T,))
        if num_axes > 1 and (axes is None or len(axes) != pairs):
            raise ValueError(f"rope_write_kv: axes has to name the axis of each of the {pairs} pairs")
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            if w is not None and not (w.dtype is bf16 and w.shape == row and w.get_device() == dev and w.is_contiguous()):
                self._want(call, name, w, bf16, row)
        if q_out is None:
            q_out = self._made((T, heads, D), stream)
            out_stride = heads * D
        else:
            out_stride = self._heads(call, "q_out", q_out, T, heads)
        if k_out is not None:
            self._want(call, "k_out", k_out, bf16, rows)
        elif self.dtype == B.EKV_E4M3:
            k_out = self._made(rows, stream)
        rope = B.Rope(2 * pairs, num_axes, B.EKV_ROPE_ADJACENT if interleaved else 0, factor, eps, weight_offset, inv_freq.data_ptr(),
                      positions.data_ptr(), bytes(axes) if num_axes > 1 else None, q_weight.data_ptr() if q_weight is not None else None,
                      k_weight.data_ptr() if k_weight is not None else None)
        B._check(B.load_library().ekv_rope_write_kv(self.handle, layer, rope, q.data_ptr(), qs[0], k.data_ptr(), ks[0], v.data_ptr(), vs[0], q_out.data_ptr(), out_stride,
                            None if k_out is None else k_out.data_ptr(), slot_mapping.data_ptr(), T, self._current(stream)))
        return q_out

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
            with contextlib.nullcontext() if stream is None else self._on(stream):
                out = torch.empty_like(q)
        if workspace is None:
            workspace = self.workspace(int(seq_lens.shape[0]), int(block_tables.shape[1]) * self.block_size)
        B.ekv_attn_decode(self.handle, layer, q, out, block_tables, seq_lens, scale, workspace, stream)
        return out

    def attn_prefill_chunk(self, layer, q, block_tables, cu_q_lens, cu_q_lens_host, seq_lens, scale, out=None,
                           stream=None):
        if out is None:
            with contextlib.nullcontext() if stream is None else self._on(stream):
                out = torch.empty_like(q)
        B.ekv_attn_prefill_chunk(self.handle, layer, q, out, block_tables, cu_q_lens, cu_q_lens_host, seq_lens,
                                 scale, stream)
        return out

    # -- scores with a cap, a distance bias, a window, a prefix; batches that share prefixes
    def _check_attn(self, call, q, out, block_tables, seq_lens, T, stream):
        """Shape of the block tables; an output if none is given."""
        at, shape, i32, bf16, dev = block_tables.shape, (T, self.num_q_heads, self.head_dim), torch.int32, torch.bfloat16, self.device.index
        if out is None:
            out = self._made(shape, stream)
        if not (len(at) == 2 and block_tables.dtype is i32 and seq_lens.dtype is i32 and q.dtype is bf16 and out.dtype is bf16
                and seq_lens.shape == at[:1] and q.shape == shape and out.shape == shape and block_tables.is_contiguous() and seq_lens.is_contiguous()
                and q.is_contiguous() and out.is_contiguous() and block_tables.get_device() == dev and seq_lens.get_device() == dev
                and q.get_device() == dev and out.get_device() == dev):
            if len(at) != 2:
                B._refuse(call, "block_tables", block_tables, "int32 [requests, max_blocks_per_seq]")
            self._want(call, "block_tables", block_tables, i32, at)
            self._want(call, "seq_lens", seq_lens, i32, at[:1])
            self._want(call, "q", q, bf16, shape)
            self._want(call, "out", out, bf16, shape)
        return at[1], out

    def _scores(self, call, n, cap, window, slopes, prefix_lens):
        if slopes is not None:
            self._want(call, "slopes", slopes, torch.float32, (self.num_q_heads,))
        if prefix_lens is not None:
            self._want(call, "prefix_lens", prefix_lens, torch.int32, (n,))
        return B.Scores(cap, window, None if slopes is None else slopes.data_ptr(), None if prefix_lens is None else prefix_lens.data_ptr())

    def _launch(self, call, need, workspace, stream):
        """call(workspace, its bytes, stream), with the workspace that was handed in.  Without one: a captured call gets memory of its graph, so that
        two graphs share none; others share one for each stream, which grows when the library says that it is too small."""
        if workspace is not None:
            B._check(call(workspace.data_ptr(), workspace.numel() * workspace.element_size(), self._current(stream)))
        elif stream is None and torch.cuda.current_device() == self.device.index:
            self._launch_here(call, need, self._current(None))
        else:
            with self._on(stream):
                self._launch_here(call, need, self._current(stream))

    def _launch_here(self, call, need, stream):
        if torch.cuda.is_current_stream_capturing():
            own = torch.empty(max(need(), 1), dtype=torch.uint8, device=self.device)
            return B._check(call(own.data_ptr(), own.numel(), stream))
        with self._lock:
            kept = self._parts.get(stream)
            st = call(kept[-1].data_ptr(), kept[-1].numel(), stream) if kept else B.Status.ERR_WORKSPACE
            if st == B.Status.ERR_WORKSPACE:  # (the ones that were too small stay: calls that are under way use them)
                kept = self._parts.setdefault(stream, [])
                kept.append(torch.empty(max(need(), 2 * kept[-1].numel() if kept else 1 << 20), dtype=torch.uint8, device=self.device))
                st = call(kept[-1].data_ptr(), kept[-1].numel(), stream)
        B._check(st)

    def attn_decode_scored(self, layer, q, block_tables, seq_lens, scale, cap=0.0, window=0, slopes=None, prefix_lens=None, out=None,
                           workspace=None, stream=None):
        """attn_decode with x = cap * tanh(x / cap), a bias of -slopes[head] * distance, a window of that many keys, and the keys below prefix_lens
        always seen; any of them."""
        n, lib = seq_lens.shape[0], B.load_library()
        width, out = self._check_attn("attn_decode_scored", q, out, block_tables, seq_lens, n, stream)
        scores = self._scores("attn_decode_scored", n, cap, window, slopes, prefix_lens)
        self._launch(lambda ws, size, stream: lib.ekv_attn_decode_scored(self.handle, layer, q.data_ptr(), out.data_ptr(), block_tables.data_ptr(), width,
                                                                         seq_lens.data_ptr(), n, scale, scores, ws, size, stream),
                     lambda: lib.ekv_attn_workspace_bytes(self.handle, n, width * self.block_size), workspace, stream)
        return out

    def attn_prefill_chunk_scored(self, layer, q, block_tables, cu_q_lens, cu_q_lens_host, seq_lens, scale, cap=0.0, window=0, slopes=None,
                                  prefix_lens=None, out=None, workspace=None, stream=None):
        """attn_prefill_chunk with scores and masks as in attn_decode_scored, for every row at its own position."""
        call, n, T, lib = "attn_prefill_chunk_scored", seq_lens.shape[0], q.shape[0], B.load_library()
        if cu_q_lens_host.dtype is not torch.int32 or cu_q_lens_host.is_cuda or cu_q_lens_host.numel() != n + 1 or not cu_q_lens_host.is_contiguous():
            B._refuse(call, "cu_q_lens_host", cu_q_lens_host, f"contiguous int32 ({n + 1},) on the host")
        self._want(call, "cu_q_lens", cu_q_lens, torch.int32, (n + 1,))
        width, out = self._check_attn(call, q, out, block_tables, seq_lens, T, stream)
        if T < cu_q_lens_host[n].item():
            B._refuse(call, "q", q, f"of at least {cu_q_lens_host[n].item()} rows")
        scores = self._scores(call, n, cap, window, slopes, prefix_lens)
        self._launch(lambda ws, size, stream: lib.ekv_attn_prefill_chunk_scored(self.handle, layer, q.data_ptr(), out.data_ptr(), block_tables.data_ptr(), width,
                                                                                cu_q_lens.data_ptr(), cu_q_lens_host.data_ptr(), seq_lens.data_ptr(), n, scale,
                                                                                scores, ws, size, stream),
                     lambda: lib.ekv_attn_prefill_scored_workspace_bytes(self.handle), workspace, stream)
        return out

    def attn_decode_shared(self, layer, q, block_tables, seq_lens, group_starts, shared_lens, scale, out=None, workspace=None, stream=None):
        """attn_decode of a batch whose requests share prefixes: group_starts [G+1] and shared_lens [G] are int32 on the host.  The shared
        tokens' blocks stand in every request's table; they are read once a group."""
        call, n, G, lib = "attn_decode_shared", seq_lens.shape[0], shared_lens.numel(), B.load_library()
        if not (group_starts.dtype is shared_lens.dtype is torch.int32 and group_starts.numel() == G + 1 and not group_starts.is_cuda
                and not shared_lens.is_cuda and group_starts.is_contiguous() and shared_lens.is_contiguous()):
            for name, t, size in (("group_starts", group_starts, G + 1), ("shared_lens", shared_lens, G)):
                if t.dtype is not torch.int32 or t.is_cuda or t.numel() != size or not t.is_contiguous():
                    B._refuse(call, name, t, f"contiguous int32 ({size},) on the host")
        width, out = self._check_attn(call, q, out, block_tables, seq_lens, n, stream)
        starts, shared = group_starts.data_ptr(), shared_lens.data_ptr()
        self._launch(lambda ws, size, stream: lib.ekv_attn_decode_shared(self.handle, layer, q.data_ptr(), out.data_ptr(), block_tables.data_ptr(), width,
                                                                         seq_lens.data_ptr(), n, starts, shared, G, scale, ws, size, stream),
                     lambda: lib.ekv_attn_decode_shared_workspace_bytes(self.handle, starts, shared, G, width), workspace, stream)
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
