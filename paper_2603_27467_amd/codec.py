"""Convenience wrapper: a codec object over the C ABI, taking torch tensors."""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np

from . import _capi as C


@dataclass(frozen=True)
class LayerCfg:
    """Codebooks of one layer (section 3.2) and its K/V norm storage (section 3.3)."""
    n_k: int
    n_v: int
    norm_bits_k: int = 8
    norm_bits_v: int = 4
    norm_mode_k: int = C.TVQ_NORM_LINEAR
    norm_mode_v: int = C.TVQ_NORM_LOG


def _stream_handle(stream) -> int:
    import torch
    if stream is None:
        # the current stream's handle without a Stream object around it (2 us a call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def desc_of(t, layers: Optional[int] = None) -> C.tvq_tensor_desc:
    """Descriptor of a [L, B, H, T, d] torch tensor (d contiguous)."""
    shape, s = t.shape, t.stride()
    if len(shape) != 5 or s[4] != 1:
        raise ValueError("expected a [L, B, H, T, d] tensor with d contiguous")
    return C.tvq_tensor_desc(shape[1], shape[3], s[0], s[1], s[2], s[3])


def _check_bytes(buf, lay: C.tvq_layout, what: str) -> None:
    """buf must be a contiguous uint8 GPU tensor holding at least the layout's bytes (the
    kernels address it from the layout alone)."""
    import torch
    if buf.dtype != torch.uint8 or not buf.is_contiguous():
        raise ValueError(f"{what} must be a contiguous uint8 GPU tensor")
    if buf.numel() < lay.total_bytes:
        raise ValueError(f"{what} holds {buf.numel()} bytes, the layout needs {lay.total_bytes}")


def _on_gpu(*tensors) -> None:
    for t in tensors:
        if not t.is_cuda:
            raise ValueError("tensors must be on the GPU")


@functools.lru_cache(maxsize=None)
def _dtypes() -> dict:
    import torch
    return {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}


class Codec:
    def __init__(self, num_layers: int, num_heads: int, head_dim: int,
                 layers: Sequence, seed: int = 0, shared_signs: bool = False,
                 signs: Optional[np.ndarray] = None, angle_packing: int = 0):
        """angle_packing = 1: group packing of non-power-of-two codebooks (tvq_config)."""
        self.L, self.H, self.d = num_layers, num_heads, head_dim
        self.layers = list(layers)
        arr = (C.tvq_layer_cfg * num_layers)()
        for i, lc in enumerate(self.layers):
            arr[i] = C.tvq_layer_cfg(lc.n_k, lc.n_v, lc.norm_bits_k, lc.norm_bits_v,
                                     lc.norm_mode_k, lc.norm_mode_v)
        self._arr = arr
        self._signs = None
        sp = None
        if signs is not None:
            self._signs = np.ascontiguousarray(signs, np.int8)
            sp = self._signs.ctypes.data_as(ctypes.POINTER(ctypes.c_int8))
        self.cfg = C.tvq_config(num_layers, num_heads, head_dim, 1 if shared_signs else 0,
                                seed & (2**64 - 1), arr, sp, angle_packing)
        self.handle = C.tvq_create(self.cfg)

    def close(self):
        if getattr(self, "handle", 0):
            C.tvq_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check_kv(self, t, what: str) -> None:
        """t must be a [L, B, H, T, d] GPU tensor of this codec's L, H and d (the kernels take
        L, H and d from the codec, so a smaller tensor would be read or written past its end)."""
        s = t.shape
        if len(s) != 5:
            raise ValueError(f"{what} must be a [L, B, H, T, d] GPU tensor")
        if s[0] != self.L or s[2] != self.H or s[4] != self.d:
            raise ValueError(f"{what} has shape {tuple(s)}; the codec needs "
                             f"[{self.L}, B, {self.H}, T, {self.d}]")

    def _check_q(self, q, out) -> None:
        s = q.shape
        if len(s) != 3 or out.shape != s or not q.is_contiguous() or not out.is_contiguous():
            raise ValueError("q and out must be contiguous [B, Hq, d] GPU tensors")
        if s[2] != self.d:
            raise ValueError(f"q has head dim {s[2]}, the codec {self.d}")

    def layout(self, batch: int, capacity_tokens: int) -> C.tvq_layout:
        return C.tvq_cache_layout(self.handle, batch, capacity_tokens)

    def alloc_cache(self, lay: C.tvq_layout, device="cuda"):
        import torch
        return torch.empty(lay.total_bytes, dtype=torch.uint8, device=device)

    def encode(self, k, v, cache, lay: C.tvq_layout, t_begin: int = 0, stream=None) -> None:
        import torch
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise ValueError("k and v must share shape, strides and dtype")
        dt = {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}.get(k.dtype)
        if dt is None:
            raise ValueError("k/v must be bf16 or fp32")
        self._check_kv(k, "k")
        _check_bytes(cache, lay, "cache")
        _on_gpu(k, v, cache)
        C.tvq_encode(self.handle, dt, k.data_ptr(), v.data_ptr(), desc_of(k), t_begin,
                     cache.data_ptr(), lay, _stream_handle(stream))

    def encode_mfma(self, k, v, cache, lay: C.tvq_layout, t_begin: int = 0,
                    stream=None) -> None:
        """encode with the matrix-core transform schedule (tvq_encode_mfma; bf16, d = 128)."""
        import torch
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != torch.bfloat16 or \
                v.dtype != torch.bfloat16:
            raise ValueError("k and v must be bf16 and share shape and strides")
        self._check_kv(k, "k")
        _check_bytes(cache, lay, "cache")
        _on_gpu(k, v, cache)
        C.tvq_encode_mfma(self.handle, k.data_ptr(), v.data_ptr(), desc_of(k), t_begin,
                          cache.data_ptr(), lay, _stream_handle(stream))

    def decode(self, cache, lay: C.tvq_layout, t_begin: int, t_end: int, k_out, v_out,
               stream=None) -> None:
        import torch
        if k_out.shape != v_out.shape or k_out.stride() != v_out.stride() or \
                k_out.dtype != v_out.dtype:
            raise ValueError("k_out and v_out must share shape, strides and dtype")
        dt = {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}.get(k_out.dtype)
        if dt is None:
            raise ValueError("outputs must be bf16 or fp32")
        self._check_kv(k_out, "k_out")
        _check_bytes(cache, lay, "cache")
        _on_gpu(k_out, v_out, cache)
        C.tvq_decode(self.handle, cache.data_ptr(), lay, t_begin, t_end, dt, k_out.data_ptr(),
                     v_out.data_ptr(), desc_of(k_out), _stream_handle(stream))

    def attention_workspace_bytes(self, batch: int, num_q_heads: int, t_end: int) -> int:
        return C.tvq_attention_workspace(self.handle, batch, num_q_heads, t_end)

    def attention(self, cache, lay: C.tvq_layout, layer: int, t_end: int, q, out,
                  scale: float, workspace=None, stream=None) -> None:
        """Attention of q ([B][Hq][d]) over tokens [0, t_end) of `layer` into out, from the
        codes (tvq_attention_decode).  `workspace` (a uint8 device tensor) is allocated when
        not given."""
        import torch
        self._check_q(q, out)
        _check_bytes(cache, lay, "cache")
        _on_gpu(q, out, cache)
        dts = {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}
        if q.dtype not in dts or out.dtype not in dts:
            raise ValueError("q/out must be bf16 or fp32")
        if workspace is None:       # the call itself checks the size of a given one
            need = self.attention_workspace_bytes(q.shape[0], q.shape[1], t_end)
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        elif workspace.dtype != torch.uint8 or not workspace.is_cuda or \
                not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 GPU tensor")
        C.tvq_attention_decode(self.handle, cache.data_ptr(), lay, layer, t_end, q.shape[1],
                               scale, dts[q.dtype], q.data_ptr(), dts[out.dtype], out.data_ptr(),
                               workspace.data_ptr(), workspace.numel(), _stream_handle(stream))

    def attention_noalloc(self, cache, lay: C.tvq_layout, layer: int, t_end: int, q, out,
                          scale: float, stream=None) -> None:
        """attention without a workspace (tvq_attention_decode_noalloc): the partials go to
        the library's static scratch; nothing is allocated, by the library or here."""
        import torch
        self._check_q(q, out)
        _check_bytes(cache, lay, "cache")
        _on_gpu(q, out, cache)
        dts = {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}
        if q.dtype not in dts or out.dtype not in dts:
            raise ValueError("q/out must be bf16 or fp32")
        C.tvq_attention_decode_noalloc(self.handle, cache.data_ptr(), lay, layer, t_end,
                                       q.shape[1], scale, dts[q.dtype], q.data_ptr(),
                                       dts[out.dtype], out.data_ptr(), _stream_handle(stream))

    # ---- paged pools (tvq_encode_paged / tvq_decode_paged / tvq_attention_paged) ----
    def pool_layout(self, n_blocks: int, block_tokens: int) -> C.tvq_layout:
        """Layout of a paged pool of n_blocks blocks of block_tokens slots."""
        return C.tvq_cache_layout(self.handle, n_blocks, block_tokens)

    @staticmethod
    def _i32(t, what):
        import torch
        if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous int32 GPU tensor")
        return t.data_ptr()

    def encode_paged(self, k, v, positions, block_table, pool, pool_lay: C.tvq_layout,
                     stream=None) -> None:
        """k, v: [L, B, T, ...] as for encode; token t of sequence b goes to position
        positions[b] + t through block_table ([B, max_blocks] int32)."""
        import torch
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise ValueError("k and v must share shape, strides and dtype")
        dt = {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}.get(k.dtype)
        if dt is None:
            raise ValueError("k/v must be bf16 or fp32")
        self._check_kv(k, "k")
        _check_bytes(pool, pool_lay, "pool")
        _on_gpu(k, v, pool)
        if block_table.dim() != 2 or positions.shape != (k.shape[1],) or \
                block_table.shape[0] != k.shape[1]:
            raise ValueError("positions [B] and block_table [B, max_blocks] must match k")
        C.tvq_encode_paged(self.handle, dt, k.data_ptr(), v.data_ptr(), desc_of(k),
                           self._i32(positions, "positions"),
                           self._i32(block_table, "block_table"), block_table.shape[1],
                           pool.data_ptr(), pool_lay, _stream_handle(stream))

    def decode_paged(self, pool, pool_lay: C.tvq_layout, block_table, t_begin: int, t_end: int,
                     k_out, v_out, stream=None) -> None:
        import torch
        if k_out.shape != v_out.shape or k_out.stride() != v_out.stride() or \
                k_out.dtype != v_out.dtype:
            raise ValueError("k_out and v_out must share shape, strides and dtype")
        dt = {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}.get(k_out.dtype)
        if dt is None:
            raise ValueError("outputs must be bf16 or fp32")
        self._check_kv(k_out, "k_out")
        _check_bytes(pool, pool_lay, "pool")
        _on_gpu(k_out, v_out, pool)
        if block_table.dim() != 2 or block_table.shape[0] != k_out.shape[1]:
            raise ValueError("block_table must be [B, max_blocks]")
        C.tvq_decode_paged(self.handle, pool.data_ptr(), pool_lay,
                           self._i32(block_table, "block_table"), block_table.shape[1], t_begin,
                           t_end, dt, k_out.data_ptr(), v_out.data_ptr(), desc_of(k_out),
                           _stream_handle(stream))

    def attention_paged_workspace_bytes(self, batch: int, num_q_heads: int, max_ctx: int,
                                        block_tokens: int) -> int:
        return C.tvq_attention_paged_workspace(self.handle, batch, num_q_heads, max_ctx,
                                               block_tokens)

    def attention_paged(self, pool, pool_lay: C.tvq_layout, block_table, ctx_lens, max_ctx: int,
                        layer: int, q, out, scale: float, workspace=None, stream=None) -> None:
        """Attention of q ([B, Hq, d]) of sequence b over its positions [0, ctx_lens[b])."""
        import torch
        self._check_q(q, out)
        _check_bytes(pool, pool_lay, "pool")
        _on_gpu(q, out, pool, block_table, ctx_lens)
        dts = {torch.bfloat16: C.TVQ_BF16, torch.float32: C.TVQ_F32}
        if q.dtype not in dts or out.dtype not in dts:
            raise ValueError("q/out must be bf16 or fp32")
        B = q.shape[0]
        if block_table.dim() != 2 or block_table.shape[0] != B or ctx_lens.shape != (B,):
            raise ValueError("block_table [B, max_blocks] and ctx_lens [B] must match q")
        if workspace is None:       # the call itself checks the size of a given one
            need = self.attention_paged_workspace_bytes(B, q.shape[1], max_ctx,
                                                        pool_lay.capacity_tokens)
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        elif workspace.dtype != torch.uint8 or not workspace.is_cuda or \
                not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 GPU tensor")
        C.tvq_attention_paged(self.handle, pool.data_ptr(), pool_lay,
                              self._i32(block_table, "block_table"), block_table.shape[1],
                              self._i32(ctx_lens, "ctx_lens"), max_ctx, B, layer, q.shape[1],
                              scale, dts[q.dtype], q.data_ptr(), dts[out.dtype], out.data_ptr(),
                              workspace.data_ptr(), workspace.numel(), _stream_handle(stream))

    # ---- many new tokens (tvq_attention_prefill / tvq_attention_prefill_paged) ----
    def attention_prefill_workspace_bytes(self, batch: int, num_q_heads: int, tokens: int,
                                          max_ctx: int) -> int:
        return C.tvq_attention_prefill_workspace(self.handle, batch, num_q_heads, tokens, max_ctx)

    def _check_rows(self, q, out) -> None:
        s = q.shape
        if len(s) != 4 or out.shape != s or q.stride(-1) != 1 or out.stride(-1) != 1:
            raise ValueError("q and out must be [B, Hq, T, d] GPU tensors with d contiguous")
        if s[3] != self.d:
            raise ValueError(f"q has head dim {s[3]}, the codec {self.d}")

    @staticmethod
    def _io_dtypes(q, out):
        dts = _dtypes()
        dq, do = dts.get(q.dtype), dts.get(out.dtype)
        if dq is None or do is None:
            raise ValueError("q/out must be bf16 or fp32")
        return dq, do

    @staticmethod
    def _rows_desc(t) -> C.tvq_tensor_desc:
        s = t.stride()
        return C.tvq_tensor_desc(t.shape[0], t.shape[2], 0, s[0], s[1], s[2])

    @staticmethod
    def _workspace(workspace, need, device, stream):
        """The given workspace (the call itself checks its size) or a new one of need() bytes,
        allocated for the stream that the call runs on."""
        import torch
        if workspace is None:
            if stream is None:
                return torch.empty(need(), dtype=torch.uint8, device=device)
            if not isinstance(stream, torch.cuda.Stream):
                handle = _stream_handle(stream)
                stream = torch.cuda.ExternalStream(handle, device=device) if handle else \
                    torch.cuda.default_stream(device)
            with torch.cuda.stream(stream):
                return torch.empty(need(), dtype=torch.uint8, device=device)
        if workspace.dtype != torch.uint8 or not workspace.is_cuda or \
                not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 GPU tensor")
        return workspace

    def attention_prefill(self, cache, lay: C.tvq_layout, layer: int, t_end: int, q, out,
                          scale: float, workspace=None, stream=None) -> None:
        """Causal attention of the newest T tokens of every sequence, q [B, Hq, T, d] (any strides
        with d contiguous), into out: token j stands at position t_end - T + j and attends to the
        positions up to its own."""
        self._check_rows(q, out)
        _check_bytes(cache, lay, "cache")
        _on_gpu(q, out, cache)
        dq, do = self._io_dtypes(q, out)
        B, Hq, T, _ = q.shape
        workspace = self._workspace(
            workspace, lambda: self.attention_prefill_workspace_bytes(B, Hq, T, t_end), q.device,
            stream)
        C.tvq_attention_prefill(self.handle, cache.data_ptr(), lay, layer, t_end, Hq, scale, dq,
                                q.data_ptr(), self._rows_desc(q), do, out.data_ptr(),
                                self._rows_desc(out), workspace.data_ptr(), workspace.numel(),
                                _stream_handle(stream))

    def attention_prefill_paged(self, pool, pool_lay: C.tvq_layout, block_table, ctx_lens,
                                max_ctx: int, layer: int, q, out, scale: float, q_lens=None,
                                workspace=None, stream=None) -> None:
        """attention_prefill over a paged pool: sequence b has q_lens[b] new tokens (all T without
        q_lens; rows behind them are not written), the last at position ctx_lens[b] - 1."""
        self._check_rows(q, out)
        _check_bytes(pool, pool_lay, "pool")
        _on_gpu(q, out, pool, block_table, ctx_lens)
        dq, do = self._io_dtypes(q, out)
        B, Hq, T, _ = q.shape
        if block_table.dim() != 2 or block_table.shape[0] != B or ctx_lens.shape != (B,) or \
                (q_lens is not None and q_lens.shape != (B,)):
            raise ValueError("block_table [B, max_blocks], ctx_lens [B] and q_lens [B] must match q")
        workspace = self._workspace(
            workspace, lambda: self.attention_prefill_workspace_bytes(B, Hq, T, max_ctx), q.device,
            stream)
        C.tvq_attention_prefill_paged(self.handle, pool.data_ptr(), pool_lay,
                                      self._i32(block_table, "block_table"), block_table.shape[1],
                                      self._i32(ctx_lens, "ctx_lens"), max_ctx,
                                      0 if q_lens is None else self._i32(q_lens, "q_lens"), layer,
                                      Hq, scale, dq, q.data_ptr(), self._rows_desc(q), do,
                                      out.data_ptr(), self._rows_desc(out), workspace.data_ptr(),
                                      workspace.numel(), _stream_handle(stream))

    # ---- part of a long context (tvq_key_bounds_paged / tvq_select_blocks / tvq_attention_blocks)
    def alloc_key_bounds(self, pool_lay: C.tvq_layout, device="cuda"):
        """Room for the key bounds of a pool, [L, n_blocks, H, 2, d] bf16 (lo, hi)."""
        import torch
        C.tvq_key_bounds_bytes(self.handle, pool_lay)        # refuses another codec's layout
        return torch.empty((self.L, pool_lay.batch, self.H, 2, self.d), dtype=torch.bfloat16,
                           device=device)

    def _check_bounds(self, bounds, pool_lay: C.tvq_layout) -> None:
        import torch
        want = (self.L, pool_lay.batch, self.H, 2, self.d)
        if bounds.dtype != torch.bfloat16 or bounds.shape != want or not bounds.is_contiguous():
            raise ValueError(f"bounds must be a contiguous bf16 GPU tensor of shape {want}")

    def key_bounds_paged(self, k, positions, block_table, bounds, pool_lay: C.tvq_layout,
                         stream=None) -> None:
        """Bring the key bounds of the pool's blocks up to date with the keys of an encode_paged
        call (the same k, positions and block_table)."""
        dt = _dtypes().get(k.dtype)
        if dt is None:
            raise ValueError("k must be bf16 or fp32")
        self._check_kv(k, "k")
        self._check_bounds(bounds, pool_lay)
        _on_gpu(k, bounds)
        desc, table = desc_of(k), block_table.shape
        if len(table) != 2 or table[0] != desc.batch or positions.shape != (desc.batch,):
            raise ValueError("positions [B] and block_table [B, max_blocks] must match k")
        C.tvq_key_bounds_paged(self.handle, dt, k.data_ptr(), desc,
                               self._i32(positions, "positions"),
                               self._i32(block_table, "block_table"), table[1],
                               bounds.data_ptr(), pool_lay, _stream_handle(stream))

    def select_blocks_workspace_bytes(self, batch: int, max_ctx: int, block_tokens: int) -> int:
        return C.tvq_select_blocks_workspace(self.handle, batch, max_ctx, block_tokens)

    def select_blocks(self, bounds, pool_lay: C.tvq_layout, block_table, ctx_lens, max_ctx: int,
                      layer: int, q, blocks, sel_lens, n_first: int = 1, n_last: int = 1,
                      workspace=None, stream=None) -> None:
        """For q ([B, Hq, d]) and each KV head, the blocks of the context whose keys can score
        highest, into blocks ([B, H, n_sel] int32, ascending, -1 behind them) and their tokens into
        sel_lens ([B, H] int32).  The first n_first and last n_last blocks are always among them."""
        shape, table, lists = q.shape, block_table.shape, blocks.shape
        if len(shape) != 3 or shape[2] != self.d or not q.is_contiguous():
            raise ValueError(f"q must be a contiguous [B, Hq, {self.d}] GPU tensor")
        self._check_bounds(bounds, pool_lay)
        _on_gpu(q, bounds, block_table, ctx_lens, blocks, sel_lens)
        dt = _dtypes().get(q.dtype)
        if dt is None:
            raise ValueError("q must be bf16 or fp32")
        B, Hq, _ = shape
        if len(table) != 2 or table[0] != B or ctx_lens.shape != (B,):
            raise ValueError("block_table [B, max_blocks] and ctx_lens [B] must match q")
        if len(lists) != 3 or lists[0] != B or lists[1] != self.H or sel_lens.shape != lists[:2]:
            raise ValueError("blocks [B, H, n_sel] and sel_lens [B, H] must match q and the codec")
        workspace = self._workspace(
            workspace, lambda: self.select_blocks_workspace_bytes(B, max_ctx,
                                                                  pool_lay.capacity_tokens),
            q.device, stream)
        C.tvq_select_blocks(self.handle, bounds.data_ptr(), pool_lay,
                            self._i32(block_table, "block_table"), table[1],
                            self._i32(ctx_lens, "ctx_lens"), max_ctx, B, layer, Hq, dt,
                            q.data_ptr(), lists[2], n_first, n_last,
                            self._i32(blocks, "blocks"), self._i32(sel_lens, "sel_lens"),
                            workspace.data_ptr(), workspace.numel(), _stream_handle(stream))

    def attention_blocks_workspace_bytes(self, batch: int, num_q_heads: int, n_sel: int,
                                         block_tokens: int) -> int:
        return C.tvq_attention_blocks_workspace(self.handle, batch, num_q_heads, n_sel,
                                                block_tokens)

    def attention_blocks(self, pool, pool_lay: C.tvq_layout, block_table, blocks, sel_lens,
                         layer: int, q, out, scale: float, workspace=None, stream=None) -> None:
        """Attention of q ([B, Hq, d]) over listed blocks: KV head h of sequence b attends to the
        first sel_lens[b, h] slots of blocks[b, h, 0], blocks[b, h, 1], ..."""
        self._check_q(q, out)
        _check_bytes(pool, pool_lay, "pool")
        _on_gpu(q, out, pool, block_table, blocks, sel_lens)
        dq, do = self._io_dtypes(q, out)
        (B, Hq, _), table, lists = q.shape, block_table.shape, blocks.shape
        if len(table) != 2 or table[0] != B:
            raise ValueError("block_table [B, max_blocks] must match q")
        if len(lists) != 3 or lists[0] != B or lists[1] != self.H or sel_lens.shape != lists[:2]:
            raise ValueError("blocks [B, H, n_sel] and sel_lens [B, H] must match q and the codec")
        n_sel = lists[2]
        workspace = self._workspace(
            workspace, lambda: self.attention_blocks_workspace_bytes(B, Hq, n_sel,
                                                                     pool_lay.capacity_tokens),
            q.device, stream)
        C.tvq_attention_blocks(self.handle, pool.data_ptr(), pool_lay,
                               self._i32(block_table, "block_table"), table[1],
                               self._i32(blocks, "blocks"), n_sel, self._i32(sel_lens, "sel_lens"),
                               B, layer, Hq, scale, dq, q.data_ptr(), do, out.data_ptr(),
                               workspace.data_ptr(), workspace.numel(), _stream_handle(stream))

    def bits_per_element(self, accounting: int = 0) -> float:
        return C.tvq_bits_per_element(self.handle, accounting)
