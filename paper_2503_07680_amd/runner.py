"""Plumbing around the C ABI: torch device buffers for one pack, plan upload, fwd/bwd calls.

Holds no arithmetic: planning happens in ``hbp_pack_plan`` and all attention math in the HIP
kernels.  Used by the tests, the smoke check and the benchmark.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B


class PackedAttention:
    """One packed buffer: plan on the host, buffers on ``cuda:0``, kernels through the C ABI."""

    def __init__(self, lengths: Sequence[int], pack_len: int, n_q_heads: int, n_kv_heads: int,
                 d_qk: int, d_v: int, softmax_scale: float = 0.0, device: str = "cuda:0",
                 with_profile: bool = False, fwd_tile_rows: Optional[int] = None, row_pad: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("PackedAttention needs a GPU: there is no CPU fallback")
        B.load_library()
        self.device = torch.device(device)
        self.rows_fwd = B.hbp_tile_rows(d_qk, d_v, B.HBP_FWD)
        self.rows_bwd = B.hbp_tile_rows(d_qk, d_v, B.HBP_BWD)
        self.cu, self.n_consumed, self.q_tiles, self.q_cost, self.pack_cost = B.hbp_pack_plan(
            lengths, pack_len, self.rows_fwd, B.HBP_TILES_QUERY)
        # the forward's own list when the head layout prefers larger query tiles (odd group sizes)
        self.rows_fwd_pref = B.hbp_fwd_tile_rows(B.AttnDesc(n_q_heads=n_q_heads, n_kv_heads=n_kv_heads,
                                                            d_qk=d_qk, d_v=d_v))
        self.fwd_tiles, self.fwd_cost = self.q_tiles, self.q_cost
        if fwd_tile_rows is None:
            fwd_tile_rows = self.rows_fwd_pref
        if fwd_tile_rows != self.rows_fwd:
            _, _, self.fwd_tiles, self.fwd_cost, _ = B.hbp_pack_plan(lengths, pack_len, fwd_tile_rows,
                                                                     B.HBP_TILES_QUERY)
        _, _, self.kv_tiles, self.kv_cost, _ = B.hbp_pack_plan(
            lengths, pack_len, self.rows_bwd, B.HBP_TILES_KEY)
        self.T = int(self.cu[-1])
        self.n_samples = len(self.cu) - 1
        self.Hq, self.Hkv, self.d_qk, self.d_v = n_q_heads, n_kv_heads, d_qk, d_v
        self.desc = B.AttnDesc(total_tokens=self.T, n_samples=self.n_samples, n_q_heads=n_q_heads,
                               n_kv_heads=n_kv_heads, d_qk=d_qk, d_v=d_v,
                               softmax_scale=float(softmax_scale),
                               fwd_tile_rows=0 if fwd_tile_rows == self.rows_fwd else int(fwd_tile_rows))
        # row_pad: extra elements (a multiple of 8) at the end of every token row of every tensor, so that
        # the row stride is not a power of two; 0 = dense [T, H, dim]
        self.row_pad = int(row_pad)
        if self.row_pad:
            self.desc.q_stride_t = n_q_heads * d_qk + self.row_pad
            self.desc.k_stride_t = n_kv_heads * d_qk + self.row_pad
            self.desc.v_stride_t = n_kv_heads * d_v + self.row_pad
            self.desc.o_stride_t = n_q_heads * d_v + self.row_pad
        dev = self.device
        # The plan's query tiles go to the GPU in the order in which they are best served.  8192 tokens in 20 samples,
        # 32/8 heads of 128, against the plan's order: forward 105 -> 91 us, dQ 106 -> 97.  The order depends on the
        # pack alone: sorted on the GPU in front of every call it cost launches of even tiles up to 13 % (16384 tokens
        # in 128 samples, 8 heads of 64: forward 33.8 -> 39.1 us) and the kernels the registers of the look-up.
        # One copy for all lists (16 bytes a tile, so every list starts on a tile's alignment).
        own_fwd = self.fwd_tiles is not self.q_tiles
        lists = [B.hbp_order_query_tiles(self.cu, self.q_tiles), self.kv_tiles]
        if own_fwd:
            lists.append(B.hbp_order_query_tiles(self.cu, self.fwd_tiles))
        n_tiles = [len(x) for x in lists]
        plan = torch.from_numpy(np.concatenate([x.ravel() for x in lists] + [self.cu])).to(dev)
        *on_gpu, self.cu_dev = plan.split([4 * n for n in n_tiles] + [len(self.cu)])
        self.q_tiles_dev, self.kv_tiles_dev, *rest = [x.view(-1, 4) for x in on_gpu]
        self.fwd_tiles_dev = rest[0] if own_fwd else self.q_tiles_dev
        self.ws_fwd = torch.empty(B.hbp_workspace_bytes(self.desc, B.HBP_FWD), dtype=torch.uint8, device=dev)
        self.ws_bwd = None
        self.prof_fwd = self.prof_bwd = self.prof_dq = None
        if with_profile:
            n = B.hbp_profile_capacity(self.desc, B.HBP_FWD)
            self.prof_fwd = torch.zeros(n * B.PROFILE_DTYPE.itemsize, dtype=torch.uint8, device=dev)
            n = B.hbp_profile_capacity(self.desc, B.HBP_BWD)
            self.prof_bwd = torch.zeros(n * B.PROFILE_DTYPE.itemsize, dtype=torch.uint8, device=dev)
            n = B.hbp_profile_capacity(self.desc, B.HBP_BWD_DQ)
            self.prof_dq = torch.zeros(n * B.PROFILE_DTYPE.itemsize, dtype=torch.uint8, device=dev)
        T = max(self.T, 1)
        bf = torch.bfloat16
        self.o = self.buffer(n_q_heads, d_v)
        self.lse = torch.zeros((n_q_heads, T), dtype=torch.float32, device=dev)
        self.dq = self.dk = self.dv = None

    # -- buffers ------------------------------------------------------------------------------
    def buffer(self, heads: int, dim: int) -> torch.Tensor:
        """Zeroed bf16 [T, heads, dim] tensor in this object's row layout (a view when rows are padded)."""
        T = max(self.T, 1)
        if not self.row_pad:
            return torch.zeros((T, heads, dim), dtype=torch.bfloat16, device=self.device)
        base = torch.zeros((T, heads * dim + self.row_pad), dtype=torch.bfloat16, device=self.device)
        return base[:, :heads * dim].view(T, heads, dim)

    # -- inputs -------------------------------------------------------------------------------
    def to_device_bf16(self, bits: np.ndarray) -> torch.Tensor:
        """uint16 bf16 bit patterns [T,H,dim] -> bf16 tensor on the device."""
        t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(self.device).view(torch.bfloat16)
        if not self.row_pad:
            return t
        out = self.buffer(t.shape[1], t.shape[2])
        out.copy_(t)
        return out

    # -- calls --------------------------------------------------------------------------------
    def _stream(self) -> int:
        return int(torch.cuda.current_stream(self.device).cuda_stream)

    def forward(self, q, k, v, profile: bool = False):
        B.hbp_varlen_attn_fwd(self.desc, q, k, v, self.cu_dev, self.fwd_tiles_dev, len(self.fwd_tiles),
                              self.o, self.lse, self.ws_fwd, self.prof_fwd if profile else None,
                              self._stream())
        return self.o, self.lse

    def alloc_backward(self):
        if self.ws_bwd is None:
            dev, bf, T = self.device, torch.bfloat16, max(self.T, 1)
            self.ws_bwd = torch.empty(B.hbp_workspace_bytes(self.desc, B.HBP_BWD), dtype=torch.uint8, device=dev)
            self.dq = self.buffer(self.Hq, self.d_qk)
            self.dk = self.buffer(self.Hkv, self.d_qk)
            self.dv = self.buffer(self.Hkv, self.d_v)

    def backward(self, q, k, v, d_o, profile: bool = False):
        self.alloc_backward()
        B.hbp_varlen_attn_bwd(self.desc, q, k, v, self.o, self.lse, d_o, self.cu_dev,
                              self.q_tiles_dev, len(self.q_tiles), self.kv_tiles_dev, len(self.kv_tiles),
                              self.dq, self.dk, self.dv, self.ws_bwd,
                              self.prof_bwd if profile else None, self.prof_dq if profile else None,
                              self._stream())
        return self.dq, self.dk, self.dv

    def profile_records(self, which: int) -> np.ndarray:
        buf = {B.HBP_FWD: self.prof_fwd, B.HBP_BWD: self.prof_bwd, B.HBP_BWD_DQ: self.prof_dq}[which]
        return np.frombuffer(buf.cpu().numpy().tobytes(), dtype=B.PROFILE_DTYPE)


_TYPES = {torch.bfloat16: B.HBP_BF16, torch.float32: B.HBP_F32}


def _check(name: str, t, device: torch.device, dtype, shape) -> None:
    """A tensor on the object's device, of the type and shape that it was made for; rows may have a stride."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.device == device:
        return
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise ValueError("%s: a tensor on %s is wanted" % (name, device))
    raise ValueError("%s: %s %s is wanted, got %s %s" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))


def _on(device: torch.device, call, *args) -> None:
    """``call(*args, stream)`` on the device's current stream, the device being the current one meanwhile.  The stream's
    raw handle and a look at the current device: 0.4 us a call, 3.4 with a torch.cuda.Stream and a device context."""
    stream = torch._C._cuda_getCurrentRawStream(device.index)
    if torch.cuda.current_device() == device.index:
        call(*args, stream)
    else:
        with torch.cuda.device(device):
            call(*args, stream)


def _device(device) -> torch.device:
    if not torch.cuda.is_available():
        raise RuntimeError("a GPU is needed: there is no CPU fallback")
    B.load_library()
    d = torch.device(device)
    return d if d.index is not None else torch.device(d.type, torch.cuda.current_device())


class PackedCrossAttention:
    """Cross attention of a pack: the query rows of sample i (``q_lengths[i]`` of them) attend to all of its
    ``kv_lengths[i]`` keys; both sides packed, either may be empty for a sample.  Plans on the host, calls on the
    device's current stream; like PackedAttention the object holds its outputs, the next call writes them again."""

    def __init__(self, q_lengths: Sequence[int], kv_lengths: Sequence[int], n_q_heads: int, n_kv_heads: int,
                 d_qk: int, d_v: int, softmax_scale: float = 0.0, device: str = "cuda:0"):
        self.device = _device(device)
        self.Hq, self.Hkv, self.d_qk, self.d_v = int(n_q_heads), int(n_kv_heads), int(d_qk), int(d_v)
        self.Tq, self.Tk = int(sum(q_lengths)), int(sum(kv_lengths))
        self.desc = B.CrossDesc(total_queries=self.Tq, total_keys=self.Tk, n_samples=len(q_lengths),
                                n_q_heads=self.Hq, n_kv_heads=self.Hkv, d_qk=self.d_qk, d_v=self.d_v,
                                softmax_scale=float(softmax_scale),
                                longest_keys=max((int(k) for q, k in zip(q_lengths, kv_lengths) if q), default=0),
                                longest_queries=max((int(q) for q, k in zip(q_lengths, kv_lengths) if k), default=0))
        self.cu_q, self.cu_kv, q_tiles, self.pairs = B.hbp_cross_plan(
            q_lengths, kv_lengths, B.hbp_cross_tile_rows(self.desc, B.HBP_FWD), B.HBP_TILES_QUERY)
        _, _, kv_tiles, _ = B.hbp_cross_plan(
            q_lengths, kv_lengths, B.hbp_cross_tile_rows(self.desc, B.HBP_BWD), B.HBP_TILES_KEY)
        self.n_q_tiles, self.n_kv_tiles = len(q_tiles), len(kv_tiles)
        self.desc.pairs = self.pairs
        # one copy; 16 bytes a tile, so both lists start on a tile's alignment
        plan = torch.from_numpy(np.concatenate([q_tiles.ravel(), kv_tiles.ravel(), self.cu_q, self.cu_kv])).to(self.device)
        self.q_tiles_dev, self.kv_tiles_dev, self.cu_q_dev, self.cu_kv_dev = plan.split(
            [q_tiles.size, kv_tiles.size, self.cu_q.size, self.cu_kv.size])
        dev, bf = self.device, torch.bfloat16
        self.o = torch.empty((self.Tq, self.Hq, self.d_v), dtype=bf, device=dev)
        self.lse = torch.empty((self.Hq, self.Tq), dtype=torch.float32, device=dev)
        self.ws_fwd = torch.empty(B.hbp_cross_workspace_bytes(self.desc, B.HBP_FWD), dtype=torch.uint8, device=dev)
        self.ws_bwd = self.dq = self.dk = self.dv = None

    def _dense(self, name: str, t: torch.Tensor, shape) -> None:
        _check(name, t, self.device, torch.bfloat16, shape)
        if not t.is_contiguous():
            raise ValueError("%s: a contiguous tensor is wanted" % name)

    def _inputs(self, q, k, v) -> None:
        self._dense("q", q, (self.Tq, self.Hq, self.d_qk))
        self._dense("k", k, (self.Tk, self.Hkv, self.d_qk))
        self._dense("v", v, (self.Tk, self.Hkv, self.d_v))

    def forward(self, q, k, v):
        """(o [Tq, Hq, d_v], lse [Hq, Tq]); rows of a sample without keys: zeros and -inf."""
        self._inputs(q, k, v)
        _on(self.device, B.hbp_cross_attn_fwd, self.desc, q, k, v, self.cu_q_dev, self.cu_kv_dev, self.q_tiles_dev,
            self.n_q_tiles, self.o, self.lse, self.ws_fwd)
        return self.o, self.lse

    def alloc_backward(self):
        if self.ws_bwd is None:
            dev, bf = self.device, torch.bfloat16
            self.ws_bwd = torch.empty(B.hbp_cross_workspace_bytes(self.desc, B.HBP_BWD), dtype=torch.uint8, device=dev)
            self.dq = torch.empty((self.Tq, self.Hq, self.d_qk), dtype=bf, device=dev)
            self.dk = torch.empty((self.Tk, self.Hkv, self.d_qk), dtype=bf, device=dev)
            self.dv = torch.empty((self.Tk, self.Hkv, self.d_v), dtype=bf, device=dev)

    def backward(self, q, k, v, d_o):
        """(dq, dk, dv) of the last forward."""
        self._inputs(q, k, v)
        self._dense("d_o", d_o, (self.Tq, self.Hq, self.d_v))
        self.alloc_backward()
        _on(self.device, B.hbp_cross_attn_bwd, self.desc, q, k, v, self.o, self.lse, d_o, self.cu_q_dev, self.cu_kv_dev,
            self.q_tiles_dev, self.n_q_tiles, self.kv_tiles_dev, self.n_kv_tiles, self.dq, self.dk, self.dv, self.ws_bwd)
        return self.dq, self.dk, self.dv


class PackedEmbedding:
    """Token embedding of packs of ``total_tokens`` tokens, and its gradient.  Tokens are int32; one outside
    [0, vocab) is none: a row of zeros, no gradient.  Calls run on the device's current stream."""

    def __init__(self, total_tokens: int, vocab: int, dim: int, scale: float = 1.0,
                 table_type: torch.dtype = torch.bfloat16, out_type: torch.dtype = torch.bfloat16,
                 device: str = "cuda:0"):
        if table_type not in _TYPES or out_type not in _TYPES:
            raise ValueError("types: torch.bfloat16 or torch.float32")
        self.device = _device(device)
        self.T, self.vocab, self.dim = int(total_tokens), int(vocab), int(dim)
        self.table_type, self.out_type = table_type, out_type
        self.desc = B.EmbedDesc(total_tokens=self.T, vocab=self.vocab, dim=self.dim, table_type=_TYPES[table_type],
                                row_type=_TYPES[out_type], scale=float(scale))
        self.ws_bytes = B.hbp_embed_bwd_workspace_bytes(self.desc)
        self.strides = (0, 0)  # the descriptor's
        self.ws = self.out = None

    def _rows(self, name: str, t: torch.Tensor, dtype, n: int) -> int:
        """Stride of [n, dim] rows in elements; overlapping or scattered rows are refused."""
        _check(name, t, self.device, dtype, (n, self.dim))
        row, column = t.stride()
        if (self.dim > 1 and column != 1) or (n > 1 and row < self.dim):
            raise ValueError("%s: rows of adjacent elements are wanted" % name)
        return row if n > 1 else self.dim

    def _operands(self, table: torch.Tensor, rows: torch.Tensor, tokens: torch.Tensor) -> None:
        _check("tokens", tokens, self.device, torch.int32, (self.T,))
        if not tokens.is_contiguous():
            raise ValueError("tokens: a contiguous tensor is wanted")
        strides = (self._rows("table", table, self.table_type, self.vocab), self._rows("rows", rows, self.out_type, self.T))
        if strides != self.strides:
            self.desc.table_stride, self.desc.row_stride = self.strides = strides

    def forward(self, table: torch.Tensor, tokens: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """scale * table[tokens]; into this object's buffer unless ``out`` is given."""
        if out is None:
            if self.out is None:
                self.out = torch.empty((self.T, self.dim), dtype=self.out_type, device=self.device)
            out = self.out
        self._operands(table, out, tokens)
        _on(self.device, B.hbp_embed_fwd, self.desc, table, tokens, out)
        return out

    def backward(self, d_out: torch.Tensor, tokens: torch.Tensor, d_table: torch.Tensor,
                 accumulate: bool = False) -> torch.Tensor:
        """The table's gradient into ``d_table``, added to what it holds with ``accumulate``."""
        self._operands(d_table, d_out, tokens)
        if self.ws is None:
            self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
        _on(self.device, B.hbp_embed_bwd, self.desc, d_out, tokens, accumulate, d_table, self.ws)
        return d_table


class GradientClip:
    """The norm of a list of gradients over all their elements, and clipping to it, in place or into ``outs``.  The
    tensors (contiguous, bf16 or fp32) are held and named by their addresses: make another object when the list
    changes."""

    def __init__(self, tensors: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None,
                 device: str = "cuda:0"):
        self.device = _device(device)
        self.tensors, self.outs = list(tensors), None if outs is None else list(outs)
        if self.outs is not None and len(self.outs) != len(self.tensors):
            raise ValueError("outs: one for each tensor")
        for i, t in enumerate(self.tensors + (self.outs or [])):
            like = self.tensors[i % max(1, len(self.tensors))]
            if not isinstance(t, torch.Tensor) or t.device != self.device or t.dtype not in _TYPES or not t.is_contiguous():
                raise ValueError("gradients: contiguous bf16 or fp32 tensors on %s are wanted" % self.device)
            if t.dtype != like.dtype or t.shape != like.shape:
                raise ValueError("outs: the tensors' types and shapes are wanted")
        self.list = B.GradList([t.data_ptr() for t in self.tensors], [t.numel() for t in self.tensors],
                               [_TYPES[t.dtype] for t in self.tensors],
                               None if self.outs is None else [t.data_ptr() for t in self.outs])
        self.sumsq_buf = torch.zeros(1, dtype=torch.float64, device=self.device)
        self.norm = torch.zeros((), dtype=torch.float32, device=self.device)
        self.ws = torch.empty(B.hbp_grad_workspace_bytes(self.list.n), dtype=torch.uint8, device=self.device)

    def sumsq(self, accumulate: bool = False) -> torch.Tensor:
        """Sum of the squares of all elements (fp64, on the device); ranks with different gradients add it up before
        ``clip_with``."""
        _on(self.device, B.hbp_grad_sumsq, self.list, accumulate, self.sumsq_buf, self.ws)
        return self.sumsq_buf

    def clip_with(self, sumsq: torch.Tensor, max_norm: float) -> torch.Tensor:
        """Clips to ``max_norm``, the sum of squares given; returns the norm (fp32, on the device)."""
        _check("sumsq", sumsq, self.device, torch.float64, (1,))
        _on(self.device, B.hbp_grad_clip, self.list, sumsq, max_norm, self.norm)
        return self.norm

    def clip(self, max_norm: float) -> torch.Tensor:
        """Norm of this object's tensors, and clipping to it; returns the norm (fp32, on the device)."""
        _on(self.device, B.hbp_grad_clip_norm, self.list, max_norm, self.sumsq_buf, self.norm, self.ws)
        return self.norm


def bf16_tensor_to_f32_numpy(t: torch.Tensor) -> np.ndarray:
    return t.detach().float().cpu().numpy()
