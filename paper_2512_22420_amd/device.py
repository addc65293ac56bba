"""Device-memory plumbing for the binding: upload a model, a paged cache and a
step's inputs as torch tensors and build the C structs that point at them.
PyTorch is used for allocation and streams only; all compute is in the HIP
library.
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional

import numpy as np
import torch

from . import binding as nb


def _to_dev(a, device) -> torch.Tensor:
    if isinstance(a, torch.Tensor):  # already resident (bf16 bits as int16, or fp32/int32)
        return a
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    return torch.from_numpy(a).to(device)


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def pack_weight(w: torch.Tensor, stream: Optional[int] = None) -> torch.Tensor:
    """Packed copy (the layout of nightjar_pack_weight) of a bf16 [N][K]
    weight matrix resident on the device as int16 bits."""
    N, K = w.shape
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    out = torch.empty(nb.packed_weight_elems(N, K), dtype=torch.int16, device=w.device)
    nb.pack_weight(w.data_ptr(), out.data_ptr(), N, K, s)
    return out


def model_desc(shape) -> nb.ModelDesc:
    return nb.ModelDesc(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.head_dim,
                        shape.ffn_dim, shape.vocab, shape.block_size, shape.rms_eps, shape.rope_theta,
                        nb.NJ_BF16 if shape.dtype == "bf16" else nb.NJ_F32)


class DeviceModel:
    """Weights resident on the device, plus the descriptor structs."""

    def __init__(self, shape, weights: Dict, device="cuda"):
        self.shape = shape
        self.desc = model_desc(shape)
        # bf16 GEMM weights go to the packed layout the GEMM kernels read
        mat = (lambda a: pack_weight(_to_dev(a, device))) if shape.dtype == "bf16" else (lambda a: _to_dev(a, device))
        self.embed = _to_dev(weights["embed"], device)
        self.final_norm = _to_dev(weights["final_norm"], device)
        self.lm_head = mat(weights["lm_head"])
        names = ("attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gate_up", "w_down")
        self.layers = [{n: (mat(lw[n]) if n.startswith("w_") else _to_dev(lw[n], device)) for n in names}
                       for lw in weights["layers"]]
        self._c_layers = (nb.LayerWeights * shape.n_layers)(
            *[nb.LayerWeights(*[_ptr(l[n]) for n in names]) for l in self.layers])
        self.c = nb.Weights(_ptr(self.embed), _ptr(self.final_norm), _ptr(self.lm_head),
                            ctypes.cast(self._c_layers, ctypes.POINTER(nb.LayerWeights)))


class DeviceCache:
    """Paged KV cache and block table on the device."""

    def __init__(self, ctx: Dict, device="cuda"):
        self.k_pages = [_to_dev(a, device) for a in ctx["k_pages"]]
        self.v_pages = [_to_dev(a, device) for a in ctx["v_pages"]]
        self.block_table = _to_dev(ctx["block_table"], device)
        self.context_lens = _to_dev(ctx["context_lens"], device)
        self.num_blocks = int(ctx["num_blocks"])
        self.max_blocks = int(ctx["block_table"].shape[1])
        self._kp = (ctypes.c_void_p * len(self.k_pages))(*[_ptr(t) for t in self.k_pages])
        self._vp = (ctypes.c_void_p * len(self.v_pages))(*[_ptr(t) for t in self.v_pages])
        self.c = nb.KvCache(ctypes.cast(self._kp, ctypes.POINTER(ctypes.c_void_p)),
                            ctypes.cast(self._vp, ctypes.POINTER(ctypes.c_void_p)), self.num_blocks)


class Workspace:
    def __init__(self, shape, max_B: int, max_k: int, device="cuda", stream: int = 0):
        self.nbytes = nb.workspace_bytes(model_desc(shape), max_B, max_k)
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        nb.workspace_init(self.ptr, self.nbytes, stream)

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr()


class StepIO:
    """One step's inputs and outputs on the device."""

    def __init__(self, shape, drafts: Dict, device="cuda", keep_logits: bool = True):
        B, k = drafts["draft_tokens"].shape
        self.B, self.k = B, k
        self.last_tokens = _to_dev(drafts["last_tokens"], device)
        self.draft_tokens = _to_dev(drafts["draft_tokens"], device) if k else None
        self.draft_probs = _to_dev(drafts["draft_probs"], device) if k else None
        self.uniforms = _to_dev(drafts["uniforms"], device)
        self.accepted_len = torch.full((B,), -7, dtype=torch.int32, device=device)
        self.next_tokens = torch.full((B, k + 1), -7, dtype=torch.int32, device=device)
        self.logits = torch.empty((B, k + 1, shape.vocab), dtype=torch.float32, device=device) if keep_logits else None


def _expect(t: Optional[torch.Tensor], dtype, numel: int, name: str) -> None:
    """The C ABI takes raw pointers: a tensor of another dtype or size would be
    reinterpreted, so it is refused here."""
    if t is None:
        return
    if t.dtype != dtype or t.numel() != numel or not t.is_contiguous():
        raise TypeError(f"{name}: need a contiguous {dtype} tensor of {numel} elements, "
                        f"got {t.dtype} {tuple(t.shape)}")


def verify(model: DeviceModel, cache: DeviceCache, io: StepIO, ws: Workspace, stream: Optional[int] = None):
    B, k, V = io.B, io.k, model.shape.vocab
    _expect(io.last_tokens, torch.int32, B, "last_tokens")
    _expect(io.draft_tokens, torch.int32, B * k, "draft_tokens")
    _expect(io.draft_probs, torch.float32, B * k * V, "draft_probs")
    _expect(io.uniforms, torch.float32, B * (k + 1), "uniforms")
    _expect(io.accepted_len, torch.int32, B, "accepted_len")
    _expect(io.next_tokens, torch.int32, B * (k + 1), "next_tokens")
    _expect(io.logits, torch.float32, B * (k + 1) * V, "logits")
    _expect(cache.context_lens, torch.int32, B, "context_lens")
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    nb.verify_step(model.desc, model.c, cache.c, _ptr(cache.block_table), cache.max_blocks, _ptr(cache.context_lens),
                   _ptr(io.last_tokens), _ptr(io.draft_tokens), _ptr(io.draft_probs), _ptr(io.uniforms), io.B, io.k,
                   _ptr(io.accepted_len), _ptr(io.next_tokens), _ptr(io.logits), ws.ptr, ws.nbytes, s)


def kv_append(model: DeviceModel, cache: DeviceCache, io: StepIO, ws: Workspace, stream: Optional[int] = None):
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    nb.kv_append(model.desc, cache.c, _ptr(cache.block_table), cache.max_blocks, _ptr(cache.context_lens),
                 _ptr(io.accepted_len), io.B, io.k, ws.ptr, ws.nbytes, s)


def device_error(ws: Workspace, stream: Optional[int] = None) -> int:
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    return nb.device_error(ws.ptr, ws.nbytes, s)


def _stream_on(stream: Optional[int], *tensors) -> int:
    """The stream to enqueue on: the given one, or the current one.  The kernels read these tensors where they are: all
    on the current GPU.  (No torch.device or torch.cuda.Stream is built: either takes longer than the checks.)"""
    dev = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise TypeError(f"need tensors on the current GPU (cuda:{dev}), got one on {t.device}")
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream


class KvLayer:
    """One layer's paged cache for the chunk calls: k [num_blocks][Hkv][16][D] and
    v [num_blocks][Hkv][D][16], fp32, bf16 (or its bits as int16), or e4m3 codes
    as uint8 with a scale byte per (block, head, slot)."""

    _DTYPES = {torch.float32: nb.NJ_F32, torch.bfloat16: nb.NJ_BF16, torch.int16: nb.NJ_BF16, torch.uint8: nb.NJ_E4M3}

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        if k.dtype not in self._DTYPES or v.dtype != k.dtype or k.dim() != 4 or v.dim() != 4:
            raise TypeError("k and v: need 4-d tensors of one page type (float32, bfloat16 or int16 bits, uint8 codes)")
        nb_, hkv, bs, D = k.shape
        if tuple(v.shape) != (nb_, hkv, D, bs):
            raise TypeError(f"v: need shape {(nb_, hkv, D, bs)}, got {tuple(v.shape)}")
        for t, n in ((k, "k"), (v, "v")):
            _expect(t, k.dtype, nb_ * hkv * bs * D, n)
        if (k.dtype == torch.uint8) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            raise TypeError("k_scale and v_scale: needed for e4m3 pages, and for no others")
        for t, n in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _expect(t, torch.uint8, nb_ * hkv * bs, n)
        if any(t is not None and t.device != k.device for t in (v, k_scale, v_scale)):
            raise TypeError("k, v and their scales: need one device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.hkv, self.head_dim = hkv, D
        self.c = nb.KvLayer(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), nb_, self._DTYPES[k.dtype])


class ChunkBatch:
    """A ragged batch of chunks (nj_chunk_batch)."""

    def __init__(self, starts: torch.Tensor, context_lens: torch.Tensor, block_table: torch.Tensor, rows: int,
                 max_chunk: int):
        B = context_lens.numel()
        _expect(starts, torch.int32, B + 1, "starts")
        _expect(context_lens, torch.int32, B, "context_lens")
        _expect(block_table, torch.int32, B * block_table.shape[-1], "block_table")
        if starts.device != context_lens.device or starts.device != block_table.device:
            raise TypeError("starts, context_lens and block_table: need one device")
        self.starts, self.context_lens, self.block_table = starts, context_lens, block_table
        self.B, self.rows, self.max_chunk = B, rows, max_chunk
        self.c = nb.ChunkBatch(_ptr(starts), _ptr(context_lens), _ptr(block_table), block_table.shape[-1], B, rows,
                               max_chunk)


class Scratch:
    """A caller-owned workspace, prepared for its calls."""

    def __init__(self, nbytes: int, device="cuda", stream: Optional[int] = None):
        self.nbytes = nbytes
        self.buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.ptr = self.buf.data_ptr()
        nb.workspace_init(self.ptr, nbytes, torch.cuda.current_stream().cuda_stream if stream is None else stream)


def chunk_workspace(desc, batch: ChunkBatch, device="cuda", stream: Optional[int] = None) -> Scratch:
    """A workspace for the chunk calls on this batch and every smaller one."""
    return Scratch(nb.chunk_attn_workspace_bytes(desc, batch.B, batch.rows, batch.max_chunk), device, stream)


def sample_workspace(rows: int, vocab: int, device="cuda", stream: Optional[int] = None) -> Scratch:
    return Scratch(nb.sample_workspace_bytes(rows, vocab), device, stream)


def _expect_row(t: torch.Tensor, desc, numel: int, name: str) -> None:
    if desc.dtype == nb.NJ_F32:
        _expect(t, torch.float32, numel, name)
    else:
        _expect(t, torch.int16 if t.dtype == torch.int16 else torch.bfloat16, numel, name)


def _expect_layer(desc, layer: KvLayer) -> None:
    if (layer.hkv, layer.head_dim) != (desc.n_kv_heads, desc.head_dim):
        raise TypeError(f"cache: need {desc.n_kv_heads} KV heads of {desc.head_dim} dims, got {layer.hkv} of {layer.head_dim}")


def chunk_store(desc, layer: KvLayer, batch: ChunkBatch, qkv: torch.Tensor, ws: Scratch,
                q_out: Optional[torch.Tensor] = None, stream: Optional[int] = None):
    """RoPE on the chunk's q and k, its K and V into the pages (nightjar_chunk_store).  qkv: fp32
    [rows, (H + 2 Hkv) * D], rows may be strided."""
    width = (desc.n_heads + 2 * desc.n_kv_heads) * desc.head_dim
    if qkv.dtype != torch.float32 or tuple(qkv.shape) != (batch.rows, width) or qkv.stride(1) != 1:
        raise TypeError(f"qkv: need a float32 tensor [{batch.rows}, {width}] with contiguous rows, got {qkv.dtype} {tuple(qkv.shape)}")
    _expect_layer(desc, layer)
    if q_out is not None:
        _expect_row(q_out, desc, batch.rows * desc.n_heads * desc.head_dim, "q_out")
    s = _stream_on(stream, qkv, q_out, layer.k, batch.starts, ws.buf)
    nb.chunk_store(desc, layer.c, batch.c, qkv.data_ptr(), qkv.stride(0) if batch.rows > 1 else width, _ptr(q_out),
                   ws.ptr, ws.nbytes, s)


def chunk_load(desc, layer: KvLayer, batch: ChunkBatch, k_out: torch.Tensor, v_out: torch.Tensor, ws: Scratch,
               stream: Optional[int] = None):
    """The chunk's K and V rows read back from the pages (nightjar_chunk_load)."""
    _expect_layer(desc, layer)
    for t, n in ((k_out, "k_out"), (v_out, "v_out")):
        _expect_row(t, desc, batch.rows * desc.n_kv_heads * desc.head_dim, n)
    s = _stream_on(stream, k_out, v_out, layer.k, batch.starts, ws.buf)
    nb.chunk_load(desc, layer.c, batch.c, k_out.data_ptr(), v_out.data_ptr(), ws.ptr, ws.nbytes, s)


def chunk_attn(desc, layer: KvLayer, batch: ChunkBatch, q: torch.Tensor, out: torch.Tensor, ws: Scratch,
               stream: Optional[int] = None):
    """Attention of the chunk's rows over the paged cache (nightjar_chunk_attn)."""
    _expect_layer(desc, layer)
    for t, n in ((q, "q"), (out, "out")):
        _expect_row(t, desc, batch.rows * desc.n_heads * desc.head_dim, n)
    s = _stream_on(stream, q, out, layer.k, batch.starts, ws.buf)
    nb.chunk_attn(desc, layer.c, batch.c, q.data_ptr(), out.data_ptr(), ws.ptr, ws.nbytes, s)


def sample(logits: torch.Tensor, uniforms: torch.Tensor, tokens: torch.Tensor, ws: Scratch,
           temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
           top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
           probs: Optional[torch.Tensor] = None, stream: Optional[int] = None):
    """One token per row of logits (nightjar_sample).  logits and probs: fp32 [rows, vocab], rows may be strided."""
    if logits.dim() != 2:
        raise TypeError(f"logits: need [rows, vocab], got {tuple(logits.shape)}")
    R, V = logits.shape
    for t, n in ((logits, "logits"), (probs, "probs")):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (R, V) or (V > 1 and t.stride(1) != 1)):
            raise TypeError(f"{n}: need a float32 tensor [{R}, {V}] with contiguous rows, got {t.dtype} {tuple(t.shape)}")
    for t, n in ((uniforms, "uniforms"), (temperature, "temperature"), (top_p, "top_p"), (min_p, "min_p")):
        _expect(t, torch.float32, R, n)
    _expect(tokens, torch.int32, R, "tokens")
    _expect(top_k, torch.int32, R, "top_k")
    s = _stream_on(stream, logits, uniforms, tokens, temperature, top_k, top_p, min_p, probs, ws.buf)
    nb.sample(logits.data_ptr(), logits.stride(0) if R > 1 else V, R, V, _ptr(temperature), _ptr(top_k), _ptr(top_p),
              _ptr(min_p), _ptr(uniforms), _ptr(tokens), _ptr(probs), 0 if probs is None else probs.stride(0) if R > 1 else V,
              ws.ptr, ws.nbytes, s)
