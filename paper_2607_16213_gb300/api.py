"""Torch-facing helpers around the C ABI: allocate device tensors and workspaces with torch,
then call selkv_compress / selkv_decode_attn.  No arithmetic of the method happens here."""
from __future__ import annotations

import contextlib
import math
from dataclasses import dataclass, field
from typing import Optional, Sequence

import torch

from . import _binding as B

_TORCH_DTYPE = {B.SELKV_BF16: torch.bfloat16, B.SELKV_FP32: torch.float32}
_DTYPE_CODE = {"bf16": B.SELKV_BF16, "fp32": B.SELKV_FP32}


def dtype_code(name: str) -> int:
    return _DTYPE_CODE[name]


def torch_dtype(code: int) -> torch.dtype:
    return _TORCH_DTYPE[code]


def make_shape(dtype: str, batch: int, num_q_heads: int, num_kv_heads: int, head_dim: int,
               obs_window: int, n_cap: int, m_cap: int) -> B.selkv_shape:
    return B.selkv_shape(_DTYPE_CODE[dtype], batch, num_q_heads, num_kv_heads, head_dim,
                         obs_window, n_cap, m_cap)


def capacity(n_max: int, rho: float, extra: int = 0, align: int = 64) -> int:
    """A row capacity that holds floor(rho * n_max) compressed rows plus `extra` appended rows."""
    need = int(math.floor(float(rho) * float(n_max))) + extra
    return max(align, ((need + align - 1) // align) * align)


class Workspace:
    """A zero-initialised device workspace of at least `nbytes` (256-byte aligned)."""

    def __init__(self, nbytes: int, device="cuda", stream=None):
        self.nbytes = max(256, int(nbytes))
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        B.check(B.selkv_workspace_init(self.buf, self.nbytes, stream), "selkv_workspace_init")

    def ptr(self) -> int:
        return self.buf.data_ptr()

    def errors(self, stream=None) -> int:
        st, flags = B.selkv_workspace_error(self.buf, stream)
        return flags


@dataclass
class CompressedCache:
    shape: B.selkv_shape
    K_c: torch.Tensor
    V_c: torch.Tensor
    bias: torch.Tensor
    lengths: torch.Tensor
    debug: dict = field(default_factory=dict)


def alloc_compressed(shape: B.selkv_shape, device="cuda") -> CompressedCache:
    dt = _TORCH_DTYPE[shape.dtype]
    Bn, H, m, d = shape.batch, shape.num_kv_heads, shape.m_cap, shape.head_dim
    return CompressedCache(shape=shape,
                           K_c=torch.zeros((Bn, H, m, d), dtype=dt, device=device),
                           V_c=torch.zeros((Bn, H, m, d), dtype=dt, device=device),
                           bias=torch.zeros((Bn, H, m), dtype=torch.float32, device=device),
                           lengths=torch.zeros((Bn,), dtype=torch.int32, device=device))


def alloc_debug(shape: B.selkv_shape, device="cuda", per_head: bool = False) -> dict:
    """Debug outputs of selkv_compress (kept_idx is per KV head in the per-head mode)."""
    Bn, H, n, m = shape.batch, shape.num_kv_heads, shape.n_cap, shape.m_cap
    return dict(
        attn=torch.zeros((Bn, H, n), dtype=torch.float32, device=device),
        score=torch.zeros((Bn, H, n), dtype=torch.float32, device=device),
        topk=torch.zeros((Bn, H, n), dtype=torch.uint8, device=device),
        kept_idx=torch.full((Bn, H, m) if per_head else (Bn, m), -1, dtype=torch.int32, device=device),
        target=torch.full((Bn, H, n), -7, dtype=torch.int32, device=device),
        gate=torch.zeros((Bn, H, n), dtype=torch.float32, device=device),
        decision=torch.full((Bn, H, n), 9, dtype=torch.uint8, device=device),
        ratio=torch.zeros((Bn, H, m), dtype=torch.float32, device=device),
    )


def compress(shape: B.selkv_shape, n_len: Sequence[int], rho: float, K: torch.Tensor,
             V: torch.Tensor, Q_obs: torch.Tensor, params: Optional[B.selkv_params] = None,
             out: Optional[CompressedCache] = None, debug: bool = False,
             workspace: Optional[Workspace] = None, stream=None) -> CompressedCache:
    """selkv_compress on device tensors; returns the compressed cache (and debug outputs)."""
    params = params or B.selkv_params.defaults()
    out = out or alloc_compressed(shape, K.device)
    dbg = alloc_debug(shape, K.device, per_head=params.select_mode == B.SELKV_SELECT_PER_HEAD) if debug else None
    ws = workspace or Workspace(B.selkv_compress_workspace_size(shape), K.device, stream)
    st = B.selkv_compress(shape, n_len, rho, params, K, V, Q_obs, out.K_c, out.V_c, out.bias,
                          out.lengths, dbg, ws.buf, ws.nbytes, stream)
    B.check(st, "selkv_compress")
    if dbg is not None:
        out.debug = dbg
    return out


def decode(cache: CompressedCache, q: torch.Tensor, k_new: Optional[torch.Tensor] = None,
           v_new: Optional[torch.Tensor] = None, use_bias: bool = True,
           out: Optional[torch.Tensor] = None, workspace: Optional[Workspace] = None,
           stream=None) -> torch.Tensor:
    """selkv_decode_attn over a compressed cache (optionally appending k_new / v_new)."""
    shape = cache.shape
    out = out if out is not None else torch.empty_like(q)
    ws = workspace or Workspace(B.selkv_decode_workspace_size(shape), q.device, stream)
    st = B.selkv_decode_attn(shape, q, cache.K_c, cache.V_c, cache.bias if use_bias else None,
                             cache.lengths, k_new, v_new, out, ws.buf, ws.nbytes, stream)
    B.check(st, "selkv_decode_attn")
    return out


# ---- caches held in 8 bits ----------------------------------------------------------------------
_QTYPE = {"e4m3": B.SELKV_Q_E4M3, "int8": B.SELKV_Q_INT8}
_CODE_DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _bad(what: str) -> None:
    raise B.SelKVError(B.SELKV_ERR_INVALID_ARG, what)


def _tensor(t: torch.Tensor, name: str, shape, dtype, device) -> None:
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device.index or not t.is_contiguous():
        _bad("%s: a contiguous %s tensor %s on %s is wanted, not %s %s on %s"
             % (name, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))


@dataclass(frozen=True, eq=False)
class QuantCache:
    """A cache held in 8 bits (see selkv_qcache in include/selkv.h): codes [B][Hkv][m_cap][d] in
    float8_e4m3fn ("e4m3") or int8 ("int8"), a scale for each `block` rows, compensation per row or
    None, and the rows held.  Contiguous tensors of one device, looked over once: they are written in
    place, not replaced."""
    shape: B.selkv_shape
    cache_type: str
    block: int
    K: torch.Tensor
    V: torch.Tensor
    K_scale: torch.Tensor
    V_scale: torch.Tensor
    bias: Optional[torch.Tensor]
    lengths: torch.Tensor

    def __post_init__(self):
        s = self.shape
        if self.cache_type not in _QTYPE or self.block not in (16, 32, 64, 128):
            _bad("QuantCache: cache_type is e4m3 or int8, block 16, 32, 64 or 128")
        dev, code = self.K.device, _CODE_DTYPE[self.cache_type]
        if dev.type != "cuda":
            _bad("QuantCache: tensors of a CUDA device")
        rows = (s.batch, s.num_kv_heads, s.m_cap)
        scales = (s.batch, s.num_kv_heads, -(-s.m_cap // self.block))
        for name, t, want, dt in (("K", self.K, rows + (s.head_dim,), code), ("V", self.V, rows + (s.head_dim,), code),
                                  ("K_scale", self.K_scale, scales, torch.float32),
                                  ("V_scale", self.V_scale, scales, torch.float32),
                                  ("bias", self.bias, rows, torch.float32), ("lengths", self.lengths, (s.batch,), torch.int32)):
            if t is not None or name != "bias":
                _tensor(t, "QuantCache." + name, want, dt, dev)
        for name, x in (("_dtype", _TORCH_DTYPE[s.dtype]), ("_bias", self._struct(self.bias)), ("_plain", self._struct(None))):
            object.__setattr__(self, name, x)

    def _struct(self, bias) -> B.selkv_qcache:
        return B.selkv_qcache(_QTYPE[self.cache_type], self.block, self.K.data_ptr(), self.V.data_ptr(),
                              self.K_scale.data_ptr(), self.V_scale.data_ptr(),
                              bias.data_ptr() if bias is not None else None, self.lengths.data_ptr())


def alloc_quant(shape: B.selkv_shape, cache_type: str = "e4m3", block: int = 64, bias: bool = True,
                device="cuda") -> QuantCache:
    """An empty 8-bit cache."""
    if cache_type not in _QTYPE or block not in (16, 32, 64, 128):
        _bad("alloc_quant: cache_type is e4m3 or int8, block 16, 32, 64 or 128")
    rows = (shape.batch, shape.num_kv_heads, shape.m_cap)
    scales = (shape.batch, shape.num_kv_heads, -(-shape.m_cap // block))
    codes = [torch.zeros(rows + (shape.head_dim,), dtype=torch.int8, device=device).view(_CODE_DTYPE[cache_type])
             for _ in range(2)]
    return QuantCache(shape, cache_type, block, *codes,
                      *(torch.zeros(scales, dtype=torch.float32, device=device) for _ in range(2)),
                      torch.zeros(rows, dtype=torch.float32, device=device) if bias else None,
                      torch.zeros((shape.batch,), dtype=torch.int32, device=device))


# (torch.cuda.current_stream() builds an object: 2.9 us a call against 0.2)
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _elsewhere(device: torch.device, stream) -> bool:
    return stream is not None or _current_device() != device.index


def _space(workspace: Optional[Workspace], size, shape, device: torch.device, stream) -> Workspace:
    if workspace is None:
        return Workspace(size(shape), device, stream)
    if workspace.buf.get_device() != device.index:
        _bad("a workspace on %s is wanted, not on %s" % (device, workspace.buf.device))
    return workspace


@contextlib.contextmanager
def _on(device: torch.device, stream):
    """The cache's device current, and allocations made on the stream that the call runs on."""
    with torch.cuda.device(device):
        with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
            yield


def quant_append(cache: QuantCache, K_new: torch.Tensor, V_new: torch.Tensor, bias_new: Optional[torch.Tensor] = None,
                 counts: Optional[torch.Tensor] = None, workspace: Optional[Workspace] = None, stream=None) -> QuantCache:
    """selkv_qcache_append: rows [B][Hkv][T][d] (the first counts[b] of each sequence) behind those of
    the cache, in place."""
    s, dev = cache.shape, cache.K.device
    if _elsewhere(dev, stream):
        with _on(dev, stream):
            return quant_append(cache, K_new, V_new, bias_new, counts, workspace)
    st = _raw_stream(dev.index)
    T = K_new.shape[2] if K_new.dim() == 4 else 0
    want = (s.batch, s.num_kv_heads, T, s.head_dim)
    _tensor(K_new, "quant_append: K_new", want, cache._dtype, dev)
    _tensor(V_new, "quant_append: V_new", want, cache._dtype, dev)
    if bias_new is not None:
        _tensor(bias_new, "quant_append: bias_new", want[:3], torch.float32, dev)
    if counts is not None:
        _tensor(counts, "quant_append: counts", (s.batch,), torch.int32, dev)
    ws = _space(workspace, B.selkv_qcache_workspace_size, s, dev, st)
    B.check(B.selkv_qcache_append(s, cache._bias, T, K_new, V_new, bias_new, counts, ws.buf, ws.nbytes, st),
            "selkv_qcache_append")
    return cache


def quantize(cache: CompressedCache, cache_type: str = "e4m3", block: int = 64, workspace: Optional[Workspace] = None,
             stream=None) -> QuantCache:
    """The compressed cache in 8 bits: its rows, compensation and lengths in a QuantCache of its capacity."""
    dev = cache.K_c.device
    if _elsewhere(dev, stream):
        with _on(dev, stream):
            return quantize(cache, cache_type, block, workspace)
    q = alloc_quant(cache.shape, cache_type, block, True, dev)
    return quant_append(q, cache.K_c, cache.V_c, cache.bias, cache.lengths[:cache.shape.batch], workspace)


def quant_read(cache: QuantCache, row0: int = 0, rows: Optional[int] = None, out=None,
               workspace: Optional[Workspace] = None, stream=None):
    """selkv_qcache_read: (K, V) of rows row0 .. row0 + rows - 1, [B][Hkv][rows][d] (with `out` given its
    rows behind the lengths stay, else they are zeros)."""
    s, dev = cache.shape, cache.K.device
    if _elsewhere(dev, stream):
        with _on(dev, stream):
            return quant_read(cache, row0, rows, out, workspace)
    st = _raw_stream(dev.index)
    if rows is None:
        rows = out[0].shape[2] if out is not None else s.m_cap - row0
    want = (s.batch, s.num_kv_heads, rows, s.head_dim)
    if out is None:
        if rows < 1:
            _bad("quant_read: rows")
        out = tuple(torch.zeros(want, dtype=cache._dtype, device=dev) for _ in range(2))
    K, V = out
    _tensor(K, "quant_read: K", want, cache._dtype, dev)
    _tensor(V, "quant_read: V", want, cache._dtype, dev)
    ws = _space(workspace, B.selkv_qcache_workspace_size, s, dev, st)
    B.check(B.selkv_qcache_read(s, cache._bias, row0, rows, K, V, ws.buf, ws.nbytes, st), "selkv_qcache_read")
    return K, V


def decode_quant(cache: QuantCache, q: torch.Tensor, k_new: Optional[torch.Tensor] = None,
                 v_new: Optional[torch.Tensor] = None, use_bias: bool = True, out: Optional[torch.Tensor] = None,
                 workspace: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """selkv_decode_attn_q: one token [B][Hq][d] over an 8-bit cache (optionally appending k_new / v_new
    [B][Hkv][d]).  A row is not appended with use_bias off to a cache that has a bias: its bias would be left unset
    (a QuantCache of the same tensors without the bias takes it)."""
    s, dev = cache.shape, cache.K.device
    if _elsewhere(dev, stream):
        with _on(dev, stream):
            return decode_quant(cache, q, k_new, v_new, use_bias, out, workspace)
    st = _raw_stream(dev.index)
    want, dt = (s.batch, s.num_q_heads, s.head_dim), cache._dtype
    _tensor(q, "decode_quant: q", want, dt, dev)
    if k_new is not None and v_new is not None:
        new = (s.batch, s.num_kv_heads, s.head_dim)
        _tensor(k_new, "decode_quant: k_new", new, dt, dev)
        _tensor(v_new, "decode_quant: v_new", new, dt, dev)
        if not use_bias and cache.bias is not None:
            _bad("decode_quant: a row appended without the cache's bias")
    if out is None:
        out = torch.empty_like(q)
    else:
        _tensor(out, "decode_quant: out", want, dt, dev)
    ws = _space(workspace, B.selkv_decode_q_workspace_size, s, dev, st)
    B.check(B.selkv_decode_attn_q(s, cache._bias if use_bias else cache._plain, q, k_new, v_new, out, ws.buf, ws.nbytes, st),
            "selkv_decode_attn_q")
    return out
