"""PyTorch-facing binding of the ART decode-attention library.

PyTorch provides device memory and the stream; every step of the computation
runs in the HIP kernels of libart.so (include/art.h).  This module only
checks tensor layouts, builds the ABI structs and passes pointers.
"""
from __future__ import annotations

import math
import threading
from typing import NamedTuple, Optional

import torch

from . import _lib
from ._lib import ArtError, DecodeOpts, DecodeShape

_ws_lock = threading.Lock()
_ws_cache: dict = {}


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else int(t.data_ptr())


def _require_cuda(t: torch.Tensor, name: str, dtype=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")


def make_shape(q, k_cache, v_cache, page_table, *, block_size: int, block_list=None,
               list_per_head: bool = True) -> DecodeShape:
    """ABI shape from tensors: q [B][Hq][D], caches [P][Hkv][Ps][D] (any
    strides with a unit head-dim stride), page_table [B][max_pages]."""
    B, Hq, D = q.shape
    P, Hkv, Ps, D2 = k_cache.shape
    if D2 != D or tuple(v_cache.shape) != tuple(k_cache.shape):
        raise ValueError("k_cache/v_cache must both be [pages][kv_heads][page_size][head_dim]")
    if k_cache.stride(3) != 1 or v_cache.stride(3) != 1:
        raise ValueError("head_dim must be the innermost (unit-stride) dimension")
    ks, vs = k_cache.stride(), v_cache.stride()
    return DecodeShape(
        batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, block_size=int(block_size),
        page_size=Ps, num_pages=P, max_pages_per_seq=int(page_table.shape[1]),
        max_blocks_per_list=0 if block_list is None else int(block_list.shape[-1]),
        list_per_head=1 if list_per_head else 0,
        k_stride_page=ks[0], k_stride_head=ks[1], k_stride_token=ks[2],
        v_stride_page=vs[0], v_stride_head=vs[1], v_stride_token=vs[2])


def make_opts(*, softmax_scale: float, tau: float, phi: float, patience: int,
              dense_order: int = 0, out_dtype=torch.float32, chunk_blocks: int = 0,
              probe_stride: int = 1, scale_of_accumulator: bool = False,
              no_detector: bool = False, max_wait_polls: int = 0,
              per_head_stop: bool = False, max_ahead_chunks: int = 0) -> DecodeOpts:
    od = _lib.OUT_BF16 if out_dtype == torch.bfloat16 else _lib.OUT_F32
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be float32 or bfloat16")
    return DecodeOpts(softmax_scale=float(softmax_scale), tau=float(tau), phi=float(phi),
                      patience=int(patience), dense_order=int(dense_order), out_dtype=od,
                      chunk_blocks=int(chunk_blocks), probe_stride=int(probe_stride),
                      scale_of_accumulator=1 if scale_of_accumulator else 0,
                      no_detector=1 if no_detector else 0,
                      max_wait_polls=int(max_wait_polls),
                      per_head_stop=1 if per_head_stop else 0,
                      max_ahead_chunks=int(max_ahead_chunks))


def workspace_bytes(shape: DecodeShape, opts: DecodeOpts) -> int:
    return _lib.workspace_bytes(shape, opts)


def new_workspace(nbytes: int, device) -> torch.Tensor:
    """A zero-filled workspace (the state art_workspace_init leaves)."""
    n = max(256, (int(nbytes) + 255) // 256 * 256)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    _lib.workspace_init(_ptr(ws), n, torch.cuda.current_stream(ws.device).cuda_stream)
    return ws


def _cached_workspace(nbytes: int, device, stream) -> torch.Tensor:
    key = (device.index if device.index is not None else torch.cuda.current_device(),
           int(stream))
    with _ws_lock:
        ws = _ws_cache.get(key)
        if ws is None or ws.numel() < nbytes:
            ws = new_workspace(max(nbytes, 1 << 20), device)
            _ws_cache[key] = ws
        return ws


def decode_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     page_table: torch.Tensor, seq_lens: torch.Tensor, *,
                     block_size: int, tau: float, phi: float, patience: int,
                     softmax_scale: Optional[float] = None, dense_order: int = 0,
                     block_list: Optional[torch.Tensor] = None,
                     block_list_len: Optional[torch.Tensor] = None,
                     list_per_head: bool = True, out_dtype=torch.float32,
                     chunk_blocks: int = 0, probe_stride: int = 1,
                     scale_of_accumulator: bool = False, no_detector: bool = False,
                     max_wait_polls: int = 0, per_head_stop: bool = False,
                     max_ahead_chunks: int = 0,
                     workspace: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     stop_block: Optional[torch.Tensor] = None):
    """ART decode attention on the current stream.

    Returns (out [B][Hq][D] out_dtype, lse [B][Hq] fp32, stop_block [B][Hkv]
    int32).  ``workspace`` (uint8, zero-filled before its first use, e.g. by
    ``new_workspace``) defaults to a per-(device, stream) cached buffer.
    ``probe_stride`` s > 1 makes the stability test look at every s-th
    coordinate of each head's output only (Sec. 3.2's subsampled probe).
    ``scale_of_accumulator`` takes d_scale on the unnormalised accumulator
    l(t) o(t) instead of o(t).  ``no_detector`` runs without the stability
    test at all (full attention over the traversal).  ``max_wait_polls``
    n > 0 makes every wait of the kernel give up after n polls (the call then
    reports ART_ERR_DEVICE_TIMEOUT through ``workspace_status``).
    ``per_head_stop`` gives every query head its own patience counter and stop
    (out and lse at the head's own stop; stop_block is then [B][Hq], each
    head's stop).  ``max_ahead_chunks`` n > 0 bounds the reads past a stop:
    a chunk of a traversal is loaded only once the chunk n before it has been
    through the stability test (the results are the same bits).
    """
    _require_cuda(q, "q", torch.bfloat16)
    _require_cuda(k_cache, "k_cache", torch.bfloat16)
    _require_cuda(v_cache, "v_cache", torch.bfloat16)
    _require_cuda(page_table, "page_table", torch.int32)
    _require_cuda(seq_lens, "seq_lens", torch.int32)
    if not q.is_contiguous() or not page_table.is_contiguous() or not seq_lens.is_contiguous():
        raise ValueError("q, page_table and seq_lens must be contiguous")
    if (block_list is None) != (block_list_len is None):
        raise ValueError("block_list and block_list_len go together")
    if block_list is not None:
        _require_cuda(block_list, "block_list", torch.int32)
        _require_cuda(block_list_len, "block_list_len", torch.int32)
        if not block_list.is_contiguous() or not block_list_len.is_contiguous():
            raise ValueError("block_list and block_list_len must be contiguous")
    B, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(D)
    shape = make_shape(q, k_cache, v_cache, page_table, block_size=block_size,
                       block_list=block_list, list_per_head=list_per_head)
    opts = make_opts(softmax_scale=softmax_scale, tau=tau, phi=phi, patience=patience,
                     dense_order=dense_order, out_dtype=out_dtype, chunk_blocks=chunk_blocks,
                     probe_stride=probe_stride, scale_of_accumulator=scale_of_accumulator,
                     no_detector=no_detector, max_wait_polls=max_wait_polls,
                     per_head_stop=per_head_stop, max_ahead_chunks=max_ahead_chunks)
    dev = q.device
    if out is None:
        out = torch.empty((B, Hq, D), dtype=out_dtype, device=dev)
    if lse is None:
        lse = torch.empty((B, Hq), dtype=torch.float32, device=dev)
    if stop_block is None:
        stop_block = torch.empty((B, Hq if per_head_stop else Hkv), dtype=torch.int32, device=dev)
    stream = torch.cuda.current_stream(dev).cuda_stream
    need = workspace_bytes(shape, opts)
    ws = workspace if workspace is not None else _cached_workspace(need, dev, stream)
    st = _lib.decode_attention(shape, opts, _ptr(q), _ptr(k_cache), _ptr(v_cache),
                               _ptr(page_table), _ptr(seq_lens), _ptr(block_list),
                               _ptr(block_list_len), _ptr(out), _ptr(lse), _ptr(stop_block),
                               _ptr(ws), ws.numel(), stream)
    if st != _lib.OK:
        raise ArtError(st, "art_decode_attention")
    return out, lse, stop_block


def decode_workload(wl, *, tau=None, phi=None, patience=None, dense_order=None,
                    out_dtype=torch.float32, chunk_blocks: int = 0, workspace=None, **kw):
    """decode_attention on a ``workloads.Workload`` resident on the GPU."""
    s = wl.spec
    return decode_attention(
        wl.q, wl.k_cache, wl.v_cache, wl.page_table, wl.seq_lens,
        block_size=s.block_size, softmax_scale=s.softmax_scale,
        tau=s.tau if tau is None else tau, phi=s.phi if phi is None else phi,
        patience=s.patience if patience is None else patience,
        dense_order=s.dense_order if dense_order is None else dense_order,
        block_list=wl.block_list, block_list_len=wl.block_list_len,
        out_dtype=out_dtype, chunk_blocks=chunk_blocks, workspace=workspace, **kw)


def validate_inputs(q, k_cache, v_cache, page_table, seq_lens, *, block_size: int,
                    block_list=None, block_list_len=None, list_per_head: bool = True):
    """Checked mode (synchronous): returns (status, bad_index, where)."""
    shape = make_shape(q, k_cache, v_cache, page_table, block_size=block_size,
                       block_list=block_list, list_per_head=list_per_head)
    opts = make_opts(softmax_scale=1.0, tau=0.0, phi=0.0, patience=1)
    stream = torch.cuda.current_stream(q.device).cuda_stream
    return _lib.validate_inputs(shape, opts, _ptr(page_table), _ptr(seq_lens),
                                _ptr(block_list), _ptr(block_list_len), stream)


def workspace_status(ws: torch.Tensor) -> int:
    """ART_OK or ART_ERR_DEVICE_TIMEOUT for calls that used ``ws`` (syncs)."""
    return _lib.workspace_status(_ptr(ws), ws.numel(), torch.cuda.current_stream(ws.device).cuda_stream)


def build_block_list(q: torch.Tensor, k_cache: torch.Tensor, page_table: torch.Tensor,
                     seq_lens: torch.Tensor, *, block_size: int, budget: int,
                     policy: int = _lib.LIST_IMPORTANCE, score_kind: int = _lib.SCORE_KEY_NORM,
                     sink_blocks: int = 0, keep_last: bool = False,
                     max_list: Optional[int] = None, return_scores: bool = False):
    """Traversal lists for decode_attention (Sec. 3.4), built on the current
    stream: importance-first (block scores, top-`budget` with forced sink /
    last blocks, descending score) or streaming (sinks first, then the
    `budget` most recent blocks).

    q bf16 [B][Hq][D] (the shape source; read for the query bound only),
    k_cache bf16 [P][Hkv][Ps][D], page_table int32 [B][max_pages], seq_lens
    int32 [B].  Returns (block_list int32 [B][Hkv][max_list], block_list_len
    int32 [B][Hkv]) and, with return_scores, the fp64 block scores
    [B][Hkv][max_blocks].  Entries past a row's length are -1.
    """
    _require_cuda(q, "q", torch.bfloat16)
    _require_cuda(k_cache, "k_cache", torch.bfloat16)
    _require_cuda(page_table, "page_table", torch.int32)
    _require_cuda(seq_lens, "seq_lens", torch.int32)
    if not q.is_contiguous() or not page_table.is_contiguous() or not seq_lens.is_contiguous():
        raise ValueError("q, page_table and seq_lens must be contiguous")
    B, Hq, D = q.shape
    P, Hkv, Ps, _ = k_cache.shape
    max_blocks = (int(page_table.shape[1]) * Ps + block_size - 1) // block_size
    if max_list is None:
        max_list = max(1, max_blocks)
    dev = q.device
    # the call writes every entry of the rows and every length
    bl = torch.empty((B, Hkv, max_list), dtype=torch.int32, device=dev)
    bll = torch.empty((B, Hkv), dtype=torch.int32, device=dev)
    shape = make_shape(q, k_cache, k_cache, page_table, block_size=block_size, block_list=bl)
    opts = _lib.ListOpts(policy=int(policy), score_kind=int(score_kind), budget=int(budget),
                         sink_blocks=int(sink_blocks), keep_last=1 if keep_last else 0)
    _lib.block_list_workspace_bytes(shape, opts)  # raises on invalid input
    # scores of blocks past a sequence's end are not written: NaN for a caller
    # who gets them, never read otherwise
    scores = torch.empty((B, Hkv, max(1, max_blocks)), dtype=torch.float64, device=dev)
    if return_scores:
        scores.fill_(float("nan"))
    stream = torch.cuda.current_stream(dev).cuda_stream
    st = _lib.build_block_list(shape, opts, _ptr(q), _ptr(k_cache), _ptr(page_table),
                               _ptr(seq_lens), _ptr(bl), _ptr(bll), _ptr(scores), 0, 0, stream,
                               padded=True)
    if st != _lib.OK:
        raise ArtError(st, "art_build_block_list")
    return (bl, bll, scores) if return_scores else (bl, bll)


# ---- a cache held in 8 bits -----------------------------------------------------

_QUANT_FORMATS = {torch.float8_e4m3fn: _lib.QUANT_E4M3, torch.int8: _lib.QUANT_INT8}
_ROWS_TYPES = {torch.bfloat16: _lib.ROWS_BF16, torch.float16: _lib.ROWS_F16,
               torch.float32: _lib.ROWS_F32}


class QuantCache(NamedTuple):
    """A paged K/V cache of 8-bit codes: ``k`` and ``v`` [P][Hkv][Ps][D],
    float8_e4m3fn or int8 (any strides with a unit head-dim stride), and a fp32
    scale for every run of slots, ``k_scale`` and ``v_scale`` [P][Hkv][Ps / run]
    (unit stride of the last dimension).  A token's values are code * scale.
    """
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    @property
    def scale_tokens(self) -> int:
        """Slots that share a scale."""
        return self.k.shape[2] // max(1, self.k_scale.shape[2])


def new_quant_cache(num_pages: int, num_kv_heads: int, page_size: int, *,
                    dtype=torch.float8_e4m3fn, scale_tokens: Optional[int] = None,
                    head_dim: int = 128, device="cuda") -> QuantCache:
    """An empty 8-bit cache (codes and scales zero) with a scale for every
    ``scale_tokens`` slots (default: the whole page, at most 64)."""
    if dtype not in _QUANT_FORMATS:
        raise ValueError("dtype must be float8_e4m3fn or int8")
    run = min(page_size, 64) if scale_tokens is None else int(scale_tokens)
    if run < 1 or page_size % run:
        raise ValueError("scale_tokens must divide page_size")
    pool = lambda: torch.zeros((num_pages, num_kv_heads, page_size, head_dim),  # noqa: E731
                               dtype=torch.uint8, device=device).view(dtype)
    scale = lambda: torch.zeros((num_pages, num_kv_heads, page_size // run),  # noqa: E731
                                dtype=torch.float32, device=device)
    return QuantCache(pool(), pool(), scale(), scale())


# These calls may serve single tokens, where a call's host side is most of its
# time: every tensor is looked at once, and the structures are filled by
# position.

def _check(t, name, dtype, dev, shape):
    """A contiguous index or output array of ``shape`` on GPU ``dev``."""
    if t.dtype is not dtype or t.get_device() != dev:
        _require_cuda(t, name, dtype)
        raise ValueError(f"{name} must be on the cache's device (cuda:{dev}), got {t.device}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)}")


def _quant_spec(cache: QuantCache):
    """(device index, pool shape, pool strides of K and V, art_quant_cache) of a
    cache, its tensors checked."""
    k, v, ks, vs = cache
    dev, fmt = k.get_device(), _QUANT_FORMATS.get(k.dtype)
    if fmt is None or v.dtype is not k.dtype:
        raise ValueError("the cache must be float8_e4m3fn or int8")
    if dev < 0 or v.get_device() != dev or ks.get_device() != dev or vs.get_device() != dev:
        for t, name in ((k, "k"), (v, "v"), (ks, "k_scale"), (vs, "v_scale")):
            _require_cuda(t, name)
        raise ValueError("the cache's tensors must be on one device")
    if ks.dtype is not torch.float32 or vs.dtype is not torch.float32:
        raise ValueError("k_scale and v_scale must be float32")
    if k.dim() != 4 or v.shape != k.shape:
        raise ValueError("k/v must both be [pages][kv_heads][page_size][head_dim]")
    pool, a, b = k.shape, k.stride(), v.stride()
    if a[3] != 1 or b[3] != 1:
        raise ValueError("head_dim must be the innermost (unit-stride) dimension")
    runs = ks.shape[2] if ks.dim() == 3 else 0
    if not runs or ks.shape != (pool[0], pool[1], runs) or vs.shape != ks.shape or pool[2] % runs:
        raise ValueError("k_scale/v_scale must both be [pages][kv_heads][page_size / run]")
    c, d = ks.stride(), vs.stride()
    if runs > 1 and (c[2] != 1 or d[2] != 1):
        raise ValueError("the runs of a page must be the scales' innermost (unit-stride) dimension")
    return dev, pool, a, b, _lib.QuantCacheSpec(fmt, pool[2] // runs, c[0], c[1], d[0], d[1])


def quant_spec(cache: QuantCache) -> _lib.QuantCacheSpec:
    """ABI description of a cache (its tensors checked), for raw calls."""
    return _quant_spec(cache)[4]


def _on_device(dev, call, *args) -> int:
    """call(*args, the current stream of GPU ``dev``) with that GPU current."""
    stream = torch._C._cuda_getCurrentRawStream(dev)
    if torch.cuda.current_device() == dev:
        return call(*args, stream)
    with torch.cuda.device(dev):
        return call(*args, stream)


def decode_attention_quant(q: torch.Tensor, cache: QuantCache, page_table: torch.Tensor,
                           seq_lens: torch.Tensor, *, block_size: int, tau: float, phi: float,
                           patience: int, softmax_scale: Optional[float] = None,
                           dense_order: int = 0, block_list: Optional[torch.Tensor] = None,
                           block_list_len: Optional[torch.Tensor] = None,
                           list_per_head: bool = True, out_dtype=torch.float32,
                           chunk_blocks: int = 0, probe_stride: int = 1,
                           scale_of_accumulator: bool = False, no_detector: bool = False,
                           max_wait_polls: int = 0, per_head_stop: bool = False,
                           max_ahead_chunks: int = 0, workspace: Optional[torch.Tensor] = None,
                           out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None,
                           stop_block: Optional[torch.Tensor] = None):
    """``decode_attention`` over a cache held in 8 bits: K and V are the
    cache's code * scale; everything else (options, lists, workspace, results)
    is as there."""
    dev, (P, Hkv, Ps, D), a, b, spec = _quant_spec(cache)
    if q.dim() != 3 or page_table.dim() != 2:
        raise ValueError("q must be [batch][q_heads][head_dim], page_table [batch][max_pages]")
    B, Hq, _ = q.shape
    _check(q, "q", torch.bfloat16, dev, (B, Hq, D))
    _check(page_table, "page_table", torch.int32, dev, (B, page_table.shape[1]))
    _check(seq_lens, "seq_lens", torch.int32, dev, (B,))
    if (block_list is None) != (block_list_len is None):
        raise ValueError("block_list and block_list_len go together")
    max_list = 0
    if block_list is not None:
        # [B][Hkv][n], or one list a sequence as [B][1][n] or [B][n]
        rows, max_list = ((B, Hkv) if list_per_head else (B,)), block_list.shape[-1]
        if not list_per_head and block_list.dim() == 3:
            rows = (B, 1)
        _check(block_list, "block_list", torch.int32, dev, (*rows, max_list))
        if block_list_len.numel() != math.prod(rows):
            raise ValueError(f"block_list_len must hold {math.prod(rows)} lengths")
        _check(block_list_len, "block_list_len", torch.int32, dev, block_list_len.shape)
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(D)
    shape = DecodeShape(B, Hq, Hkv, D, int(block_size), Ps, P, page_table.shape[1], max_list,
                        1 if list_per_head else 0, a[0], a[1], a[2], b[0], b[1], b[2])
    opts = make_opts(softmax_scale=softmax_scale, tau=tau, phi=phi, patience=patience,
                     dense_order=dense_order, out_dtype=out_dtype, chunk_blocks=chunk_blocks,
                     probe_stride=probe_stride, scale_of_accumulator=scale_of_accumulator,
                     no_detector=no_detector, max_wait_polls=max_wait_polls,
                     per_head_stop=per_head_stop, max_ahead_chunks=max_ahead_chunks)
    heads = Hq if per_head_stop and not no_detector else Hkv
    if out is None:
        out = torch.empty((B, Hq, D), dtype=out_dtype, device=q.device)
    else:
        _check(out, "out", out_dtype, dev, (B, Hq, D))
    if lse is None:
        lse = torch.empty((B, Hq), dtype=torch.float32, device=q.device)
    else:
        _check(lse, "lse", torch.float32, dev, (B, Hq))
    if stop_block is None:
        stop_block = torch.empty((B, heads), dtype=torch.int32, device=q.device)
    else:
        _check(stop_block, "stop_block", torch.int32, dev, (B, heads))
    need = _lib.workspace_bytes(shape, opts)
    ws = workspace
    if ws is None:
        ws = _ws_cache.get((dev, torch._C._cuda_getCurrentRawStream(dev)))
        if ws is None or ws.numel() < need:
            with torch.cuda.device(dev):
                ws = _cached_workspace(need, q.device, torch.cuda.current_stream(dev).cuda_stream)
    elif ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError("workspace must be contiguous and on the cache's device")
    st = _on_device(dev, _lib.decode_attention_quant, shape, opts, spec, q.data_ptr(),
                    cache.k.data_ptr(), cache.v.data_ptr(), cache.k_scale.data_ptr(),
                    cache.v_scale.data_ptr(), page_table.data_ptr(), seq_lens.data_ptr(),
                    _ptr(block_list), _ptr(block_list_len), out.data_ptr(), lse.data_ptr(),
                    stop_block.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size())
    if st != _lib.OK:
        raise ArtError(st, "art_decode_attention_quant")
    return out, lse, stop_block


def _quant_rows_call(cache, k_rows, v_rows, page_table, positions, token_offsets):
    """(device index, shape, spec, rows) of an append or a read, its tensors
    checked."""
    dev, (P, H, Ps, D), a, b, spec = _quant_spec(cache)
    kind = _ROWS_TYPES.get(k_rows.dtype)
    if kind is None:
        raise ValueError("rows must be bfloat16, float16 or float32")
    if k_rows.get_device() != dev or v_rows.get_device() != dev or v_rows.dtype is not k_rows.dtype:
        for t, name in ((k_rows, "k"), (v_rows, "v")):
            _require_cuda(t, name, k_rows.dtype)
        raise ValueError("k and v must be on the cache's device")
    if k_rows.dim() != 3 or k_rows.shape[1:] != (H, D) or v_rows.shape != k_rows.shape:
        raise ValueError(f"k and v must both be [rows][{H}][{D}]")
    c, d = k_rows.stride(), v_rows.stride()
    if c[2] != 1 or d[2] != 1:
        raise ValueError("head_dim must be the innermost (unit-stride) dimension")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [batch][max_pages]")
    B, width = page_table.shape
    _check(page_table, "page_table", torch.int32, dev, (B, width))
    if positions is not None:
        _check(positions, "positions", torch.int32, dev, (B,))
    if token_offsets is not None:
        _check(token_offsets, "token_offsets", torch.int32, dev, (B + 1,))
    shape = DecodeShape(B, H, H, D, 64, Ps, P, width, 0, 1, a[0], a[1], a[2], b[0], b[1], b[2])
    return dev, shape, spec, _lib.QuantRows(kind, k_rows.shape[0], c[0], c[1], d[0], d[1])


def quant_append(cache: QuantCache, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor,
                 positions: Optional[torch.Tensor], *,
                 token_offsets: Optional[torch.Tensor] = None) -> None:
    """Quantise new tokens into the cache, on the current stream.

    ``k`` and ``v`` [rows][Hkv][D] (bf16, fp16 or fp32) hold the new tokens of
    all sequences, packed: rows token_offsets[b] .. token_offsets[b + 1] - 1 are
    sequence b's tokens positions[b], positions[b] + 1, ... (``token_offsets``
    int32 [B + 1]; without it every sequence has rows / B of them).
    ``positions`` int32 [B]: the tokens that each sequence holds already (None:
    none; negative: an unused row of a padded batch).  A run of slots gets the
    smallest power-of-two scale that holds its tokens; one that holds older
    tokens keeps its scale unless it has to grow, and its old codes are then
    rounded anew.  ``seq_lens`` stays the caller's to advance.
    """
    dev, shape, spec, rows = _quant_rows_call(cache, k, v, page_table, positions, token_offsets)
    st = _on_device(dev, _lib.quant_append, shape, spec, rows, k.data_ptr(), v.data_ptr(),
                    _ptr(token_offsets), _ptr(positions), page_table.data_ptr(),
                    cache.k.data_ptr(), cache.v.data_ptr(), cache.k_scale.data_ptr(),
                    cache.v_scale.data_ptr())
    if st != _lib.OK:
        raise ArtError(st, "art_quant_append")


def quant_read(cache: QuantCache, page_table: torch.Tensor, positions: Optional[torch.Tensor], *,
               token_offsets: Optional[torch.Tensor] = None, rows: Optional[int] = None,
               dtype=torch.bfloat16, k: Optional[torch.Tensor] = None,
               v: Optional[torch.Tensor] = None):
    """Bring stored tokens back as packed rows, on the current stream.

    Rows token_offsets[b] .. token_offsets[b + 1] - 1 receive sequence b's
    tokens positions[b], positions[b] + 1, ... (as in ``quant_append``).
    Returns (k, v) [rows][Hkv][D] in ``dtype`` (bf16, fp16 or fp32; the fp32
    product code * scale rounded to it); ``rows`` sizes them where they are not given.  Rows of no
    token are left as they were (not initialised, where they are not given).
    """
    if k is None or v is None:
        if rows is None:
            raise ValueError("rows is needed where k and v are not given")
        size, on = (int(rows), cache.k.shape[1], cache.k.shape[3]), cache.k.device
        k = torch.empty(size, dtype=dtype, device=on) if k is None else k
        v = torch.empty(size, dtype=dtype, device=on) if v is None else v
    dev, shape, spec, packed = _quant_rows_call(cache, k, v, page_table, positions, token_offsets)
    st = _on_device(dev, _lib.quant_read, shape, spec, packed, cache.k.data_ptr(),
                    cache.v.data_ptr(), cache.k_scale.data_ptr(), cache.v_scale.data_ptr(),
                    _ptr(token_offsets), _ptr(positions), page_table.data_ptr(), k.data_ptr(),
                    v.data_ptr())
    if st != _lib.OK:
        raise ArtError(st, "art_quant_read")
    return k, v


# ---- drafted tokens over the bf16 cache -------------------------------------------
#
# The nodes of all sequences are packed rows: rows token_offsets[b] ..
# token_offsets[b + 1] - 1 are sequence b's nodes 0, 1, ... (int32 [B + 1]; without
# it every sequence has rows / B of them), node i in slot context_lens[b] + i of the
# cache.  A sequence with a negative context is an unused one of a padded batch.

_ROPE_LAYOUTS = {"half": _lib.ROPE_HALF, "interleaved": _lib.ROPE_INTERLEAVED}


class Rope(NamedTuple):
    """Rotary positions: pair i of a head's first 2 len(freqs) dims turns by
    position * freqs[i] radians and is multiplied by ``scale``.  ``freqs`` fp64 on
    the GPU; ``layout`` "half" (dims i and i + len(freqs)) or "interleaved"
    (dims 2i and 2i + 1)."""
    freqs: torch.Tensor
    layout: str = "half"
    scale: float = 1.0


def rope_frequencies(rot_dim: int = 128, *, base: float = 10000.0, layout: str = "half",
                     factor: float = 1.0, original_len: Optional[int] = None,
                     beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda") -> Rope:
    """The usual frequencies, base ** (-2i / rot_dim), as a ``Rope``.

    ``factor`` > 1 scales them for contexts that many times as long: all alike
    (positions divided by it), or with ``original_len`` the way of YaRN
    (arXiv 2309.00071): pairs that turn more than ``beta_fast`` times over the
    original length keep their frequency, those of fewer than ``beta_slow`` turns
    have it divided, with a linear ramp over the pairs between them, and rotated
    values are multiplied by 0.1 ln(factor) + 1.
    """
    if rot_dim < 2 or rot_dim % 2 or rot_dim > 128 or factor < 1.0:
        raise ValueError("rot_dim must be even, 2 .. 128, and factor at least 1")
    half = rot_dim // 2
    i = torch.arange(half, dtype=torch.float64)
    freqs, scale = base ** (-i / half), 1.0
    if original_len is None:
        freqs = freqs / factor
    else:
        # the pair that turns n times over the original length
        pair = lambda n: half * math.log(original_len / (2 * math.pi * n)) / math.log(base)  # noqa: E731
        low, high = max(math.floor(pair(beta_fast)), 0), min(math.ceil(pair(beta_slow)), rot_dim - 1)
        ramp = ((i - low) / max(high - low, 1e-3)).clamp(0, 1)
        freqs, scale = freqs * (1 - ramp) + freqs / factor * ramp, 0.1 * math.log(factor) + 1.0
    return Rope(freqs.to(device), layout, scale)


def _rope_spec(rope: Rope, dev: int) -> _lib.RopeSpec:
    freqs, layout, scale = rope
    if layout not in _ROPE_LAYOUTS:
        raise ValueError('layout must be "half" or "interleaved"')
    _check(freqs, "freqs", torch.float64, dev, (freqs.numel(),))
    return _lib.RopeSpec(_ROPE_LAYOUTS[layout], 2 * freqs.numel(), float(scale))


def _packed_rows(t: torch.Tensor, name: str, dev: int) -> _lib.Rows:
    """ABI description of rows [rows][heads][head_dim] on GPU ``dev``."""
    kind, size, stride = _ROWS_TYPES.get(t.dtype), t.shape, t.stride()
    if kind is None or dev < 0 or t.get_device() != dev or len(size) != 3 or size[2] != 128 or stride[2] != 1:
        if kind is None:
            raise ValueError(f"{name} must be bfloat16, float16 or float32")
        _require_cuda(t, name)
        if t.get_device() != dev:
            raise ValueError(f"{name} must be on cuda:{dev}, got {t.device}")
        raise ValueError(f"{name} must be [rows][heads][128] with a unit head-dim stride")
    return _lib.Rows(kind, size[1], stride[0], stride[1])


def _bf16_pools(k_cache, v_cache, page_table):
    """(device index, heads, batch, shape fields from page_size on) of a bf16
    cache and its table, checked."""
    dev, pool = k_cache.get_device(), k_cache.shape
    if (dev < 0 or v_cache.get_device() != dev or k_cache.dtype is not torch.bfloat16
            or v_cache.dtype is not torch.bfloat16):
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            _require_cuda(t, name, torch.bfloat16)
        raise ValueError("the cache's tensors must be on one device")
    if len(pool) != 4 or v_cache.shape != pool:
        raise ValueError("k_cache/v_cache must both be [pages][kv_heads][page_size][head_dim]")
    a, b = k_cache.stride(), v_cache.stride()
    if a[3] != 1 or b[3] != 1:
        raise ValueError("head_dim must be the innermost (unit-stride) dimension")
    table = page_table.shape
    if len(table) != 2:
        raise ValueError("page_table must be [batch][max_pages]")
    B, width = table
    _check(page_table, "page_table", torch.int32, dev, table)
    P, H, Ps, _ = pool
    return dev, H, B, (Ps, P, width, 0, 1, a[0], a[1], a[2], b[0], b[1], b[2])


def rope_rows(x: torch.Tensor, positions: torch.Tensor, rope: Rope, *,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotate rows ``x`` [rows][heads][128] (bf16, fp16 or fp32) to ``positions``
    (int32 [rows]), on the current stream.  ``out`` (default: like ``x``) may be
    ``x`` itself, or of another of the three types.  Keys of an 8-bit cache are
    rotated so before ``quant_append``.  ``Rope(-freqs, layout, scale)`` gives the
    gradient of a rotation, which is the way back where scale is 1."""
    dev = x.get_device()
    x_rows = _packed_rows(x, "x", dev)
    _check(positions, "positions", torch.int32, dev, (x.shape[0],))
    spec = _rope_spec(rope, dev)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    elif out.shape != x.shape:
        raise ValueError("out must have the shape of x")
    st = _on_device(dev, _lib.rope_rows, spec, x.shape[0], x_rows, x.data_ptr(),
                    _packed_rows(out, "out", dev), out.data_ptr(), positions.data_ptr(),
                    rope.freqs.data_ptr())
    if st != _lib.OK:
        raise ArtError(st, "art_rope_rows")
    return out


def rope_append(k_cache: torch.Tensor, v_cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                page_table: torch.Tensor, context_lens: torch.Tensor, *, rope: Optional[Rope] = None,
                q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                token_offsets: Optional[torch.Tensor] = None,
                row_positions: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Append new tokens to the bf16 cache, on the current stream: keys rotated
    on the way, values as they are, both rounded to bf16.

    ``k`` and ``v`` [rows][Hkv][128] (bf16, fp16 or fp32) are the packed nodes (or
    prompts) of all sequences, ``context_lens`` int32 [B] the tokens that each holds
    already.  A row's position is its slot, or row_positions[row] (int32, e.g. from
    ``tree_layout``).  With ``q`` [rows][Hq][128], of the type of ``k``, the queries are
    rotated too; returns them in bf16 (``q_out``, or new), else None.  ``rope`` None:
    no rotation.  ``context_lens`` stays the caller's to advance.
    """
    dev, H, B, fields = _bf16_pools(k_cache, v_cache, page_table)
    k_rows, v_rows, size = _packed_rows(k, "k", dev), _packed_rows(v, "v", dev), k.shape
    if size[1] != H or v.shape != size or v.dtype is not k.dtype:
        raise ValueError(f"k and v must both be [rows][{H}][128] of one type")
    rows = size[0]
    _check(context_lens, "context_lens", torch.int32, dev, (B,))
    if token_offsets is not None:
        _check(token_offsets, "token_offsets", torch.int32, dev, (B + 1,))
    if row_positions is not None:
        _check(row_positions, "row_positions", torch.int32, dev, (rows,))
    q_rows = out_rows = None
    heads = H
    if q is not None:
        q_rows, size = _packed_rows(q, "q", dev), q.shape
        heads = size[1]
        if size[0] != rows or q.dtype is not k.dtype:
            raise ValueError("q must have the rows and the type of k")
        if q_out is None:
            q_out = torch.empty(size, dtype=torch.bfloat16, device=q.device)
            out_rows = _lib.Rows(_lib.ROWS_BF16, heads, 128 * heads, 128)
        elif q_out.shape != size or q_out.dtype is not torch.bfloat16:
            raise ValueError("q_out must be bfloat16 of the shape of q")
        else:
            out_rows = _packed_rows(q_out, "q_out", dev)
    elif q_out is not None:
        raise ValueError("q_out goes with q")
    spec = None if rope is None else _rope_spec(rope, dev)
    shape = DecodeShape(B, heads, H, k_cache.shape[3], 64, *fields)
    st = _on_device(dev, _lib.rope_append, shape, spec, rows, q_rows, _ptr(q), out_rows, _ptr(q_out),
                    k_rows, k.data_ptr(), v_rows, v.data_ptr(), _ptr(token_offsets),
                    context_lens.data_ptr(), _ptr(row_positions),
                    0 if rope is None else rope.freqs.data_ptr(), page_table.data_ptr(),
                    k_cache.data_ptr(), v_cache.data_ptr())
    if st != _lib.OK:
        raise ArtError(st, "art_rope_append")
    return q_out


def tree_layout(parents: torch.Tensor, context_lens: torch.Tensor, *, mask_words: int = 1,
                token_offsets: Optional[torch.Tensor] = None):
    """Masks and positions of trees of nodes, on the current stream.

    ``parents`` int32 [rows]: the parent's number within the sequence, -1 for node
    0.  Returns (mask int64 [rows][mask_words], positions int32 [rows]): bit j % 64
    of word j / 64 is set for the node and its ancestors j; a node's position is
    its sequence's context plus its depth.  Rows of no sequence are not written, nor
    those of sequences of more than 1024 nodes or of context + nodes > 2^31.
    """
    dev, B = parents.get_device(), context_lens.shape[0]
    rows = parents.shape[0]
    _check(parents, "parents", torch.int32, dev, (rows,))
    _check(context_lens, "context_lens", torch.int32, dev, (B,))
    if dev < 0:
        _require_cuda(parents, "parents")
    if token_offsets is not None:
        _check(token_offsets, "token_offsets", torch.int32, dev, (B + 1,))
    mask = torch.empty((rows, int(mask_words)), dtype=torch.int64, device=parents.device)
    positions = torch.empty_like(parents)
    st = _on_device(dev, _lib.tree_layout, B, rows, parents.data_ptr(), _ptr(token_offsets),
                    context_lens.data_ptr(), int(mask_words), mask.data_ptr(), positions.data_ptr())
    if st != _lib.OK:
        raise ArtError(st, "art_tree_layout")
    return mask, positions


def _call_workspace(workspace, need: int, dev: int, device) -> torch.Tensor:
    """The caller's workspace, or one of this call's own: the allocator orders its
    reuse on the stream, and under capture it belongs to the graph."""
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on cuda:{dev}")
    return workspace


def tree_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                   page_table: torch.Tensor, context_lens: torch.Tensor, *,
                   mask: Optional[torch.Tensor] = None,
                   token_offsets: Optional[torch.Tensor] = None,
                   softmax_scale: Optional[float] = None, out_dtype=torch.float32,
                   workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   lse: Optional[torch.Tensor] = None):
    """Full attention of several new tokens a sequence over the bf16 cache, which
    holds their keys and values already, on the current stream.

    ``q`` bf16 [rows][Hq][128] are the packed nodes' queries.  A node sees its
    sequence's context and the nodes that its row of ``mask`` (int64
    [rows][words], as from ``tree_layout``) has a bit for; without a mask node i sees
    nodes 0 .. i (a chain of drafts, a chunk of a prompt).  Returns (out
    [rows][Hq][128] out_dtype, lse [rows][Hq] fp32); a row that sees nothing gets 0
    and -inf, and rows of no sequence are not written.  Sums are held in fp32 and
    probabilities with 24 bits; with ``out_dtype`` bfloat16 these have 16, or 8 (as the
    output itself) where a KV head has, on average, more than 64 rows of queries of a
    sequence (rows / B, rounded up, times Hq / Hkv).  ``workspace`` (uint8 of
    ``_lib.tree_workspace_bytes``, needs no initialisation) defaults to one of the
    call's own.
    """
    dev, H, B, fields = _bf16_pools(k_cache, v_cache, page_table)
    if q.dim() != 3 or q.dtype is not torch.bfloat16 or q.get_device() != dev:
        _require_cuda(q, "q", torch.bfloat16)
        raise ValueError(f"q must be [rows][q_heads][head_dim] on cuda:{dev}")
    rows, Hq, D = q.shape
    if D != k_cache.shape[3] or q.stride(2) != 1:
        raise ValueError("head_dim must be that of the cache, and innermost (unit stride)")
    _check(context_lens, "context_lens", torch.int32, dev, (B,))
    if token_offsets is not None:
        _check(token_offsets, "token_offsets", torch.int32, dev, (B + 1,))
    words = 0
    if mask is not None:
        words = mask.shape[-1] if mask.dim() else 0
        if words < 1:
            raise ValueError("mask must be [rows][words] with a word at least")
        _check(mask, "mask", torch.int64, dev, (rows, words))
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be float32 or bfloat16")
    if out is None:
        out = torch.empty((rows, Hq, D), dtype=out_dtype, device=q.device)
    else:
        _check(out, "out", out_dtype, dev, (rows, Hq, D))
    if lse is None:
        lse = torch.empty((rows, Hq), dtype=torch.float32, device=q.device)
    else:
        _check(lse, "lse", torch.float32, dev, (rows, Hq))
    shape = DecodeShape(B, Hq, H, D, 64, *fields)
    opts = _lib.TreeOpts(1.0 / math.sqrt(D) if softmax_scale is None else float(softmax_scale),
                         _lib.OUT_BF16 if out_dtype is torch.bfloat16 else _lib.OUT_F32, rows, words,
                         q.stride(0), q.stride(1))
    ws = _call_workspace(workspace, _lib.tree_workspace_bytes(shape, opts), dev, q.device)
    st = _on_device(dev, _lib.tree_attention, shape, opts, q.data_ptr(), k_cache.data_ptr(),
                    v_cache.data_ptr(), page_table.data_ptr(), context_lens.data_ptr(),
                    _ptr(token_offsets), _ptr(mask), out.data_ptr(), lse.data_ptr(), ws.data_ptr(),
                    ws.numel() * ws.element_size())
    if st != _lib.OK:
        raise ArtError(st, "art_tree_attention")
    return out, lse


def verify_drafts(target: torch.Tensor, tokens: torch.Tensor, parents: torch.Tensor,
                  uniforms: torch.Tensor, last_uniforms: torch.Tensor, *,
                  draft: Optional[torch.Tensor] = None,
                  token_offsets: Optional[torch.Tensor] = None, max_path: Optional[int] = None,
                  workspace: Optional[torch.Tensor] = None):
    """Verify drafted tokens against the target's probabilities, on the current
    stream, so that the accepted tokens and the one that follows are distributed as
    tokens drawn from the target.

    ``target`` [rows][V] (fp32, bf16 or fp16): row r holds the probabilities of the
    token that follows node r.  ``draft``, likewise and of the same type: those from
    which node r's children were drawn (independently); without it the drafts are
    taken as given.  ``tokens`` and ``parents`` int32 [rows] (node 0, parent -1, is
    the sequence's newest token), ``uniforms`` fp32 [rows] and ``last_uniforms`` fp32
    [B] random numbers in [0, 1).  One-hot rows verify greedily.  Returns (accepted
    int32 [B][max_path], the accepted nodes in order and -1 behind them; counts int32
    [B]; next_tokens int32 [B]).  ``max_path`` defaults to rows / B (needed with
    ``token_offsets``).
    """
    dev, kind = target.get_device(), _ROWS_TYPES.get(target.dtype)
    if kind is None or dev < 0:
        _require_cuda(target, "target")
        raise ValueError("target must be bfloat16, float16 or float32")
    if target.dim() != 2 or target.stride(1) != 1:
        raise ValueError("target must be [rows][vocab] with a unit vocab stride")
    rows, vocab = target.shape
    B = last_uniforms.shape[0]
    if draft is not None:
        if draft.get_device() != dev or draft.dtype is not target.dtype:
            _require_cuda(draft, "draft", target.dtype)
            raise ValueError("draft must be on the target's device")
        if draft.shape != target.shape or draft.stride(1) != 1:
            raise ValueError("draft must have the shape of target, with a unit vocab stride")
    _check(tokens, "tokens", torch.int32, dev, (rows,))
    _check(parents, "parents", torch.int32, dev, (rows,))
    _check(uniforms, "uniforms", torch.float32, dev, (rows,))
    _check(last_uniforms, "last_uniforms", torch.float32, dev, (B,))
    if token_offsets is not None:
        _check(token_offsets, "token_offsets", torch.int32, dev, (B + 1,))
    if max_path is None:
        if token_offsets is not None:
            raise ValueError("max_path is needed with token_offsets")
        max_path = max(1, rows // max(1, B))
    # (the stride of a single row says nothing)
    strides = [max(t.stride(0), vocab) if rows < 2 else t.stride(0)
               for t in (target, target if draft is None else draft)]
    opts = _lib.VerifyOpts(B, rows, vocab, int(max_path), kind, *strides)
    ws = _call_workspace(workspace, _lib.verify_workspace_bytes(opts), dev, target.device)
    accepted, counts, following = tokens.new_empty((B, int(max_path))), tokens.new_empty(B), tokens.new_empty(B)
    st = _on_device(dev, _lib.verify_drafts, opts, target.data_ptr(), _ptr(draft), tokens.data_ptr(),
                    parents.data_ptr(), _ptr(token_offsets), uniforms.data_ptr(),
                    last_uniforms.data_ptr(), accepted.data_ptr(), counts.data_ptr(),
                    following.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size())
    if st != _lib.OK:
        raise ArtError(st, "art_verify_drafts")
    return accepted, counts, following


def keep_accepted(k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor,
                  context_lens: torch.Tensor, accepted: torch.Tensor, counts: torch.Tensor) -> None:
    """Move the accepted nodes' keys and values up to the context's end, on the
    current stream: node accepted[b][j] to slot context_lens[b] + j for j <
    counts[b] (as ``verify_drafts`` returns them).  The sequence then holds
    context_lens[b] + counts[b] tokens; ``context_lens`` stays the caller's to
    advance."""
    dev, H, B, fields = _bf16_pools(k_cache, v_cache, page_table)
    _check(context_lens, "context_lens", torch.int32, dev, (B,))
    if accepted.dim() != 2:
        raise ValueError("accepted must be [batch][max_path]")
    _check(accepted, "accepted", torch.int32, dev, (B, accepted.shape[1]))
    _check(counts, "counts", torch.int32, dev, (B,))
    shape = DecodeShape(B, H, H, k_cache.shape[3], 64, *fields)
    st = _on_device(dev, _lib.keep_accepted, shape, accepted.shape[1], accepted.data_ptr(),
                    counts.data_ptr(), context_lens.data_ptr(), page_table.data_ptr(),
                    k_cache.data_ptr(), v_cache.data_ptr())
    if st != _lib.OK:
        raise ArtError(st, "art_keep_accepted")
