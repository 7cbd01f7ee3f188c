"""Decode attention with shaped scores, the packed (4-bit) KV cache, and eviction.

Beside plain decode attention over bf16 caches, a program that decodes long or
many contexts needs scores that are capped, biased by distance or masked, a
smaller cache, and a way to drop the tokens that matter least:

* ``shaped_decode_attention`` (bf16 caches) and ``packed_decode_attention``
  (packed caches): for the tokens t that request b sees (``t < prefix_lens[b]`` or
  ``t >= starts[b]``, below its length L),
  ``x = scale * q.k``, ``x = softcap * tanh(x / softcap)``,
  ``x += slopes[h] * (t - (L - 1))``, then softmax and the weighted values;
* ``new_packed_kv_cache``, ``packed_append``, ``packed_gather``: uint8
  ``[num_blocks, num_kv_heads, 2176]``, 4-bit numbers with a power of two for every 32
  dims of a token, 0.27 of the bf16 bytes;
* ``add_attention_weights`` / ``packed_add_attention_weights`` and ``kv_evict`` /
  ``packed_evict``: running sums of the attention weights, and the move of the tokens
  with the largest ones to new blocks.

Like the package's other calls, these run the library's HIP kernels on torch's
current stream (or ``stream``) without synchronising, and raise without a GPU.
"""
from __future__ import annotations

import ctypes
import math

import paper_2411_01142_amd as _neo

__all__ = [
    "shaped_decode_attention", "packed_decode_attention", "new_packed_kv_cache",
    "packed_append", "packed_gather", "add_attention_weights",
    "packed_add_attention_weights", "kv_evict", "packed_evict", "PACKED_RECORD_BYTES",
]

PACKED_RECORD_BYTES = 2176
_BLOCK, _DIM = 16, 128
_SCALE = 1.0 / math.sqrt(_DIM)


class _ScoreShape(ctypes.Structure):
    _fields_ = [("softcap", ctypes.c_float), ("slopes", ctypes.c_void_p),
                ("starts", ctypes.c_void_p), ("prefix_lens", ctypes.c_void_p)]


def declare(lib):
    """The C signatures of this module's entry points."""
    P, I, F, S, L = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t,
                     ctypes.c_int64)
    shape = ctypes.POINTER(_ScoreShape)
    signatures = {
        "neo_shaped_decode_attention": [P, P, P, P, P, I, I, I, I, F, shape, P, P, I, I, I, L, P,
                                        S, P],
        "neo_packed_decode_attention": [P, P, P, P, I, I, I, I, F, shape, P, P, I, I, I, L, P, S,
                                        P],
        "neo_packed_append": [P, P, P, P, I, L, L, L, L, P, P, I, I, I, I, I, I, L, P],
        "neo_packed_gather": [P, P, I, P, P, I, I, I, I, I, I, L, P, P, P],
        "neo_add_attention_weights": [P, P, L, P, P, P, P, P, I, I, I, I, F, shape, I, I, I, L,
                                      P],
        "neo_packed_add_attention_weights": [P, P, L, P, P, P, P, P, I, I, I, I, F, shape, I, I,
                                             I, L, P],
        "neo_kv_evict": [P, P, P, P, P, L, P, I, P, I, P, P, P, I, I, I, I, I, I, L, P],
        "neo_packed_evict": [P, P, P, P, L, P, I, P, I, P, P, P, I, I, I, I, I, I, L, P],
    }
    for name, args in signatures.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int


# ------------------------------------------------------------------ checks

# As in the package's own calls, a kernel can be shorter than the Python around it, so
# the checks are written for the tensors that pass them: plain attributes compared once.
# What does not pass goes through the full ones, which say what is wrong.

_torch_module = None


def _t():
    global _torch_module
    if _torch_module is None:
        _torch_module = _neo._torch()
    return _torch_module


def _want(t, name, dtype, shape, device):
    """t's address if it is a contiguous tensor of this type and shape on ``device``."""
    if (type(t) is _t().Tensor and t.dtype is dtype and t.shape == shape and t.device == device
            and t.is_contiguous()):
        return t.data_ptr()
    _neo._require(t, name, dtype, len(shape))
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {shape} (got {tuple(t.shape)})")
    if t.device != device:
        raise ValueError(f"{name} must be on {device} (got {t.device})")
    return t.data_ptr()


def _device_of(t, name):
    if not isinstance(t, _t().Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU (got {t.device}); there is no CPU path")
    return t.device


def _bf16_caches(k_cache, v_cache):
    """(blocks, kv heads, block stride in elements); v_cache may be None."""
    torch = _t()
    shape, stride = k_cache.shape, k_cache.stride()
    if (k_cache.dtype is torch.bfloat16 and len(shape) == 5 and shape[2:] == (16, 16, 8)
            and stride[1:] == (2048, 128, 8, 1) and stride[0] % 8 == 0
            and stride[0] >= shape[1] * 2048):
        if v_cache is None:
            return shape[0], shape[1], stride[0]
        if (type(v_cache) is torch.Tensor and v_cache.dtype is torch.bfloat16
                and v_cache.shape == (shape[0], shape[1], _DIM, _BLOCK)
                and v_cache.stride() == (stride[0], 2048, 16, 1)
                and v_cache.device == k_cache.device):
            return shape[0], shape[1], stride[0]
    if v_cache is None:
        block_stride = _neo._require_cache(k_cache, "k_cache", 5)
    else:
        block_stride = _neo._shared_stride(k_cache, "k_cache", v_cache, "v_cache")
    nb, hkv = k_cache.shape[:2]
    if tuple(k_cache.shape[2:]) != (_DIM // 8, _BLOCK, 8):
        raise ValueError(f"k_cache must be [blocks, kv heads, 16, 16, 8] (got {tuple(k_cache.shape)})")
    if v_cache is not None:
        if tuple(v_cache.shape) != (nb, hkv, _DIM, _BLOCK):
            raise ValueError(f"v_cache shape {tuple(v_cache.shape)} != {(nb, hkv, _DIM, _BLOCK)}")
        if v_cache.device != k_cache.device:
            raise ValueError("k_cache and v_cache must be on one device")
    return nb, hkv, block_stride


def _packed_cache(cache):
    """(blocks, kv heads, block stride in bytes)."""
    shape, stride = cache.shape, cache.stride()
    if cache.dtype is not _t().uint8:
        raise TypeError(f"cache must be torch.uint8 (got {cache.dtype})")
    if len(shape) != 3 or shape[2] != PACKED_RECORD_BYTES:
        raise ValueError(f"cache must be [blocks, kv heads, {PACKED_RECORD_BYTES}] "
                         f"(got {tuple(shape)})")
    if (stride[1:] != (PACKED_RECORD_BYTES, 1) or stride[0] < shape[1] * PACKED_RECORD_BYTES
            or stride[0] % 16 != 0):
        raise ValueError("cache must be dense within each block, with a block stride that is a "
                         f"multiple of 16 bytes of at least one block (strides {stride})")
    return shape[0], shape[1], stride[0]


def _tables(block_table, seq_lens, device):
    """(batch, table width, addresses of both)."""
    torch = _t()
    if not isinstance(block_table, torch.Tensor):
        raise TypeError("block_table must be a torch.Tensor")
    shape = block_table.shape
    if len(shape) != 2:
        raise ValueError(f"block_table must have 2 dims (got shape {tuple(shape)})")
    B, width = shape
    return (B, width, _want(block_table, "block_table", torch.int32, (B, width), device),
            _want(seq_lens, "seq_lens", torch.int32, (B,), device))


def _queries(q, B, device):
    """(query heads, address)."""
    torch = _t()
    if not isinstance(q, torch.Tensor):
        raise TypeError("q must be a torch.Tensor")
    if q.dim() != 3:
        raise ValueError(f"q must have 3 dims (got shape {tuple(q.shape)})")
    hq = q.shape[1]
    return hq, _want(q, "q", torch.bfloat16, (B, hq, _DIM), device)


def _score_shape(softcap, slopes, starts, prefix_lens, B, hq, device):
    """The C structure, or None where scores are plain."""
    if softcap is None and slopes is None and starts is None and prefix_lens is None:
        return None
    torch = _t()
    return _ScoreShape(
        0.0 if softcap is None else softcap,
        None if slopes is None else _want(slopes, "slopes", torch.float32, (hq,), device),
        None if starts is None else _want(starts, "starts", torch.int32, (B,), device),
        None if prefix_lens is None else _want(prefix_lens, "prefix_lens", torch.int32, (B,),
                                               device))


def _new(shape, dtype, device, stream):
    """A tensor of the pool of the stream that is going to write it."""
    torch = _t()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _capturing(stream):
    torch = _t()
    if stream is None:
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


# --------------------------------------------------------------- attention

def _attend(packed, q, caches, block_table, seq_lens, scale, out, softcap, slopes, starts,
            prefix_lens, lse, workspace, stream):
    torch = _t()
    lib = _neo._lib or _neo.load_library()
    device = _device_of(caches[0], "cache" if packed else "k_cache")
    nb, hkv, stride = _packed_cache(*caches) if packed else _bf16_caches(*caches)
    B, width, table_at, lens_at = _tables(block_table, seq_lens, device)
    hq, q_at = _queries(q, B, device)
    shape = _score_shape(softcap, slopes, starts, prefix_lens, B, hq, device)
    if out is None:
        out = _new((B, hq, _DIM), torch.float32, device, stream)
        out_at = out.data_ptr()
    else:
        out_at = _want(out, "out", torch.float32, (B, hq, _DIM), device)
    lse_at = None if lse is None else _want(lse, "lse", torch.float32, (B, hq), device)
    need = _neo._cached_workspace_bytes(B, hq, hkv, _DIM)
    if B == 0:
        return out
    handle = _neo._raw_stream(torch, stream, device)
    if workspace is None:
        if _capturing(stream):
            raise ValueError("a call that is captured in a graph needs a workspace of its own "
                             "(new_workspace)")
        workspace = _neo._workspaces.get((device.index, handle))
        if workspace is None or workspace.numel() < need:
            workspace = _neo._workspace(need, device, _neo._stream_of(stream, device))
    else:
        _neo._require(workspace, "workspace", torch.uint8, 1)
        if workspace.device != device:
            raise ValueError("all tensors must be on one device")
    fn = lib.neo_packed_decode_attention if packed else lib.neo_shaped_decode_attention
    args = (q_at, *(c.data_ptr() for c in caches), table_at, lens_at, hq, hkv, _DIM, _BLOCK,
            _SCALE if scale is None else scale, shape, out_at, lse_at, B,
            width, nb, stride, workspace.data_ptr(), workspace.numel(), handle)
    _neo._check(_neo._on_device(torch, device, fn, args))
    return out


def shaped_decode_attention(q, k_cache, v_cache, block_table, seq_lens, scale=None, out=None, *,
                            softcap=None, slopes=None, starts=None, prefix_lens=None, lse=None,
                            workspace=None, stream=None):
    """Decode attention over bf16 caches with shaped scores; returns ``out`` (fp32 [B, Hq, 128]).

    ``softcap`` (None or 0: none) caps scores by a tanh; ``slopes`` (fp32 [Hq]) biases
    them by distance; ``starts`` and ``prefix_lens`` (int32 [B]) are the tokens that a
    request sees: ``t < prefix_lens[b]`` or ``t >= starts[b]``. ``lse`` (fp32 [B, Hq]), if
    given, receives the rows' log-sum-exps. A request that sees nothing gets zeros and
    minus infinity. The other arguments are ``decode_attention``'s; a workspace may serve
    both, and a call captured in a graph needs one of its own.
    """
    return _attend(False, q, (k_cache, v_cache), block_table, seq_lens, scale, out, softcap,
                   slopes, starts, prefix_lens, lse, workspace, stream)


def packed_decode_attention(q, cache, block_table, seq_lens, scale=None, out=None, *,
                            softcap=None, slopes=None, starts=None, prefix_lens=None, lse=None,
                            workspace=None, stream=None):
    """``shaped_decode_attention`` over a packed cache (``new_packed_kv_cache``)."""
    return _attend(True, q, (cache,), block_table, seq_lens, scale, out, softcap, slopes, starts,
                   prefix_lens, lse, workspace, stream)


# ------------------------------------------------------------ packed cache

def new_packed_kv_cache(num_blocks: int, num_kv_heads: int, device="cuda"):
    """A packed cache: uint8 ``[num_blocks, num_kv_heads, 2176]``, K and V of a block and kv
    head in one record (a quarter of the bf16 bytes and a sixteenth). Uninitialised."""
    torch = _t()
    return torch.empty((num_blocks, num_kv_heads, PACKED_RECORD_BYTES), dtype=torch.uint8,
                       device=device)


def _row_strides(t, name, rows, hkv, device):
    """(row stride, head stride) in elements of bf16 rows [rows, Hkv, 128] that may be a view
    into something larger, such as a fused projection's output."""
    torch = _t()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} must be on {device} (got {t.device})")
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name} must be torch.bfloat16 (got {t.dtype})")
    shape = t.shape
    if len(shape) != 3 or (rows is not None and shape[0] != rows) or shape[1:] != (hkv, _DIM):
        raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, {hkv}, {_DIM}] "
                         f"(got {tuple(shape)})")
    r, h, d = t.stride()
    if d != 1 or r % 8 != 0 or h % 8 != 0 or t.data_ptr() % 16 != 0:
        raise ValueError(f"{name} must have its dims in a run, strides that are multiples of 8 "
                         f"and 16-byte alignment (strides {t.stride()})")
    return (r if shape[0] > 1 else 0), (h if hkv > 1 else 0)


def packed_append(cache, k_new, v_new, block_table, seq_lens, row_starts=None, *, stream=None):
    """Write new tokens (k_new, v_new: bf16 [rows, Hkv, 128], possibly strided) into a packed
    cache, in place. Without ``row_starts`` row b is request b's newest token; with it (int32
    [B + 1], ascending), rows ``row_starts[b] .. row_starts[b + 1] - 1`` are its last tokens,
    as after a prompt. ``seq_lens`` counts them. Rows past ``row_starts[B]`` are skipped."""
    torch = _t()
    lib = _neo._lib or _neo.load_library()
    device = _device_of(cache, "cache")
    nb, hkv, stride = _packed_cache(cache)
    B, width, table_at, lens_at = _tables(block_table, seq_lens, device)
    starts_at = None
    if row_starts is not None:
        starts_at = _want(row_starts, "row_starts", torch.int32, (B + 1,), device)
    kr, kh = _row_strides(k_new, "k_new", None if row_starts is not None else B, hkv, device)
    rows = k_new.shape[0]
    vr, vh = _row_strides(v_new, "v_new", rows, hkv, device)
    args = (cache.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), starts_at, rows, kr, kh, vr, vh,
            table_at, lens_at, B, width, hkv, _DIM, _BLOCK, nb, stride,
            _neo._raw_stream(torch, stream, device))
    _neo._check(_neo._on_device(torch, device, lib.neo_packed_append, args))


def packed_gather(cache, block_table, seq_lens, row_starts=None, k_out=None, v_out=None, *,
                  rows=None, stream=None):
    """(k, v) bf16 [rows, Hkv, 128]: the tokens that ``packed_append`` with the same
    ``row_starts`` and lengths would write, read back exactly. The number of rows is that of
    ``k_out`` and ``v_out``, or ``rows``, or without ``row_starts`` the batch. Rows that have no
    token are left as they were (new outputs: zero)."""
    torch = _t()
    lib = _neo._lib or _neo.load_library()
    device = _device_of(cache, "cache")
    nb, hkv, stride = _packed_cache(cache)
    B, width, table_at, lens_at = _tables(block_table, seq_lens, device)
    starts_at = None
    if row_starts is not None:
        starts_at = _want(row_starts, "row_starts", torch.int32, (B + 1,), device)
    for t in (k_out, v_out):
        if t is not None and rows is None:
            rows = t.shape[0]
    if rows is None:
        if row_starts is not None:
            raise ValueError("rows (or k_out and v_out) must be given with row_starts")
        rows = B
    outs = []
    for t, name in ((k_out, "k_out"), (v_out, "v_out")):
        if t is None:
            t = _new((rows, hkv, _DIM), torch.bfloat16, device, stream)
            if stream is None:
                t.zero_()
            else:
                with torch.cuda.stream(stream):
                    t.zero_()
        _want(t, name, torch.bfloat16, (rows, hkv, _DIM), device)
        outs.append(t)
    args = (cache.data_ptr(), starts_at, rows, table_at, lens_at, B, width, hkv, _DIM, _BLOCK, nb,
            stride, outs[0].data_ptr(), outs[1].data_ptr(),
            _neo._raw_stream(torch, stream, device))
    _neo._check(_neo._on_device(torch, device, lib.neo_packed_gather, args))
    return tuple(outs)


# ---------------------------------------------------------------- eviction

def _sums_stride(sums, name, B, hkv, width, device):
    torch = _t()
    if not isinstance(sums, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if sums.dim() != 3 or sums.shape[2] < width * _BLOCK:
        raise ValueError(f"{name} must be [batch, kv heads, at least {width * _BLOCK}] "
                         f"(got {tuple(sums.shape)})")
    _want(sums, name, torch.float32, (B, hkv, sums.shape[2]), device)
    return sums.shape[2]


def _add_weights(packed, sums, lse, q, cache, block_table, seq_lens, scale, out, softcap, slopes,
                 starts, prefix_lens, stream):
    torch = _t()
    lib = _neo._lib or _neo.load_library()
    device = _device_of(cache, "cache" if packed else "k_cache")
    nb, hkv, stride = _packed_cache(cache) if packed else _bf16_caches(cache, None)
    B, width, table_at, lens_at = _tables(block_table, seq_lens, device)
    hq, q_at = _queries(q, B, device)
    S = _sums_stride(sums, "sums", B, hkv, width, device)
    if out is None:
        out = sums
    else:
        _want(out, "out", torch.float32, (B, hkv, S), device)
        a, b, n = sums.data_ptr(), out.data_ptr(), 4 * sums.numel()
        if a != b and a < b + n and b < a + n:
            raise ValueError("out must be sums or not overlap it")
    lse_at = _want(lse, "lse", torch.float32, (B, hq), device)
    shape = _score_shape(softcap, slopes, starts, prefix_lens, B, hq, device)
    fn = lib.neo_packed_add_attention_weights if packed else lib.neo_add_attention_weights
    args = (sums.data_ptr(), out.data_ptr(), S, lse_at, q_at, cache.data_ptr(), table_at, lens_at,
            hq, hkv, _DIM, _BLOCK, _SCALE if scale is None else scale, shape,
            B, width, nb, stride, _neo._raw_stream(torch, stream, device))
    _neo._check(_neo._on_device(torch, device, fn, args))
    return out


def add_attention_weights(sums, lse, q, k_cache, block_table, seq_lens, scale=None, out=None, *,
                          softcap=None, slopes=None, starts=None, prefix_lens=None, stream=None):
    """Add one step's attention weights to ``sums`` (fp32 [B, Hkv, S], S at least 16 times the
    table's width): for every token that a request sees, the sum over the kv head's query heads of
    ``exp(score - lse)``. ``lse`` is what ``shaped_decode_attention`` wrote for the same
    arguments. Writes ``out`` (default: ``sums``, in place), elsewhere leaving it as it was, and
    returns it."""
    return _add_weights(False, sums, lse, q, k_cache, block_table, seq_lens, scale, out, softcap,
                        slopes, starts, prefix_lens, stream)


def packed_add_attention_weights(sums, lse, q, cache, block_table, seq_lens, scale=None, out=None,
                                 *, softcap=None, slopes=None, starts=None, prefix_lens=None,
                                 stream=None):
    """``add_attention_weights`` for a packed cache."""
    return _add_weights(True, sums, lse, q, cache, block_table, seq_lens, scale, out, softcap,
                        slopes, starts, prefix_lens, stream)


def _evict(packed, caches, block_table, seq_lens, sums, budgets, new_table, recent, stream):
    torch = _t()
    lib = _neo._lib or _neo.load_library()
    device = _device_of(caches[0], "cache" if packed else "k_cache")
    nb, hkv, stride = _packed_cache(*caches) if packed else _bf16_caches(*caches)
    B, width, table_at, lens_at = _tables(block_table, seq_lens, device)
    S = _sums_stride(sums, "sums", B, hkv, width, device)
    budgets_at = _want(budgets, "budgets", torch.int32, (B,), device)
    if not isinstance(new_table, torch.Tensor):
        raise TypeError("new_table must be a torch.Tensor")
    if new_table.dim() != 2:
        raise ValueError(f"new_table must have 2 dims (got shape {tuple(new_table.shape)})")
    new_width = new_table.shape[1]
    new_at = _want(new_table, "new_table", torch.int32, (B, new_width), device)
    new_lens = _new((B,), torch.int32, device, stream)
    kept = _new((B, hkv, new_width * _BLOCK), torch.int32, device, stream)
    new_sums = _new((B, hkv, new_width * _BLOCK), torch.float32, device, stream)
    fn = lib.neo_packed_evict if packed else lib.neo_kv_evict
    args = (*(c.data_ptr() for c in caches), table_at, lens_at, sums.data_ptr(), S, budgets_at,
            int(recent), new_at, new_width, new_lens.data_ptr(), kept.data_ptr(),
            new_sums.data_ptr(), B, width, hkv, _DIM, _BLOCK, nb, stride,
            _neo._raw_stream(torch, stream, device))
    _neo._check(_neo._on_device(torch, device, fn, args))
    return new_lens, kept, new_sums


def kv_evict(k_cache, v_cache, block_table, seq_lens, sums, budgets, new_table, *, recent=0,
             stream=None):
    """Keep ``min(L, budgets[b])`` tokens of each request and kv head: the newest ``recent`` and
    those with the largest ``sums`` (equal ones: the lower token), copied in their order to the
    blocks of ``new_table`` (int32 [B, new width], distinct blocks of the same caches that
    ``block_table`` does not name; a budget above 16 times its width is cut to that). The old
    blocks are only read and are the caller's to free.
    Returns (new_lens int32 [B], kept int32 [B, Hkv, 16 * new width], new_sums fp32 likewise):
    the tokens' former positions and their sums, then -1 and 0."""
    return _evict(False, (k_cache, v_cache), block_table, seq_lens, sums, budgets, new_table,
                  recent, stream)


def packed_evict(cache, block_table, seq_lens, sums, budgets, new_table, *, recent=0, stream=None):
    """``kv_evict`` for a packed cache."""
    return _evict(True, (cache,), block_table, seq_lens, sums, budgets, new_table, recent, stream)
