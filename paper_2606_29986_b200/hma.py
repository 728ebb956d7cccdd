"""ctypes binding of libhma.so: the same entry points as include/hma.h, argument marshalling only.

Tensors are torch CUDA tensors (torch provides device memory and streams); every step of the
path runs inside the library's kernels.  Loading fails loudly when the library has not been
built: there is no fallback of any kind.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libhma.so")

HMA_OK = 0
HMA_ERR_INVALID_ARG, HMA_ERR_UNSUPPORTED_SHAPE, HMA_ERR_ALIGNMENT = 1, 2, 3
HMA_ERR_WORKSPACE_TOO_SMALL, HMA_ERR_CUDA = 4, 5
HMA_ERR_STATIC_LIMIT = 7
HMA_KV_BFP8, HMA_KV_BF16, HMA_KV_BFP4 = 0, 1, 2
HMA_WIRE_TILE32, HMA_WIRE_ROWMAJOR, HMA_WIRE_BF16_ROWS = 0, 1, 2
HMA_OUT_BF16, HMA_OUT_F32 = 0, 1
HMA_KEYS_AS_QUERIES, HMA_KEYS_INTERLEAVED = 0, 1
HMA_FLAG_BAD_PAGE_ATTENTION, HMA_FLAG_BAD_PAGE_INGEST, HMA_FLAG_BAD_PAGE_DEQUANT, HMA_FLAG_WAIT_TIMEOUT = 1, 2, 4, 8
HMA_FLAG_BAD_VALUE_ENCODE, HMA_FLAG_EXPONENT_RANGE, HMA_FLAG_BAD_PLAN = 16, 32, 64
HMA_FLAG_NO_PAGES, HMA_FLAG_BAD_LENGTHS, HMA_FLAG_BAD_POSITION = 128, 256, 512


class CacheDesc(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32), ("bfp_block", ctypes.c_int32),
                ("num_pages", ctypes.c_int64), ("format", ctypes.c_int32), ("key_layout", ctypes.c_int32)]


class HmaError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        detail = ""
        if status == HMA_ERR_CUDA:
            detail = ": " + hma_last_cuda_error()
        super().__init__("%s: %s (status %d)%s" % (where, status_string(status), status, detail))


_lib = None


def lib():
    """The loaded C-ABI library.  Raises if libhma.so is missing (build it with build.py)."""
    global _lib
    if _lib is None:
        # HMA_LIBRARY selects another build of the same sources (the instrumented libhma_trace.so), nothing else
        path = os.environ.get("HMA_LIBRARY") or _LIB_PATH
        if not os.path.exists(path):
            raise ImportError("%s is not built: run `python -m paper_2606_29986_b200.build`" % os.path.basename(path))
        L = ctypes.CDLL(path)
        vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        L.hma_cache_layer_bytes.restype = sz
        L.hma_cache_layer_bytes.argtypes = [ctypes.POINTER(CacheDesc)]
        L.hma_cache_create.restype = i32
        L.hma_cache_create.argtypes = [ctypes.POINTER(CacheDesc), ctypes.POINTER(vp), ctypes.POINTER(vp)]
        L.hma_cache_destroy.restype = None
        L.hma_cache_destroy.argtypes = [vp]
        L.hma_kv_ingest_layer.restype = i32
        L.hma_kv_ingest_layer.argtypes = [vp, i32, vp, vp, i32, i32, i32, vp, i64, i64, vp]
        L.hma_kv_ingest_layer_shards.restype = i32
        L.hma_kv_ingest_layer_shards.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), i32,
                                                 ctypes.POINTER(i32), ctypes.POINTER(i32), vp, i64, i64, vp]
        L.hma_kv_ingest_request_shards.restype = i32
        L.hma_kv_ingest_request_shards.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), sz, i32,
                                                   ctypes.POINTER(i32), ctypes.POINTER(i32), vp, i64, i64, vp]
        L.hma_step_tables.restype = i32
        L.hma_step_tables.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, i64, vp, vp]
        L.hma_release_pages.restype = i32
        L.hma_release_pages.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, vp]
        L.hma_rope_table.restype = i32
        L.hma_rope_table.argtypes = [ctypes.POINTER(ctypes.c_double), i32, i64, i64, ctypes.c_double, vp, vp]
        L.hma_kv_append.restype = i32
        L.hma_kv_append.argtypes = [vp, i32, vp, vp, i32, i64, i64, vp, i64, vp]
        L.hma_qk_norm_rope.restype = i32
        L.hma_qk_norm_rope.argtypes = [vp, i32, vp, i32, i64, i64, vp, vp, f32, vp, i64, i32, i32, vp, vp, vp, vp, vp]
        L.hma_decode_attention_workspace_bytes.restype = sz
        L.hma_decode_attention_workspace_bytes.argtypes = [ctypes.POINTER(CacheDesc), i32]
        L.hma_decode_attention_workspace_init.restype = i32
        L.hma_decode_attention_workspace_init.argtypes = [vp, sz, vp]
        L.hma_decode_attention.restype = i32
        L.hma_decode_attention.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, i32, f32, vp, sz, vp]
        L.hma_decode_attention_multi.restype = i32
        L.hma_decode_attention_multi.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, i32, i32, f32, vp, sz, vp]
        L.hma_decode_attention_window.restype = i32
        L.hma_decode_attention_window.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, i32, i32, i32, i32, f32, vp, sz, vp]
        L.hma_decode_attention_plan_bytes.restype = sz
        L.hma_decode_attention_plan_bytes.argtypes = [i32]
        L.hma_decode_attention_plan.restype = i32
        L.hma_decode_attention_plan.argtypes = [vp, vp, i32, vp, i32, i32, vp, sz, vp]
        L.hma_decode_attention_planned.restype = i32
        L.hma_decode_attention_planned.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, i32, i32, f32, vp, vp, sz, vp]
        L.hma_decode_attention_static.restype = i32
        L.hma_decode_attention_static.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, i32, f32, vp]
        L.hma_decode_attention_static_limit_bytes.restype = sz
        L.hma_decode_attention_static_limit_bytes.argtypes = []
        L.hma_kv_read_probe.restype = i32
        L.hma_kv_read_probe.argtypes = [vp, i32, vp, i32, vp, i32, vp, sz, vp]
        L.hma_hbm_read_probe.restype = i32
        L.hma_hbm_read_probe.argtypes = [vp, sz, vp, vp]
        L.hma_hbm_copy_probe.restype = i32
        L.hma_hbm_copy_probe.argtypes = [vp, sz, vp, sz, vp]
        L.hma_attention_alu_probe.restype = i32
        L.hma_attention_alu_probe.argtypes = [vp, i32, vp, i32, vp, i32, vp, sz, vp]
        L.hma_decode_attention_mixed.restype = i32
        L.hma_decode_attention_mixed.argtypes = [vp, vp, i32, vp, vp, i32, vp, i32, vp, vp, i32, vp, i32, f32, vp, sz, vp]
        L.hma_decode_attention_mixed_planned.restype = i32
        L.hma_decode_attention_mixed_planned.argtypes = [vp, vp, i32, vp, vp, i32, vp, i32, vp, vp, i32, vp, i32, f32, vp, vp, vp, sz, vp]
        L.hma_decode_attention_simple.restype = i32
        L.hma_decode_attention_simple.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, i32, f32, vp]
        L.hma_bfp8_dequant_bf16.restype = i32
        L.hma_bfp8_dequant_bf16.argtypes = [vp, i32, i32, vp, i64, i64, vp, vp]
        L.hma_bfp8_dequant_bf16_naive.restype = i32
        L.hma_bfp8_dequant_bf16_naive.argtypes = [vp, i32, i32, vp, i64, i64, vp, vp]
        L.hma_bfp8_rebuild_request.restype = i32
        L.hma_bfp8_rebuild_request.argtypes = [vp, vp, i64, i64, vp, vp]
        L.hma_bfp8_encode_rows.restype = i32
        L.hma_bfp8_encode_rows.argtypes = [vp, vp, i32, i64, vp, vp]
        L.hma_bfp8_dequant_blocks_bf16.restype = i32
        L.hma_bfp8_dequant_blocks_bf16.argtypes = [vp, vp, i64, vp, vp]
        L.hma_error_flags.restype = i32
        L.hma_error_flags.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32), vp]
        L.hma_status_string.restype = ctypes.c_char_p
        L.hma_status_string.argtypes = [i32]
        L.hma_last_cuda_error.restype = ctypes.c_char_p
        L.hma_last_cuda_error.argtypes = []
        L.hma_launch_count.restype = i64
        L.hma_launch_count.argtypes = []
        _lib = L
    return _lib


def status_string(status):
    return lib().hma_status_string(int(status)).decode()


def _check(status, where):
    if status != HMA_OK:
        raise HmaError(status, where)


def _stream(stream):
    """The cudaStream_t of `stream`, or of the current device's current stream (torch.cuda.current_stream() builds a Python object for
    it, 3 us a call; the raw handle is all that is needed)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _device():
    """The current device's number (-2 without a GPU: no tensor is there)."""
    try:
        return torch._C._cuda_getDevice()
    except RuntimeError:
        return -2


def _stream_of(dev, stream):
    """_stream for a call that knows the current device already."""
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _ptr(t):
    return t.data_ptr() if t is not None else None


def make_desc(num_layers, num_q_heads, num_kv_heads, num_pages, fmt=HMA_KV_BFP8, head_dim=128, page_tokens=16, bfp_block=16,
              key_layout=0):
    return CacheDesc(num_layers, num_q_heads, num_kv_heads, head_dim, page_tokens, bfp_block, num_pages, fmt, key_layout)


def hma_cache_layer_bytes(desc):
    return int(lib().hma_cache_layer_bytes(ctypes.byref(desc)))


def _fit(dev, *tensors):
    """Whether every (tensor, type, numbers it has to hold) is a contiguous tensor of that type on CUDA device `dev`; None, an argument
    that was left out, is.  (One call for all: the checks are what a small call's host time consists of, 0.25 us a tensor.)"""
    for t, dtype, n in tensors:
        if t is not None and (t.dtype is not dtype or t.get_device() != dev or t.numel() < n or not t.is_contiguous()):
            return False
    return True


def _refuse(where):
    raise HmaError(HMA_ERR_INVALID_ARG, where)


class KVCache:
    """Owns the torch uint8 layer buffers and the library's cache handle.  `layers` adopts existing buffers (one contiguous uint8
    CUDA tensor of hma_cache_layer_bytes per layer) instead of allocating them."""

    def __init__(self, desc, device="cuda", fill=None, layers=None):
        self.desc = desc
        nbytes = hma_cache_layer_bytes(desc)
        if nbytes == 0:
            raise HmaError(HMA_ERR_UNSUPPORTED_SHAPE, "hma_cache_layer_bytes")
        self.layers = []
        if layers is not None:
            if len(layers) != desc.num_layers:
                raise HmaError(HMA_ERR_INVALID_ARG, "KVCache")
            if not _fit(_device(), *[(t, torch.uint8, nbytes) for t in layers]):
                _refuse("KVCache")
            self.layers = list(layers)
        for _ in range(desc.num_layers - len(self.layers)):
            t = torch.empty(nbytes, dtype=torch.uint8, device=device)
            if fill is not None:
                t.fill_(fill)
            self.layers.append(t)
        ptrs = (ctypes.c_void_p * desc.num_layers)(*[t.data_ptr() for t in self.layers])
        handle = ctypes.c_void_p()
        _check(lib().hma_cache_create(ctypes.byref(desc), ptrs, ctypes.byref(handle)), "hma_cache_create")
        self.handle = handle

    def close(self):
        if getattr(self, "handle", None):
            lib().hma_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def hma_kv_ingest_layer(cache, layer, k_wire, v_wire, wire_layout, head_begin, head_count, page_ids,
                        token_begin, n_tokens, stream=None):
    _check(lib().hma_kv_ingest_layer(cache.handle, layer, _ptr(k_wire), _ptr(v_wire), wire_layout, head_begin,
                                     head_count, _ptr(page_ids), token_begin, n_tokens, _stream(stream)),
           "hma_kv_ingest_layer")


def hma_kv_ingest_layer_shards(cache, layer, k_wires, v_wires, wire_layout, head_begins, head_counts, page_ids,
                               token_begin, n_tokens, stream=None):
    """All producer shards of one layer in one launch; k_wires / v_wires are lists of tensors, one per shard."""
    n = len(k_wires)
    kp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in k_wires])
    vp_ = (ctypes.c_void_p * n)(*[t.data_ptr() for t in v_wires])
    hb = (ctypes.c_int32 * n)(*head_begins)
    hc = (ctypes.c_int32 * n)(*head_counts)
    _check(lib().hma_kv_ingest_layer_shards(cache.handle, layer, n, kp, vp_, wire_layout, hb, hc, _ptr(page_ids),
                                            token_begin, n_tokens, _stream(stream)), "hma_kv_ingest_layer_shards")


def hma_kv_ingest_request_shards(cache, k_wires, v_wires, layer_stride_bytes, wire_layout, head_begins, head_counts, page_ids,
                                 token_begin, n_tokens, stream=None):
    """Every layer of the cache in one call: k_wires / v_wires are lists (one per shard) of layer 0's wire tensors; layer l's
    wire starts l * layer_stride_bytes further on in the same allocation."""
    n = len(k_wires)
    kp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in k_wires])
    vp_ = (ctypes.c_void_p * n)(*[t.data_ptr() for t in v_wires])
    hb = (ctypes.c_int32 * n)(*head_begins)
    hc = (ctypes.c_int32 * n)(*head_counts)
    _check(lib().hma_kv_ingest_request_shards(cache.handle, n, kp, vp_, layer_stride_bytes, wire_layout, hb, hc, _ptr(page_ids),
                                              token_begin, n_tokens, _stream(stream)), "hma_kv_ingest_request_shards")


def hma_step_tables(cache, past_lens, new_lens, block_table, free_pages, free_count, context_lens, row_starts, positions, slots,
                    free_count_out=None, stream=None):
    """Pages, context lengths, row starts, positions and slots of one step's new tokens (see include/hma.h).  positions and slots
    are as long as the (padded) token buffer; free_count_out defaults to free_count, in place."""
    b, n, dev, i32 = past_lens.shape[0], positions.numel(), _device(), torch.int32
    left = free_count if free_count_out is None else free_count_out
    if not (_fit(dev, (past_lens, i32, b), (new_lens, i32, b), (block_table, i32, 0), (free_pages, i32, cache.desc.num_pages), (free_count, i32, 1),
                 (context_lens, i32, b), (row_starts, i32, b + 1), (positions, i32, n), (slots, torch.int64, n), (left, i32, 1)) and
            block_table.dim() == 2 and block_table.shape[0] >= b):
        _refuse("hma_step_tables")
    _check(lib().hma_step_tables(cache.handle, past_lens.data_ptr(), new_lens.data_ptr(), b, block_table.data_ptr(), block_table.shape[1],
                                 free_pages.data_ptr(), free_count.data_ptr(), context_lens.data_ptr(), row_starts.data_ptr(),
                                 positions.data_ptr(), slots.data_ptr(), n, left.data_ptr(), _stream_of(dev, stream)), "hma_step_tables")


def hma_release_pages(cache, finished, context_lens, block_table, free_pages, free_count, stream=None):
    """Pages of the sequences with finished[b] != 0 go back to the free list."""
    b, dev, i32 = context_lens.shape[0], _device(), torch.int32
    if not (_fit(dev, (finished, i32, b), (context_lens, i32, b), (block_table, i32, 0), (free_pages, i32, cache.desc.num_pages), (free_count, i32, 1)) and
            block_table.dim() == 2 and block_table.shape[0] >= b):
        _refuse("hma_release_pages")
    _check(lib().hma_release_pages(cache.handle, _ptr(finished), _ptr(context_lens), b, _ptr(block_table), block_table.shape[1],
                                   _ptr(free_pages), _ptr(free_count), _stream_of(dev, stream)), "hma_release_pages")


def hma_rope_table(inv_freq, n_pos, first_pos=0, scale=1.0, table=None, device="cuda", stream=None):
    """fp32 [n_pos][rotary_dim] table (cosines, then sines) for hma_qk_norm_rope; inv_freq: rotary_dim / 2 floats."""
    f = [float(x) for x in inv_freq]
    if table is None:
        table = torch.empty((n_pos, 2 * len(f)), dtype=torch.float32, device=device)
    if not _fit(_device(), (table, torch.float32, n_pos * 2 * len(f))):
        _refuse("hma_rope_table")
    _check(lib().hma_rope_table((ctypes.c_double * len(f))(*f), 2 * len(f), first_pos, n_pos, float(scale), _ptr(table), _stream(stream)),
           "hma_rope_table")
    return table


def _in_dtype(where, t, dev):
    """hma_out_dtype_t of an input tensor; anything but BF16 and F32 on device `dev` is refused."""
    if t.get_device() == dev:
        if t.dtype is torch.bfloat16:
            return HMA_OUT_BF16
        if t.dtype is torch.float32:
            return HMA_OUT_F32
    _refuse(where)


def hma_kv_append(cache, layer, k, v, slots, stream=None):
    """K and V rows [tokens][kv heads][128] (BF16 or FP32; the token stride is free, so slices of a projection's output do) into
    the cache at slots (int64 [tokens], -1 skips a row)."""
    n, heads, dev = slots.numel(), cache.desc.num_kv_heads, _device()
    dt = _in_dtype("hma_kv_append", k, dev)
    if not _fit(dev, (slots, torch.int64, n)):
        _refuse("hma_kv_append")
    st, sv = k.stride(), v.stride()
    if (v.dtype is not k.dtype or v.get_device() != dev or k.shape != (n, heads, 128) or v.shape != (n, heads, 128) or
            st[2] != 1 or sv[2] != 1 or (heads > 1 and (st[1] != 128 or sv[1] != 128))):
        _refuse("hma_kv_append")
    _check(lib().hma_kv_append(cache.handle, layer, k.data_ptr(), v.data_ptr(), dt, st[0], sv[0], slots.data_ptr(), n,
                               _stream_of(dev, stream)), "hma_kv_append")


def hma_qk_norm_rope(cache, layer, qkv, q_weight, k_weight, eps, rope_table, positions, q_out, k_out=None, slots=None,
                     interleaved=False, stream=None):
    """qkv [tokens][(q heads + 2 kv heads) * 128] (BF16 or FP32, free token stride) -> normed and rotated queries in q_out, keys in
    k_out and / or keys and values in the cache at slots.  rope_table: hma_rope_table's, or None for no rotation."""
    n, d, dev, where = qkv.shape[0], cache.desc, _device(), "hma_qk_norm_rope"
    dt, hq, hkv = _in_dtype(where, qkv, dev), d.num_q_heads, d.num_kv_heads
    st, rows, rotary = qkv.stride(), 0, 0
    if rope_table is not None:
        if rope_table.dim() != 2 or positions is None:
            _refuse(where)
        rows, rotary = rope_table.shape
    if not (len(st) == 2 and st[1] == 1 and qkv.shape[1] == (hq + 2 * hkv) * 128 and
            _fit(dev, (q_out, torch.bfloat16, n * hq * 128), (k_out, torch.bfloat16, n * hkv * 128), (slots, torch.int64, n), (q_weight, qkv.dtype, 128),
                 (k_weight, qkv.dtype, 128), (rope_table, torch.float32, 0), (positions if rotary else None, torch.int32, n))):
        _refuse(where)
    _check(lib().hma_qk_norm_rope(cache.handle, layer, qkv.data_ptr(), dt, st[0], n, _ptr(q_weight), _ptr(k_weight), eps, _ptr(rope_table),
                                  rows, rotary, 1 if interleaved else 0, _ptr(positions), _ptr(slots), q_out.data_ptr(), _ptr(k_out),
                                  _stream_of(dev, stream)), where)


def hma_decode_attention_workspace_bytes(desc, batch):
    return int(lib().hma_decode_attention_workspace_bytes(ctypes.byref(desc), batch))


def hma_decode_attention_workspace_init(workspace, stream=None):
    """Zero-fills a workspace (required once before its first use; calls leave it ready for the next one)."""
    _check(lib().hma_decode_attention_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "hma_decode_attention_workspace_init")


def new_workspace(desc, batch, device="cuda", copies=1):
    """A torch uint8 tensor sized for hma_decode_attention on `batch` sequences (`copies` = 2 for the two-cache call,
    each half rounded up to 256 bytes) and initialised through hma_decode_attention_workspace_init."""
    n = (hma_decode_attention_workspace_bytes(desc, batch) + 255) // 256 * 256
    ws = torch.empty(copies * n, dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):
        hma_decode_attention_workspace_init(ws)
    return ws


def hma_decode_attention(cache, layer, q, out, block_table, context_lens, sm_scale, workspace, stream=None):
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    _check(lib().hma_decode_attention(cache.handle, layer, _ptr(q), _ptr(out), out_dtype, _ptr(block_table),
                                      block_table.shape[1], _ptr(context_lens), q.shape[0], float(sm_scale),
                                      _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "hma_decode_attention")


def hma_decode_attention_multi(cache, layer, q, out, block_table, context_lens, sm_scale, workspace, stream=None):
    """q, out: [batch][q_len][Hq][128]; the last q_len cached tokens of each sequence are the query tokens (causal)."""
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    _check(lib().hma_decode_attention_multi(cache.handle, layer, _ptr(q), _ptr(out), out_dtype, _ptr(block_table),
                                            block_table.shape[1], _ptr(context_lens), q.shape[0], q.shape[1], float(sm_scale),
                                            _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "hma_decode_attention_multi")


def _int32(n):
    """`n` as an int32 of the C ABI, numbers beyond its range held at its ends (ctypes would drop their upper bits)."""
    return max(-1 << 31, min(int(n), (1 << 31) - 1))


def hma_decode_attention_window(cache, layer, q, out, block_table, context_lens, window, sinks, sm_scale, workspace, stream=None):
    """Attention over the last `window` tokens and the first `sinks` ones; q, out: [batch][Hq][128], or [batch][q_len][Hq][128] with the
    last q_len cached tokens of each sequence as the query tokens, each with a window of its own.  Either number may exceed the context by
    any amount."""
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    shape, n, dev, where = q.shape, q.numel(), _device(), "hma_decode_attention_window"
    b, q_len = shape[0], shape[1] if len(shape) == 4 else 1
    if not (len(shape) in (3, 4) and shape[-2] == cache.desc.num_q_heads and shape[-1] == 128 and block_table.dim() == 2 and
            _fit(dev, (q, torch.bfloat16, n), (out, torch.float32 if out_dtype == HMA_OUT_F32 else torch.bfloat16, n), (context_lens, torch.int32, b),
                 (block_table, torch.int32, 0)) and block_table.shape[0] >= b and workspace.get_device() == dev):
        raise HmaError(HMA_ERR_UNSUPPORTED_SHAPE if b * q_len > 1024 else HMA_ERR_INVALID_ARG, where)
    _check(lib().hma_decode_attention_window(cache.handle, layer, _ptr(q), _ptr(out), out_dtype, _ptr(block_table),
                                             block_table.shape[1], _ptr(context_lens), b, q_len, _int32(window), _int32(sinks),
                                             float(sm_scale), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                             _stream_of(dev, stream)), where)


def hma_decode_attention_plan_bytes(rows):
    """Bytes of a plan for `rows` = sequences x query tokens per sequence."""
    return int(lib().hma_decode_attention_plan_bytes(rows))


def hma_decode_attention_plan(cache, block_table, context_lens, q_len=1, plan=None, stream=None):
    """Runs the attention kernel's set-up for this block table and these context lengths once and returns the plan (a uint8
    device tensor, reused when given); valid for every layer until the table or the lengths change."""
    batch = context_lens.shape[0]
    need = hma_decode_attention_plan_bytes(batch * q_len)
    if plan is None:
        plan = torch.empty(need, dtype=torch.uint8, device=context_lens.device)
    _check(lib().hma_decode_attention_plan(cache.handle, _ptr(block_table), block_table.shape[1], _ptr(context_lens), batch, q_len,
                                           _ptr(plan), plan.numel(), _stream(stream)), "hma_decode_attention_plan")
    return plan


def hma_decode_attention_planned(cache, layer, q, out, block_table, context_lens, sm_scale, plan, workspace, stream=None):
    """hma_decode_attention (q, out: [batch][Hq][128]) or hma_decode_attention_multi (q, out: [batch][q_len][Hq][128]) with the
    set-up taken from `plan` (hma_decode_attention_plan with the same table, lengths and q_len)."""
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    q_len = q.shape[1] if q.dim() == 4 else 1
    _check(lib().hma_decode_attention_planned(cache.handle, layer, _ptr(q), _ptr(out), out_dtype, _ptr(block_table),
                                              block_table.shape[1], _ptr(context_lens), q.shape[0], q_len, float(sm_scale),
                                              _ptr(plan), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                              _stream(stream)), "hma_decode_attention_planned")


def hma_decode_attention_static(cache, layer, q, out, block_table, context_lens, sm_scale, stream=None):
    """hma_decode_attention without a workspace argument, for callers that cannot allocate device memory.

    The scratch is an array inside the library (hma_decode_attention_static_limit_bytes() bytes on every GPU
    that loads it).  Raises HmaError(HMA_ERR_STATIC_LIMIT) when batch * kv heads is too large for it.  Calls
    on one device share the array: keep them on one stream.  Make the first call outside stream capture."""
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    _check(lib().hma_decode_attention_static(cache.handle, layer, _ptr(q), _ptr(out), out_dtype, _ptr(block_table),
                                             block_table.shape[1], _ptr(context_lens), q.shape[0], float(sm_scale),
                                             _stream(stream)), "hma_decode_attention_static")


def hma_decode_attention_static_limit_bytes():
    return int(lib().hma_decode_attention_static_limit_bytes())


def hma_kv_read_probe(cache, layer, block_table, context_lens, workspace, stream=None):
    _check(lib().hma_kv_read_probe(cache.handle, layer, _ptr(block_table), block_table.shape[1], _ptr(context_lens),
                                   context_lens.shape[0], _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream)), "hma_kv_read_probe")


def hma_attention_alu_probe(cache, layer, block_table, context_lens, workspace, stream=None):
    _check(lib().hma_attention_alu_probe(cache.handle, layer, _ptr(block_table), block_table.shape[1], _ptr(context_lens),
                                         context_lens.shape[0], _ptr(workspace), workspace.numel() * workspace.element_size(),
                                         _stream(stream)), "hma_attention_alu_probe")


def hma_hbm_read_probe(src, sink, stream=None):
    """Contiguous streaming read of the whole tensor `src` (a read-only memory ceiling); `sink` is a 4-byte device tensor."""
    _check(lib().hma_hbm_read_probe(_ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream(stream)), "hma_hbm_read_probe")


def hma_hbm_copy_probe(src, read_bytes, dst, write_bytes, stream=None):
    """Streaming read of `read_bytes` of `src` mixed with a streaming write of `write_bytes` of `dst` (a copy-like ceiling)."""
    assert read_bytes <= src.numel() * src.element_size() and write_bytes <= dst.numel() * dst.element_size()
    _check(lib().hma_hbm_copy_probe(_ptr(src), read_bytes, _ptr(dst), write_bytes, _stream(stream)), "hma_hbm_copy_probe")


def hma_decode_attention_mixed(prefix, tail, layer, q, out, prefix_table, prefix_lens, tail_table, tail_lens, sm_scale,
                               workspace, stream=None):
    """Attention over a BFP8 prefix cache and a BF16 tail cache (see include/hma.h)."""
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    _check(lib().hma_decode_attention_mixed(prefix.handle, tail.handle, layer, _ptr(q), _ptr(out), out_dtype,
                                            _ptr(prefix_table), prefix_table.shape[1], _ptr(prefix_lens),
                                            _ptr(tail_table), tail_table.shape[1], _ptr(tail_lens), q.shape[0],
                                            float(sm_scale), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                            _stream(stream)), "hma_decode_attention_mixed")


def hma_decode_attention_mixed_planned(prefix, tail, layer, q, out, prefix_table, prefix_lens, tail_table, tail_lens, sm_scale,
                                       prefix_plan, tail_plan, workspace, stream=None):
    """hma_decode_attention_mixed with both launches' set-up taken from plans (one per cache, hma_decode_attention_plan)."""
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    _check(lib().hma_decode_attention_mixed_planned(prefix.handle, tail.handle, layer, _ptr(q), _ptr(out), out_dtype,
                                                    _ptr(prefix_table), prefix_table.shape[1], _ptr(prefix_lens),
                                                    _ptr(tail_table), tail_table.shape[1], _ptr(tail_lens), q.shape[0],
                                                    float(sm_scale), _ptr(prefix_plan), _ptr(tail_plan), _ptr(workspace),
                                                    workspace.numel() * workspace.element_size(), _stream(stream)),
           "hma_decode_attention_mixed_planned")


def hma_decode_attention_simple(cache, layer, q, out, block_table, context_lens, sm_scale, stream=None):
    out_dtype = HMA_OUT_F32 if out.dtype == torch.float32 else HMA_OUT_BF16
    _check(lib().hma_decode_attention_simple(cache.handle, layer, _ptr(q), _ptr(out), out_dtype, _ptr(block_table),
                                             block_table.shape[1], _ptr(context_lens), q.shape[0], float(sm_scale),
                                             _stream(stream)), "hma_decode_attention_simple")


def hma_bfp8_dequant_bf16(cache, layer, which, page_ids, token_begin, n_tokens, out_bf16, stream=None):
    _check(lib().hma_bfp8_dequant_bf16(cache.handle, layer, which, _ptr(page_ids), token_begin, n_tokens,
                                       _ptr(out_bf16), _stream(stream)), "hma_bfp8_dequant_bf16")


def hma_bfp8_dequant_bf16_naive(cache, layer, which, page_ids, token_begin, n_tokens, out_bf16, stream=None):
    """Elementwise strawman of hma_bfp8_dequant_bf16 (same bits, one thread per element)."""
    _check(lib().hma_bfp8_dequant_bf16_naive(cache.handle, layer, which, _ptr(page_ids), token_begin, n_tokens,
                                             _ptr(out_bf16), _stream(stream)), "hma_bfp8_dequant_bf16_naive")


def hma_bfp8_rebuild_request(cache, page_ids, token_begin, n_tokens, out_bf16, stream=None):
    """Every layer, K and V, of one request in a single launch -> out_bf16 [layers][2][n_tokens][Hkv][128]."""
    _check(lib().hma_bfp8_rebuild_request(cache.handle, _ptr(page_ids), token_begin, n_tokens, _ptr(out_bf16), _stream(stream)),
           "hma_bfp8_rebuild_request")


def hma_bfp8_encode_rows(cache, x, wire_rowmajor, stream=None):
    """x: float32 or bfloat16 tensor [..., 128] -> ROWMAJOR BFP8 rows in wire_rowmajor (uint8 [..., 136])."""
    n_rows = x.numel() // 128
    _check(lib().hma_bfp8_encode_rows(cache.handle, _ptr(x), 1 if x.dtype == torch.bfloat16 else 0, n_rows,
                                      _ptr(wire_rowmajor), _stream(stream)), "hma_bfp8_encode_rows")


def hma_bfp8_dequant_blocks_bf16(exps, mants, n_blocks, out_bf16, stream=None):
    _check(lib().hma_bfp8_dequant_blocks_bf16(_ptr(exps), _ptr(mants), n_blocks, _ptr(out_bf16), _stream(stream)),
           "hma_bfp8_dequant_blocks_bf16")


def hma_error_flags(cache, stream=None):
    v = ctypes.c_uint32(0)
    _check(lib().hma_error_flags(cache.handle, ctypes.byref(v), _stream(stream)), "hma_error_flags")
    return int(v.value)


def hma_last_cuda_error():
    return lib().hma_last_cuda_error().decode()


def hma_launch_count():
    return int(lib().hma_launch_count())
