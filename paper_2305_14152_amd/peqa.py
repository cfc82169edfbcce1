"""Thin ctypes binding over the C-ABI library (include/peqa.h), same names, argument
marshalling only.  PyTorch supplies device memory and the HIP stream; every step of the
computation runs inside libpeqa_hip.so.  There is no fallback: a missing library raises."""
import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpeqa_hip.so")

PEQA_OK = 0
PEQA_ERR_NULL, PEQA_ERR_SHAPE, PEQA_ERR_BITS, PEQA_ERR_GROUP = 1, 2, 3, 4
PEQA_ERR_ALIGN, PEQA_ERR_WORKSPACE, PEQA_ERR_DEVICE, PEQA_ERR_PARAM = 5, 6, 7, 8
PEQA_OP_FWD, PEQA_OP_BWD, PEQA_OP_FWD_KEEP, PEQA_OP_BWD_KEPT, PEQA_OP_FWD_Z, PEQA_OP_BWD_Z = 0, 1, 2, 3, 4, 5
PEQA_OPT_GEMM_WAVES, PEQA_OPT_BWD_PAIR, PEQA_OPT_GROUPED_DDS = 0, 1, 2

EXPORTS = ["peqa_check_layout", "peqa_packed_words", "peqa_num_scales", "peqa_workspace_bytes",
           "peqa_status_string", "peqa_bit_location", "peqa_quantize", "peqa_linear_fwd",
           "peqa_linear_bwd", "peqa_scale_update", "peqa_trace_begin", "peqa_trace_end",
           "peqa_workspace_bytes_fused", "peqa_linear_fwd_fused", "peqa_linear_fwd_keep", "peqa_linear_bwd_kept",
           "peqa_linear_fwd_z", "peqa_linear_bwd_z", "peqa_quantize_search",
           "peqa_scale_update_multi", "peqa_device_info",
           "peqa_row_sums", "peqa_linear_fwd_fused_rs", "peqa_linear_bwd_rs",
           "peqa_set_option", "peqa_get_option", "peqa_linear_fwd_static",
           "peqa_block_workspace_bytes", "peqa_block_fwd", "peqa_block_bwd", "peqa_trace_select",
           "peqa_check_cache", "peqa_rope_append", "peqa_paged_attention_workspace_bytes", "peqa_paged_attention",
           "peqa_token_logprobs_workspace_bytes", "peqa_token_logprobs", "peqa_token_logprobs_bwd"]


class Layout(ctypes.Structure):
    _fields_ = [("n_out", ctypes.c_int32), ("k_in", ctypes.c_int32),
                ("bits", ctypes.c_int32), ("group_size", ctypes.c_int32)]

    @property
    def groups(self):
        return self.k_in // self.group_size if self.group_size else 1


class AdamW(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float), ("step", ctypes.c_int32)]


PEQA_CACHE_BF16, PEQA_CACHE_FP8 = 0, 1
PEQA_LOGITS_BF16, PEQA_LOGITS_F32 = 0, 1
PEQA_MAX_TOP = 32


class KVCache(ctypes.Structure):
    """peqa_kv_cache; made by kv_cache(), which keeps the tensors that it points into."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("table", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("slot_stride", ctypes.c_int64), ("table_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_seqs", ctypes.c_int32), ("n_blocks", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class PeqaError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__("%s: %s (status %d)" % (what, status_string(status), status))


_lib = None


def lib():
    """Loads libpeqa_hip.so; raises if it has not been built (python -m paper_2305_14152_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libpeqa_hip.so is missing: build it with __graft_entry__.build() "
                              "or `python paper_2305_14152_amd/build.py`; there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        LP = ctypes.POINTER(Layout)
        L.peqa_check_layout.argtypes = [LP]
        L.peqa_check_layout.restype = i32
        L.peqa_packed_words.argtypes = [LP]
        L.peqa_packed_words.restype = sz
        L.peqa_num_scales.argtypes = [LP]
        L.peqa_num_scales.restype = sz
        L.peqa_workspace_bytes.argtypes = [LP, i32, i32]
        L.peqa_workspace_bytes.restype = sz
        L.peqa_status_string.argtypes = [i32]
        L.peqa_status_string.restype = ctypes.c_char_p
        L.peqa_bit_location.argtypes = [LP, i32, i32, i32, ctypes.POINTER(sz), ctypes.POINTER(i32)]
        L.peqa_bit_location.restype = i32
        L.peqa_quantize.argtypes = [LP, vp, vp, vp, vp, vp]
        L.peqa_quantize.restype = i32
        L.peqa_quantize_search.argtypes = [LP, vp, i32, ctypes.c_float, vp, vp, vp, vp]
        L.peqa_quantize_search.restype = i32
        L.peqa_linear_fwd.argtypes = [LP, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
        L.peqa_linear_fwd.restype = i32
        L.peqa_linear_fwd_static.argtypes = [LP, vp, vp, vp, vp, vp, i32, vp, vp]
        L.peqa_linear_fwd_static.restype = i32
        L.peqa_linear_bwd.argtypes = [LP, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.peqa_linear_bwd.restype = i32
        L.peqa_linear_fwd_keep.argtypes = [LP, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.peqa_linear_fwd_keep.restype = i32
        L.peqa_linear_bwd_kept.argtypes = [LP, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.peqa_linear_bwd_kept.restype = i32
        L.peqa_linear_fwd_z.argtypes = [LP, vp, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
        L.peqa_linear_fwd_z.restype = i32
        L.peqa_linear_bwd_z.argtypes = [LP, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.peqa_linear_bwd_z.restype = i32
        L.peqa_scale_update.argtypes = [sz, vp, vp, vp, vp, vp, ctypes.POINTER(AdamW), vp]
        L.peqa_scale_update.restype = i32
        L.peqa_scale_update_multi.argtypes = [i32, vp, ctypes.POINTER(AdamW), vp]
        L.peqa_scale_update_multi.restype = i32
        L.peqa_row_sums.argtypes = [vp, i32, i32, vp, vp]
        L.peqa_row_sums.restype = i32
        L.peqa_linear_fwd_fused_rs.argtypes = [i32, vp, vp, vp, i32, vp, sz, vp]
        L.peqa_linear_fwd_fused_rs.restype = i32
        L.peqa_linear_bwd_rs.argtypes = [LP, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.peqa_linear_bwd_rs.restype = i32
        L.peqa_workspace_bytes_fused.argtypes = [i32, vp, i32]
        L.peqa_workspace_bytes_fused.restype = sz
        L.peqa_linear_fwd_fused.argtypes = [i32, vp, vp, i32, vp, sz, vp]
        L.peqa_linear_fwd_fused.restype = i32
        L.peqa_set_option.argtypes = [i32, i32]
        L.peqa_set_option.restype = i32
        L.peqa_get_option.argtypes = [i32]
        L.peqa_get_option.restype = i32
        L.peqa_block_workspace_bytes.argtypes = [i32, vp, i32, i32]
        L.peqa_block_workspace_bytes.restype = sz
        L.peqa_block_fwd.argtypes = [i32, vp, i32, vp, sz, vp]
        L.peqa_block_fwd.restype = i32
        L.peqa_block_bwd.argtypes = [i32, vp, i32, vp, sz, vp]
        L.peqa_block_bwd.restype = i32
        L.peqa_trace_select.argtypes = [ctypes.c_char_p]
        L.peqa_trace_select.restype = i32
        L.peqa_trace_begin.argtypes = [i32]
        L.peqa_trace_begin.restype = i32
        L.peqa_trace_end.argtypes = [i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(i32),
                                     ctypes.POINTER(ctypes.c_float)]
        L.peqa_trace_end.restype = i32
        i64, CP = ctypes.c_int64, ctypes.POINTER(KVCache)
        L.peqa_check_cache.argtypes = [CP]
        L.peqa_check_cache.restype = i32
        L.peqa_rope_append.argtypes = [CP, i32, vp, vp, vp, vp, i32, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]
        L.peqa_rope_append.restype = i32
        L.peqa_paged_attention_workspace_bytes.argtypes = [CP, i32, i32, i32, i32]
        L.peqa_paged_attention_workspace_bytes.restype = sz
        L.peqa_paged_attention.argtypes = [CP, i32, i32, vp, i64, vp, vp, i32, i32, ctypes.c_float, vp, i64, vp, vp, sz, vp]
        L.peqa_paged_attention.restype = i32
        L.peqa_token_logprobs_workspace_bytes.argtypes = [i32, i32, i32]
        L.peqa_token_logprobs_workspace_bytes.restype = sz
        L.peqa_token_logprobs.argtypes = [vp, i32, i32, i32, i64, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.peqa_token_logprobs.restype = i32
        L.peqa_token_logprobs_bwd.argtypes = [vp, i32, i32, i32, i64, vp, vp, vp, vp, vp, vp, i64, vp]
        L.peqa_token_logprobs_bwd.restype = i32
        _lib = L
    return _lib


def status_string(status):
    return lib().peqa_status_string(int(status)).decode()


def _check(status, what):
    if status != PEQA_OK:
        raise PeqaError(status, what)


def _ptr(t):
    """Device (or raw integer) pointer of a torch tensor; None -> NULL."""
    if t is None or isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors must be contiguous"
    return t.data_ptr()


_current_stream = None


def _stream(stream):
    # The raw handle of torch's current stream.  Building a torch.cuda.Stream object to ask for it took 2.7 us, more than the
    # rest of the marshalling: with this and the items below as bytes, a training step of a 256 x 256 layer 32.1 -> 26.4 us,
    # a fused forward of three small layers 10.6 -> 7.4.
    global _current_stream
    if stream is None:
        if _current_stream is None:
            import torch
            torch.cuda.current_device()        # (initialises torch's side, which the calls below take for granted)
            raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
            _current_stream = lambda: raw(device())
        return _current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def layout(n_out, k_in, bits, group_size=0):
    return Layout(int(n_out), int(k_in), int(bits), int(group_size))


def check_layout(L):
    return int(lib().peqa_check_layout(ctypes.byref(L)))


def packed_words(L):
    return int(lib().peqa_packed_words(ctypes.byref(L)))


def num_scales(L):
    return int(lib().peqa_num_scales(ctypes.byref(L)))


def workspace_bytes(L, T, op):
    return int(lib().peqa_workspace_bytes(ctypes.byref(L), int(T), int(op)))


def bit_location(L, i, k, t):
    w, b = ctypes.c_size_t(), ctypes.c_int32()
    _check(lib().peqa_bit_location(ctypes.byref(L), i, k, t, ctypes.byref(w), ctypes.byref(b)), "peqa_bit_location")
    return int(w.value), int(b.value)


def quantize(L, W0, packed, s0, z0, stream=None):
    _check(lib().peqa_quantize(ctypes.byref(L), _ptr(W0), _ptr(packed), _ptr(s0), _ptr(z0), _stream(stream)),
           "peqa_quantize")


class UpdateItem(ctypes.Structure):
    _fields_ = [("n_scales", ctypes.c_size_t), ("ds", ctypes.c_void_p), ("d_ds", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("s0", ctypes.c_void_p)]


_UPDATE_ITEM = struct.Struct("@N5P")
assert _UPDATE_ITEM.size == ctypes.sizeof(UpdateItem)


def scale_update_multi(tensors, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, stream=None):
    """tensors: sequence of (n_scales, ds, d_ds, m, v, s0)."""
    try:
        items = b"".join([_UPDATE_ITEM.pack(int(n), _ptr(ds) or 0, _ptr(d_ds) or 0, _ptr(m) or 0, _ptr(v) or 0, _ptr(s0) or 0)
                          for n, ds, d_ds, m, v, s0 in tensors])
    except struct.error:                       # numbers that C takes modulo 2^64 (a negative n_scales: refused by the library)
        items = b"".join([bytes(UpdateItem(int(n), *map(_ptr, t))) for n, *t in tensors])
    opt = AdamW(lr, beta1, beta2, eps, weight_decay, int(step))
    _check(lib().peqa_scale_update_multi(len(tensors), items, ctypes.byref(opt), _stream(stream)),
           "peqa_scale_update_multi")


def device_info():
    """(compute units, peak engine clock in kHz) of the current device."""
    cus, khz = ctypes.c_int32(0), ctypes.c_int32(0)
    f = lib().peqa_device_info
    f.argtypes = [ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
    f.restype = ctypes.c_int32
    _check(f(ctypes.byref(cus), ctypes.byref(khz)), "peqa_device_info")
    return cus.value, khz.value


def row_sums(X, T, K, rs, stream=None):
    _check(lib().peqa_row_sums(_ptr(X), int(T), int(K), _ptr(rs), _stream(stream)), "peqa_row_sums")


def linear_fwd_fused_rs(layers, X, rs, T, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_fwd_fused_rs(len(layers), _items(layers), _ptr(X), _ptr(rs), int(T),
                                          _ptr(workspace), int(workspace_bytes_), _stream(stream)),
           "peqa_linear_fwd_fused_rs")


def linear_bwd_rs(L, packed, s0, ds, z0, X, rs, dY, T, dX, d_ds, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_bwd_rs(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(X), _ptr(rs),
                                    _ptr(dY), int(T), _ptr(dX), _ptr(d_ds), _ptr(workspace), int(workspace_bytes_),
                                    _stream(stream)), "peqa_linear_bwd_rs")


def quantize_search(L, W0, n_ratios, min_ratio, packed, s0, z0, stream=None):
    _check(lib().peqa_quantize_search(ctypes.byref(L), _ptr(W0), int(n_ratios), float(min_ratio), _ptr(packed),
                                      _ptr(s0), _ptr(z0), _stream(stream)), "peqa_quantize_search")


def linear_fwd(L, packed, s0, ds, z0, X, T, Y, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_fwd(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(X), int(T),
                                 _ptr(Y), _ptr(workspace), int(workspace_bytes_), _stream(stream)),
           "peqa_linear_fwd")


STATIC_SCRATCH_BYTES = 16 << 20


def linear_fwd_static(L, packed, s0, ds, z0, X, T, Y, stream=None):
    _check(lib().peqa_linear_fwd_static(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(X), int(T),
                                        _ptr(Y), _stream(stream)), "peqa_linear_fwd_static")


class FwdItem(ctypes.Structure):
    _fields_ = [("layout", Layout), ("packed", ctypes.c_void_p), ("s0", ctypes.c_void_p), ("ds", ctypes.c_void_p),
                ("z0", ctypes.c_void_p), ("Y", ctypes.c_void_p)]


_FWD_ITEM = struct.Struct("@%ds5P" % ctypes.sizeof(Layout))
assert _FWD_ITEM.size == ctypes.sizeof(FwdItem)


def _items(layers):
    """layers: sequence of (L, packed, s0, ds, z0, Y).  The bytes of an array of FwdItem (made field by field as ctypes
    structures they took 3.4 us for three, and take 2.4)."""
    try:
        return b"".join([_FWD_ITEM.pack(bytes(L) if type(L) is Layout else bytes(FwdItem(L).layout),   # (a tuple, or TypeError)
                                        _ptr(packed) or 0, _ptr(s0) or 0, _ptr(ds) or 0, _ptr(z0) or 0, _ptr(Y) or 0)
                         for L, packed, s0, ds, z0, Y in layers])
    except struct.error:                       # numbers that C takes modulo 2^64
        return b"".join([bytes(FwdItem(L, *map(_ptr, t))) for L, *t in layers])


def workspace_bytes_fused(layers, T):
    return int(lib().peqa_workspace_bytes_fused(len(layers), _items(layers), int(T)))


def linear_fwd_fused(layers, X, T, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_fwd_fused(len(layers), _items(layers), _ptr(X), int(T), _ptr(workspace),
                                       int(workspace_bytes_), _stream(stream)), "peqa_linear_fwd_fused")


def linear_bwd(L, packed, s0, ds, z0, X, dY, T, dX, d_ds, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_bwd(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(X), _ptr(dY),
                                 int(T), _ptr(dX), _ptr(d_ds), _ptr(workspace), int(workspace_bytes_),
                                 _stream(stream)), "peqa_linear_bwd")


def linear_fwd_keep(L, packed, s0, ds, z0, X, T, Y, P, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_fwd_keep(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(X), int(T),
                                      _ptr(Y), _ptr(P), _ptr(workspace), int(workspace_bytes_), _stream(stream)),
           "peqa_linear_fwd_keep")


def linear_bwd_kept(L, packed, s0, ds, z0, P, dY, T, dX, d_ds, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_bwd_kept(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(P), _ptr(dY),
                                      int(T), _ptr(dX), _ptr(d_ds), _ptr(workspace), int(workspace_bytes_),
                                      _stream(stream)), "peqa_linear_bwd_kept")


def linear_fwd_z(L, packed, s0, ds, z0, dz, X, T, Y, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_fwd_z(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(dz), _ptr(X),
                                   int(T), _ptr(Y), _ptr(workspace), int(workspace_bytes_), _stream(stream)),
           "peqa_linear_fwd_z")


def linear_bwd_z(L, packed, s0, ds, z0, dz, X, dY, T, dX, d_ds, d_dz, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_linear_bwd_z(ctypes.byref(L), _ptr(packed), _ptr(s0), _ptr(ds), _ptr(z0), _ptr(dz), _ptr(X),
                                   _ptr(dY), int(T), _ptr(dX), _ptr(d_ds), _ptr(d_dz), _ptr(workspace),
                                   int(workspace_bytes_), _stream(stream)), "peqa_linear_bwd_z")


def scale_update(n_scales, ds, d_ds, m, v, s0, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1,
                 stream=None):
    opt = AdamW(lr, beta1, beta2, eps, weight_decay, int(step))
    _check(lib().peqa_scale_update(int(n_scales), _ptr(ds), _ptr(d_ds), _ptr(m), _ptr(v), _ptr(s0),
                                   ctypes.byref(opt), _stream(stream)), "peqa_scale_update")


class BlockItem(ctypes.Structure):
    _fields_ = [("layout", Layout), ("packed", ctypes.c_void_p), ("s0", ctypes.c_void_p), ("ds", ctypes.c_void_p),
                ("z0", ctypes.c_void_p), ("X", ctypes.c_void_p), ("Y", ctypes.c_void_p), ("dY", ctypes.c_void_p),
                ("dX", ctypes.c_void_p), ("d_ds", ctypes.c_void_p), ("row_sums", ctypes.c_void_p)]


def block_items(layers):
    """layers: sequence of dicts with keys L, packed, s0, z0 and optionally ds, X, Y, dY, dX, d_ds, row_sums."""
    arr = (BlockItem * len(layers))()
    for i, d in enumerate(layers):
        arr[i] = BlockItem(d["L"], _ptr(d["packed"]), _ptr(d["s0"]), _ptr(d.get("ds")), _ptr(d["z0"]), _ptr(d.get("X")),
                           _ptr(d.get("Y")), _ptr(d.get("dY")), _ptr(d.get("dX")), _ptr(d.get("d_ds")),
                           _ptr(d.get("row_sums")))
    return arr


def block_workspace_bytes(items, T, op):
    return int(lib().peqa_block_workspace_bytes(len(items), ctypes.addressof(items), int(T), int(op)))


def block_fwd(items, T, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_block_fwd(len(items), ctypes.addressof(items), int(T), _ptr(workspace), int(workspace_bytes_),
                                _stream(stream)), "peqa_block_fwd")


def block_bwd(items, T, workspace, workspace_bytes_, stream=None):
    _check(lib().peqa_block_bwd(len(items), ctypes.addressof(items), int(T), _ptr(workspace), int(workspace_bytes_),
                                _stream(stream)), "peqa_block_bwd")


def set_option(option, value):
    _check(lib().peqa_set_option(int(option), int(value)), "peqa_set_option")


def get_option(option):
    return int(lib().peqa_get_option(int(option)))


def trace_begin(max_launches, prefix=None):
    """Brackets the library's launches with HIP events until trace_end(); `prefix` restricts it to kernels whose
    name starts with it."""
    _check(lib().peqa_trace_select(prefix.encode() if prefix else None), "peqa_trace_select")
    _check(lib().peqa_trace_begin(int(max_launches)), "peqa_trace_begin")


def trace_end(max_kernels=32):
    names = (ctypes.c_char_p * max_kernels)()
    launches = (ctypes.c_int32 * max_kernels)()
    total_ms = (ctypes.c_float * max_kernels)()
    n = lib().peqa_trace_end(max_kernels, names, launches, total_ms)
    return {names[i].decode(): (int(launches[i]), float(total_ms[i])) for i in range(n)}


class _Kinds(dict):
    """Names of tensors' types, each formed once: this module takes tensors without importing what they are made by."""
    def __missing__(self, dtype):
        self[dtype] = name = str(dtype).rpartition(".")[2]
        return name


_kind = _Kinds()
_BF16 = ("bfloat16", "int16", "uint16")        # bf16, or its 16-bit pattern
_FP8 = ("float8_e4m3fn", "uint8")              # the cache's 8-bit floats, or their bytes


def kv_cache(k, v, table, k_scale=None, v_scale=None):
    """The cache of two pools [pages, kv_heads, page_size, head_dim] (any strides, the same of both, the last 1) of bf16 or
    torch.float8_e4m3fn, or of their bits as 16- or 8-bit integers, and a table [sequences, blocks] of int32.  k_scale, v_scale [kv_heads]
    fp32 or None."""
    assert k.shape == v.shape and k.dim() == 4 and k.stride() == v.stride() and k.stride(3) == 1 and k.dtype == v.dtype, \
        "pools [pages, kv_heads, page_size, head_dim] of one type with the same strides, the last 1"
    assert table.dim() == 2 and table.stride(1) == 1 and _kind[table.dtype] == "int32", "table [sequences, blocks] of int32"
    n_seqs, n_blocks = table.shape             # (a single row may have any stride)
    assert n_seqs == 1 or table.stride(0) >= n_blocks, "table [sequences, blocks] whose rows do not overlap"
    fp8 = _kind[k.dtype] in _FP8
    assert fp8 or _kind[k.dtype] in _BF16, "pools of bf16 or float8_e4m3fn"
    for scale in (k_scale, v_scale):
        assert scale is None or isinstance(scale, int) or (_kind[scale.dtype] == "float32" and scale.numel() == k.shape[1]), \
            "scales [kv_heads] of fp32"
    c = KVCache(k.data_ptr(), v.data_ptr(), table.data_ptr(), _ptr(k_scale), _ptr(v_scale), k.stride(0), k.stride(1), k.stride(2),
                table.stride(0) if n_seqs > 1 else n_blocks, k.shape[0], k.shape[2], k.shape[1], k.shape[3], n_seqs, n_blocks,
                PEQA_CACHE_FP8 if fp8 else PEQA_CACHE_BF16, 0)
    c.tensors = (k, v, table, k_scale, v_scale)
    return c


def check_cache(cache):
    return int(lib().peqa_check_cache(ctypes.byref(cache)))


_ROWS = "tensors [rows, heads, head_dim] of bf16 whose rows are contiguous"


def _rows(x, heads, dim):
    """(pointer, row stride) of such a tensor with more than one row.  (Every attribute of a tensor that is asked for takes some 0.1 us of a
    call's 6 to 8, and a function called as much.)"""
    s0, s1, s2 = x.stride()
    assert s2 == 1 and (s1 == dim or heads == 1) and _kind[x.dtype] in _BF16, _ROWS
    return x.data_ptr(), s0


def _index(t, n=None):
    """Pointer of n positions, lengths, sequences, words or alternatives (of a shape that was compared: n is left out); None -> NULL."""
    if t is None:
        return None
    assert _kind[t.dtype] == "int32" and t.is_contiguous() and (n is None or t.numel() == n), "a contiguous tensor of int32, one of each"
    return t.data_ptr()


def _floats(t, n=0):
    """Pointer of n fp32 numbers at least (of a shape that was compared: n is left out); None -> NULL, a device address as it is."""
    if t is None or isinstance(t, int):
        return t
    assert _kind[t.dtype] == "float32" and t.is_contiguous() and (n == 0 or t.numel() >= n), "a contiguous tensor of float32, one of each"
    return t.data_ptr()


def _room(t, n):
    """Pointer of a workspace of n bytes; None -> NULL (refused where one is needed), a device address as it is."""
    if t is None or isinstance(t, int):
        return t
    assert t.nbytes >= n and t.is_contiguous(), "a contiguous workspace of %d bytes" % n
    return t.data_ptr()


def rope_append(cache, q, k, v, pos, cos, sin, q_out, seq=None, interleaved=False, stream=None):
    """q, q_out [T, heads, head_dim] or None, k, v [T, kv_heads, head_dim], pos, seq [T] int32, cos, sin [positions, rot / 2] fp32
    or None (no rotation)."""
    T, kv_heads, dim = shape = k.shape
    assert kv_heads == cache.kv_heads and dim == cache.head_dim and v.shape == shape, "k and v [T, kv_heads, head_dim] of the cache"
    kp, ks = _rows(k, kv_heads, dim)
    vp, vs = _rows(v, kv_heads, dim)
    heads, qp, qs, op, os_ = 0, None, 0, None, 0
    if q is not None:
        n, heads, d = shape = q.shape
        assert n == T and d == dim
        qp, qs = _rows(q, heads, dim)
        if q_out is not None:
            assert q_out.shape == shape
            op, os_ = _rows(q_out, heads, dim)
    elif q_out is not None:
        op = q_out.data_ptr()                  # (refused by the library)
    if T == 1:                                 # (a single row may have any stride)
        ks = vs = kv_heads * dim
        qs = os_ = heads * dim
    n_pos = half = 0
    if cos is not None:
        n_pos, half = shape = cos.shape
        assert sin is None or sin.shape == shape
    status = (_lib or lib()).peqa_rope_append(cache, T, _index(pos, T), _index(seq, T), _floats(cos), _floats(sin), n_pos,
                                              2 * half, interleaved, heads, qp, qs, kp, ks, vp, vs, op, os_, _stream(stream))
    if status:
        raise PeqaError(status, "peqa_rope_append")


def paged_attention_workspace_bytes(cache, heads, rows, max_len, window=0):
    return int(lib().peqa_paged_attention_workspace_bytes(ctypes.byref(cache), int(rows), int(heads), int(max_len), int(window)))


def paged_attention(cache, q, lens, max_len, scale, out, workspace, workspace_bytes_, lse=None, seq=None, window=0, stream=None):
    """q, out [rows, heads, head_dim], lens, seq [rows] int32, lse [rows, heads] fp32."""
    rows, heads, dim = shape = q.shape
    assert out.shape == shape and dim == cache.head_dim
    assert lse is None or lse.shape == (rows, heads)
    qp, qs = _rows(q, heads, dim)
    op, os_ = _rows(out, heads, dim)
    if rows == 1:                              # (a single row may have any stride)
        qs = os_ = heads * dim
    status = (_lib or lib()).peqa_paged_attention(cache, rows, heads, qp, qs, _index(lens, rows), _index(seq, rows), max_len, window, scale, op, os_,
                                                  _floats(lse), _room(workspace, workspace_bytes_), workspace_bytes_, _stream(stream))
    if status:
        raise PeqaError(status, "peqa_paged_attention")


def _logits(x):
    """(pointer, type, rows, words, row stride) of logits [T, vocab]."""
    (T, V), (s0, s1), kind = x.shape, x.stride(), _kind[x.dtype]
    assert (s1 == 1 or V == 1) and (kind == "float32" or kind in _BF16), "logits [T, vocab] of bf16 or fp32 with contiguous rows"
    return x.data_ptr(), PEQA_LOGITS_F32 if kind == "float32" else PEQA_LOGITS_BF16, T, V, s0 if T > 1 else V


def token_logprobs_workspace_bytes(T, vocab, top=0):
    return int(lib().peqa_token_logprobs_workspace_bytes(int(T), int(vocab), int(top)))


def token_logprobs(logits, targets, logp, entropy, lse, top_logp, top_ids, workspace, workspace_bytes_, stream=None):
    """logits [T, vocab], targets [T] int32, logp, entropy, lse [T] fp32 or None, top_logp, top_ids [T, top] or None."""
    xp, dtype, T, V, stride = _logits(logits)
    top = 0
    if top_ids is not None:
        n, top = top_ids.shape
        assert n == T and top_logp.shape == (T, top)
    status = (_lib or lib()).peqa_token_logprobs(xp, dtype, T, V, stride, _index(targets, T), top, _floats(logp, T), _floats(entropy, T),
                                                 _floats(lse, T), _floats(top_logp), _index(top_ids), _room(workspace, workspace_bytes_),
                                                 workspace_bytes_, _stream(stream))
    if status:
        raise PeqaError(status, "peqa_token_logprobs")


def token_logprobs_bwd(logits, targets, lse, entropy, d_logp, d_entropy, d_logits, stream=None):
    """d_logits [T, vocab], the gradient of sum(d_logp * logp + d_entropy * entropy); may be `logits` itself."""
    xp, dtype, T, V, stride = _logits(logits)
    dp, d_dtype, dT, dV, d_stride = _logits(d_logits)
    assert (d_dtype, dT, dV) == (dtype, T, V)
    status = (_lib or lib()).peqa_token_logprobs_bwd(xp, dtype, T, V, stride, _index(targets, T), _floats(lse, T), _floats(entropy, T),
                                                     _floats(d_logp, T), _floats(d_entropy, T), dp, d_stride, _stream(stream))
    if status:
        raise PeqaError(status, "peqa_token_logprobs_bwd")
