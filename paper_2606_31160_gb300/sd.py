"""ctypes binding of libsd.so: the C ABI of include/sd.h with torch tensors.

Argument marshalling only: every function checks shapes / dtypes / devices,
passes `tensor.data_ptr()` and torch's current CUDA stream to the C entry
point of the same name, and raises SDError on a non-zero status. All the
arithmetic of the verify step runs in the CUDA kernels of libsd.so; there is
no CPU fallback, and loading fails loudly when the library is missing.
"""

import ctypes
import functools
import os
import re

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsd.so")
HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "sd.h")

SD_BF16, SD_F32 = 0, 1
SD_ERR_WORKSPACE = 3
SD_DEVERR_KV_OVERFLOW = 0x1
SD_DEVERR_ROLLBACK = 0x2
SD_DEVERR_TOKEN_RANGE = 0x4
SD_DEVERR_LENGTH = 0x8
SD_DEVERR_TIMEOUT = 0x10
SD_DEVERR_TREE = 0x20
SD_DEVERR_PAGE = 0x40


class SDError(RuntimeError):
    def __init__(self, what, status):
        super().__init__("%s failed: %s" % (what, status_str(status)))
        self.status = status


class KVCacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class KV8CacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("len", ctypes.c_void_p), ("ticket", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("capacity", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32)]


class PagedCacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("table", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("ticket", ctypes.c_void_p), ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("page", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


_lib = None

_vp, _i, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_ll = ctypes.c_longlong
_SIGNATURES = {
    "sd_status_str": ([_i], ctypes.c_char_p),
    "sd_version": ([], ctypes.c_char_p),
    "sd_rope_apply": ([_vp, _vp, _i, _i, _i, _i, _i, _vp, ctypes.POINTER(ctypes.c_int32), _i, _f, _vp], _i),
    "sd_rope_apply_1d": ([_vp, _vp, _i, _i, _i, _i, _i, _vp, _f, _vp], _i),
    "sd_kv_append": ([ctypes.POINTER(KVCacheStruct), _vp, _vp, _i, _vp], _i),
    "sd_kv_rollback": ([_vp, _i, _i, _vp, _i, _vp], _i),
    "sd_verify_attention_workspace": ([_i, _i, _i, _i, _i, _i], _sz),
    "sd_verify_attention": ([_vp, ctypes.POINTER(KVCacheStruct), _vp, _i, _i, _f, _vp, _sz, _vp], _i),
    "sd_verify_attention_ex": ([_vp, ctypes.POINTER(KVCacheStruct), _vp, _i, _i, _f, _i, _vp, _sz, _vp], _i),
    "sd_verify_layer_workspace": ([_i, _i, _i, _i, _i, _i], _sz),
    "sd_verify_layer": ([_vp, _vp, _vp, _vp, ctypes.POINTER(ctypes.c_int32), _i, _f,
                         ctypes.POINTER(KVCacheStruct), _vp, _i, _i, _f, _vp, _sz, _i, _vp], _i),
    "sd_accept_greedy_workspace": ([_i, _i, _i], _sz),
    "sd_accept_greedy": ([_vp, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _sz, _vp], _i),
    "sd_accept_greedy_noalloc": ([_vp, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp], _i),
    "sd_accept_greedy_noalloc_max_bytes": ([], _sz),
    "sd_accept_sample_workspace": ([_i, _i, _i], _sz),
    "sd_accept_sample": ([_vp, _vp, _i, _i, _i, _f, _vp, _vp, _vp, _vp, _vp, _sz, _vp], _i),
    "sd_get_device_error": ([_vp, ctypes.POINTER(ctypes.c_uint32)], _i),
    "sd_set_cluster_size": ([_i], _i),
    "sd_verify_kernel": ([_i, _i, _i, _i, _i, _i, _i], ctypes.c_char_p),
    "sd_verify_cluster_size": ([_i, _i, _i, _i, _i, _i, _i], _i),
    "sd_attention_budget": ([_vp, ctypes.POINTER(KVCacheStruct), _i, _i, _f, _vp, _vp, _vp, _vp], _i),
    "sd_kv8_append": ([ctypes.POINTER(KV8CacheStruct), _vp, _vp, _i, _vp], _i),
    "sd_kv8_store": ([ctypes.POINTER(KV8CacheStruct), ctypes.POINTER(KVCacheStruct), _vp], _i),
    "sd_kv8_attention_workspace": ([_i, _i, _i, _i, _i, _i], _sz),
    "sd_kv8_attention_ex": ([_vp, ctypes.POINTER(KV8CacheStruct), _vp, _i, _i, _f, _i, _vp, _sz, _vp], _i),
    "sd_kv8_attention": ([_vp, ctypes.POINTER(KV8CacheStruct), _vp, _i, _i, _f, _i, _vp], _i),
    "sd_attention_weights_workspace": ([_i, _i, _i, _i, _i, _i], _sz),
    "sd_attention_weights_ex": ([_vp, ctypes.POINTER(KVCacheStruct), _i, _i, _f, _vp, _vp, _f, _vp, _vp, _sz, _vp], _i),
    "sd_attention_weights": ([_vp, ctypes.POINTER(KVCacheStruct), _i, _i, _f, _vp, _vp, _f, _vp, _vp], _i),
    "sd_kv_evict": ([ctypes.POINTER(KVCacheStruct), _vp, _i, _i, _i, ctypes.POINTER(KVCacheStruct), _vp, _vp, _vp], _i),
    "sd_paged_append": ([ctypes.POINTER(PagedCacheStruct), _vp, _ll, _vp, _ll, _vp, _ll, _vp, _i, _i, _vp,
                         ctypes.POINTER(ctypes.c_int32), _i, _f, _vp, _vp], _i),
    "sd_tree_attention_workspace": ([_i, _i, _i, _i, _i, _i], _sz),
    "sd_tree_attention": ([_vp, _ll, ctypes.POINTER(PagedCacheStruct), _vp, _vp, _vp, _i, _i, _f, _vp, _sz, _vp], _i),
    "sd_accept_tree_workspace": ([_i, _i, _i], _sz),
    "sd_accept_tree": ([_vp, _i, _i, _i, _i, _ll, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp], _i),
    "sd_paged_commit": ([ctypes.POINTER(PagedCacheStruct), _i, _vp, _vp, _vp, _i, _vp], _i),
    "sd_token_logprobs": ([_vp, _i, _i, _i, ctypes.c_longlong, _vp, _f, _i, _vp, _vp, _vp, _vp, _vp], _i),
}


def lib():
    """Load libsd.so (built in-tree by paper_2606_31160_gb300.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libsd.so not found at %s: run paper_2606_31160_gb300.build.build() "
                               "(there is no CPU fallback)" % LIB_PATH)
        handle = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.argtypes = args
            fn.restype = res
        _lib = handle
    return _lib


def header_symbols():
    """Names of every function include/sd.h declares."""
    with open(HEADER_PATH) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(sd_[a-z0-9_]+)\s*\(", text)))


def status_str(status):
    return lib().sd_status_str(int(status)).decode()


def version():
    return lib().sd_version().decode()


def _check(status, what):
    if status != 0:
        raise SDError(what, status)


# private to torch: looked up once, and done without where a torch has them not
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    """Handle of torch's current stream on the current device (where torch offers it
    without the Stream object that torch.cuda.current_stream() builds, ~1 us a call)."""
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


_Tensor = torch.Tensor


def _dev(t, name, dtype=None, ndim=None):
    """The checked tensor's device address (an int: the declared argument types
    convert it; a c_void_p object an argument cost as much as its checks)."""
    if t.__class__ is _Tensor and t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype is dtype) and ndim is None:
        return t.data_ptr()
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on a CUDA device (no CPU path exists)" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if ndim is not None and t.dim() != ndim:
        raise ValueError("%s must have %d dims, got %s" % (name, ndim, tuple(t.shape)))
    return t.data_ptr()


@functools.lru_cache(maxsize=64)
def _sections(sections):
    return (ctypes.c_int32 * 3)(*sections)


def workspace(nbytes, device=None):
    """A zero-filled device workspace of at least nbytes (16-byte aligned)."""
    return torch.zeros(max(int(nbytes), 16), dtype=torch.uint8,
                       device=device if device is not None else torch.cuda.current_device())


# ----------------------------------------------------------------------- RoPE

def rope_apply(q, k, pos, sections, interleaved=0, base=1e6):
    """In-place M-RoPE of q [B,R,Hq,D] and k [B,R,Hkv,D] (bf16) at pos [B,R,3] int32."""
    B, R, Hq, D = q.shape
    Hkv = k.shape[2]
    if tuple(k.shape) != (B, R, Hkv, D) or tuple(pos.shape) != (B, R, 3):
        raise ValueError("shape mismatch")
    sec = _sections(tuple(int(s) for s in sections))
    _check(lib().sd_rope_apply(_dev(q, "q", torch.bfloat16), _dev(k, "k", torch.bfloat16), B, R, Hq,
                               Hkv, D, _dev(pos, "pos", torch.int32), sec, int(interleaved),
                               float(base), _stream()), "sd_rope_apply")


def rope_apply_1d(q, k, pos1d, base=1e6):
    """In-place FlatRoPE / 1D RoPE at sequence positions pos1d [B,R] int32."""
    B, R, Hq, D = q.shape
    Hkv = k.shape[2]
    if tuple(k.shape) != (B, R, Hkv, D) or tuple(pos1d.shape) != (B, R):
        raise ValueError("shape mismatch")
    _check(lib().sd_rope_apply_1d(_dev(q, "q", torch.bfloat16), _dev(k, "k", torch.bfloat16), B, R,
                                  Hq, Hkv, D, _dev(pos1d, "pos1d", torch.int32), float(base),
                                  _stream()), "sd_rope_apply_1d")


# ------------------------------------------------------------------ KV cache

class KVCache:
    """One layer's bf16 KV cache [B, Hkv, cap, D] plus its device lengths [B]."""

    def __init__(self, k, v, lens):
        if k.shape != v.shape or k.dim() != 4:
            raise ValueError("k and v must both be [B, Hkv, cap, D]")
        _dev(k, "k", torch.bfloat16)
        _dev(v, "v", torch.bfloat16)
        _dev(lens, "len", torch.int32, 1)
        self.k, self.v, self.len = k, v, lens
        B, H, cap, D = k.shape
        self._struct = KVCacheStruct(k.data_ptr(), v.data_ptr(), lens.data_ptr(), B, H, cap, D)
        # what a call reads, fixed with the struct
        self._ref, self._shape = ctypes.byref(self._struct), (B, H, cap, D)

    @classmethod
    def empty(cls, B, Hkv, cap, D, device="cuda"):
        k = torch.zeros((B, Hkv, cap, D), dtype=torch.bfloat16, device=device)
        return cls(k, torch.zeros_like(k), torch.zeros(B, dtype=torch.int32, device=device))

    @property
    def struct(self):
        return self._ref

    @property
    def shape(self):
        return self._shape


def kv_append(cache, k_new, v_new):
    """Write k_new / v_new [B,R,Hkv,D] at len[b] .. len[b]+R-1; len += R."""
    B, H, _, D = cache.shape
    R = k_new.shape[1]
    if tuple(k_new.shape) != (B, R, H, D) or k_new.shape != v_new.shape:
        raise ValueError("shape mismatch")
    _check(lib().sd_kv_append(cache.struct, _dev(k_new, "k_new", torch.bfloat16),
                              _dev(v_new, "v_new", torch.bfloat16), R, _stream()), "sd_kv_append")


def kv_rollback(lens, committed, n_appended):
    """lens [..., B] (one or more layers' length arrays, contiguous) -= n_appended - committed[b]."""
    B = committed.numel()
    _check(lib().sd_kv_rollback(_dev(lens, "len", torch.int32), lens.numel(), B,
                                _dev(committed, "committed", torch.int32), int(n_appended), _stream()),
           "sd_kv_rollback")


# ----------------------------------------------------------------- attention

def attention_workspace_bytes(B, R, Hq, Hkv, D, capacity):
    return int(lib().sd_verify_attention_workspace(B, R, Hq, Hkv, D, capacity))


_attn_ws = {}


SD_ATTN_BLOCK_MASK = 1
SD_ATTN_PREFIX_EARLY = 2
SD_LAYER_BLOCK_MASK = 2


def verify_attention(q, cache, out=None, scale=0.0, ws=None, block=False, early=False):
    """Causal GQA verify attention of q [B,R,Hq,D] (rotated) over the cache (appended).
    ws: the split-merge workspace (see sd_verify_attention_workspace); when None a
    zero-filled one is kept per (device, shape) and reused by later calls.
    block=True sets SD_ATTN_BLOCK_MASK; early=True sets SD_ATTN_PREFIX_EARLY (the
    previous kernel on the stream writes neither this cache nor its len)."""
    B, R, Hq, D = q.shape
    if cache.shape[0] != B or cache.shape[3] != D:
        raise ValueError("q and cache disagree")
    if out is None:
        out = torch.empty_like(q)
    if ws is None:
        need = attention_workspace_bytes(B, R, Hq, cache.shape[1], D, cache.shape[2])
        key = (q.device.index, need)
        if need and key not in _attn_ws:
            _attn_ws[key] = workspace(need, q.device)
        ws = _attn_ws.get(key)
    wp = _dev(ws, "ws") if ws is not None else ctypes.c_void_p(0)
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check(lib().sd_verify_attention_ex(_dev(q, "q", torch.bfloat16), cache.struct,
                                        _dev(out, "out", torch.bfloat16), R, Hq, float(scale),
                                        (SD_ATTN_BLOCK_MASK if block else 0) | (SD_ATTN_PREFIX_EARLY if early else 0),
                                        wp, nbytes, _stream()),
           "sd_verify_attention")
    return out


def attention_budget(q, cache, n_visual, scale=0.0, mass=None, entropy=None):
    """Per (scene, row, head): attention mass on the visual, trajectory / text and
    generated keys, and the normalised entropy over the non-visual keys.
    q [B,R,Hq,D] (rotated), cache appended, n_visual int32 [B] -> (mass [B,R,Hq,3],
    entropy [B,R,Hq]) float32."""
    B, R, Hq, D = q.shape
    if mass is None:
        mass = torch.empty((B, R, Hq, 3), dtype=torch.float32, device=q.device)
    if entropy is None:
        entropy = torch.empty((B, R, Hq), dtype=torch.float32, device=q.device)
    _check(lib().sd_attention_budget(_dev(q, "q", torch.bfloat16), cache.struct, R, Hq, float(scale),
                                     _dev(n_visual, "n_visual", torch.int32), _dev(mass, "mass", torch.float32),
                                     _dev(entropy, "entropy", torch.float32), _stream()),
           "sd_attention_budget")
    return mass, entropy


SD_LAYER_PREFIX_EARLY = 1


def layer_workspace_bytes(B, R, Hq, Hkv, D, capacity):
    return int(lib().sd_verify_layer_workspace(B, R, Hq, Hkv, D, capacity))


def verify_layer(q, k_new, v_new, pos, sections, cache, interleaved=0, base=1e6, out=None, scale=0.0,
                 ws=None, early=False, block=False):
    """sd_verify_layer: M-RoPE of q / k_new (in place), append of k_new / v_new at
    len[b] (the prefix length on entry; len += R) and the verify attention; returns out.
    early=True sets SD_LAYER_PREFIX_EARLY (the previous kernel on the stream writes
    neither this layer's cache nor its len); block=True sets SD_LAYER_BLOCK_MASK."""
    B, R, Hq, D = q.shape
    Hkv = k_new.shape[2]
    if tuple(k_new.shape) != (B, R, Hkv, D) or k_new.shape != v_new.shape or tuple(pos.shape) != (B, R, 3):
        raise ValueError("shape mismatch")
    if cache.shape[0] != B or cache.shape[1] != Hkv or cache.shape[3] != D:
        raise ValueError("q and cache disagree")
    if out is None:
        out = torch.empty_like(q)
    if ws is None:
        # one workspace per layer cache: calls with early=True overlap the
        # previous layer's kernel, so layers must not share their tickets
        need = layer_workspace_bytes(B, R, Hq, Hkv, D, cache.shape[2])
        ws = getattr(cache, "_layer_ws", None)
        if ws is None or ws.numel() < need:
            ws = workspace(need, q.device)
            cache._layer_ws = ws
    sec = _sections(tuple(int(x) for x in sections))
    _check(lib().sd_verify_layer(_dev(q, "q", torch.bfloat16), _dev(k_new, "k_new", torch.bfloat16),
                                 _dev(v_new, "v_new", torch.bfloat16), _dev(pos, "pos", torch.int32), sec,
                                 int(interleaved), float(base), cache.struct, _dev(out, "out", torch.bfloat16),
                                 R, Hq, float(scale), _dev(ws, "ws"), ws.numel() * ws.element_size(),
                                 (SD_LAYER_PREFIX_EARLY if early else 0) | (SD_LAYER_BLOCK_MASK if block else 0),
                                 _stream()), "sd_verify_layer")
    return out


# ----------------------------------------------------------- 8-bit KV cache

class KV8Cache:
    """One layer's 8-bit KV cache: e4m3 codes [B, Hkv, cap, D] (torch.float8_e4m3fn), fp32
    scales [B, Hkv, ceil(cap / block)] and device lengths [B]; value = code * scale of the
    row's block."""

    def __init__(self, k, v, k_scale, v_scale, lens, block=64):
        if k.shape != v.shape or k.dim() != 4:
            raise ValueError("k and v must both be [B, Hkv, cap, D]")
        B, H, cap, D = k.shape
        block = int(block)
        if block <= 0:
            raise ValueError("block must be positive")
        want = (B, H, -(-cap // block))
        if k_scale.shape != want or v_scale.shape != want or lens.shape != (B,):
            raise ValueError("scales must be %s and len (%d,)" % (want, B))
        for t, name in ((k, "k"), (v, "v")):
            _dev(t, name, torch.float8_e4m3fn)
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _dev(t, name, torch.float32)
        _dev(lens, "len", torch.int32)
        _same_device(k, v, k_scale, v_scale, lens)
        self.k, self.v, self.k_scale, self.v_scale, self.len, self.block = k, v, k_scale, v_scale, lens, block
        self._ticket = torch.zeros(max(B, 1), dtype=torch.int32, device=k.device)
        self._struct = KV8CacheStruct(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                      lens.data_ptr(), self._ticket.data_ptr(), B, H, cap, D, block)
        self._ref, self._shape = ctypes.byref(self._struct), (B, H, cap, D)

    @classmethod
    def empty(cls, B, Hkv, cap, D, block=64, device="cuda"):
        if int(block) <= 0:
            raise ValueError("block must be positive")
        k = torch.zeros((B, Hkv, cap, D), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
        s = torch.ones((B, Hkv, -(-cap // block)), dtype=torch.float32, device=device)
        return cls(k, torch.zeros_like(k), s, s.clone(), torch.zeros(B, dtype=torch.int32, device=device), block)

    @property
    def struct(self):
        return self._ref

    @property
    def shape(self):
        return self._shape


def _same_device(*tensors):
    for t in tensors[1:]:
        if t.device != tensors[0].device:
            raise ValueError("all tensors must be on one device")


def kv8_append(cache, k_new, v_new):
    """Quantise and write k_new / v_new [B,R,Hkv,D] bf16 at len[b] .. len[b]+R-1; len += R."""
    B, H, _, D = cache._shape
    shape = k_new.shape
    if len(shape) != 4 or shape != (B, shape[1], H, D) or v_new.shape != shape:
        raise ValueError("shape mismatch")
    _check(lib().sd_kv8_append(cache._ref, _dev(k_new, "k_new", torch.bfloat16), _dev(v_new, "v_new", torch.bfloat16),
                               shape[1], _stream()), "sd_kv8_append")


def kv8_store(cache, src):
    """Quantise a whole bf16 KVCache into the 8-bit cache, its lengths included."""
    if (cache.shape[0], cache.shape[1], cache.shape[3]) != (src.shape[0], src.shape[1], src.shape[3]):
        raise ValueError("the caches disagree")
    _check(lib().sd_kv8_store(cache.struct, src.struct, _stream()), "sd_kv8_store")


def kv8_attention_workspace_bytes(B, R, Hq, Hkv, D, capacity):
    return int(lib().sd_kv8_attention_workspace(B, R, Hq, Hkv, D, capacity))


def kv8_attention(q, cache, out=None, scale=0.0, block=False, ws=None):
    """Verify attention of q [B,R,Hq,D] bf16 (rotated) over an 8-bit cache (rows appended):
    verify_attention on the keys and values that the codes stand for. block=True selects
    the block mask. ws: kv8_attention_workspace_bytes of device memory; when None a batch
    that takes one has it from torch's allocator, on the current stream."""
    B, R, Hq, D = q.shape
    _, Hkv, cap, dim = cache.shape
    if cache.shape[0] != B or dim != D:
        raise ValueError("q and cache disagree")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape:
        raise ValueError("out must have q's shape")
    if ws is None and B > 1:
        need = lib().sd_kv8_attention_workspace(B, R, Hq, Hkv, D, cap)
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    args = (_dev(q, "q", torch.bfloat16), cache.struct, _dev(out, "out", torch.bfloat16), R, Hq, float(scale),
            SD_ATTN_BLOCK_MASK if block else 0)
    if ws is None:
        _check(lib().sd_kv8_attention(*args, _stream()), "sd_kv8_attention")
    else:
        _check(lib().sd_kv8_attention_ex(*args, _dev(ws, "ws"), ws.numel() * ws.element_size(), _stream()),
               "sd_kv8_attention")
    return out


# ------------------------------------------------------ weights and eviction

def attention_weights_workspace_bytes(B, R, Hq, Hkv, D, capacity):
    return int(lib().sd_attention_weights_workspace(B, R, Hq, Hkv, D, capacity))


def attention_weights(q, cache, weights_in=None, weights=None, decay=1.0, committed=None, scale=0.0, ws=None):
    """The attention weight that each cached key gathers from the rows q [B,R,Hq,D] (keys
    appended): weights = decay * weights_in + the sum over the committed rows and the KV
    head's query heads, fp32 [B,Hkv,cap]. committed: int32 [B] rows that count, or all. ws:
    attention_weights_workspace_bytes of device memory; when None a batch that takes one
    has it from torch's allocator, on the current stream."""
    B, R, Hq, D = q.shape
    _, Hkv, cap, _ = cache.shape
    if cache.shape[0] != B or cache.shape[3] != D:
        raise ValueError("q and cache disagree")
    if weights is None:
        weights = torch.zeros((B, Hkv, cap), dtype=torch.float32, device=q.device)
    if weights.shape != (B, Hkv, cap) or (weights_in is not None and weights_in.shape != weights.shape):
        raise ValueError("weights must be [B, Hkv, cap]")
    if committed is not None and committed.shape != (B,):
        raise ValueError("committed must be [B]")
    if ws is None and B > 1:
        need = lib().sd_attention_weights_workspace(B, R, Hq, Hkv, D, cap)
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    args = (_dev(q, "q", torch.bfloat16), cache.struct, R, Hq, float(scale),
            None if committed is None else _dev(committed, "committed", torch.int32),
            None if weights_in is None else _dev(weights_in, "weights_in", torch.float32),
            float(decay), _dev(weights, "weights", torch.float32))
    if ws is None:
        _check(lib().sd_attention_weights(*args, _stream()), "sd_attention_weights")
    else:
        _check(lib().sd_attention_weights_ex(*args, _dev(ws, "ws"), ws.numel() * ws.element_size(), _stream()),
               "sd_attention_weights")
    return weights


def kv_evict(src, weights, dst, keep, sinks=0, recent=0, weights_out=None, kept=None):
    """Copy to dst the min(len, keep) keys of each KV head of src that hold the most weight
    (fp32 [B,Hkv,cap]), the first `sinks` and the last `recent` among them, in their order.
    weights_out [B,Hkv,dst cap] takes their weights, kept [B,Hkv,keep] int32 their indices."""
    B, Hkv, cap, D = src.shape
    keep = int(keep)
    if (dst.shape[0], dst.shape[1], dst.shape[3]) != (B, Hkv, D):
        raise ValueError("the caches disagree")
    if weights.shape != (B, Hkv, cap):
        raise ValueError("weights must be [B, Hkv, cap]")
    if weights_out is not None and weights_out.shape != (B, Hkv, dst.shape[2]):
        raise ValueError("weights_out must be [B, Hkv, cap of dst]")
    if kept is not None and kept.shape != (B, Hkv, keep):
        raise ValueError("kept must be [B, Hkv, keep]")
    _check(lib().sd_kv_evict(src.struct, _dev(weights, "weights", torch.float32), keep, int(sinks), int(recent), dst.struct,
                             None if weights_out is None else _dev(weights_out, "weights_out", torch.float32),
                             None if kept is None else _dev(kept, "kept", torch.int32), _stream()), "sd_kv_evict")


# ------------------------------------------------------------ log probabilities

def token_logprobs(logits, tokens, temperature=1.0, top_n=0, logprob=None, entropy=None, top_ids=None, top_logprobs=None):
    """Log probabilities of tokens [...] int32 under softmax(logits [..., V] / temperature)
    (bf16 or fp32), the rows' entropies (nats) and their top_n alternatives. A token -1
    gives 0. Returns (logprob [...], entropy [...], top_ids [..., top_n] int32,
    top_logprobs [..., top_n])."""
    shape, lead, dtype, top_n = logits.shape, tokens.shape, logits.dtype, int(top_n)
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise ValueError("logits must be bf16 or fp32")
    V, rows = shape[-1], tokens.numel()
    if shape[:-1] != lead:
        raise ValueError("tokens must be %s" % (tuple(shape[:-1]),))
    if logits.is_contiguous():
        ptr, stride = _dev(logits, "logits"), V
    else:
        ptr, stride = _padded_rows(logits, rows)
    wide, f32, i32 = (*lead, max(top_n, 0)), torch.float32, torch.int32
    if logprob is None:
        logprob = torch.empty(lead, dtype=f32, device=logits.device)
    if entropy is None:
        entropy = torch.empty(lead, dtype=f32, device=logits.device)
    if top_ids is None:
        top_ids = torch.empty(wide, dtype=i32, device=logits.device)
    if top_logprobs is None:
        top_logprobs = torch.empty(wide, dtype=f32, device=logits.device)
    if logprob.shape != lead or entropy.shape != lead or top_ids.shape != wide or top_logprobs.shape != wide:
        raise ValueError("logprob and entropy must be %s, top_ids and top_logprobs %s" % (tuple(lead), wide))
    status = lib().sd_token_logprobs(ptr, SD_BF16 if dtype is torch.bfloat16 else SD_F32, rows, V, stride,
                                     _dev(tokens, "tokens", i32), float(temperature), top_n,
                                     _dev(logprob, "logprob", f32), _dev(entropy, "entropy", f32),
                                     _dev(top_ids, "top_ids", i32), _dev(top_logprobs, "top_logprobs", f32), _stream())
    if status:
        raise SDError("sd_token_logprobs", status)
    return logprob, entropy, top_ids, top_logprobs


def _padded_rows(logits, rows):
    """Address and row stride of logits whose rows are contiguous and evenly spaced (a
    padded vocabulary)."""
    if not logits.is_cuda:
        raise ValueError("logits must be on a CUDA device (no CPU path exists)")
    lead, strides = logits.shape[:-1], logits.stride()
    step = next((s for n, s in zip(reversed(lead), reversed(strides[:-1])) if n > 1), logits.shape[-1])
    want = step
    for n, s in zip(reversed(lead), reversed(strides[:-1])):
        if n > 1 and s != want:
            raise ValueError("logits' rows must be evenly spaced")
        want *= n
    if (logits.shape[-1] > 1 and strides[-1] != 1) or step < logits.shape[-1]:
        raise ValueError("logits' rows must be contiguous")
    return logits.data_ptr(), step


# ------------------------------------------------- paged KV cache, drafted trees

class PagedKVCache:
    """One layer's paged bf16 KV cache: pools [pages, Hkv, page, D], a page table [B,
    max_pages] int32 (which may be shared between layers) and device lengths [B]; row n of
    scene b lies in page table[b, n // page]."""

    def __init__(self, k, v, table, lens):
        if k.shape != v.shape or k.dim() != 4:
            raise ValueError("k and v must both be [pages, Hkv, page, D]")
        if table.dim() != 2 or lens.shape != table.shape[:1]:
            raise ValueError("table must be [B, max_pages] and len [B]")
        for t, name, dtype in ((k, "k", torch.bfloat16), (v, "v", torch.bfloat16), (table, "table", torch.int32),
                               (lens, "len", torch.int32)):
            _dev(t, name, dtype)
        _same_device(k, v, table, lens)
        self.k, self.v, self.table, self.len = k, v, table, lens
        n_pages, H, page, D = k.shape
        B, max_pages = table.shape
        self._ticket = torch.zeros(max(B, 1), dtype=torch.int32, device=k.device)
        self._struct = PagedCacheStruct(k.data_ptr(), v.data_ptr(), table.data_ptr(), lens.data_ptr(),
                                        self._ticket.data_ptr(), B, H, n_pages, page, max_pages, D)
        # what a call reads, fixed with the struct
        self._ref, self._shape, self._device = ctypes.byref(self._struct), (B, H, max_pages * page, D), k.device.index

    @classmethod
    def empty(cls, B, Hkv, cap, D, page=64, device="cuda"):
        """Room for cap rows a scene, every scene with pages of its own."""
        if int(page) <= 0:
            raise ValueError("page must be positive")
        per = -(-cap // page)
        k = torch.zeros((B * per, Hkv, page, D), dtype=torch.bfloat16, device=device)
        table = torch.arange(B * per, dtype=torch.int32, device=device).view(B, per)
        return cls(k, torch.zeros_like(k), table, torch.zeros(B, dtype=torch.int32, device=device))

    @property
    def struct(self):
        return self._ref

    @property
    def shape(self):
        """(scenes, KV heads, rows that a scene's pages hold, head dim)"""
        return self._shape


class PagedKVCacheGroup:
    """The caches of a step's layers, as paged_commit takes them."""

    def __init__(self, caches):
        self.caches = tuple(caches)
        if not self.caches:
            raise ValueError("no caches")
        _same_device(*(c.k for c in self.caches))
        self._structs = (PagedCacheStruct * len(self.caches))(*(c._struct for c in self.caches))


def _stream_on(index):
    """The current stream, of the device that the tensors are on: kernels launch on the current one."""
    at = torch.cuda.current_device() if _raw_device is None else _raw_device()
    if index != at:
        raise ValueError("the tensors must be on the current device")
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(at)


def _ints(t, name, shape, device):
    """Address of an int32 tensor of this shape on this device, None for None."""
    if t is None:
        return None
    if t.__class__ is not _Tensor or t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        _dev(t, name, torch.int32)
        if t.shape != shape or t.get_device() != device:
            raise ValueError("%s must be %s on the caller's device" % (name, tuple(shape)))
    return t.data_ptr()


def _ws(ws, device):
    """Address and bytes of a workspace on this device."""
    ptr = _dev(ws, "ws")
    if ws.get_device() != device:
        raise ValueError("ws must be on the caller's device")
    return ptr, ws.numel() * ws.element_size()


def _row_stride(t, name, shape, device):
    """Address and row stride of bf16 rows [B, R, H, D] whose last two dims are contiguous
    and whose rows are evenly spaced (part of a projection's output)."""
    if not isinstance(t, _Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype is not torch.bfloat16 or t.shape != shape or t.get_device() != device:
        raise ValueError("%s must be %s bf16 on the caller's CUDA device" % (name, tuple(shape)))
    B, R, H, D = shape
    if t.is_contiguous():
        return t.data_ptr(), H * D
    sb, sr, sh, sd_ = t.stride()
    if (D > 1 and sd_ != 1) or (H > 1 and sh != D):
        raise ValueError("%s: a row's heads must be contiguous" % name)
    step = sr if R > 1 else sb
    if R > 1 and B > 1 and sb != R * sr:
        raise ValueError("%s's rows must be evenly spaced" % name)
    if step % 8:
        raise ValueError("%s's rows must be a multiple of 8 elements apart" % name)
    return t.data_ptr(), step


def paged_append(cache, k_new, v_new, q=None, pos=None, sections=None, interleaved=0, base=1e6, n_new=None, q_out=None):
    """Append k_new / v_new [B,R,Hkv,D] to a PagedKVCache, the keys rotated at pos [B,R,3] on
    the way, and rotate q [B,R,Hq,D] beside them: into q_out [B,R,Hq,D], or in place. pos
    None: nothing is rotated (q must be None). n_new: int32 [B] rows of each scene that
    count, or all. k_new, v_new and q may be parts of one projection's output. Returns the
    rotated queries."""
    B, H, _, D = cache._shape
    dev = cache._device
    stream = _stream_on(dev)
    if len(k_new.shape) != 4:
        raise ValueError("k_new must be [B, R, Hkv, D]")
    R = k_new.shape[1]
    kp, ks = _row_stride(k_new, "k_new", (B, R, H, D), dev)
    vp, vs = _row_stride(v_new, "v_new", (B, R, H, D), dev)
    Hq, qp, qs, op = 0, None, 0, None
    if q is not None:
        if pos is None:
            raise ValueError("q without pos")
        Hq = q.shape[2] if len(q.shape) == 4 else 0
        qp, qs = _row_stride(q, "q", (B, R, Hq, D), dev)
        if q_out is not None:
            op = _dev(q_out, "q_out", torch.bfloat16)
            if q_out.shape != q.shape or q_out.get_device() != dev:
                raise ValueError("q_out must have q's shape and device")
    elif q_out is not None:
        raise ValueError("q_out without q")
    if pos is not None and sections is None:
        raise ValueError("pos without sections")
    sec = None if pos is None else _sections(sections if sections.__class__ is tuple else tuple(int(x) for x in sections))
    _check(lib().sd_paged_append(cache._ref, kp, ks, vp, vs, qp, qs, op, R, Hq, _ints(pos, "pos", (B, R, 3), dev), sec,
                                 int(interleaved), float(base), _ints(n_new, "n_new", (B,), dev), stream),
           "sd_paged_append")
    return q if q_out is None else q_out


def tree_attention_workspace_bytes(B, R, Hq, Hkv, D, capacity):
    """The most that a call of up to B scenes, R rows and capacity (max_pages * page) rows takes."""
    return int(lib().sd_tree_attention_workspace(B, R, Hq, Hkv, D, capacity))


def tree_attention(q, cache, parents=None, n_new=None, out=None, scale=0.0, ws=None):
    """Attention of a drafted tree's rows q [B,R,Hq,D] (rotated) over a PagedKVCache that
    holds them: a row sees the prefix, its ancestors and itself. parents [B,R] int32: the
    earlier row that each row follows, -1 for the prefix; None: a chain. n_new: int32 [B]
    rows of each scene that count, or all. ws: tree_attention_workspace_bytes of device
    memory (of the largest call, where it serves several); when None a call that takes one has
    it from torch's allocator, on the current stream."""
    B, H, cap, D = cache._shape
    dev = cache._device
    stream = _stream_on(dev)
    if len(q.shape) != 4:
        raise ValueError("q must be [B, R, Hq, D]")
    R, Hq = q.shape[1], q.shape[2]
    qp, qs = _row_stride(q, "q", (B, R, Hq, D), dev)
    if out is None:
        out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    elif out.shape != q.shape or out.get_device() != dev:
        raise ValueError("out must have q's shape and device")
    args = (qp, qs, cache._ref, _ints(parents, "parents", (B, R), dev), _ints(n_new, "n_new", (B,), dev),
            _dev(out, "out", torch.bfloat16), R, Hq, float(scale))
    status = lib().sd_tree_attention(*args, *((None, 0) if ws is None else _ws(ws, dev)), stream)
    if status == SD_ERR_WORKSPACE and ws is None:  # (nothing was launched; most calls take none)
        ws = torch.empty(tree_attention_workspace_bytes(B, R, Hq, H, D, cap), dtype=torch.uint8, device=q.device)
        status = lib().sd_tree_attention(*args, *_ws(ws, dev), stream)
    _check(status, "sd_tree_attention")
    return out


def accept_tree_workspace_bytes(B, R, V):
    return int(lib().sd_accept_tree_workspace(B, R, V))


def accept_tree(logits, tokens, parents=None, n_new=None, ws=None, n_emit=None, path=None, out=None, argmax=None):
    """Greedy acceptance along a tree: from row 0 to the child whose token [B,R] int32 is the
    row's argmax of logits [B,R,V] (bf16 or fp32), while there is one. parents, n_new: as for
    tree_attention. ws: accept_tree_workspace_bytes, zero-filled before its first use.
    Returns (n_emit [B], path [B,R], out [B,R], argmax [B,R]) int32: the rows on the walk, their
    indices, then -1, and the tokens that they emit, then -1."""
    B, R, V = logits.shape
    dt = {torch.bfloat16: SD_BF16, torch.float32: SD_F32}.get(logits.dtype)
    if dt is None:
        raise ValueError("logits must be bf16 or fp32")
    if logits.is_contiguous():
        ptr, stride = _dev(logits, "logits"), V
    else:
        ptr, stride = _padded_rows(logits, B * R)
    dev = logits.device
    stream = _stream_on(dev.index)
    if ws is None:
        ws = workspace(accept_tree_workspace_bytes(B, R, V), dev)
    n_emit = torch.empty(B, dtype=torch.int32, device=dev) if n_emit is None else n_emit
    path = torch.empty((B, R), dtype=torch.int32, device=dev) if path is None else path
    out = torch.empty((B, R), dtype=torch.int32, device=dev) if out is None else out
    argmax = torch.empty((B, R), dtype=torch.int32, device=dev) if argmax is None else argmax
    wide, at = (B, R), dev.index
    _check(lib().sd_accept_tree(ptr, dt, B, R, V, stride, _ints(tokens, "tokens", wide, at), _ints(parents, "parents", wide, at),
                                _ints(n_new, "n_new", (B,), at), _ints(n_emit, "n_emit", (B,), at), _ints(path, "path", wide, at),
                                _ints(out, "out", wide, at), _ints(argmax, "argmax", wide, at), *_ws(ws, at), stream),
           "sd_accept_tree")
    return n_emit, path, out, argmax


def paged_commit(caches, path, n_emit, n_new=None):
    """Keep the rows path [B,R] int32 (n_emit [B] of them) of the R rows (n_new [B]) that were
    appended last, in a PagedKVCacheGroup, a PagedKVCache or a list of them: they move
    together behind the prefix and the lengths follow."""
    if not isinstance(caches, PagedKVCacheGroup):
        caches = PagedKVCacheGroup([caches] if isinstance(caches, PagedKVCache) else caches)
    first = caches.caches[0]
    B, dev = first._shape[0], first._device
    stream = _stream_on(dev)
    if len(path.shape) != 2:
        raise ValueError("path must be [B, R]")
    R = path.shape[1]
    _check(lib().sd_paged_commit(caches._structs, len(caches.caches), _ints(path, "path", (B, R), dev),
                                 _ints(n_emit, "n_emit", (B,), dev), _ints(n_new, "n_new", (B,), dev), R, stream),
           "sd_paged_commit")


# -------------------------------------------------------------- acceptance

def greedy_workspace_bytes(B, K, V):
    return int(lib().sd_accept_greedy_workspace(B, K, V))


def sample_workspace_bytes(B, K, V):
    return int(lib().sd_accept_sample_workspace(B, K, V))


def accept_greedy(logits, draft, ws=None, n_emit=None, tokens=None, argmax=None):
    """Greedy acceptance over logits [B,K+1,V] (bf16 or fp32) and draft [B,K] int32.
    Returns (n_emit [B], tokens [B,K+1], argmax [B,K+1]) int32 device tensors."""
    B, R, V = logits.shape
    K = R - 1
    dt = {torch.bfloat16: SD_BF16, torch.float32: SD_F32}.get(logits.dtype)
    if dt is None:
        raise ValueError("logits must be bf16 or fp32")
    dev = logits.device
    if ws is None:
        ws = workspace(greedy_workspace_bytes(B, K, V), dev)
    n_emit = torch.empty(B, dtype=torch.int32, device=dev) if n_emit is None else n_emit
    tokens = torch.empty((B, R), dtype=torch.int32, device=dev) if tokens is None else tokens
    argmax = torch.empty((B, R), dtype=torch.int32, device=dev) if argmax is None else argmax
    draft_p = _dev(draft, "draft", torch.int32) if K > 0 else ctypes.c_void_p(0)
    _check(lib().sd_accept_greedy(_dev(logits, "logits"), dt, B, K, V, draft_p,
                                  _dev(n_emit, "n_emit", torch.int32), _dev(tokens, "tokens", torch.int32),
                                  _dev(argmax, "argmax", torch.int32), _dev(ws, "ws"), ws.numel() * ws.element_size(),
                                  _stream()), "sd_accept_greedy")
    return n_emit, tokens, argmax


def accept_greedy_noalloc(logits, draft, n_emit=None, tokens=None, argmax=None):
    """sd_accept_greedy_noalloc: greedy acceptance with the library's fixed
    scratch array instead of a caller workspace (no device allocation)."""
    B, R, V = logits.shape
    K = R - 1
    dt = {torch.bfloat16: SD_BF16, torch.float32: SD_F32}.get(logits.dtype)
    if dt is None:
        raise ValueError("logits must be bf16 or fp32")
    dev = logits.device
    n_emit = torch.empty(B, dtype=torch.int32, device=dev) if n_emit is None else n_emit
    tokens = torch.empty((B, R), dtype=torch.int32, device=dev) if tokens is None else tokens
    argmax = torch.empty((B, R), dtype=torch.int32, device=dev) if argmax is None else argmax
    draft_p = _dev(draft, "draft", torch.int32) if K > 0 else ctypes.c_void_p(0)
    _check(lib().sd_accept_greedy_noalloc(_dev(logits, "logits"), dt, B, K, V, draft_p,
                                          _dev(n_emit, "n_emit", torch.int32),
                                          _dev(tokens, "tokens", torch.int32),
                                          _dev(argmax, "argmax", torch.int32), _stream()),
           "sd_accept_greedy_noalloc")
    return n_emit, tokens, argmax


def accept_sample(z_target, z_draft, draft, u, temperature, ws=None, n_emit=None, tokens=None):
    """Rejection-sampling acceptance; returns (n_emit [B], tokens [B,K+1]) int32."""
    B, R, V = z_target.shape
    K = R - 1
    dev = z_target.device
    if ws is None:
        ws = workspace(sample_workspace_bytes(B, K, V), dev)
    n_emit = torch.empty(B, dtype=torch.int32, device=dev) if n_emit is None else n_emit
    tokens = torch.empty((B, R), dtype=torch.int32, device=dev) if tokens is None else tokens
    zd = _dev(z_draft, "z_draft", torch.float32) if K > 0 else ctypes.c_void_p(0)
    dr = _dev(draft, "draft", torch.int32) if K > 0 else ctypes.c_void_p(0)
    _check(lib().sd_accept_sample(_dev(z_target, "z_target", torch.float32), zd, B, K, V,
                                  float(temperature), dr, _dev(u, "u", torch.float32),
                                  _dev(n_emit, "n_emit", torch.int32), _dev(tokens, "tokens", torch.int32),
                                  _dev(ws, "ws"), ws.numel() * ws.element_size(), _stream()),
           "sd_accept_sample")
    return n_emit, tokens


def set_cluster_size(cluster_size=0):
    """Force the tcgen05 attention cluster size (1, 2, 4, 6, 8, 16); 0 = automatic."""
    _check(lib().sd_set_cluster_size(int(cluster_size)), "sd_set_cluster_size")


def verify_kernel(B, R, Hq, Hkv, D, capacity, layer=False):
    """Name of the kernel that serves this shape on the current device
    (sd_verify_kernel): "tcgen05", "mma.sync" or "three kernels"."""
    return lib().sd_verify_kernel(B, R, Hq, Hkv, D, capacity, 1 if layer else 0).decode()


def verify_cluster_size(B, R, Hq, Hkv, D, capacity, layer=False):
    """CTAs a cluster that this shape's next call takes (sd_verify_cluster_size); 0 off the tcgen05 path."""
    return lib().sd_verify_cluster_size(B, R, Hq, Hkv, D, capacity, 1 if layer else 0)


def get_device_error():
    """Synchronise the current stream; return and clear the device error bits."""
    bits = ctypes.c_uint32(0)
    st = lib().sd_get_device_error(torch.cuda.current_stream().cuda_stream, ctypes.byref(bits))
    if st not in (0, 5, 6):
        raise SDError("sd_get_device_error", st)
    return int(bits.value)
