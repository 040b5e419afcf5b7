"""Binding of the operators in include/tst_attention.h -- same names as the C entry points, argument marshalling only, with the manners of
operators.py: what does not fit raises ValueError, what the library refuses TstgemmError."""
from __future__ import annotations

import ctypes
import math

from . import binding
from .binding import TstgemmError, _launch_stream, _load
from .operators import _dense, _on, _result, _shared, _type, _workspace

KV_BLOCK = 16   # tokens that share a scale
_vp, _ci, _i64, _sz, _f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
_SIGNATURES = {
    "tst_kv_row": [_ci],
    "tst_kv_cache_bytes": [_ci, _ci, _ci, _ci, ctypes.POINTER(_sz), ctypes.POINTER(_sz)],
    "tst_kv_append": [_vp, _vp, _ci, _vp, _vp, _vp, _ci, _vp, _vp, _vp, _vp],
    "tst_kv_read": [_vp, _vp, _ci, _vp, _vp, _vp],
    "tst_kv_attention_workspace_bytes": [_vp, _vp, _ci, ctypes.POINTER(_sz)],
    "tst_kv_attention": [_vp, _ci, _ci, _vp, _vp, _f32, _vp, _vp, _sz, _vp],
    "tst_attention": [_vp, _vp, _vp, _ci, _ci, _ci, _ci, _vp, _ci, _ci, _f32, _vp, _vp],
}
_lib = None
_native = None   # the native half (csrc/launch_attention.cpp): calls with plain tensors that bring nothing but their operands


def _ops():
    global _lib, _native
    if _lib is None:
        lib = _load()
        for name, args in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ctypes.c_int
        _lib = lib
        if binding._launch is not None:   # built, and for this torch
            from . import _launch as native
            native.bind_attention(*(ctypes.cast(getattr(lib, name), _vp).value for name in (
                "tst_kv_append", "tst_kv_read", "tst_kv_attention_workspace_bytes", "tst_kv_attention", "tst_attention")), TstgemmError, KvCache)
            _native = native
    return _lib


def _call(name, *args):
    for value, kind in zip(args, _SIGNATURES[name]):
        if kind is _ci and not -2 ** 31 <= value < 2 ** 31:   # ctypes would take its low 32 bits
            raise TstgemmError(-1, name)
    rc = getattr(_ops(), name)(*args)
    if rc != 0:
        raise TstgemmError(rc, name)


class _CacheStruct(ctypes.Structure):
    """tst_kv_cache_t of include/tst_attention.h."""
    _fields_ = [("struct_size", _sz), ("pages", _ci), ("page_tokens", _ci), ("heads", _ci), ("head_size", _ci), ("k_codes", _vp), ("v_codes", _vp),
                ("k_scale", _vp), ("v_scale", _vp)]


class _SequencesStruct(ctypes.Structure):
    """tst_sequences_t"""
    _fields_ = [("struct_size", _sz), ("sequences", _ci), ("tokens", _ci), ("offsets", _vp), ("lens", _vp), ("table", _vp), ("columns", _ci), ("table_stride", _i64)]


class _HeadsStruct(ctypes.Structure):
    """tst_heads_t"""
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class _RotationStruct(ctypes.Structure):
    """tst_rotation_t"""
    _fields_ = [("struct_size", _sz), ("cos", _vp), ("sin", _vp), ("positions", _ci), ("pairs", _ci), ("interleaved", _ci)]


def _struct(kind, what, *values):
    """A struct of the call `what`; refuses integers of which a field would take the low 32 bits."""
    for (_, field), value in zip(kind._fields_, values):
        if field is _ci and not -2 ** 31 <= value < 2 ** 31:
            raise TstgemmError(-1, what)
    return kind(*values)


def _tensor_of_cache(i, name):
    def put(self, t):   # cache.k_scale *= 2 comes here with the tensor that is there
        if t is not self._tensors[i]:
            raise AttributeError(f"{name} stays the tensor it is: copy into it, or make a KvCache of others")
    return property(lambda self: self._tensors[i], put)


class KvCache:
    """Keys and values of one layer in 8 bits (tst_kv_cache): pages of `page` tokens, a scale for each block of 16 tokens and head.

    k_codes int8 [pages, heads, page, row], v_codes int8 [pages, heads, page / 16, row, 16], k_scale and v_scale float32 [pages, heads, page / 16]; row is
    head_size padded to 64, 96, 128, 192 or 256.  What a cache is made of stays: calls go by the addresses of its tensors, so none can be
    put in another's place, and a cache whose tensors have been given other memory since is refused."""

    def __init__(self, page, head_size, k_codes, v_codes, k_scale, v_scale):
        import torch
        sizes = all(isinstance(t, torch.Tensor) for t in (k_codes, v_codes, k_scale, v_scale)) and k_codes.dim() == 4 and isinstance(page, int) and isinstance(head_size, int)
        row = _ops().tst_kv_row(head_size) if sizes and 1 <= head_size <= 256 else 0
        if not row or page not in (16, 32, 64, 128, 256):
            raise ValueError("a cache has pages of 16, 32, 64, 128 or 256 tokens, heads of 1 to 256 entries, and four tensors")
        pages, heads = k_codes.shape[:2]
        for t, name, dtype, shape in ((k_codes, "k_codes", torch.int8, (pages, heads, page, row)), (v_codes, "v_codes", torch.int8, (pages, heads, page // 16, row, 16)),
                                      (k_scale, "k_scale", torch.float32, (pages, heads, page // 16)), (v_scale, "v_scale", torch.float32, (pages, heads, page // 16))):
            _dense(t, name, dtype, shape, k_codes.get_device())
        codes, scales = _sz(), _sz()
        _call("tst_kv_cache_bytes", pages, page, heads, head_size, ctypes.byref(codes), ctypes.byref(scales))   # refuses sizes that no call takes
        self._device_index, self._tensors = k_codes.get_device(), (k_codes, v_codes, k_scale, v_scale)
        self._struct = _struct(_CacheStruct, "tst_kv_cache_bytes", ctypes.sizeof(_CacheStruct), pages, page, heads, head_size, *(t.data_ptr() for t in self._tensors))   # their addresses
        self._ref, self._raw = ctypes.byref(self._struct), ctypes.addressof(self._struct)

    pages, page = property(lambda self: self._struct.pages), property(lambda self: self._struct.page_tokens)
    heads, head_size = property(lambda self: self._struct.heads), property(lambda self: self._struct.head_size)
    device_index = property(lambda self: self._device_index)
    k_codes, v_codes, k_scale, v_scale = (_tensor_of_cache(i, name) for i, name in enumerate(("k_codes", "v_codes", "k_scale", "v_scale")))

    def _check(self):
        s = self._struct
        if tuple(t.data_ptr() for t in self._tensors) != (s.k_codes, s.v_codes, s.k_scale, s.v_scale):
            raise ValueError("the cache's tensors have been given other memory: make a KvCache of them")


def tst_kv_cache(pages: int, page: int, heads: int, head_size: int, device=None) -> KvCache:
    """A cache with nothing in it, on the current device unless another is given."""
    import torch
    codes, scales = _sz(), _sz()
    _call("tst_kv_cache_bytes", pages, page, heads, head_size, ctypes.byref(codes), ctypes.byref(scales))
    row = _ops().tst_kv_row(head_size)
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    scale = (pages, heads, page // 16)
    return KvCache(page, head_size, torch.zeros((pages, heads, page, row), dtype=torch.int8, device=device),
                   torch.zeros((*scale, row, 16), dtype=torch.int8, device=device), torch.zeros(scale, device=device), torch.zeros(scale, device=device))


def _heads(x, what, dtype=None, like=None):
    """A CUDA tensor [T, heads, size] on the current device whose heads' entries lie together; `like`: (T, size) that it has to have."""
    import torch
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 3 and (dtype is None or x.dtype == dtype)):
        raise ValueError(f"{what} must be a CUDA tensor [tokens, heads, head size]" + (f" of {dtype}" if dtype else ""))
    if x.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what} must be on the current device")
    if x.is_neg():   # a view whose memory holds the values negated
        raise ValueError(f"{what} must hold its values as they are (resolve_neg())")
    T, heads, size = x.shape
    if heads < 1 or size < 1 or (size > 1 and x.stride(2) != 1):
        raise ValueError(f"{what} must have heads whose entries lie together")
    if like is not None and (T, size) != tuple(like):
        raise ValueError(f"{what} must have {like[0]} tokens and a head size of {like[1]}")
    return _HeadsStruct(x.data_ptr(), x.stride(0) if T > 1 else 0, x.stride(1) if heads > 1 else 0)


def _int32(x, what, shape, dev):
    import torch
    return _dense(x, what, torch.int32, shape, dev)


def _sequences(cache, pages, lens, offsets, T, what):
    """tst_sequences_t of packed rows; pages may have rows that lie apart."""
    import torch
    if not isinstance(cache, KvCache) or cache.device_index != torch.cuda.current_device():
        raise ValueError("cache must be a KvCache on the current device")
    cache._check()
    dev = cache.device_index
    if not (isinstance(pages, torch.Tensor) and pages.is_cuda and pages.dtype == torch.int32 and pages.dim() == 2 and pages.shape[1] >= 1 and not pages.is_neg()
            and pages.get_device() == dev and (pages.shape[1] == 1 or pages.stride(1) == 1)):
        raise ValueError("pages must be an int32 CUDA matrix of contiguous rows on the cache's device")
    S, columns = pages.shape
    stride = pages.stride(0) if S > 1 else columns
    if stride < columns:
        raise ValueError("pages must have rows that do not overlap")
    lens_ptr = _int32(lens, "lens", (S,), dev)
    offsets_ptr = None if offsets is None else _int32(offsets, "offsets", (S + 1,), dev)
    if offsets is None and T != S:
        raise ValueError("without offsets there is a token for each sequence")
    return _struct(_SequencesStruct, what, ctypes.sizeof(_SequencesStruct), S, T, offsets_ptr, lens_ptr, pages.data_ptr(), columns, stride)


def tst_kv_append(cache: KvCache, K, V, pages, lens, offsets=None, Q=None, cos=None, sin=None, interleaved=False, keys=False, stream=None):
    """New keys and values [T, heads, head_size] (float32, bfloat16 or float16) into the cache: rows offsets[i] .. offsets[i + 1] - 1 are the last tokens of sequence i,
    which has lens[i] tokens with them; a token at position p is in page pages[i, p // page].  offsets None: a row for each sequence.  offsets, lens, pages: int32 on the GPU.

    cos, sin float32 [positions, pairs]: keys are rotated by their positions on the way, and queries Q [T, q_heads, head_size] if there are any, in halves
    (i, i + pairs) or neighbours (2 i, 2 i + 1).  Returns (Q rotated or None, K rotated if `keys` or None)."""
    if _native is not None and stream is None:
        done = _native.kv_append(cache, K, V, pages, lens, offsets, Q, cos, sin, interleaved, keys)
        if done is not None:
            return done
    import torch
    k = _heads(K, "K")
    kind, T, dev = _type(K.dtype, "K"), K.shape[0], K.get_device()
    s = _sequences(cache, pages, lens, offsets, T, "tst_kv_append")
    if K.shape[1:] != (cache.heads, cache.head_size) or not isinstance(V, torch.Tensor) or V.shape != K.shape:
        raise ValueError(f"K and V must be [tokens, {cache.heads}, {cache.head_size}]")
    v = _heads(V, "V", K.dtype)
    q = None if Q is None else _heads(Q, "Q", K.dtype, (T, cache.head_size))
    rotation = None
    if (cos is None) != (sin is None) or (cos is None and (Q is not None or keys)):
        raise ValueError("cos and sin come together, and with queries or rotated keys")
    if cos is not None:
        if not isinstance(cos, torch.Tensor) or cos.dim() != 2 or cos.shape[0] < 1 or not 1 <= cos.shape[1] <= cache.head_size // 2:
            raise ValueError("cos and sin must be [positions, pairs], with at most head_size / 2 pairs")
        rotation = _struct(_RotationStruct, "tst_kv_append", ctypes.sizeof(_RotationStruct), _dense(cos, "cos", torch.float32, cos.shape, dev), _dense(sin, "sin", torch.float32, cos.shape, dev),
                           *cos.shape, int(bool(interleaved)))
    q_out = None if Q is None else _result(None, "", K.dtype, tuple(Q.shape), stream, dev)
    k_out = _result(None, "", K.dtype, tuple(K.shape), stream, dev) if keys else None
    _call("tst_kv_append", cache._ref, ctypes.byref(s), kind, ctypes.byref(k), ctypes.byref(v), None if q is None else ctypes.byref(q), 0 if q is None else Q.shape[1],
          None if rotation is None else ctypes.byref(rotation), None if q_out is None else q_out.data_ptr(), None if k_out is None else k_out.data_ptr(), _launch_stream(stream, dev))
    _shared(stream, (*cache._tensors, K, V, Q, pages, lens, offsets, cos, sin), [t for t in (*cache._tensors, q_out, k_out) if t is not None])
    return q_out, k_out


def tst_kv_read(cache: KvCache, pages, lens, tokens: int, offsets=None, dtype=None, stream=None):
    """What the codes of the last tokens of sequences stand for: (K, V), each [tokens, heads, head_size] of dtype (bfloat16 unless another is given).  offsets, lens and
    pages as in tst_kv_append."""
    if _native is not None and stream is None:
        done = _native.kv_read(cache, pages, lens, tokens, offsets, dtype)
        if done is not None:
            return done
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    kind, tokens = _type(dtype, "dtype"), int(tokens)
    if tokens < 0:
        raise ValueError("tokens is a number of rows")
    s = _sequences(cache, pages, lens, offsets, tokens, "tst_kv_read")
    dev, shape = cache.device_index, (tokens, cache.heads, cache.head_size)
    K, V = _result(None, "", dtype, shape, stream, dev), _result(None, "", dtype, shape, stream, dev)
    _call("tst_kv_read", cache._ref, ctypes.byref(s), kind, K.data_ptr(), V.data_ptr(), _launch_stream(stream, dev))
    _shared(stream, (*cache._tensors, pages, lens, offsets), (K, V))
    return K, V


def _scale(scale, size):
    scale = 1 / math.sqrt(size) if scale is None else float(scale)
    if not abs(scale) <= 2.0 ** 127:
        raise ValueError("scale must be finite, and no more than 2^127")
    return scale


def tst_kv_attention(Q, cache: KvCache, pages, lens, offsets=None, scale=None, Y=None, workspace=None, stream=None):
    """Attention of new tokens, which have been appended, over the cache: Q [T, q_heads, head_size] float32, bfloat16 or float16, q_heads a multiple of the cache's heads ->
    Y of the same shape and type.  offsets, lens and pages as in tst_kv_append; scale: 1 / sqrt(head_size) unless another is given."""
    if _native is not None and Y is None and workspace is None and stream is None:
        done = _native.kv_attention(Q, cache, pages, lens, offsets, scale)
        if done is not None:
            return done
    q = _heads(Q, "Q")
    kind, (T, q_heads, size), dev = _type(Q.dtype, "Q"), Q.shape, Q.get_device()
    s = _sequences(cache, pages, lens, offsets, T, "tst_kv_attention")
    if size != cache.head_size or q_heads % cache.heads:
        raise ValueError(f"Q must be [tokens, a multiple of {cache.heads}, {cache.head_size}]")
    scale = _scale(scale, size)
    need = _sz()
    _call("tst_kv_attention_workspace_bytes", cache._ref, ctypes.byref(s), q_heads, ctypes.byref(need))
    Y = _result(Y, "Y", Q.dtype, (T, q_heads, size), stream, dev)
    keep, ws, n = _workspace(need.value, workspace, stream, dev)
    _call("tst_kv_attention", ctypes.byref(q), kind, q_heads, cache._ref, ctypes.byref(s), scale, Y.data_ptr(), ws, n, _launch_stream(stream, dev))
    _shared(stream, (Q, *cache._tensors, pages, lens, offsets, Y, keep), (Y,))
    return Y


def tst_attention(Q, K, V, offsets, scale=None, Y=None, stream=None):
    """Causal attention over whole prompts packed one behind another: Q [T, q_heads, head_size], K and V [T, heads, head_size] of one type, float32, bfloat16 or float16, q_heads a
    multiple of heads; offsets int32 [sequences + 1] on the GPU, rows offsets[i] .. offsets[i + 1] - 1 being sequence i.  Y: as Q; rows of no sequence are left as they are
    (in a Y that is made here: whatever the memory held).  scale: 1 / sqrt(head_size) unless another is given."""
    if _native is not None and Y is None and stream is None:
        done = _native.attention(Q, K, V, offsets, scale)
        if done is not None:
            return done
    import torch
    q = _heads(Q, "Q")
    kind, (T, q_heads, size), dev = _type(Q.dtype, "Q"), Q.shape, Q.get_device()
    k, v = _heads(K, "K", Q.dtype, (T, size)), _heads(V, "V", Q.dtype, (T, size))
    if K.shape != V.shape or q_heads % K.shape[1]:
        raise ValueError("K and V must have the same heads, and Q a multiple of them")
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("offsets must be int32 [sequences + 1]")
    S = offsets.numel() - 1
    offsets_ptr = _int32(offsets, "offsets", (S + 1,), dev)
    Y = _result(Y, "Y", Q.dtype, (T, q_heads, size), stream, dev)
    _call("tst_attention", ctypes.byref(q), ctypes.byref(k), ctypes.byref(v), kind, q_heads, K.shape[1], size, offsets_ptr, S, T, _scale(scale, size), Y.data_ptr(),
          _launch_stream(stream, dev))
    _shared(stream, (Q, K, V, offsets, Y), (Y,))
    return Y
