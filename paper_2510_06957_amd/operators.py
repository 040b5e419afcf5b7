"""Binding of the operators in include/tst_ops.h -- same names as the C entry points, argument marshalling only.

Tensors are looked over here; what does not fit raises ValueError, what the library refuses TstgemmError.  Results and workspaces are
allocated by torch on the stream the call runs on, unless they are given.
"""
from __future__ import annotations

import contextlib
import ctypes

from . import binding
from .binding import TstgemmError, _launch_stream, _load

TST_F32, TST_BF16, TST_F16 = 0, 1, 2
_vp, _ci, _i64, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
_SIGNATURES = {
    "tst_quantize": [_vp, _ci, _i64, _vp, _i64, _vp, _ci, _ci, _vp],
    "tst_w8_bytes": [_ci, _ci, ctypes.POINTER(_sz)],
    "tst_w8_pack": [_vp, _ci, _ci, _ci, _vp, _vp],
    "tst_w8_gemm": [_vp, _i64, _vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _vp],
    "tst_w8_linear_workspace_bytes": [_ci, _ci, ctypes.POINTER(_sz)],
    "tst_w8_linear": [_vp, _ci, _i64, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _vp, _sz, _vp],
    "tst_moe_workspace_bytes": [_vp, _ci, _ci, ctypes.POINTER(_sz)],
    "tst_moe": [_vp, _i64, _vp, _ci, _ci, _vp, _vp, _vp, _ci, _vp, _sz, _vp],
    "tst_logprobs_workspace_bytes": [_ci, _ci, _ci, ctypes.POINTER(_sz)],
    "tst_logprobs": [_vp, _ci, _i64, _vp, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _ci, _ci, _vp, _sz, _vp],
}
_lib = None
_native = None   # the native half (csrc/launch_ops.cpp): calls with plain tensors that bring nothing but their operands


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
            native.bind_ops(*(ctypes.cast(getattr(lib, name), _vp).value for name in (
                "tst_w8_gemm", "tst_w8_linear_workspace_bytes", "tst_w8_linear", "tst_moe_workspace_bytes", "tst_moe",
                "tst_logprobs_workspace_bytes", "tst_logprobs")), TstgemmError, W8, Moe)
            _native = native
    return _lib


def _call(name, *args):
    for value, kind in zip(args, _SIGNATURES[name]):
        if kind is _ci and not -2 ** 31 <= value < 2 ** 31:   # ctypes would take its low 32 bits
            raise TstgemmError(-1, name)
    rc = getattr(_ops(), name)(*args)
    if rc != 0:
        raise TstgemmError(rc, name)


def _bytes(name, *args) -> int:
    n = _sz()
    _call(name, *args, ctypes.byref(n))
    return n.value


def _type(dtype, what):
    import torch
    try:
        return {torch.float32: TST_F32, torch.bfloat16: TST_BF16, torch.float16: TST_F16}[dtype]
    except KeyError:
        raise ValueError(f"{what} must be float32, bfloat16 or float16") from None


def _rows(x, what, dtype=None):
    """A CUDA matrix on the current device whose rows are contiguous; returns (rows, columns, entries between rows)."""
    import torch
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 2 and (dtype is None or x.dtype == dtype)):
        raise ValueError(f"{what} must be a CUDA matrix" + (f" of {dtype}" if dtype else ""))
    if x.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what} must be on the current device")
    n, k = x.shape
    stride = x.stride(0) if n > 1 else max(k, 1)
    if x.is_neg():   # a view whose memory holds the values negated
        raise ValueError(f"{what} must hold its values as they are (resolve_neg())")
    if k < 1 or (k > 1 and x.stride(1) != 1) or stride < k:
        raise ValueError(f"{what} must have contiguous rows of at least one entry that do not overlap")
    return n, k, stride


def _dense(x, what, dtype, shape, dev):
    import torch
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == dtype and tuple(x.shape) == tuple(shape) and x.is_contiguous()
            and not x.is_neg() and x.get_device() == dev):
        raise ValueError(f"{what} must be a contiguous {dtype} CUDA tensor of shape {list(shape)} on the operands' device")
    return x.data_ptr()


def _on(stream):
    """Memory that a call allocates belongs to the stream it runs on."""
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _shared(stream, operands, results):
    """A call on a stream that was given: operands are in use there until it is done, what it made may be looked at on the current one."""
    import torch
    if stream is not None:
        here = torch.cuda.current_stream()
        for t in operands:
            if t is not None:
                t.record_stream(stream)
        for t in results:
            t.record_stream(here)


def _workspace(bytes_, given, stream, dev):
    """(tensor to keep until the call is enqueued, address, bytes)"""
    import torch
    if given is not None:
        if not (isinstance(given, torch.Tensor) and given.is_cuda and given.is_contiguous() and given.get_device() == dev):
            raise ValueError("workspace must be a contiguous CUDA tensor on the operands' device")
        return given, given.data_ptr(), given.numel() * given.element_size()
    if bytes_ == 0:
        return None, None, 0
    with _on(stream):
        ws = torch.empty(bytes_, dtype=torch.uint8, device=dev)
    return ws, ws.data_ptr(), bytes_


def _result(given, what, dtype, shape, stream, dev):
    import torch
    if given is not None:
        _dense(given, what, dtype, shape, dev)
        return given
    with _on(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


class W8:
    """8-bit weights in their device form (tst_w8_pack) with the scale of each output channel."""

    def __init__(self, K, N, count, packed, scale):
        self.K, self.N, self.count, self.packed, self.scale = K, N, count, packed, scale
        self._check()

    def _check(self):
        """The kernels go by K and N: what they read has to be there."""
        import torch
        p, s = self.packed, self.scale
        if not (isinstance(p, torch.Tensor) and isinstance(s, torch.Tensor) and p.dtype == torch.uint8 and s.dtype == torch.float32 and p.is_contiguous()
                and s.is_contiguous() and p.device == s.device and p.numel() == self.count * _bytes("tst_w8_bytes", self.K, self.N)
                and s.numel() == self.count * self.N):
            raise ValueError("packed (uint8) and scale (float32) must be those of count matrices K x N, contiguous and on one device")


def _pack(W, what, stream):
    """W: [K, N] or [count, K, N]"""
    import torch
    if not (isinstance(W, torch.Tensor) and W.is_cuda and W.dtype == torch.int8 and W.dim() in (2, 3) and W.is_contiguous() and not W.is_neg() and W.numel()):
        raise ValueError(f"{what} must be a contiguous int8 CUDA tensor [K, N] or [count, K, N]")
    dev = W.get_device()
    if dev != torch.cuda.current_device():
        raise ValueError(f"{what} must be on the current device")
    count = W.shape[0] if W.dim() == 3 else 1
    K, N = W.shape[-2:]
    size = _bytes("tst_w8_bytes", K, N)
    with _on(stream):
        packed = torch.empty(count * size, dtype=torch.uint8, device=dev)
    _call("tst_w8_pack", W.data_ptr(), count, K, N, packed.data_ptr(), _launch_stream(stream, dev))
    _shared(stream, (W,), (packed,))
    return count, K, N, packed, dev


def tst_w8_pack(W, scale, stream=None) -> W8:
    """Weights of a layer in 8 bits: W int8 [K, N], scale float32 [N] (of each output channel), both on the GPU.  A ternary matrix
    is a case of them: torch.from_numpy(tcsc_to_dense(t)).cuda()."""
    import torch
    if not isinstance(W, torch.Tensor) or W.dim() != 2:
        raise ValueError("W must be a contiguous int8 CUDA tensor [K, N]")
    count, K, N, packed, dev = _pack(W, "W", stream)
    _dense(scale, "scale", torch.float32, (N,), dev)
    return W8(K, N, count, packed, scale)


def _layer(w, b, dev):
    import torch
    if not isinstance(w, W8) or w.count != 1 or w.packed.get_device() != dev:
        raise ValueError("w must be the W8 of one matrix on the operands' device")
    w._check()
    return None if b is None else _dense(b, "b", torch.float32, (w.N,), dev)


def tst_quantize(X, Q=None, scale=None, stream=None):
    """Codes and scales of tokens: X [M, K] float32, bfloat16 or float16 -> (Q int8 [M, K], scale float32 [M]).  Q is a view of rows
    on 64-byte borders unless it is given."""
    import torch
    M, K, stride = _rows(X, "X")
    kind, dev = _type(X.dtype, "X"), X.get_device()
    if Q is None:
        with _on(stream):
            Q = torch.empty((M, (K + 63) // 64 * 64), dtype=torch.int8, device=dev)[:, :K]
    elif not (isinstance(Q, torch.Tensor) and Q.is_cuda and Q.get_device() == dev and tuple(Q.shape) == (M, K)):
        raise ValueError("Q must be an int8 CUDA matrix of X's shape on X's device")
    _, _, q_stride = _rows(Q, "Q", torch.int8)
    scale = _result(scale, "scale", torch.float32, (M,), stream, dev)
    _call("tst_quantize", X.data_ptr(), kind, stride, Q.data_ptr(), q_stride, scale.data_ptr(), M, K, _launch_stream(stream, dev))
    _shared(stream, (X, Q, scale), (Q, scale))
    return Q, scale


def tst_w8_gemm(Q, scale, w: W8, b=None, Y=None, dtype=None, stream=None):
    """Y = (Q W) scale[:, None] w.scale + b: Q int8 [M, K] with rows on 16-byte borders (as tst_quantize leaves them), scale float32
    [M], w from tst_w8_pack, b float32 [N] or None.  dtype of Y: float32 unless another or Y itself is given."""
    if _native is not None and Y is None and stream is None:
        done = _native.w8_gemm(Q, scale, w, b, dtype)
        if done is not None:
            return done
    import torch
    M, K, stride = _rows(Q, "Q", torch.int8)
    dev = Q.get_device()
    b_ptr = _layer(w, b, dev)
    if K != w.K:
        raise ValueError(f"Q has {K} columns, w {w.K} rows")
    if Q.data_ptr() % 16 or (M > 1 and stride % 16):
        raise ValueError("Q's rows must start on 16-byte borders (tst_quantize allocates them so)")
    s_ptr = _dense(scale, "scale", torch.float32, (M,), dev)
    dtype = dtype or (torch.float32 if Y is None else Y.dtype)
    kind = _type(dtype, "Y")
    Y = _result(Y, "Y", dtype, (M, w.N), stream, dev)
    _call("tst_w8_gemm", Q.data_ptr(), stride, s_ptr, w.packed.data_ptr(), w.scale.data_ptr(), b_ptr, Y.data_ptr(), kind, M, K, w.N,
          _launch_stream(stream, dev))
    _shared(stream, (Q, scale, w.packed, w.scale, b, Y), (Y,))
    return Y


def tst_w8_linear(X, w: W8, b=None, Y=None, workspace=None, stream=None):
    """tst_w8_gemm() of tst_quantize(X): X [M, K] float32, bfloat16 or float16, Y of the same type."""
    if _native is not None and Y is None and workspace is None and stream is None:
        done = _native.w8_linear(X, w, b)
        if done is not None:
            return done
    M, K, stride = _rows(X, "X")
    kind, dev = _type(X.dtype, "X"), X.get_device()
    b_ptr = _layer(w, b, dev)
    if K != w.K:
        raise ValueError(f"X has {K} columns, w {w.K} rows")
    Y = _result(Y, "Y", X.dtype, (M, w.N), stream, dev)
    keep, ws, n = _workspace(_bytes("tst_w8_linear_workspace_bytes", M, K), workspace, stream, dev)
    _call("tst_w8_linear", X.data_ptr(), kind, stride, w.packed.data_ptr(), w.scale.data_ptr(), b_ptr, Y.data_ptr(), M, K, w.N, ws, n,
          _launch_stream(stream, dev))
    _shared(stream, (X, w.packed, w.scale, b, Y, keep), (Y,))
    return Y


class _MoeStruct(ctypes.Structure):
    """tst_moe_t of include/tst_ops.h."""
    _fields_ = [("struct_size", _sz), ("type", _ci), ("experts", _ci), ("width", _ci), ("inner", _ci), ("router", _vp), ("gate", _vp),
                ("up", _vp), ("down", _vp), ("gate_scale", _vp), ("up_scale", _vp), ("down_scale", _vp)]


class Moe:
    """The weights of a mixture-of-experts layer in their device form (tst_moe_pack)."""

    def __init__(self, E, D, F, dtype, device_index, tensors, struct):
        self.E, self.D, self.F, self.dtype, self.device_index = E, D, F, dtype, device_index
        self._tensors, self._struct = tensors, struct   # the struct holds the tensors' addresses
        self._ref = ctypes.byref(struct)
        self._raw = ctypes.addressof(struct)   # for the native half


def tst_moe_pack(router, gate, gate_scale, up, up_scale, down, down_scale, stream=None) -> Moe:
    """router [E, D] float32, bfloat16 or float16 (the type of the tokens to come); gate, up int8 [E, D, F] with scales float32
    [E, F]; down int8 [E, F, D] with scales float32 [E, D]."""
    import torch
    n, D, stride = _rows(router, "router")
    kind = _type(router.dtype, "router")
    if n > 1 and stride != D:
        raise ValueError("router must be contiguous")
    dev = router.get_device()
    E, packed, F = n, [], None
    for what, W, S in (("gate", gate, gate_scale), ("up", up, up_scale), ("down", down, down_scale)):
        if not isinstance(W, torch.Tensor) or W.dim() != 3 or W.shape[0] != E or (F is not None and W.shape[1:] != ((F, D) if what == "down" else (D, F))):
            raise ValueError("gate and up must be [E, D, F], down [E, F, D]")
        _, rows, cols, p, on = _pack(W, what, stream)
        if what == "gate":
            F = cols
            if rows != D:
                raise ValueError("gate and up must be [E, D, F], down [E, F, D]")
        if on != dev:
            raise ValueError(f"{what} must be on the router's device")
        _dense(S, what + "_scale", torch.float32, (E, cols), dev)
        packed.append(p)
    s = _MoeStruct(ctypes.sizeof(_MoeStruct), kind, E, D, F, router.data_ptr(), *(p.data_ptr() for p in packed), gate_scale.data_ptr(),
                   up_scale.data_ptr(), down_scale.data_ptr())
    _bytes("tst_moe_workspace_bytes", ctypes.byref(s), 1, 1)   # refuses sizes that no call takes
    return Moe(E, D, F, router.dtype, dev, (router, *packed, gate_scale, up_scale, down_scale), s)


def tst_moe(X, moe: Moe, top_k: int, normalize=True, Y=None, ids=None, p=None, workspace=None, stream=None):
    """The layer for tokens X [T, D] of the router's type: (Y [T, D], ids int32 [T, top_k], p float32 [T, top_k]).  normalize: the
    chosen experts' weights add up to one, else they are those of the softmax over all experts."""
    if _native is not None and Y is None and ids is None and p is None and workspace is None and stream is None:
        done = _native.moe(X, moe, top_k, normalize)
        if done is not None:
            return done
    import torch
    if not isinstance(moe, Moe):
        raise ValueError("moe must be what tst_moe_pack gives")
    T, D, stride = _rows(X, "X", moe.dtype)
    dev = X.get_device()
    if D != moe.D or dev != moe.device_index:
        raise ValueError(f"X must be [T, {moe.D}] on the experts' device")
    top_k = int(top_k)
    size = _bytes("tst_moe_workspace_bytes", moe._ref, T, top_k)
    Y = _result(Y, "Y", moe.dtype, (T, D), stream, dev)
    ids = _result(ids, "ids", torch.int32, (T, top_k), stream, dev)
    p = _result(p, "p", torch.float32, (T, top_k), stream, dev)
    keep, ws, n = _workspace(size, workspace, stream, dev)
    _call("tst_moe", X.data_ptr(), stride, moe._ref, top_k, int(bool(normalize)), Y.data_ptr(), ids.data_ptr(), p.data_ptr(), T, ws, n,
          _launch_stream(stream, dev))
    _shared(stream, (X, *moe._tensors, Y, ids, p, keep), (Y, ids, p))
    return Y, ids, p


def tst_logprobs(logits, tokens=None, top=0, workspace=None, stream=None):
    """Log probabilities in rows of logits [R, V] float32, bfloat16 or float16: (of_token, entropy [R], top_ids int32 [R, top],
    of_top [R, top]).  tokens: int32 or int64 [R] or [R, C]; of_token has their shape, [R, 0] without any."""
    if _native is not None and workspace is None and stream is None:
        done = _native.logprobs(logits, tokens, top)
        if done is not None:
            return done
    import torch
    R, V, stride = _rows(logits, "logits")
    kind, dev = _type(logits.dtype, "logits"), logits.get_device()
    if tokens is None:
        shape, t_ptr, t_bytes = (R, 0), None, 8
    else:
        if not isinstance(tokens, torch.Tensor) or tokens.dtype not in (torch.int32, torch.int64) or tokens.dim() not in (1, 2) or tokens.shape[0] != R:
            raise ValueError("tokens must be int32 or int64, [R] or [R, C]")
        shape = tuple(tokens.shape)
        t_ptr, t_bytes = _dense(tokens, "tokens", tokens.dtype, shape, dev), tokens.element_size()
    C, top = (shape[1] if len(shape) == 2 else 1), int(top)
    size = _bytes("tst_logprobs_workspace_bytes", R, V, top)
    f32 = torch.float32
    of_token = _result(None, "", f32, shape, stream, dev)
    entropy = _result(None, "", f32, (R,), stream, dev)
    ids = _result(None, "", torch.int32, (R, top), stream, dev)
    of_top = _result(None, "", f32, (R, top), stream, dev)
    keep, ws, n = _workspace(size, workspace, stream, dev)
    _call("tst_logprobs", logits.data_ptr(), kind, stride, t_ptr, t_bytes, C, top, of_token.data_ptr(), entropy.data_ptr(),
          ids.data_ptr(), of_top.data_ptr(), R, V, ws, n, _launch_stream(stream, dev))
    _shared(stream, (logits, tokens, keep), (of_token, entropy, ids, of_top))
    return of_token, entropy, ids, of_top
