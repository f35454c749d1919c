"""ctypes binding of libsubspec.so: one Python function per C entry point, with the
same name and argument order.  Tensors are passed as their data pointers; a
``stream`` of None means torch's current stream on the current device."""
from __future__ import annotations

import ctypes
import os
import struct
from itertools import compress, repeat
from operator import ge, is_not

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libsubspec.so"

SUBSPEC_PATH_AUTO = 0
SUBSPEC_PATH_GEMV = 1
SUBSPEC_PATH_MFMA = 2
SUBSPEC_PATH_MFMA16 = 3
SUBSPEC_PATH_MFMA32 = 4
SUBSPEC_NOALLOC_SCRATCH_BYTES = 32 << 20  # the fixed per-device scratch of subspec_qlinear_noalloc

_STATUS = {0: "OK", -1: "EINVAL", -2: "EUNSUPPORTED", -3: "EHIP", -4: "ECAPTURE"}


class SubspecError(RuntimeError):
    def __init__(self, fn: str, status: int, message: str):
        super().__init__(f"{fn} failed with {_STATUS.get(status, status)}: {message}")
        self.status = status
        self.message = message


class _Plan(ctypes.Structure):
    _fields_ = [("path", ctypes.c_int), ("mfma_rows", ctypes.c_int), ("rows", ctypes.c_int),
                ("tiles_per_wave", ctypes.c_int),
                ("waves", ctypes.c_int),
                ("chunk_blocks", ctypes.c_int), ("ring_chunks", ctypes.c_int), ("col_groups", ctypes.c_int),
                ("full_groups", ctypes.c_int),
                ("splits", ctypes.c_int), ("blocks_per_split", ctypes.c_int),
                ("grid", ctypes.c_int), ("workspace_bytes", ctypes.c_size_t),
                ("teams", ctypes.c_int), ("row_blocks", ctypes.c_int)]


class SubspecProj(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("qweight", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("zeros", ctypes.c_void_p), ("y", ctypes.c_void_p), ("N", ctypes.c_int),
                ("K", ctypes.c_int)]


_lib = None


def library_path() -> str:
    return os.path.join(_HERE, _LIB_NAME)


def load_library():
    """Load libsubspec.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(or python -m paper_2509_18344_amd.build)")
    lib = ctypes.CDLL(path)
    P, I, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    sig = {
        "subspec_qpack_bytes": (S, [I, I, I]),
        "subspec_quantize": (I, [P, I, I, I, I, P, P, P, P]),
        "subspec_qpack": (I, [P, I, I, I, P, P]),
        "subspec_quantize_hqq": (I, [P, I, I, I, I, P, P, P, P]),
        "subspec_qpack_host": (I, [P, I, I, I, P]),
        "subspec_qlinear": (I, [P, P, P, P, I, I, I, I, I, P, P]),
        "subspec_qlinear_path": (I, [P, P, P, P, I, I, I, I, I, P, I, P]),
        "subspec_qlinear_noalloc": (I, [P, P, P, P, I, I, I, I, I, P, P]),
        "subspec_qlinear_plan": (I, [I, I, I, I, I, I, ctypes.POINTER(_Plan)]),
        "subspec_qdequant": (I, [P, P, P, I, I, I, I, P, P, P]),
        "subspec_reserve": (I, [S]),
        "subspec_workspace_info": (I, [ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_int),
                                       ctypes.POINTER(ctypes.c_ulonglong)]),
        "subspec_stack_forward": (I, [P, I, I, I, I, P]),
        "subspec_stack_capture": (I, [P, I, I, I, I, P,
                                      ctypes.POINTER(ctypes.c_void_p)]),
        "subspec_graph_launch": (I, [P, P]),
        "subspec_graph_destroy": (I, [P]),
        "subspec_tree_expand": (I, [P, P, I, I, ctypes.c_float, I, P, P, P, P]),
        "subspec_tree_workspace_bytes": (S, [I, I, I]),
        "subspec_tree_plan": (I, [I, I, I, P, P, P]),
        "subspec_tree_attention": (I, [P, P, P, P, P, P, I, I, I, I, I, I, ctypes.c_float, P, P]),
        "subspec_tree_attention_workspace_bytes": (S, [I, I, I, I, I]),
        "subspec_tree_attention_plan": (I, [I, I, I, I, I, P, P]),
        "subspec_qkv_rope": (I, [P, I, P, P, P, ctypes.c_float, P, P, I, I, I, I, I, P, P, P, P]),
        "subspec_kv4_bytes": (S, [I, I, I]),
        "subspec_kv4_append": (I, [P, P, I, P, P, I, I, I, I, I, P, P, P]),
        "subspec_kv4_read": (I, [P, P, I, I, I, I, I, P, P, P]),
        "subspec_tree_attention_kv4": (I, [P, P, P, P, I, I, I, I, I, I, I, ctypes.c_float, P, P]),
        "subspec_tree_attention_kv4_workspace_bytes": (S, [I, I, I, I, I]),
        "subspec_tree_attention_kv4_plan": (I, [I, I, I, I, I, P, P]),
        "subspec_tree_verify": (I, [P, P, P, P, I, I, ctypes.c_float, P, P, P, P]),
        "subspec_tree_verify_workspace_bytes": (S, [I, I]),
        "subspec_prefetch_create": (I, [S, I, ctypes.POINTER(ctypes.c_void_p)]),
        "subspec_prefetch_destroy": (I, [P]),
        "subspec_prefetch_begin": (I, [P, P, S, ctypes.POINTER(ctypes.c_longlong)]),
        "subspec_prefetch_acquire": (I, [P, ctypes.c_longlong, P, ctypes.POINTER(ctypes.c_void_p)]),
        "subspec_prefetch_release": (I, [P, ctypes.c_longlong, P]),
        "subspec_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _ptr(t):
    """Data pointer of a torch tensor / numpy array, or an int address, or None."""
    try:  # a tensor, the usual argument
        return t.data_ptr()
    except AttributeError:
        pass
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if hasattr(t, "ctypes"):
        return t.ctypes.data
    raise TypeError(f"cannot take the address of {type(t)}")


_torch = _raw_stream = _device = None


def _stream(s):
    if s is None:
        global _torch, _raw_stream, _device
        if _torch is None:
            import torch as _torch
            # private to torch: where a version lacks them, the public Stream object below
            _raw_stream = getattr(_torch._C, "_cuda_getCurrentRawStream", None)
            _device = getattr(_torch._C, "_cuda_getDevice", None)
        # The current stream's handle without a Stream object around it: a projection of
        # a few microseconds is bound by this marshalling (7.9 us per eager call of a
        # 512 x 256 projection with the object and a ctypes structure per field).
        if _raw_stream is not None and _device is not None and _torch.cuda.is_initialized():
            return _raw_stream(_device())
        return _torch.cuda.current_stream().cuda_stream
    if isinstance(s, int):
        return s
    return s.cuda_stream


_get_device = _is_contiguous = _data_ptr = _dtype = _numel = None

# What a tensor may hold, by what the kernel takes its elements for: numbers of that type, or integers
# of its size with their bits.
_TYPES = {"bf16": ("bfloat16", "int16", "uint16"), "i32": ("int32", "uint32"), "f32": ("float32",),
          "f64": ("float64",), "u8": ("uint8", "int8")}
_NONE = repeat(None)
_usual = {}  # a call's kinds -> the first torch type of each


def _device_args(fn: str, stream, kinds, needs, *args):
    """One call's stream handle and its tensors' data pointers.  Each tensor has to be contiguous, on
    the device the call runs on, of its kind (a name of _TYPES) and of at least as many elements as
    `needs` says: the C entry points see none of this, and a kernel that is handed anything else
    reads or writes past it (an address is taken as it is, None stays None).  torch's methods mapped
    over the tensors: a method call each is most of the binding's time at a few microseconds a kernel."""
    global _get_device, _is_contiguous, _data_ptr, _dtype, _numel
    if stream is None and _get_device is not None:
        there = [*map(is_not, args, _NONE)]
        given, types, least = args, _usual.get(kinds) or _usual_types(kinds), needs
        if not all(there):
            given, types, least = [*compress(args, there)], [*compress(types, there)], compress(needs, there)
        try:
            on = {*map(_get_device, given)}
            dev = on.pop() if on else -1
            if (not on and dev >= 0 and dev == _device() and all(map(_is_contiguous, given)) and
                    [*map(_dtype, given)] == types and all(map(ge, map(_numel, given), least))):
                ptr = map(_data_ptr, given)
                if given is args:
                    return [_raw_stream(dev), *ptr]
                return [_raw_stream(dev), *[next(ptr) if t else None for t in there]]
        except TypeError:  # addresses among them
            pass
    dev, out = _current_device(stream), []
    for t, kind, need in zip(args, kinds, needs):
        if t is None or isinstance(t, int):
            out.append(t)
            continue
        try:
            on, whole = t.get_device(), t.is_contiguous()
        except AttributeError:
            raise TypeError(f"{fn}: a device tensor or an address, not {type(t)}") from None
        if on != dev or not whole:
            raise SubspecError(fn, -1, f"a {'' if whole else 'not contiguous '}tensor on device {on}: needs a contiguous "
                               "one on the current device, and a stream of that device")
        if str(t.dtype).rpartition(".")[2] not in _TYPES[kind]:
            raise SubspecError(fn, -1, f"a tensor of {t.dtype}: needs one of {' or '.join(_TYPES[kind])}")
        if t.numel() < need:
            raise SubspecError(fn, -1, f"a tensor of {t.numel()} elements: needs {need}")
        out.append(t.data_ptr())
    handle = _stream(stream)
    if _get_device is None and _raw_stream is not None and _device is not None:
        base = getattr(_torch._C, "TensorBase", _torch.Tensor)
        _get_device, _is_contiguous, _data_ptr = base.get_device, base.is_contiguous, base.data_ptr
        _dtype, _numel = base.dtype.__get__, base.numel
    return [handle, *out]


def _usual_types(kinds):
    _usual[kinds] = [getattr(_torch, _TYPES[k][0]) for k in kinds]
    return _usual[kinds]


def _current_device(stream) -> int:
    """The device the call runs on; -2 where no tensor can be on it (no device in use yet, or
    a stream of another device)."""
    if stream is None and _device is not None and _torch.cuda.is_initialized():
        return _device()
    import torch
    if not torch.cuda.is_initialized():
        return -2
    dev = torch.cuda.current_device()
    return dev if getattr(stream, "device_index", dev) == dev else -2


def _check(fn: str, status: int) -> int:
    if status != 0:
        raise SubspecError(fn, status, subspec_last_error())
    return status


def subspec_last_error() -> str:
    return load_library().subspec_last_error().decode()


def subspec_qpack_bytes(bits: int, N: int, K: int) -> int:
    return int(load_library().subspec_qpack_bytes(bits, N, K))


def subspec_quantize(w, bits, group, N, K, codes, scales, zeros, stream=None) -> int:
    return _check("subspec_quantize", load_library().subspec_quantize(
        _ptr(w), bits, group, N, K, _ptr(codes), _ptr(scales), _ptr(zeros), _stream(stream)))


def subspec_quantize_hqq(w, bits, group, N, K, codes, scales, zeros, stream=None) -> int:
    return _check("subspec_quantize_hqq", load_library().subspec_quantize_hqq(
        _ptr(w), bits, group, N, K, _ptr(codes), _ptr(scales), _ptr(zeros), _stream(stream)))


def subspec_qpack(codes, bits, N, K, qweight, stream=None) -> int:
    return _check("subspec_qpack", load_library().subspec_qpack(
        _ptr(codes), bits, N, K, _ptr(qweight), _stream(stream)))


def subspec_qpack_host(codes, bits, N, K, qweight) -> int:
    return _check("subspec_qpack_host", load_library().subspec_qpack_host(
        _ptr(codes), bits, N, K, _ptr(qweight)))


def subspec_qlinear(x, qweight, scales, zeros, bits, group, M, N, K, y, stream=None) -> int:
    return _check("subspec_qlinear", load_library().subspec_qlinear(
        _ptr(x), _ptr(qweight), _ptr(scales), _ptr(zeros), bits, group, M, N, K, _ptr(y),
        _stream(stream)))


def subspec_qlinear_noalloc(x, qweight, scales, zeros, bits, group, M, N, K, y, stream=None) -> int:
    return _check("subspec_qlinear_noalloc", load_library().subspec_qlinear_noalloc(
        _ptr(x), _ptr(qweight), _ptr(scales), _ptr(zeros), bits, group, M, N, K, _ptr(y), _stream(stream)))


def subspec_qlinear_path(x, qweight, scales, zeros, bits, group, M, N, K, y, path,
                         stream=None) -> int:
    return _check("subspec_qlinear_path", load_library().subspec_qlinear_path(
        _ptr(x), _ptr(qweight), _ptr(scales), _ptr(zeros), bits, group, M, N, K, _ptr(y), path,
        _stream(stream)))


def subspec_qlinear_plan(M, N, K, bits, group, path=SUBSPEC_PATH_AUTO) -> dict:
    p = _Plan()
    _check("subspec_qlinear_plan", load_library().subspec_qlinear_plan(
        M, N, K, bits, group, path, ctypes.byref(p)))
    return {name: getattr(p, name) for name, _ in _Plan._fields_}


def subspec_qdequant(qweight, scales, zeros, bits, group, N, K, w_f32, w_bf16,
                     stream=None) -> int:
    return _check("subspec_qdequant", load_library().subspec_qdequant(
        _ptr(qweight), _ptr(scales), _ptr(zeros), bits, group, N, K, _ptr(w_f32), _ptr(w_bf16),
        _stream(stream)))


def subspec_reserve(nbytes: int) -> int:
    return _check("subspec_reserve", load_library().subspec_reserve(nbytes))


def subspec_workspace_info() -> dict:
    """The calling device's workspace: bytes, retired buffers held, allocations so far."""
    b, r, a = ctypes.c_size_t(), ctypes.c_int(), ctypes.c_ulonglong()
    _check("subspec_workspace_info", load_library().subspec_workspace_info(
        ctypes.byref(b), ctypes.byref(r), ctypes.byref(a)))
    return {"bytes": int(b.value), "retired": int(r.value), "allocations": int(a.value)}


_PROJ_PACK = struct.Struct("@5P2i").pack  # the layout of SubspecProj


def _projs(projs):
    """The bytes of an array of subspec_proj from dicts with keys x, qweight, scales, zeros,
    y, N, K (tensors or addresses)."""
    try:  # the structures' bytes in one go
        return b"".join([_PROJ_PACK(
            _ptr(p["x"]) or 0, _ptr(p["qweight"]) or 0, _ptr(p["scales"]) or 0, _ptr(p["zeros"]) or 0,
            _ptr(p["y"]) or 0, int(p["N"]), int(p["K"])) for p in projs])
    except (struct.error, OverflowError):  # a value outside its C type: ctypes' own conversion
        pass
    arr = (SubspecProj * len(projs))()
    for i, p in enumerate(projs):
        arr[i] = SubspecProj(_ptr(p["x"]), _ptr(p["qweight"]), _ptr(p["scales"]), _ptr(p["zeros"]),
                             _ptr(p["y"]), int(p["N"]), int(p["K"]))
    return arr


def subspec_stack_forward(projs, bits, group, M, stream=None) -> int:
    arr = _projs(projs)
    return _check("subspec_stack_forward", load_library().subspec_stack_forward(
        arr, len(projs), bits, group, M, _stream(stream)))


def subspec_stack_capture(projs, bits, group, M, stream) -> int:
    """Returns the graph handle (an address) of the captured sequence."""
    arr = _projs(projs)
    h = ctypes.c_void_p()
    _check("subspec_stack_capture", load_library().subspec_stack_capture(
        arr, len(projs), bits, group, M, _stream(stream), ctypes.byref(h)))
    return h.value


def subspec_graph_launch(graph, stream=None) -> int:
    return _check("subspec_graph_launch", load_library().subspec_graph_launch(graph, _stream(stream)))


def subspec_graph_destroy(graph) -> int:
    return _check("subspec_graph_destroy", load_library().subspec_graph_destroy(graph))


def subspec_tree_expand(logits, parent_logp, R, V, temperature, k, parent_out, token_out,
                        score_out, stream=None) -> int:
    return _check("subspec_tree_expand", load_library().subspec_tree_expand(
        _ptr(logits), _ptr(parent_logp), R, V, float(temperature), k, _ptr(parent_out),
        _ptr(token_out), _ptr(score_out), _stream(stream)))


def subspec_tree_workspace_bytes(R, V, k) -> int:
    return int(load_library().subspec_tree_workspace_bytes(R, V, k))


def subspec_tree_attention(q, k_cache, v_cache, k_new, v_new, mask, M, Hq, Hkv, S, P, T, scale, out,
                           stream=None):
    return _check("subspec_tree_attention", load_library().subspec_tree_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_new), _ptr(v_new), _ptr(mask), M, Hq, Hkv, S, P, T,
        scale, _ptr(out), _stream(stream)))


def subspec_tree_attention_workspace_bytes(M, Hq, Hkv, P, T) -> int:
    return int(load_library().subspec_tree_attention_workspace_bytes(M, Hq, Hkv, P, T))


def subspec_tree_attention_plan(M, Hq, Hkv, P, T):
    """(splits, tiles_per_split) of the tree-attention launch."""
    s, t = ctypes.c_int(), ctypes.c_int()
    _check("subspec_tree_attention_plan", load_library().subspec_tree_attention_plan(
        M, Hq, Hkv, P, T, ctypes.byref(s), ctypes.byref(t)))
    return s.value, t.value


def subspec_qkv_rope(qkv, ld, bias, q_weight, k_weight, eps, positions, inv_freq, rot, interleaved, M, Hq, Hkv,
                     q, k_new, v_new, stream=None) -> int:
    heads = Hq + 2 * Hkv
    if not rot:  # not read
        positions = inv_freq = None
    st, x, b, qw, kw, pos, freq, qo, ko, vo = _device_args(
        "subspec_qkv_rope", stream, ("bf16", "bf16", "bf16", "bf16", "i32", "f64", "bf16", "bf16", "bf16"),
        ((M - 1) * ld + heads * 128, heads * 128, 128, 128, M, rot // 2, M * Hq * 128, M * Hkv * 128, M * Hkv * 128),
        qkv, bias, q_weight, k_weight, positions, inv_freq, q, k_new, v_new)
    return _check("subspec_qkv_rope", load_library().subspec_qkv_rope(
        x, ld, b, qw, kw, eps, pos, freq, rot, int(interleaved), M, Hq, Hkv, qo, ko, vo, st))


def subspec_kv4_bytes(Hkv: int, S: int, group: int) -> int:
    return int(load_library().subspec_kv4_bytes(Hkv, S, group))


def _kv4_size(Hkv, S, group):
    """subspec_kv4_bytes without the call; of an invalid shape, which the library refuses, anything."""
    return Hkv * (S // 32) * (2304 if group == 64 else 2176)


def subspec_kv4_append(k, v, src_rows, rows, count, n, Hkv, S, pos, group, k_cache, v_cache, stream=None) -> int:
    src, cache = src_rows * Hkv * 128, _kv4_size(Hkv, S, group)
    st, pk, pv, pr, pc, ck, cv = _device_args(
        "subspec_kv4_append", stream, ("bf16", "bf16", "i32", "i32", "u8", "u8"), (src, src, n, 1, cache, cache),
        k, v, rows, count, k_cache, v_cache)
    return _check("subspec_kv4_append", load_library().subspec_kv4_append(
        pk, pv, src_rows, pr, pc, n, Hkv, S, pos, group, ck, cv, st))


def subspec_kv4_read(k_cache, v_cache, Hkv, S, pos, n, group, k, v, stream=None) -> int:
    out, cache = n * Hkv * 128, _kv4_size(Hkv, S, group)
    st, ck, cv, pk, pv = _device_args("subspec_kv4_read", stream, ("u8", "u8", "bf16", "bf16"), (cache, cache, out, out),
                                      k_cache, v_cache, k, v)
    return _check("subspec_kv4_read", load_library().subspec_kv4_read(
        ck, cv, Hkv, S, pos, n, group, pk, pv, st))


def subspec_tree_attention_kv4(q, k_cache, v_cache, mask, M, Hq, Hkv, S, P, T, group, scale, out, stream=None) -> int:
    rows, cache = M * Hq * 128, _kv4_size(Hkv, S, group)
    st, pq, ck, cv, pm, po = _device_args(
        "subspec_tree_attention_kv4", stream, ("bf16", "u8", "u8", "i32", "bf16"),
        (rows, cache, cache, M * ((T + M + 31) // 32), rows), q, k_cache, v_cache, mask, out)
    return _check("subspec_tree_attention_kv4", load_library().subspec_tree_attention_kv4(
        pq, ck, cv, pm, M, Hq, Hkv, S, P, T, group, scale, po, st))


def subspec_tree_attention_kv4_workspace_bytes(M, Hq, Hkv, P, T) -> int:
    return int(load_library().subspec_tree_attention_kv4_workspace_bytes(M, Hq, Hkv, P, T))


def subspec_tree_attention_kv4_plan(M, Hq, Hkv, P, T):
    """(splits, tiles_per_split) of the launch."""
    s, t = ctypes.c_int(), ctypes.c_int()
    _check("subspec_tree_attention_kv4_plan", load_library().subspec_tree_attention_kv4_plan(
        M, Hq, Hkv, P, T, ctypes.byref(s), ctypes.byref(t)))
    return s.value, t.value


def subspec_tree_verify(logits, parent, token, uniform, N, V, temperature, path, accepted, next_token, stream=None) -> int:
    if not temperature:  # not read
        uniform = None
    st, pl, pp, pt, pu, po, pa, pn = _device_args(
        "subspec_tree_verify", stream, ("bf16", "i32", "i32", "f32", "i32", "i32", "i32"),
        ((N + 1) * V, N, N, N + 1, N, 1, 1), logits, parent, token, uniform, path, accepted, next_token)
    return _check("subspec_tree_verify", load_library().subspec_tree_verify(
        pl, pp, pt, pu, N, V, temperature, po, pa, pn, st))


def subspec_tree_verify_workspace_bytes(N, V) -> int:
    return int(load_library().subspec_tree_verify_workspace_bytes(N, V))


class Prefetcher:
    """The library's cross-layer weight prefetcher (a ring of `slots` device buffers of
    `slot_bytes`, one copy stream): begin(host) -> ticket, acquire(ticket, stream) ->
    device address, release(ticket, stream).  Host sources must be pinned."""

    def __init__(self, slot_bytes: int, slots: int):
        h = ctypes.c_void_p()
        _check("subspec_prefetch_create", load_library().subspec_prefetch_create(slot_bytes, slots, ctypes.byref(h)))
        self._h = h.value

    def begin(self, host, nbytes=None) -> int:
        if nbytes is None:
            nbytes = host.numel() * host.element_size()
        t = ctypes.c_longlong()
        _check("subspec_prefetch_begin", load_library().subspec_prefetch_begin(self._h, _ptr(host), nbytes,
                                                                               ctypes.byref(t)))
        return t.value

    def acquire(self, ticket: int, stream=None) -> int:
        p = ctypes.c_void_p()
        _check("subspec_prefetch_acquire", load_library().subspec_prefetch_acquire(self._h, ticket, _stream(stream),
                                                                                   ctypes.byref(p)))
        return p.value

    def release(self, ticket: int, stream=None) -> None:
        _check("subspec_prefetch_release", load_library().subspec_prefetch_release(self._h, ticket, _stream(stream)))

    def close(self) -> None:
        if self._h:
            _check("subspec_prefetch_destroy", load_library().subspec_prefetch_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def subspec_tree_plan(R, V, k):
    """(chunks, chunk_len, list_len) of the expansion launch for (R, V, k)."""
    c, n, l = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check("subspec_tree_plan", load_library().subspec_tree_plan(
        R, V, k, ctypes.byref(c), ctypes.byref(n), ctypes.byref(l)))
    return c.value, n.value, l.value
