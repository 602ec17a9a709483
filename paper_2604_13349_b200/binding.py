"""Thin ctypes binding of the C ABI in ``include/obf.h``.

Argument marshalling only: every step of the compression runs in the CUDA
kernels of ``libobf_b200.so``.  PyTorch appears here for device memory and
streams, nothing else.  There is no CPU fallback: if the library has not been
built (``python -m paper_2604_13349_b200.build``) loading it raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from typing import Dict, List, Optional, Sequence

import torch

from . import build as _build

OBF_OK = 0
OBF_ERR_INVALID_ARG = 1
OBF_ERR_UNSUPPORTED = 2
OBF_ERR_WORKSPACE = 3
OBF_ERR_CUDA = 4
OBF_ERR_DEVICE_STATUS = 5

OBF_F32 = 0
OBF_BF16 = 1

OBF_DEV_NONFINITE = 0x1
OBF_DEV_NO_CONVERGE = 0x2
OBF_DEV_TIMEOUT = 0x4
OBF_DEV_INTERNAL = 0x8
OBF_DEV_SKIPPED = 0x100
OBF_DEV_SPAN_FULL = 0x200

OBF_FLAG_GENERIC_PATH = 0x1
OBF_FLAG_LAYERWISE = 0x2        # one retained set per layer (masses summed over its KV heads)
OBF_FLAG_FAST_PATH = 0x4        # three Gram subspace iterations instead of the exact eigenvectors
OBF_FLAG_ATTN_INJECT = 0x8      # the back-fill shared out by attention mass instead of uniformly (App. D.2)
OBF_FLAG_EARLY_OUT = 0x20       # span test first; the pass over V skips heads whose retained values span R^d
OBF_FLAG_MERGE = 0x10           # cache-merging baseline instead of Orthogonal BackFill (App. E)
OBF_FLAG_TEST_WAIT_EXPIRES = 0x10000   # test hook: waits of the score kernel, or of the tensor-core attention, run out


def OBF_FLAG_SINK(n: int) -> int:
    """Protected sink prefix: the first n <= 255 positions are retained besides the budget."""
    return (int(n) & 0xFF) << 8


def k_eff(T: int, budget: int, flags: int = 0) -> int:
    """Rows of K_out / V_out / idx per head for a cache of T positions."""
    s = min((flags >> 8) & 0xFF, T)
    return s + min(int(budget), T - s)
OBF_MAX_CACHES = 32

EXPORTS = ("obf_workspace_bytes", "obf_compress", "evict_only", "obf_host_arena_bytes",
           "obf_compress_host", "obf_last_device_status", "obf_status_string",
           "obf_last_launch_count", "obf_compress_profiled", "obf_phase_name",
           "evict_only_static", "obf_static_scratch_status",
           "obf_attend_workspace_bytes", "obf_attend", "obf_attend_shared", "obf_evict_by_mass")
OBF_STATIC_SCRATCH_BYTES = 8 << 20
OBF_MAX_PHASES = 16


class ObfParams(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("n_obs", ctypes.c_int32), ("rank", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("flags", ctypes.c_uint32)]


class ObfDiag(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in (
        "a_keep", "a_del", "alpha", "rcr", "delta_norm", "kth_score", "next_score",
        "lam_1", "lam_rho", "lam_next")] + [
        ("span_rank", ctypes.c_int32), ("rho_eff", ctypes.c_int32), ("status", ctypes.c_uint32),
        ("revr", ctypes.c_float), ("pc", ctypes.c_float)]


DIAG_BYTES = ctypes.sizeof(ObfDiag)
DIAG_FLOAT_FIELDS = [n for n, t in ObfDiag._fields_ if t is ctypes.c_float]


class ObfCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_obs", ctypes.c_void_p),
                ("T", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("k_out", ctypes.c_void_p), ("v_out", ctypes.c_void_p), ("idx_out", ctypes.c_void_p),
                ("diag_out", ctypes.c_void_p), ("scores_out", ctypes.c_void_p), ("delta_out", ctypes.c_void_p),
                ("lse_extra", ctypes.c_void_p), ("k_q8_out", ctypes.c_void_p), ("v_q8_out", ctypes.c_void_p),
                ("k_scale_out", ctypes.c_void_p), ("v_scale_out", ctypes.c_void_p), ("assign_out", ctypes.c_void_p)]


class ObfAttend(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "kv_heads", "q_heads", "head_dim", "n_q", "capacity", "window", "sinks", "dtype")] + [
        ("scale", ctypes.c_float), ("decay", ctypes.c_float), ("flags", ctypes.c_uint32)] + [
        (n, ctypes.c_void_p) for n in ("q", "k", "v", "out")] + [
        (n, ctypes.c_int64 * 3) for n in ("q_stride", "k_stride", "v_stride", "out_stride")] + [
        (n, ctypes.c_void_p) for n in ("lens", "q_lens", "lse_out", "mass_in", "mass_out")]


class ObfPrefix(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 2), ("v_stride", ctypes.c_int64 * 2),
                ("rows", ctypes.c_int32)]


class ObfEvict(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "kv_heads", "head_dim", "capacity", "dtype", "keep", "sinks", "recent")] + [
        (n, ctypes.c_void_p) for n in ("k", "v", "k_out", "v_out")] + [
        (n, ctypes.c_int64 * 3) for n in ("k_stride", "v_stride", "k_out_stride", "v_out_stride")] + [
        (n, ctypes.c_void_p) for n in ("mass", "lens", "idx_out", "mass_out")] + [("mass_out_rows", ctypes.c_int32), ("lens_out", ctypes.c_void_p)]


class ObfError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (status %d)" % (where, obf_status_string(code), code))


_lib = None


def library_path() -> str:
    return _build.LIB_PATH


def load() -> ctypes.CDLL:
    """Loads ``libobf_b200.so``; raises if it has not been built."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(
                "CUDA extension %s is missing; build it with `python -m paper_2604_13349_b200.build` "
                "(there is no CPU fallback)" % path)
        lib = ctypes.CDLL(path)
        pp, pc = ctypes.POINTER(ObfParams), ctypes.POINTER(ObfCache)
        lib.obf_workspace_bytes.argtypes = [pp, pc, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
        lib.obf_workspace_bytes.restype = ctypes.c_int
        lib.obf_host_arena_bytes.argtypes = [pp, pc, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
        lib.obf_host_arena_bytes.restype = ctypes.c_int
        for name in ("obf_compress", "evict_only", "obf_compress_host"):
            fn = getattr(lib, name)
            fn.argtypes = [pp, pc, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
            fn.restype = ctypes.c_int
        lib.obf_last_device_status.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_uint32)]
        lib.obf_last_device_status.restype = ctypes.c_int
        lib.obf_status_string.argtypes = [ctypes.c_int]
        lib.obf_status_string.restype = ctypes.c_char_p
        lib.obf_compress_profiled.argtypes = [pp, pc, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t,
                                              ctypes.c_void_p, ctypes.POINTER(ctypes.c_float),
                                              ctypes.POINTER(ctypes.c_int32)]
        lib.obf_compress_profiled.restype = ctypes.c_int
        lib.obf_phase_name.argtypes = [ctypes.c_int32]
        lib.obf_phase_name.restype = ctypes.c_char_p
        lib.evict_only_static.argtypes = [pp, pc, ctypes.c_int32, ctypes.c_void_p]
        lib.evict_only_static.restype = ctypes.c_int
        lib.obf_static_scratch_status.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_uint32)]
        lib.obf_static_scratch_status.restype = ctypes.c_int
        pa, px = ctypes.POINTER(ObfAttend), ctypes.POINTER(ObfPrefix)
        lib.obf_attend_workspace_bytes.argtypes = [pa, px, ctypes.POINTER(ctypes.c_size_t)]
        lib.obf_attend.argtypes = [pa, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        lib.obf_attend_shared.argtypes = [pa, px, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        lib.obf_evict_by_mass.argtypes = [ctypes.POINTER(ObfEvict), ctypes.c_void_p]
        for name in ("obf_attend_workspace_bytes", "obf_attend", "obf_attend_shared", "obf_evict_by_mass"):
            getattr(lib, name).restype = ctypes.c_int
        lib.obf_last_launch_count.argtypes = []
        lib.obf_last_launch_count.restype = ctypes.c_int32
        _lib = lib
    return _lib


def obf_status_string(code: int) -> str:
    return load().obf_status_string(int(code)).decode()


def make_params(layers: int, kv_heads: int, q_heads: int, head_dim: int, n_obs: int, rank: int,
                dtype: int, eps: float = 1e-12, flags: int = 0) -> ObfParams:
    return ObfParams(layers, kv_heads, q_heads, head_dim, n_obs, rank, dtype, eps, flags)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def make_cache(k, v, q_obs, T: int, budget: int, k_out, v_out, idx_out, diag_out=None,
               scores_out=None, delta_out=None, lse_extra=None, q8=None, assign_out=None) -> ObfCache:
    """Tensors (device or, for the host entry point, pinned/pageable CPU) or raw addresses.
    q8: (k_q8_out, v_q8_out, k_scale_out, v_scale_out) for the int8 copy of the relay, or None."""
    q8 = q8 or (None, None, None, None)
    return ObfCache(_ptr(k), _ptr(v), _ptr(q_obs), int(T), int(budget), _ptr(k_out), _ptr(v_out),
                    _ptr(idx_out), _ptr(diag_out), _ptr(scores_out), _ptr(delta_out), _ptr(lse_extra),
                    _ptr(q8[0]), _ptr(q8[1]), _ptr(q8[2]), _ptr(q8[3]), _ptr(assign_out))


def _carray(caches: Sequence[ObfCache]):
    arr = (ObfCache * len(caches))(*caches)
    return arr


def _stream_handle(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def obf_workspace_bytes(params: ObfParams, caches: Sequence[ObfCache]) -> int:
    out = ctypes.c_size_t(0)
    rc = load().obf_workspace_bytes(ctypes.byref(params), _carray(caches), len(caches), ctypes.byref(out))
    if rc != OBF_OK:
        raise ObfError(rc, "obf_workspace_bytes")
    return int(out.value)


def obf_host_arena_bytes(params: ObfParams, caches: Sequence[ObfCache]) -> int:
    out = ctypes.c_size_t(0)
    rc = load().obf_host_arena_bytes(ctypes.byref(params), _carray(caches), len(caches), ctypes.byref(out))
    if rc != OBF_OK:
        raise ObfError(rc, "obf_host_arena_bytes")
    return int(out.value)


def _call(name: str, params, caches, buf, buf_bytes, stream, check=True) -> int:
    rc = getattr(load(), name)(ctypes.byref(params), _carray(caches), len(caches),
                               _ptr(buf), int(buf_bytes), _stream_handle(stream))
    if check and rc != OBF_OK:
        raise ObfError(rc, name)
    return rc


def obf_compress(params, caches, workspace, workspace_bytes=None, stream=None, check=True) -> int:
    nb = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    return _call("obf_compress", params, caches, workspace, nb, stream, check)


def evict_only(params, caches, workspace, workspace_bytes=None, stream=None, check=True) -> int:
    nb = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    return _call("evict_only", params, caches, workspace, nb, stream, check)


def evict_only_static(params, caches, stream=None, check=True) -> int:
    """evict_only on the library's built-in scratch array, for callers that cannot allocate a
    workspace (see include/obf.h).  Inputs and outputs are device tensors as for evict_only; the
    call shape must fit OBF_STATIC_SCRATCH_BYTES; calls that overlap on the GPU race on the array."""
    rc = load().evict_only_static(ctypes.byref(params), _carray(caches), len(caches), _stream_handle(stream))
    if check and rc != OBF_OK:
        raise ObfError(rc, "evict_only_static")
    return rc


def obf_static_scratch_status(stream=None) -> int:
    """Status word left by the last evict_only_static call on the current device."""
    out = ctypes.c_uint32(0)
    rc = load().obf_static_scratch_status(_stream_handle(stream), ctypes.byref(out))
    if rc not in (OBF_OK, OBF_ERR_DEVICE_STATUS):
        raise ObfError(rc, "obf_static_scratch_status")
    return int(out.value)


def obf_compress_host(params, caches, device_arena, arena_bytes=None, stream=None, check=True) -> int:
    nb = device_arena.numel() * device_arena.element_size() if arena_bytes is None else arena_bytes
    return _call("obf_compress_host", params, caches, device_arena, nb, stream, check)


def obf_compress_profiled(params, caches, workspace, workspace_bytes=None, stream=None):
    """Runs the call with an event after every launch; returns [(kernel name, milliseconds), ...]."""
    nb = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    ms = (ctypes.c_float * OBF_MAX_PHASES)()
    n = ctypes.c_int32(0)
    rc = load().obf_compress_profiled(ctypes.byref(params), _carray(caches), len(caches), _ptr(workspace),
                                      int(nb), _stream_handle(stream), ms, ctypes.byref(n))
    if rc != OBF_OK:
        raise ObfError(rc, "obf_compress_profiled")
    return [(load().obf_phase_name(i).decode(), float(ms[i])) for i in range(n.value)]


def obf_last_device_status(workspace, stream=None) -> int:
    out = ctypes.c_uint32(0)
    rc = load().obf_last_device_status(_ptr(workspace), _stream_handle(stream), ctypes.byref(out))
    if rc not in (OBF_OK, OBF_ERR_DEVICE_STATUS):
        raise ObfError(rc, "obf_last_device_status")
    return int(out.value)


def obf_last_launch_count() -> int:
    return int(load().obf_last_launch_count())


# ---------------------------------------------------------------------------
# convenience: allocate outputs with torch and call the C ABI once
# ---------------------------------------------------------------------------
def _torch_dtype(dtype: int):
    return torch.float32 if dtype == OBF_F32 else torch.bfloat16


def parse_diag(diag_bytes: torch.Tensor) -> List[Dict[str, float]]:
    """uint8 tensor [heads, sizeof(obf_diag_t)] (any device) -> list of dicts."""
    raw = diag_bytes.detach().cpu().contiguous().numpy().tobytes()
    n = len(raw) // DIAG_BYTES
    arr = (ObfDiag * n).from_buffer_copy(raw)
    return [{name: getattr(arr[i], name) for name, _ in ObfDiag._fields_} for i in range(n)]


def compress_caches(params: ObfParams, caches_in: Sequence[Dict[str, object]], *, evict: bool = False,
                    want_scores: bool = False, want_delta: bool = True, want_diag: bool = True,
                    want_int8: bool = False, want_assign: bool = False,
                    stream=None, workspace: Optional[torch.Tensor] = None) -> List[Dict[str, object]]:
    """Compress a batch of device caches.

    ``caches_in``: dicts with device tensors ``K, V [layers, kv_heads, T, d]``,
    ``Q [layers, q_heads, n_obs, d]``, an int ``budget`` and optionally ``lse_extra [layers, q_heads, n_obs]``
    (fp32, the out-of-prompt softmax mass per observation query).  Returns one dict per
    cache with ``K_out, V_out, idx`` (and ``scores``, ``delta``, ``diag`` bytes when asked).
    """
    dt = _torch_dtype(params.dtype)
    hpc = params.layers * params.kv_heads
    outs, cs = [], []
    for ci in caches_in:
        K, V, Q = ci["K"], ci["V"], ci["Q"]
        assert K.is_cuda and K.is_contiguous() and V.is_contiguous() and Q.is_contiguous()
        assert K.dtype == dt and V.dtype == dt and Q.dtype == dt
        T = K.shape[2]
        ke = k_eff(T, ci["budget"], params.flags)
        dev = K.device
        o = {
            "K_out": torch.empty((params.layers, params.kv_heads, ke, params.head_dim), dtype=dt, device=dev),
            "V_out": torch.empty((params.layers, params.kv_heads, ke, params.head_dim), dtype=dt, device=dev),
            "idx": torch.empty((params.layers, params.kv_heads, ke), dtype=torch.int32, device=dev),
            "diag": torch.zeros((hpc, DIAG_BYTES), dtype=torch.uint8, device=dev) if want_diag else None,
            "scores": torch.empty((params.layers, params.kv_heads, T), dtype=torch.float32, device=dev)
            if want_scores else None,
            "delta": torch.zeros((params.layers, params.kv_heads, params.head_dim), dtype=torch.float32,
                                 device=dev) if want_delta else None,
        }
        q8 = None
        if want_int8:
            o["K_q8"] = torch.empty((params.layers, params.kv_heads, ke, params.head_dim), dtype=torch.int8, device=dev)
            o["V_q8"] = torch.empty_like(o["K_q8"])
            o["K_scale"] = torch.empty((params.layers, params.kv_heads, ke), dtype=torch.float32, device=dev)
            o["V_scale"] = torch.empty_like(o["K_scale"])
            q8 = (o["K_q8"], o["V_q8"], o["K_scale"], o["V_scale"])
        o["assign"] = torch.empty((params.layers, params.kv_heads, T), dtype=torch.int32, device=dev) if want_assign else None
        outs.append(o)
        cs.append(make_cache(K, V, Q, T, ci["budget"], o["K_out"], o["V_out"], o["idx"], o["diag"],
                             o["scores"], o["delta"], ci.get("lse_extra"), q8, o["assign"]))
    nb = obf_workspace_bytes(params, cs)
    if workspace is None or workspace.numel() * workspace.element_size() < nb:
        workspace = torch.empty(nb, dtype=torch.uint8, device=caches_in[0]["K"].device)
    (evict_only if evict else obf_compress)(params, cs, workspace, stream=stream)
    for o in outs:
        o["workspace"] = workspace
        o["cache_structs"] = cs                 # for a repeated call on the same buffers (profiling)
    return outs


# ---------------------------------------------------------------------------
# operators on a relayed cache
# ---------------------------------------------------------------------------
_DTYPES = {torch.float32: OBF_F32, torch.bfloat16: OBF_BF16}
_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32

# A single token's attention takes some microseconds on the device, so these wrappers hand the structs over as packed bytes
# (building a ctypes structure field by field takes longer than the kernels).
_ATTEND = struct.Struct("@9i2fI4P12q5P")
_PREFIX = struct.Struct("@2P4qi4x")
_EVICT = struct.Struct("@8i4P12q4Pi4xP")
assert (_ATTEND.size, _PREFIX.size, _EVICT.size) == (ctypes.sizeof(ObfAttend), ctypes.sizeof(ObfPrefix), ctypes.sizeof(ObfEvict))
_packed_calls: Dict[str, object] = {}
_STATUS_ONLY = 256
_status_words: Dict[int, torch.Tensor] = {}
_MOST = 0x7FFFFFFF                      # windows and numbers of first tokens beyond any position are as good


def _packed(name: str):
    """An entry point taking its structs as bytes."""
    fn = _packed_calls.get(name)
    if fn is None:
        bytes_, ptr, size = ctypes.c_char_p, ctypes.c_void_p, ctypes.c_size_t
        args = {"obf_attend_workspace_bytes": (bytes_, bytes_, ptr), "obf_attend": (bytes_, ptr, size, ptr),
                "obf_attend_shared": (bytes_, bytes_, ptr, size, ptr), "obf_evict_by_mass": (bytes_, ptr)}[name]
        fn = _packed_calls[name] = ctypes.CFUNCTYPE(ctypes.c_int, *args)((name, load()))
    return fn


def _refuse(name: str, t, shape, dtype, device) -> None:
    raise ValueError("%s: %s %s on %s expected, got %s" % (
        name, dtype, tuple(shape), device, "%s %s on %s" % (t.dtype, tuple(t.shape), t.device) if isinstance(t, torch.Tensor) else type(t).__name__))


def _rows(t: torch.Tensor, shape, dtype, device: int, name: str):
    """Checks a tensor of rows of contiguous channels and gives its strides."""
    st = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or st[-1] != 1:
        _refuse(name + " (contiguous channels)", t, shape, dtype, device)
    return st


def _dense(t: Optional[torch.Tensor], shape, dtype, device: int, name: str) -> int:
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _refuse(name + " (contiguous)", t, shape, dtype, device)
    return t.data_ptr()


def _refuse_graph(name: str) -> None:
    raise ValueError("%s has no gradients: call it under torch.no_grad() or with detached tensors" % name)


def _attend_args(q, k, v, lens, q_lens, window, sinks, scale, out, lse_out, mass_in, mass_out, decay, flags) -> bytes:
    dt, dev = q.dtype, q.get_device()
    code = OBF_BF16 if dt is _BF16 else OBF_F32 if dt is _F32 else -1
    shape_q, shape_k = q.shape, k.shape
    if code < 0 or dev < 0 or len(shape_q) != 4 or len(shape_k) != 4:
        raise ValueError("q, k: float32 or bfloat16 device tensors [batch, heads, rows, head_dim] expected")
    B, hq, n_q, d = shape_q
    b, kv, cap, dk = shape_k
    sq, sk, sv, so = q.stride(), k.stride(), v.stride(), out.stride()
    if not (b == B and dk == d and v.shape == shape_k and out.shape == shape_q and k.dtype is dt and v.dtype is dt and out.dtype is dt and
            k.get_device() == dev and v.get_device() == dev and out.get_device() == dev and sq[3] == sk[3] == sv[3] == so[3] == 1):
        for t, shape, name in ((q, shape_q, "q"), (k, (B, kv, cap, d), "k"), (v, (B, kv, cap, d), "v"), (out, shape_q, "out")):
            _rows(t, shape, dt, dev, name)                       # names the one that is wrong
    return _ATTEND.pack(
        B, kv, hq, d, n_q, cap, min(window, _MOST), min(sinks, _MOST), code, scale, decay, flags, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
        sq[0], sq[1], sq[2], sk[0], sk[1], sk[2], sv[0], sv[1], sv[2], so[0], so[1], so[2],
        0 if lens is None else _dense(lens, (B,), _I32, dev, "lens"), 0 if q_lens is None else _dense(q_lens, (B,), _I32, dev, "q_lens"),
        0 if lse_out is None else _dense(lse_out, shape_q[:3], _F32, dev, "lse_out"),
        0 if mass_in is None else _dense(mass_in, shape_k[:3], _F32, dev, "mass_in"),
        0 if mass_out is None else _dense(mass_out, shape_k[:3], _F32, dev, "mass_out"))


def _enqueue(name: str, device: int, args, stream) -> None:
    """The call with the tensors' device current, on the given stream or the device's current one."""
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(device)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            rc = _packed(name)(*args, stream)
    else:
        rc = _packed(name)(*args, stream)
    if rc != OBF_OK:
        raise ObfError(rc, name)


def _attend_call(name, args, prefix, q, out, lse_out, mass_out, workspace, want_status, stream):
    if workspace is None:
        nb = ctypes.c_size_t(0)
        rc = _packed("obf_attend_workspace_bytes")(args, prefix, ctypes.addressof(nb))
        if rc != OBF_OK:
            raise ObfError(rc, name)
        size = nb.value
        if size <= _STATUS_ONLY and not want_status:                # a status word that nobody asks for: one per device does for all
            workspace = _status_words.get(q.get_device())
            if workspace is None:
                workspace = torch.zeros(_STATUS_ONLY, dtype=torch.uint8, device=q.device)
                if not torch.cuda.is_current_stream_capturing():          # (a graph's memory goes with the graph)
                    _status_words[q.get_device()] = workspace
        elif stream is None:
            workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
        else:
            with _allocating(stream, q.device):
                workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    else:
        if workspace.device != q.device or not workspace.is_contiguous():
            raise ValueError("workspace: contiguous memory on %s expected" % q.device)
        size = workspace.numel() * workspace.element_size()
    call = (args, workspace.data_ptr(), size) if prefix is None else (args, prefix, workspace.data_ptr(), size)
    _enqueue(name, q.get_device(), call, stream)
    got = {"out": out}
    if lse_out is not None:
        got["lse"] = lse_out
    if mass_out is not None:
        got["mass"] = mass_out
    if want_status:
        got["workspace"] = workspace
    return got


def _allocating(stream, device: torch.device):
    """Memory for a call on `stream` is allocated, and cleared, on that stream."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream)


def _attend_outputs(q, q_lens, out, lse_out, want_lse, stream):
    if out is None or (lse_out is None and want_lse):
        make = torch.empty if q_lens is None else torch.zeros    # what lies behind a sequence's queries is not written
        with _allocating(stream, q.device):
            if out is None:
                out = make(q.shape, dtype=q.dtype, device=q.device)
            if lse_out is None and want_lse:
                lse_out = make(q.shape[:3], dtype=torch.float32, device=q.device)
    return out, lse_out


def attend(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, lens: Optional[torch.Tensor] = None, q_lens: Optional[torch.Tensor] = None,
           window: int = 0, sinks: int = 0, scale: float = 0.0, out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
           want_lse: bool = False, mass_in: Optional[torch.Tensor] = None, mass_out: Optional[torch.Tensor] = None, decay: float = 1.0,
           flags: int = 0, workspace: Optional[torch.Tensor] = None, want_status: bool = False, stream=None) -> Dict[str, torch.Tensor]:
    """Causal attention of ``q [batch, q_heads, n_q, d]`` over caches ``k, v [batch, kv_heads, capacity, d]`` with an optional sliding
    window whose first ``sinks`` keys stay visible (``obf_attend`` in include/obf.h).

    ``lens``, ``q_lens``: int32 device tensors ``[batch]``, the rows of a sequence's cache and its queries that count (None: all);
    the queries are the last tokens of the cache.  Any strides with contiguous channels.  ``mass_out [batch, kv_heads, capacity]``
    (fp32) receives ``decay * mass_in`` plus the attention mass of every key; it may be ``mass_in``.  ``workspace``: one that
    ``attend_workspace`` made for these shapes; else one is allocated for the call.  Returns ``out`` and, where asked for,
    ``lse [batch, q_heads, n_q]`` (natural log), ``mass`` and, with ``want_status``, the call's ``workspace``:
    ``obf_last_device_status`` waits for the stream and reads there whether a length was out of range (``OBF_DEV_INTERNAL``) or a
    wait on the device ran out (``OBF_DEV_TIMEOUT``: the results are not to be used).  Without it nothing reports either.  There are
    no gradients: where autograd records, tensors that require one are refused.
    """
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or (mass_in is not None and mass_in.requires_grad)):
        _refuse_graph("attend")
    out, lse_out = _attend_outputs(q, q_lens, out, lse_out, want_lse, stream)
    args = _attend_args(q, k, v, lens, q_lens, window, sinks, scale, out, lse_out, mass_in, mass_out, decay, flags)
    return _attend_call("obf_attend", args, None, q, out, lse_out, mass_out, workspace, want_status, stream)


def attend_shared(q: torch.Tensor, k_prefix: torch.Tensor, v_prefix: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *,
                  lens: Optional[torch.Tensor] = None, q_lens: Optional[torch.Tensor] = None, scale: float = 0.0,
                  out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None, want_lse: bool = False, flags: int = 0,
                  workspace: Optional[torch.Tensor] = None, want_status: bool = False, stream=None) -> Dict[str, torch.Tensor]:
    """The same for a batch whose sequences all see ``k_prefix, v_prefix [kv_heads, rows, d]`` before their own keys
    (``obf_attend_shared``): the prefix is read once for all of them."""
    if torch.is_grad_enabled() and (q.requires_grad or k_prefix.requires_grad or v_prefix.requires_grad or k.requires_grad or v.requires_grad):
        _refuse_graph("attend_shared")
    out, lse_out = _attend_outputs(q, q_lens, out, lse_out, want_lse, stream)
    args = _attend_args(q, k, v, lens, q_lens, 0, 0, scale, out, lse_out, None, None, 1.0, flags)
    if k_prefix.dim() != 3:
        raise ValueError("k_prefix: [kv_heads, rows, head_dim] expected")
    rows = k_prefix.shape[1]
    shape = (k.shape[1], rows, q.shape[3])
    sk, sv = _rows(k_prefix, shape, q.dtype, q.get_device(), "k_prefix"), _rows(v_prefix, shape, q.dtype, q.get_device(), "v_prefix")
    prefix = _PREFIX.pack(k_prefix.data_ptr(), v_prefix.data_ptr(), sk[0], sk[1], sv[0], sv[1], rows)
    return _attend_call("obf_attend_shared", args, prefix, q, out, lse_out, None, workspace, want_status, stream)


def attend_workspace(q: torch.Tensor, k: torch.Tensor, *, window: int = 0, sinks: int = 0, mass: bool = False, prefix_rows: int = 0,
                     flags: int = 0) -> torch.Tensor:
    """A workspace for ``attend`` (``prefix_rows`` 0) or ``attend_shared`` calls of these shapes."""
    B, hq, n_q, d = q.shape
    kv, cap = k.shape[1], k.shape[2]
    args = _ATTEND.pack(B, kv, hq, d, n_q, cap, min(window, _MOST), min(sinks, _MOST), _DTYPES.get(q.dtype, -1), 0.0, 1.0, flags, *([0] * 16), 0, 0, 0, 0, 1 if mass else 0)
    prefix = _PREFIX.pack(0, 0, 0, 0, 0, 0, prefix_rows) if prefix_rows else None
    nb = ctypes.c_size_t(0)
    rc = _packed("obf_attend_workspace_bytes")(args, prefix, ctypes.addressof(nb))
    if rc != OBF_OK:
        raise ObfError(rc, "obf_attend_workspace_bytes")
    return torch.zeros(nb.value, dtype=torch.uint8, device=q.device)


def obf_attend_workspace_bytes(args: ObfAttend, prefix: Optional[ObfPrefix] = None) -> int:
    out = ctypes.c_size_t(0)
    rc = load().obf_attend_workspace_bytes(ctypes.byref(args), ctypes.byref(prefix) if prefix is not None else None, ctypes.byref(out))
    if rc != OBF_OK:
        raise ObfError(rc, "obf_attend_workspace_bytes")
    return int(out.value)


def evict_by_mass(k: torch.Tensor, v: torch.Tensor, mass: torch.Tensor, keep: int, *, lens: Optional[torch.Tensor] = None, sinks: int = 0,
                  recent: int = 0, k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None,
                  idx_out: Optional[torch.Tensor] = None, mass_out: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
                  stream=None) -> Dict[str, torch.Tensor]:
    """Brings caches ``k, v [batch, kv_heads, capacity, d]`` down to ``keep`` rows per head by their accumulated masses
    ``[batch, kv_heads, capacity]``: the first ``sinks``, the last ``recent`` and the heaviest others, in ascending order
    (``obf_evict_by_mass`` in include/obf.h).  ``k_out, v_out`` and ``mass_out`` may have more rows than ``keep``: the cache goes on
    there.  Returns ``K_out, V_out, idx, mass, lens``."""
    if torch.is_grad_enabled() and (k.requires_grad or v.requires_grad or mass.requires_grad):
        _refuse_graph("evict_by_mass")
    dt, dev, at = k.dtype, k.device, k.get_device()
    code = OBF_BF16 if dt is _BF16 else OBF_F32 if dt is _F32 else -1
    shape = k.shape
    if code < 0 or at < 0 or len(shape) != 4:
        raise ValueError("k: a float32 or bfloat16 device tensor [batch, kv_heads, capacity, head_dim] expected")
    B, kv, cap, d = shape
    if k_out is None or v_out is None or idx_out is None or mass_out is None or lens_out is None:
        make = torch.zeros if lens is not None or keep > cap else torch.empty    # rows behind a sequence's last one are not written
        with _allocating(stream, dev):
            if k_out is None:
                k_out = make((B, kv, keep, d), dtype=dt, device=dev)
            if v_out is None:
                v_out = make((B, kv, keep, d), dtype=dt, device=dev)
            if idx_out is None:
                idx_out = make((B, kv, keep), dtype=_I32, device=dev)
            if mass_out is None:
                mass_out = make((B, kv, keep), dtype=_F32, device=dev)
            if lens_out is None:
                lens_out = torch.empty((B,), dtype=_I32, device=dev)
    shape_ko, shape_vo, mo = k_out.shape, v_out.shape, mass_out.shape[-1]
    ko, vo = shape_ko[-2], shape_vo[-2]
    if min(ko, vo, mo) < keep:
        raise ValueError("k_out, v_out and mass_out: at least `keep` rows expected")
    sk, sv, s1, s2 = k.stride(), v.stride(), k_out.stride(), v_out.stride()
    if not (v.shape == shape and shape_ko == (B, kv, ko, d) and shape_vo == (B, kv, vo, d) and v.dtype is dt and k_out.dtype is dt and v_out.dtype is dt and
            v.get_device() == at and k_out.get_device() == at and v_out.get_device() == at and sk[3] == sv[3] == s1[3] == s2[3] == 1):
        for t, want, name in ((k, shape, "k"), (v, shape, "v"), (k_out, (B, kv, ko, d), "k_out"), (v_out, (B, kv, vo, d), "v_out")):
            _rows(t, want, dt, at, name)                         # names the one that is wrong
    args = _EVICT.pack(
        B, kv, d, cap, code, keep, sinks, recent, k.data_ptr(), v.data_ptr(), k_out.data_ptr(), v_out.data_ptr(),
        sk[0], sk[1], sk[2], sv[0], sv[1], sv[2], s1[0], s1[1], s1[2], s2[0], s2[1], s2[2],
        _dense(mass, shape[:3], _F32, at, "mass"), 0 if lens is None else _dense(lens, (B,), _I32, at, "lens"),
        _dense(idx_out, (B, kv, keep), _I32, at, "idx_out"), _dense(mass_out, (B, kv, mo), _F32, at, "mass_out"), mo,
        _dense(lens_out, (B,), _I32, at, "lens_out"))
    _enqueue("obf_evict_by_mass", at, (args,), stream)
    return {"K_out": k_out, "V_out": v_out, "idx": idx_out, "mass": mass_out, "lens": lens_out}
