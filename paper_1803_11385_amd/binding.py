"""ctypes binding of libhch.so: the same names as the C entry points, arguments marshalled
from numpy arrays (HOST) and torch tensors (DEVICE).  No arithmetic happens here."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

__all__ = [
    "HchError", "Levels", "LevelInfo", "HCH_F32", "HCH_BF16",
    "HCH_WS_FWD", "HCH_WS_BWD_DATA", "HCH_WS_BWD_WEIGHT", "HCH_WS_MIN",
    "HCH_ALGO_COLUMNS", "HCH_ALGO_FUSED", "HCH_ALGO_COLUMNS_RESIDENT", "HCH_ALGO_FUSED_DENSE",
    "library_path", "load_library", "exported_symbols",
    "hch_build_levels", "hch_build_levels_device", "hch_build_tables_host", "hch_build_neighbours",
    "hch_build_neighbours_range", "hch_build_index_lists", "hch_hash2col", "hch_col2hash", "hch_conv_workspace_bytes", "hch_conv_fwd", "hch_conv_bwd_data",
    "hch_conv_bwd_weight", "hch_pool_fwd", "hch_pool_bwd", "hch_relu_fwd", "hch_relu_bwd", "hch_relu_pool_fwd",
    "hch_pool_relu_bwd", "hch_pool_relu_bwd_pooled", "hch_deconv_fwd", "hch_deconv_bwd_data", "hch_deconv_bwd_weight",
    "hch_unpool_fwd", "hch_unpool_bwd", "hch_kernel_count", "hch_kernel_name", "hch_profile_enable", "hch_profile_read",
    "hch_profile_reset", "hch_field_build", "hch_sconv_workspace_bytes", "hch_sconv_fwd", "hch_sconv_bwd_weight",
    "hch_sconv_bwd_data", "hch_avgpool_fwd", "hch_avgpool_bwd", "hch_build_levels_ratios",
    "hch_spool_max_fwd", "hch_spool_max_bwd", "hch_spool_avg_fwd", "hch_spool_avg_bwd", "hch_build_tap_major",
    "hch_conv_bwd_weight_noalloc", "HCH_NOALLOC_SCRATCH_BYTES", "hch_probe_mfma", "hch_set_lean_loops",
    "hch_layernorm_fwd", "hch_layernorm_workspace_bytes", "hch_layernorm_bwd", "hch_rope_fwd", "hch_rope_bwd",
    "hch_attn_workspace_bytes", "hch_attn_fwd", "hch_attn_bwd",
]

HCH_F32, HCH_BF16 = 0, 1
HCH_WS_FWD, HCH_WS_BWD_DATA, HCH_WS_BWD_WEIGHT, HCH_WS_MIN = 0, 1, 2, 3
HCH_ALGO_COLUMNS, HCH_ALGO_FUSED, HCH_ALGO_COLUMNS_RESIDENT, HCH_ALGO_FUSED_DENSE = 0, 1, 2, 3

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIBPATH = os.path.join(_HERE, "libhch.so")

# every symbol include/hch.h declares
exported_symbols = [
    "hch_last_error", "hch_build_levels", "hch_build_levels_device", "hch_build_tables_host", "hch_free_levels",
    "hch_num_levels", "hch_level_info", "hch_build_neighbours", "hch_build_neighbours_range", "hch_build_index_lists", "hch_hash2col",
    "hch_col2hash",
    "hch_conv_workspace_bytes", "hch_conv_fwd", "hch_conv_bwd_data", "hch_conv_bwd_weight",
    "hch_pool_fwd", "hch_pool_bwd", "hch_relu_fwd", "hch_relu_bwd", "hch_relu_pool_fwd",
    "hch_pool_relu_bwd", "hch_pool_relu_bwd_pooled", "hch_deconv_fwd", "hch_deconv_bwd_data", "hch_deconv_bwd_weight",
    "hch_unpool_fwd", "hch_unpool_bwd", "hch_kernel_count", "hch_kernel_name", "hch_profile_enable", "hch_profile_read",
    "hch_profile_reset", "hch_field_build", "hch_sconv_workspace_bytes", "hch_sconv_fwd", "hch_sconv_bwd_weight",
    "hch_sconv_bwd_data", "hch_avgpool_fwd", "hch_avgpool_bwd", "hch_build_levels_ratios",
    "hch_spool_max_fwd", "hch_spool_max_bwd", "hch_spool_avg_fwd", "hch_spool_avg_bwd", "hch_build_tap_major",
    "hch_conv_bwd_weight_noalloc",
    "hch_probe_mfma", "hch_set_lean_loops",
    "hch_layernorm_fwd", "hch_layernorm_workspace_bytes", "hch_layernorm_bwd", "hch_rope_fwd", "hch_rope_bwd",
    "hch_attn_workspace_bytes", "hch_attn_fwd", "hch_attn_bwd",
]


class HchError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"hch status {status}: {message}")
        self.status = status


class _Desc(C.Structure):
    _fields_ = [("ubar", C.c_int32), ("batch", C.c_int32), ("n_total", C.c_int64),
                ("m_total", C.c_int64), ("r_total", C.c_int64), ("nbr_valid", C.c_int64),
                ("mbar", C.c_void_p), ("rbar", C.c_void_p), ("attempts", C.c_void_p),
                ("M", C.c_void_p), ("R", C.c_void_p), ("N", C.c_void_p),
                ("coords_host", C.c_void_p), ("H_host", C.c_void_p), ("T_host", C.c_void_p),
                ("Phi_host", C.c_void_p), ("V_host", C.c_void_p),
                ("H", C.c_void_p), ("T", C.c_void_p), ("Phi", C.c_void_p), ("V", C.c_void_p),
                ("coords", C.c_void_p), ("nbr27", C.c_void_p), ("child8", C.c_void_p),
                ("row_order", C.c_void_p), ("tile_taps", C.c_void_p)]


class _KernelStats(C.Structure):
    _fields_ = [("launches", C.c_int64), ("ms", C.c_double), ("bytes", C.c_double),
                ("flops", C.c_double)]


class _AttnDesc(C.Structure):
    _fields_ = [("dtype", C.c_int), ("batch", C.c_int32), ("heads_q", C.c_int32), ("heads_kv", C.c_int32),
                ("head_dim", C.c_int32), ("scale", C.c_float), ("n_q", C.c_int64), ("n_k", C.c_int64),
                ("q_offsets", C.c_void_p), ("k_offsets", C.c_void_p), ("key_mask", C.c_void_p),
                ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_v", C.c_int64), ("ld_o", C.c_int64),
                ("ld_do", C.c_int64), ("ld_dq", C.c_int64), ("ld_dk", C.c_int64), ("ld_dv", C.c_int64)]


_lib = None


def library_path():
    return _LIBPATH


def load_library():
    """Load libhch.so (built by paper_1803_11385_amd.build.build_library).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIBPATH):
        raise ImportError(f"{_LIBPATH} is missing: run `python -c 'import __graft_entry__ as g; "
                          "g.build()'` (hipcc --offload-arch=gfx950) first; there is no fallback")
    # torch brings a HIP runtime of its own: whichever comes first serves both, and a process with two finds no GPU
    try:
        import torch  # noqa: F401
    except ImportError:
        pass                                # the host entries need none
    L = C.CDLL(_LIBPATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.hch_last_error.restype = C.c_char_p
    L.hch_build_levels.argtypes = [vp, vp, i32, i32, i32, vp, C.POINTER(vp)]
    L.hch_build_levels_device.argtypes = [vp, vp, i32, i32, i32, vp, C.POINTER(vp)]
    L.hch_build_tables_host.argtypes = [vp, vp, i32, i32, i32, C.POINTER(vp)]
    L.hch_build_levels_ratios.argtypes = [vp, vp, i32, i32, i32, vp, i32, vp, C.POINTER(vp)]
    L.hch_spool_max_fwd.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, i32, vp]
    L.hch_spool_max_bwd.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp]
    L.hch_spool_avg_fwd.argtypes = [vp, i32, i32, i32, vp, vp, vp, i32, vp]
    L.hch_spool_avg_bwd.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, i32, vp]
    L.hch_free_levels.argtypes = [vp]
    L.hch_free_levels.restype = None
    L.hch_num_levels.argtypes = [vp]
    L.hch_num_levels.restype = i32
    L.hch_level_info.argtypes = [vp, i32, C.POINTER(_Desc)]
    L.hch_build_neighbours.argtypes = [vp, i32, vp]
    L.hch_build_neighbours_range.argtypes = [vp, i32, i32, vp]
    L.hch_build_index_lists.argtypes = [vp, i32, i32, vp]
    L.hch_build_tap_major.argtypes = [vp, i32, vp]
    L.hch_hash2col.argtypes = [vp, i32, C.c_int, vp, i32, i64, i64, vp, vp]
    L.hch_col2hash.argtypes = [vp, i32, vp, i32, vp, vp]
    L.hch_conv_workspace_bytes.argtypes = [vp, i32, i32, i32, C.c_int, C.c_int, C.c_int]
    L.hch_conv_workspace_bytes.restype = sz
    L.hch_field_build.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp]
    L.hch_sconv_workspace_bytes.argtypes = [vp, i32, i32, i32, i32, i32, C.c_int, C.c_int]
    L.hch_sconv_workspace_bytes.restype = sz
    for name in ("hch_sconv_fwd", "hch_sconv_bwd_weight", "hch_sconv_bwd_data"):
        getattr(L, name).argtypes = [vp, i32, i32, i32, C.c_int, vp, vp, vp, vp, i32, i32, vp, sz, vp]
    L.hch_avgpool_fwd.argtypes = [vp, i32, vp, vp, i32, vp]
    L.hch_avgpool_bwd.argtypes = [vp, i32, vp, vp, i32, vp]
    L.hch_unpool_fwd.argtypes = [vp, i32, vp, vp, vp, i32, vp]
    L.hch_unpool_bwd.argtypes = [vp, i32, vp, vp, vp, i32, vp]
    for name in ("hch_conv_fwd", "hch_conv_bwd_data", "hch_conv_bwd_weight",
                 "hch_deconv_fwd", "hch_deconv_bwd_data", "hch_deconv_bwd_weight"):
        getattr(L, name).argtypes = [vp, i32, C.c_int, vp, vp, vp, i32, i32, vp, sz, C.c_int, vp]
    L.hch_conv_bwd_weight_noalloc.argtypes = [vp, i32, C.c_int, vp, vp, vp, i32, i32, vp]
    L.hch_pool_fwd.argtypes = [vp, i32, vp, vp, vp, i32, vp]
    L.hch_pool_bwd.argtypes = [vp, i32, vp, vp, vp, i32, vp]
    L.hch_relu_pool_fwd.argtypes = [vp, i32, vp, vp, vp, vp, i32, vp]
    L.hch_pool_relu_bwd.argtypes = [vp, i32, vp, vp, vp, vp, i32, vp]
    L.hch_pool_relu_bwd_pooled.argtypes = [vp, i32, vp, vp, vp, vp, i32, vp]
    L.hch_relu_fwd.argtypes = [vp, vp, i64, vp]
    L.hch_relu_bwd.argtypes = [vp, vp, vp, i64, vp]
    L.hch_layernorm_fwd.argtypes = [C.c_int, vp, vp, vp, vp, vp, C.c_int, vp, vp, i64, i32, C.c_float, vp]
    L.hch_layernorm_workspace_bytes.argtypes = [i64, i32]
    L.hch_layernorm_workspace_bytes.restype = sz
    L.hch_layernorm_bwd.argtypes = [C.c_int, vp, vp, vp, C.c_int, vp, vp, vp, vp, vp, i64, i32, vp, sz, vp]
    for name in ("hch_rope_fwd", "hch_rope_bwd"):
        getattr(L, name).argtypes = [C.c_int, vp, i64, C.c_int, vp, i64, vp, i64, i32, i32, i32, vp, C.c_float, C.c_float, vp]
    L.hch_attn_workspace_bytes.argtypes = [C.POINTER(_AttnDesc), C.c_int]
    L.hch_attn_workspace_bytes.restype = sz
    L.hch_attn_fwd.argtypes = [C.POINTER(_AttnDesc), vp, vp, vp, vp, vp, vp, sz, vp]
    L.hch_attn_bwd.argtypes = [C.POINTER(_AttnDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.hch_probe_mfma.argtypes = [C.c_int, i32, i32, vp, vp]
    L.hch_set_lean_loops.argtypes = [i32]
    L.hch_set_lean_loops.restype = i32
    L.hch_kernel_count.restype = i32
    L.hch_kernel_name.argtypes = [i32]
    L.hch_kernel_name.restype = C.c_char_p
    L.hch_profile_enable.argtypes = [i32, i32]
    L.hch_profile_read.argtypes = [i32, C.POINTER(_KernelStats)]
    _lib = L
    return L


def _check(st):
    if st != 0:
        raise HchError(st, load_library().hch_last_error().decode())


def _host_array(ptr, shape, dtype):
    n = int(np.prod(shape))
    if n == 0 or not ptr:
        return np.zeros(shape, dtype)
    buf = (C.c_char * (n * np.dtype(dtype).itemsize)).from_address(ptr)
    return np.frombuffer(buf, dtype=dtype).reshape(shape).copy()


class LevelInfo:
    """Python view of hch_level_desc.  Host arrays are copied into numpy; device arrays are
    exposed as raw addresses (ints) plus `device_*()` helpers that copy them back via torch."""

    def __init__(self, d: _Desc):
        b = d.batch
        self.ubar, self.batch = d.ubar, b
        self.n_total, self.m_total, self.r_total = d.n_total, d.m_total, d.r_total
        self.nbr_valid = d.nbr_valid
        self.mbar = _host_array(d.mbar, (b,), np.int32)
        self.rbar = _host_array(d.rbar, (b,), np.int32)
        self.attempts = _host_array(d.attempts, (b,), np.int32)
        self.M = _host_array(d.M, (b + 1,), np.int64)
        self.R = _host_array(d.R, (b + 1,), np.int64)
        self.N = _host_array(d.N, (b + 1,), np.int64)
        self._d = d

    # host copies of the tables
    def coords_host(self):
        return _host_array(self._d.coords_host, (self.n_total, 3), np.int32)

    def H_host(self):
        return _host_array(self._d.H_host, (self.m_total,), np.int32)

    def T_host(self):
        return _host_array(self._d.T_host, (self.m_total, 3), np.uint16)

    def Phi_host(self):
        return _host_array(self._d.Phi_host, (self.r_total, 3), np.uint8)

    def V_host(self):
        return _host_array(self._d.V_host, (self.m_total,), np.int32)

    # device arrays copied back to numpy
    def _dev(self, ptr, shape, dtype):
        import torch
        n = int(np.prod(shape))
        out = np.empty(shape, dtype)
        if n == 0:
            return out
        if not ptr:
            raise HchError(1, "device table is NULL")
        nbytes = n * np.dtype(dtype).itemsize
        t = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        import ctypes
        hip = _hip()
        st = hip.hipMemcpy(C.c_void_p(t.data_ptr()), C.c_void_p(ptr), C.c_size_t(nbytes), 3)
        if st != 0:
            raise HchError(4, f"hipMemcpy failed ({st})")
        return np.frombuffer(t.cpu().numpy().tobytes(), dtype=dtype).reshape(shape).copy()

    def device_H(self):
        return self._dev(self._d.H, (self.m_total,), np.int32)

    def device_T(self):
        return self._dev(self._d.T, (self.m_total, 3), np.uint16)

    def device_Phi(self):
        return self._dev(self._d.Phi, (self.r_total, 3), np.uint8)

    def device_V(self):
        return self._dev(self._d.V, (self.m_total,), np.int32)

    def device_coords(self):
        return self._dev(self._d.coords, (self.n_total, 3), np.int32)

    def device_nbr27(self):
        return self._dev(self._d.nbr27, (self.n_total, 27), np.int32)

    def device_child8(self):
        return self._dev(self._d.child8, (self.n_total, 8), np.int32)

    def device_row_order(self):
        return self._dev(self._d.row_order, (self.n_total,), np.int32)

    def device_tile_taps(self):
        return self._dev(self._d.tile_taps, ((self.n_total + 63) // 64,), np.uint32)


_hiplib = None


def _hip():
    global _hiplib
    if _hiplib is None:
        for name in ("libamdhip64.so", "/opt/rocm/lib/libamdhip64.so"):
            try:
                _hiplib = C.CDLL(name)
                break
            except OSError:
                continue
        if _hiplib is None:
            raise ImportError("libamdhip64.so not found")
        _hiplib.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
    return _hiplib


class Levels:
    """Owner of an hch_levels handle."""

    def __init__(self, handle):
        self._h = handle
        self._n = {}

    @property
    def handle(self):
        if not self._h:
            raise HchError(1, "levels already freed")
        return self._h

    @property
    def n_levels(self):
        return load_library().hch_num_levels(self.handle)

    def info(self, level):
        d = _Desc()
        _check(load_library().hch_level_info(self.handle, level, C.byref(d)))
        return LevelInfo(d)

    def n(self, level):
        """N_l, the number of voxels (rows of every feature tensor) of `level`."""
        if level not in self._n:
            self._n[level] = int(self.info(level).n_total)
        return self._n[level]

    def device_offsets(self, level, device="cuda"):
        """First row of each shape of `level`, and behind the last: [batch + 1] int32 on `device`, as hch_attn_* take it."""
        import torch
        return torch.from_numpy(self.info(level).N.astype(np.int32)).to(device)

    def device_positions(self, level, device="cuda"):
        """Voxel positions of `level` in data order, [n][3] int32 on `device`, as hch_rope_* take them."""
        import torch
        return torch.from_numpy(self.info(level).coords_host()).to(device)

    def free(self):
        if self._h:
            load_library().hch_free_levels(self._h)
            self._h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


_torch = None


def _th():
    """torch, imported by the first call that has a tensor to check."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _stream(stream):
    """The stream's address; None: torch's current one (by its raw accessor where there is one: 0.1 us in place of 1)."""
    if stream is not None:
        return int(stream)
    th = _torch or _th()
    raw = getattr(th._C, "_cuda_getCurrentRawStream", None)
    return raw(th.cuda.current_device()) if raw else th.cuda.current_stream().cuda_stream


# Every DEVICE argument is checked here, on the host, before its address goes to the library: a
# CPU tensor, a wrong element type, a non-contiguous view or a buffer shorter than the call will
# read or write would otherwise become an out-of-bounds access on the GPU instead of an error.
_F32, _I32 = "f32", "i32"


def _dp(t, what="tensor", kind=None, numel=0):
    """Address of a DEVICE tensor (None -> NULL).  kind: _F32, _I32, an hch_dtype (HCH_F32 / HCH_BF16:
    float32, or any 2-byte element type holding bfloat16 bit patterns), or None (bytes)."""
    if t is None:
        return None
    th = _torch or _th()
    if not isinstance(t, th.Tensor) or not t.is_cuda:
        raise HchError(1, f"{what}: must be a torch tensor in GPU memory")
    if not t.is_contiguous():
        raise HchError(1, f"{what}: must be contiguous")
    if kind == _F32 or kind == HCH_F32:
        ok = t.dtype == th.float32
    elif kind == _I32:
        ok = t.dtype == th.int32
    elif kind == HCH_BF16:
        ok = t.element_size() == 2
    else:
        ok = True
    if not ok:
        raise HchError(1, f"{what}: wrong element type {t.dtype}")
    if t.numel() < numel:
        raise HchError(1, f"{what}: {t.numel()} elements, the call needs {int(numel)}")
    return t.data_ptr()


def _nbytes(ws):
    return ws.numel() * ws.element_size() if ws is not None else 0


def _in_dtype(dtype):
    if dtype not in (HCH_F32, HCH_BF16):
        raise HchError(1, "unknown dtype")
    return dtype


def _level_n(levels, level, what="level"):
    if not isinstance(level, int) or level < 0 or level >= levels.n_levels:
        raise HchError(1, f"{what} out of range")
    return levels.n(level)


def _out_level(levels, level_in, stride):
    """Rows of the level a field of this stride writes, for the argument checks only; the library
    decides (and rejects a stride that no level matches)."""
    n_in = _level_n(levels, level_in, "level_in")
    if stride == 1:
        return n_in, n_in
    u = levels.info(level_in).ubar
    for l in range(level_in + 1, levels.n_levels):
        if levels.info(l).ubar * stride >= u > (levels.info(l).ubar - 1) * stride:
            return n_in, levels.n(l)
    raise HchError(1, "no level of this set is `stride` times coarser than level_in")


def _host_inputs(coords, model_offsets):
    coords = np.ascontiguousarray(coords, dtype=np.int32)
    offs = np.ascontiguousarray(model_offsets, dtype=np.int64)
    if coords.ndim != 2 or coords.shape[1] != 3 or offs.ndim != 1 or offs.size < 2:
        raise HchError(1, "coords must be [n,3] and model_offsets [b+1]")
    if coords.shape[0] != offs[-1]:
        raise HchError(1, "model_offsets[-1] must equal the number of coordinates")
    return coords, offs


def hch_build_levels(coords, model_offsets, resolution, n_levels, stream=None):
    coords, offs = _host_inputs(coords, model_offsets)
    h = C.c_void_p()
    _check(load_library().hch_build_levels(coords.ctypes.data, offs.ctypes.data, offs.size - 1,
                                           int(resolution), int(n_levels), _stream(stream),
                                           C.byref(h)))
    return Levels(h)


def hch_build_levels_device(coords, model_offsets, resolution, n_levels, stream=None):
    coords, offs = _host_inputs(coords, model_offsets)
    h = C.c_void_p()
    _check(load_library().hch_build_levels_device(coords.ctypes.data, offs.ctypes.data, offs.size - 1,
                                                  int(resolution), int(n_levels), _stream(stream),
                                                  C.byref(h)))
    return Levels(h)


def hch_build_levels_ratios(coords, model_offsets, resolution, ratios, device_tables=False, stream=None):
    """Levels 0 .. len(ratios): level l+1 is ratios[l] times coarser than level l."""
    coords, offs = _host_inputs(coords, model_offsets)
    r = np.ascontiguousarray(np.asarray(ratios, dtype=np.int32).reshape(-1))
    h = C.c_void_p()
    _check(load_library().hch_build_levels_ratios(coords.ctypes.data, offs.ctypes.data, offs.size - 1,
                                                  int(resolution), int(r.size) + 1,
                                                  r.ctypes.data if r.size else None,
                                                  1 if device_tables else 0, _stream(stream), C.byref(h)))
    return Levels(h)


def hch_build_tables_host(coords, model_offsets, resolution, n_levels):
    coords, offs = _host_inputs(coords, model_offsets)
    h = C.c_void_p()
    _check(load_library().hch_build_tables_host(coords.ctypes.data, offs.ctypes.data,
                                                offs.size - 1, int(resolution), int(n_levels),
                                                C.byref(h)))
    return Levels(h)


def hch_build_neighbours(levels, level, stream=None):
    _check(load_library().hch_build_neighbours(levels.handle, level, _stream(stream)))


def hch_build_tap_major(levels, level=-1, stream=None):
    _check(load_library().hch_build_tap_major(levels.handle, level, _stream(stream)))


def hch_build_neighbours_range(levels, first, count, stream=None):
    _check(load_library().hch_build_neighbours_range(levels.handle, first, count, _stream(stream)))


def hch_build_index_lists(levels, first, count, stream=None):
    _check(load_library().hch_build_index_lists(levels.handle, first, count, _stream(stream)))


def hch_hash2col(levels, level, dtype, X, c_in, row_begin, row_count, col, stream=None):
    n, dt = _level_n(levels, level), _in_dtype(dtype)
    _check(load_library().hch_hash2col(levels.handle, level, dtype, _dp(X, "X", dt, n * c_in), c_in, row_begin,
                                       row_count, _dp(col, "col", dt, max(0, row_count) * 27 * c_in), _stream(stream)))


def hch_col2hash(levels, level, dcol, c_in, dX, stream=None):
    n = _level_n(levels, level)
    _check(load_library().hch_col2hash(levels.handle, level, _dp(dcol, "dcol", _F32, n * 27 * c_in), c_in,
                                       _dp(dX, "dX", _F32, n * c_in), _stream(stream)))


def hch_conv_workspace_bytes(levels, level, c_in, c_out, dtype, kind, algo=HCH_ALGO_COLUMNS):
    return int(load_library().hch_conv_workspace_bytes(levels.handle, level, c_in, c_out, dtype,
                                                       kind, algo))


def _conv_like(name, levels, level, dtype, a, a_c, b, b_c, out, out_c, c_in, c_out, workspace, algo, stream):
    """a, b: inputs of `dtype`; out: float32.  *_c: channels per voxel row, or None for a weight
    tensor of 27 * c_in * c_out elements."""
    n, dt = _level_n(levels, level), _in_dtype(dtype)
    wn = 27 * c_in * c_out
    size = lambda c: wn if c is None else n * c
    _check(getattr(load_library(), name)(levels.handle, level, dtype, _dp(a, "first input", dt, size(a_c)),
                                         _dp(b, "second input", dt, size(b_c)), _dp(out, "output", _F32, size(out_c)),
                                         c_in, c_out, _dp(workspace, "workspace"), _nbytes(workspace), algo,
                                         _stream(stream)))


def hch_conv_fwd(levels, level, dtype, X, W, Y, c_in, c_out, workspace, algo=HCH_ALGO_COLUMNS, stream=None):
    _conv_like("hch_conv_fwd", levels, level, dtype, X, c_in, W, None, Y, c_out, c_in, c_out, workspace, algo, stream)


def hch_conv_bwd_data(levels, level, dtype, dY, W, dX, c_in, c_out, workspace, algo=HCH_ALGO_COLUMNS, stream=None):
    _conv_like("hch_conv_bwd_data", levels, level, dtype, dY, c_out, W, None, dX, c_in, c_in, c_out, workspace, algo, stream)


def hch_conv_bwd_weight(levels, level, dtype, X, dY, dW, c_in, c_out, workspace, algo=HCH_ALGO_COLUMNS, stream=None):
    _conv_like("hch_conv_bwd_weight", levels, level, dtype, X, c_in, dY, c_out, dW, None, c_in, c_out, workspace, algo, stream)


HCH_NOALLOC_SCRATCH_BYTES = 32 << 20


def hch_conv_bwd_weight_noalloc(levels, level, dtype, X, dY, dW, c_in, c_out, stream=None):
    n, dt = _level_n(levels, level), _in_dtype(dtype)
    _check(load_library().hch_conv_bwd_weight_noalloc(levels.handle, level, dtype, _dp(X, "X", dt, n * c_in),
                                                      _dp(dY, "dY", dt, n * c_out),
                                                      _dp(dW, "dW", _F32, 27 * c_in * c_out), c_in, c_out,
                                                      _stream(stream)))


def hch_deconv_fwd(levels, level, dtype, X, W, Y, c_in, c_out, workspace, algo=HCH_ALGO_COLUMNS, stream=None):
    _conv_like("hch_deconv_fwd", levels, level, dtype, X, c_in, W, None, Y, c_out, c_in, c_out, workspace, algo, stream)


def hch_deconv_bwd_data(levels, level, dtype, dY, W, dX, c_in, c_out, workspace, algo=HCH_ALGO_COLUMNS,
                        stream=None):
    _conv_like("hch_deconv_bwd_data", levels, level, dtype, dY, c_out, W, None, dX, c_in, c_in, c_out, workspace, algo, stream)


def hch_deconv_bwd_weight(levels, level, dtype, X, dY, dW, c_in, c_out, workspace, algo=HCH_ALGO_COLUMNS,
                          stream=None):
    _conv_like("hch_deconv_bwd_weight", levels, level, dtype, X, c_in, dY, c_out, dW, None, c_in, c_out, workspace, algo, stream)


def _pool_rows(levels, level_in):
    """(N_fine, N_coarse) of a pooling between level_in and level_in + 1."""
    return _level_n(levels, level_in, "level_in"), _level_n(levels, level_in + 1, "level_in + 1")


def hch_unpool_fwd(levels, level_out, Xc, argmax, Y, c, stream=None):
    nf, nc = _pool_rows(levels, level_out)
    _check(load_library().hch_unpool_fwd(levels.handle, level_out, _dp(Xc, "Xc", _F32, nc * c),
                                         _dp(argmax, "argmax", _I32, nc * c), _dp(Y, "Y", _F32, nf * c), c,
                                         _stream(stream)))


def hch_unpool_bwd(levels, level_out, dY, argmax, dXc, c, stream=None):
    nf, nc = _pool_rows(levels, level_out)
    _check(load_library().hch_unpool_bwd(levels.handle, level_out, _dp(dY, "dY", _F32, nf * c),
                                         _dp(argmax, "argmax", _I32, nc * c), _dp(dXc, "dXc", _F32, nc * c), c,
                                         _stream(stream)))


def hch_pool_fwd(levels, level_in, X, Y, argmax, c, stream=None):
    nf, nc = _pool_rows(levels, level_in)
    _check(load_library().hch_pool_fwd(levels.handle, level_in, _dp(X, "X", _F32, nf * c), _dp(Y, "Y", _F32, nc * c),
                                       _dp(argmax, "argmax", _I32, nc * c), c, _stream(stream)))


def hch_pool_bwd(levels, level_in, dY, argmax, dX, c, stream=None):
    nf, nc = _pool_rows(levels, level_in)
    _check(load_library().hch_pool_bwd(levels.handle, level_in, _dp(dY, "dY", _F32, nc * c),
                                       _dp(argmax, "argmax", _I32, nc * c), _dp(dX, "dX", _F32, nf * c), c,
                                       _stream(stream)))


def hch_relu_pool_fwd(levels, level_in, Y, A, P, argmax, c, stream=None):
    nf, nc = _pool_rows(levels, level_in)
    _check(load_library().hch_relu_pool_fwd(levels.handle, level_in, _dp(Y, "Y", _F32, nf * c), _dp(A, "A", _F32, nf * c),
                                            _dp(P, "P", _F32, nc * c), _dp(argmax, "argmax", _I32, nc * c), c,
                                            _stream(stream)))


def hch_pool_relu_bwd(levels, level_in, dP, argmax, A, dY, c, stream=None):
    nf, nc = _pool_rows(levels, level_in)
    _check(load_library().hch_pool_relu_bwd(levels.handle, level_in, _dp(dP, "dP", _F32, nc * c),
                                            _dp(argmax, "argmax", _I32, nc * c), _dp(A, "A", _F32, nf * c),
                                            _dp(dY, "dY", _F32, nf * c), c, _stream(stream)))


def hch_pool_relu_bwd_pooled(levels, level_in, dP, argmax, P, dY, c, stream=None):
    nf, nc = _pool_rows(levels, level_in)
    _check(load_library().hch_pool_relu_bwd_pooled(levels.handle, level_in, _dp(dP, "dP", _F32, nc * c),
                                                   _dp(argmax, "argmax", _I32, nc * c), _dp(P, "P", _F32, nc * c),
                                                   _dp(dY, "dY", _F32, nf * c), c, _stream(stream)))


def hch_field_build(levels, level_in, F, stride, pad, field, field_t, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _check(load_library().hch_field_build(levels.handle, level_in, F, stride, pad,
                                          _dp(field, "field", _I32, n_out * F ** 3),
                                          _dp(field_t, "field_t", _I32, n_in * F ** 3), _stream(stream)))


def hch_sconv_workspace_bytes(levels, level_in, F, stride, c_in, c_out, dtype, kind):
    return int(load_library().hch_sconv_workspace_bytes(levels.handle, level_in, F, stride, c_in, c_out, dtype, kind))


def _sconv(name, levels, level_in, F, stride, dtype, a, a_n, b, b_n, out, out_n, idx, idx_n, c_in, c_out, workspace,
           stream):
    dt = _in_dtype(dtype)
    _check(getattr(load_library(), name)(levels.handle, level_in, F, stride, dtype, _dp(a, "first input", dt, a_n),
                                         _dp(b, "second input", dt, b_n), _dp(out, "output", _F32, out_n),
                                         _dp(idx, "index rows", _I32, idx_n), c_in, c_out, _dp(workspace, "workspace"),
                                         _nbytes(workspace), _stream(stream)))


def hch_sconv_fwd(levels, level_in, F, stride, dtype, X, W, Y, field, c_in, c_out, workspace, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _sconv("hch_sconv_fwd", levels, level_in, F, stride, dtype, X, n_in * c_in, W, F ** 3 * c_in * c_out, Y,
           n_out * c_out, field, n_out * F ** 3, c_in, c_out, workspace, stream)


def hch_sconv_bwd_weight(levels, level_in, F, stride, dtype, X, dY, dW, field, c_in, c_out, workspace, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _sconv("hch_sconv_bwd_weight", levels, level_in, F, stride, dtype, X, n_in * c_in, dY, n_out * c_out, dW,
           F ** 3 * c_in * c_out, field, n_out * F ** 3, c_in, c_out, workspace, stream)


def hch_sconv_bwd_data(levels, level_in, F, stride, dtype, dY, W, dX, field_t, c_in, c_out, workspace, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _sconv("hch_sconv_bwd_data", levels, level_in, F, stride, dtype, dY, n_out * c_out, W, F ** 3 * c_in * c_out, dX,
           n_in * c_in, field_t, n_in * F ** 3, c_in, c_out, workspace, stream)


def hch_avgpool_fwd(levels, level_in, X, Y, c, stream=None):
    nf, nc = _pool_rows(levels, level_in)
    _check(load_library().hch_avgpool_fwd(levels.handle, level_in, _dp(X, "X", _F32, nf * c), _dp(Y, "Y", _F32, nc * c),
                                          c, _stream(stream)))


def hch_avgpool_bwd(levels, level_in, dY, dX, c, stream=None):
    nf, nc = _pool_rows(levels, level_in)
    _check(load_library().hch_avgpool_bwd(levels.handle, level_in, _dp(dY, "dY", _F32, nc * c),
                                          _dp(dX, "dX", _F32, nf * c), c, _stream(stream)))


def hch_spool_max_fwd(levels, level_in, F, stride, X, field, Y, argmax, c, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _check(load_library().hch_spool_max_fwd(levels.handle, level_in, F, stride, _dp(X, "X", _F32, n_in * c),
                                            _dp(field, "field", _I32, n_out * F ** 3), _dp(Y, "Y", _F32, n_out * c),
                                            _dp(argmax, "argmax", _I32, n_out * c), c, _stream(stream)))


def hch_spool_max_bwd(levels, level_in, F, stride, pad, dY, argmax, field, field_t, dX, c, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _check(load_library().hch_spool_max_bwd(levels.handle, level_in, F, stride, pad, _dp(dY, "dY", _F32, n_out * c),
                                            _dp(argmax, "argmax", _I32, n_out * c),
                                            _dp(field, "field", _I32, n_out * F ** 3),
                                            _dp(field_t, "field_t", _I32, n_in * F ** 3), _dp(dX, "dX", _F32, n_in * c),
                                            c, _stream(stream)))


def hch_spool_avg_fwd(levels, level_in, F, stride, X, field, Y, c, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _check(load_library().hch_spool_avg_fwd(levels.handle, level_in, F, stride, _dp(X, "X", _F32, n_in * c),
                                            _dp(field, "field", _I32, n_out * F ** 3), _dp(Y, "Y", _F32, n_out * c), c,
                                            _stream(stream)))


def hch_spool_avg_bwd(levels, level_in, F, stride, pad, dY, field, field_t, dX, c, stream=None):
    n_in, n_out = _out_level(levels, level_in, stride)
    _check(load_library().hch_spool_avg_bwd(levels.handle, level_in, F, stride, pad, _dp(dY, "dY", _F32, n_out * c),
                                            _dp(field, "field", _I32, n_out * F ** 3),
                                            _dp(field_t, "field_t", _I32, n_in * F ** 3), _dp(dX, "dX", _F32, n_in * c),
                                            c, _stream(stream)))


def hch_relu_fwd(x, y, n, stream=None):
    _check(load_library().hch_relu_fwd(_dp(x, "x", _F32, n), _dp(y, "y", _F32, n), n, _stream(stream)))


def hch_relu_bwd(y, dy, dx, n, stream=None):
    _check(load_library().hch_relu_bwd(_dp(y, "y", _F32, n), _dp(dy, "dy", _F32, n), _dp(dx, "dx", _F32, n), n,
                                       _stream(stream)))


def hch_layernorm_fwd(x_dtype, X, R, S, gamma, beta, y_dtype, Y, stats, n, c, eps=1e-5, stream=None):
    """s = X + R (kept in S; both None: s = X), Y = norm(s) * gamma + beta, stats = mean and 1 / deviation per row."""
    tx, ty, e = _in_dtype(x_dtype), _in_dtype(y_dtype), n * c
    _check(load_library().hch_layernorm_fwd(tx, _dp(X, "X", tx, e), _dp(R, "R", tx, e), _dp(S, "S", tx, e),
                                            _dp(gamma, "gamma", _F32, c), _dp(beta, "beta", _F32, c), ty,
                                            _dp(Y, "Y", ty, e), _dp(stats, "stats", _F32, 2 * n), n, c, eps,
                                            _stream(stream)))


def hch_layernorm_workspace_bytes(n, c):
    return int(load_library().hch_layernorm_workspace_bytes(n, c))


def hch_layernorm_bwd(x_dtype, X, stats, gamma, dy_dtype, dY, dS, dX, dgamma, dbeta, n, c, workspace, stream=None):
    """Gradients of hch_layernorm_fwd from the rows it normalised and their stats; dX = that of the norm + dS."""
    tx, ty, e = _in_dtype(x_dtype), _in_dtype(dy_dtype), n * c
    _check(load_library().hch_layernorm_bwd(tx, _dp(X, "X", tx, e), _dp(stats, "stats", _F32, 2 * n),
                                            _dp(gamma, "gamma", _F32, c), ty, _dp(dY, "dY", ty, e),
                                            _dp(dS, "dS", tx, e), _dp(dX, "dX", tx, e),
                                            _dp(dgamma, "dgamma", _F32, c), _dp(dbeta, "dbeta", _F32, c), n, c,
                                            _dp(workspace, "workspace"), _nbytes(workspace), _stream(stream)))


def _rows(t, what, dtype, n, width):
    """Address and row stride of n rows of `width` elements: a 2-D tensor, or a part of the columns of one."""
    th = _torch or _th()
    if not isinstance(t, th.Tensor) or not t.is_cuda:
        raise HchError(1, f"{what}: must be a torch tensor in GPU memory")
    if t.dtype != th.float32 if dtype == HCH_F32 else t.element_size() != 2:
        raise HchError(1, f"{what}: wrong element type {t.dtype}")
    shape = t.shape
    if len(shape) != 2 or shape[0] < n or shape[1] < width:
        raise HchError(1, f"{what}: needs {n} rows of {width} elements, has {tuple(shape)}")
    if n == 0:
        return t.data_ptr(), width
    ld, step = t.stride()
    if (step != 1 and width > 1) or (n > 1 and ld < width):
        raise HchError(1, f"{what}: the elements of a row must lie side by side and rows must not overlap")
    return t.data_ptr(), ld if n > 1 else width     # nothing lies behind the only row


def _rope(name, x_dtype, X, y_dtype, Y, coords, n, heads, rot_heads, head_dim, sections, base, scale, stream):
    tx, ty, w = _in_dtype(x_dtype), _in_dtype(y_dtype), heads * head_dim
    if len(sections) != 3:
        raise HchError(1, "sections: the pairs of three axes")
    x, ld_x = _rows(X, "first tensor", tx, n, w)
    y, ld_y = _rows(Y, "second tensor", ty, n, w)
    _check(getattr(load_library(), name)(tx, x, ld_x, ty, y, ld_y, _dp(coords, "coords", _I32, 3 * n), n, heads,
                                         rot_heads, head_dim, (C.c_int32 * 3)(*sections), base, scale, _stream(stream)))


def hch_rope_fwd(x_dtype, X, y_dtype, Y, coords, n, heads, rot_heads, head_dim, sections, base=10000.0, scale=1.0,
                 stream=None):
    """Rotary positions from coords [n][3]; X and Y are [n][heads * head_dim], or columns of wider rows."""
    _rope("hch_rope_fwd", x_dtype, X, y_dtype, Y, coords, n, heads, rot_heads, head_dim, sections, base, scale, stream)


def hch_rope_bwd(dy_dtype, dY, dx_dtype, dX, coords, n, heads, rot_heads, head_dim, sections, base=10000.0, scale=1.0,
                 stream=None):
    _rope("hch_rope_bwd", dy_dtype, dY, dx_dtype, dX, coords, n, heads, rot_heads, head_dim, sections, base, scale, stream)


def hch_attn_workspace_bytes(kind, dtype, batch, n_q, n_k, heads_q, heads_kv, head_dim):
    """kind: HCH_WS_FWD for hch_attn_fwd, HCH_WS_BWD_DATA for hch_attn_bwd."""
    d = _AttnDesc(dtype=_in_dtype(dtype), batch=batch, heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim, n_q=n_q,
                  n_k=n_k)
    return int(load_library().hch_attn_workspace_bytes(C.byref(d), kind))


def _attn_desc(dtype, Q, K, q_offsets, k_offsets, key_mask, heads_q, heads_kv, head_dim, scale):
    """Description of a call without its row strides, and the lengths of a query's and of a key's row."""
    th = _torch or _th()
    dt = _in_dtype(dtype)
    for t, what in ((Q, "Q"), (K, "K")):
        if not isinstance(t, th.Tensor) or t.dim() != 2:
            raise HchError(1, f"{what}: must be a torch tensor of rows")
    n_q, n_k = Q.shape[0], K.shape[0]
    qo, ko, mask = _dp(q_offsets, "q_offsets", _I32), _dp(k_offsets, "k_offsets", _I32), None
    batch = q_offsets.numel() - 1 if qo is not None and ko is not None else -1
    if batch < 0 or k_offsets.numel() != batch + 1:
        raise HchError(1, "q_offsets and k_offsets: batch + 1 entries each")
    if key_mask is not None:
        mask = _dp(key_mask, "key_mask", None, n_k)
        if key_mask.element_size() != 1:
            raise HchError(1, "key_mask: must have elements of one byte")
    return _AttnDesc(dt, batch, heads_q, heads_kv, head_dim, scale, n_q, n_k, qo, ko, mask), heads_q * head_dim, heads_kv * head_dim


def hch_attn_fwd(dtype, Q, K, V, O, lse, q_offsets, k_offsets, key_mask, heads_q, heads_kv, head_dim, scale, workspace,
                 stream=None):
    """Attention inside each shape: Q, O are [n_q][heads_q * head_dim], K, V [n_k][heads_kv * head_dim], or columns of
    wider rows; offsets [batch + 1] int32 on the device; lse [n_q][heads_q] float or None; key_mask [n_k] bytes or None."""
    d, wq, wk = _attn_desc(dtype, Q, K, q_offsets, k_offsets, key_mask, heads_q, heads_kv, head_dim, scale)
    q, d.ld_q = _rows(Q, "Q", dtype, d.n_q, wq)
    k, d.ld_k = _rows(K, "K", dtype, d.n_k, wk)
    v, d.ld_v = _rows(V, "V", dtype, d.n_k, wk)
    o, d.ld_o = _rows(O, "O", dtype, d.n_q, wq)
    _check(load_library().hch_attn_fwd(C.byref(d), q, k, v, o, _dp(lse, "lse", _F32, d.n_q * heads_q),
                                       _dp(workspace, "workspace"), _nbytes(workspace), _stream(stream)))


def hch_attn_bwd(dtype, Q, K, V, O, lse, dO, dQ, dK, dV, q_offsets, k_offsets, key_mask, heads_q, heads_kv, head_dim, scale,
                 workspace, stream=None):
    """Gradients of hch_attn_fwd, from its inputs, its O and its lse."""
    d, wq, wk = _attn_desc(dtype, Q, K, q_offsets, k_offsets, key_mask, heads_q, heads_kv, head_dim, scale)
    n_q, n_k = d.n_q, d.n_k
    q, d.ld_q = _rows(Q, "Q", dtype, n_q, wq)
    k, d.ld_k = _rows(K, "K", dtype, n_k, wk)
    v, d.ld_v = _rows(V, "V", dtype, n_k, wk)
    o, d.ld_o = _rows(O, "O", dtype, n_q, wq)
    do, d.ld_do = _rows(dO, "dO", dtype, n_q, wq)
    dq, d.ld_dq = _rows(dQ, "dQ", dtype, n_q, wq)
    dk, d.ld_dk = _rows(dK, "dK", dtype, n_k, wk)
    dv, d.ld_dv = _rows(dV, "dV", dtype, n_k, wk)
    _check(load_library().hch_attn_bwd(C.byref(d), q, k, v, o, _dp(lse, "lse", _F32, n_q * heads_q), do, dq, dk, dv,
                                       _dp(workspace, "workspace"), _nbytes(workspace), _stream(stream)))


def hch_probe_mfma(dtype, iters, workgroups, sink, stream=None):
    _check(load_library().hch_probe_mfma(_in_dtype(dtype), int(iters), int(workgroups),
                                         _dp(sink, "sink", _F32, workgroups * 256), _stream(stream)))


def hch_set_lean_loops(enabled):
    return int(load_library().hch_set_lean_loops(1 if enabled else 0))


def hch_kernel_count():
    return int(load_library().hch_kernel_count())


def hch_kernel_name(kernel_id):
    return load_library().hch_kernel_name(kernel_id).decode()


def hch_profile_enable(kernel_id, on):
    _check(load_library().hch_profile_enable(int(kernel_id), int(bool(on))))


def hch_profile_read(kernel_id):
    st = _KernelStats()
    _check(load_library().hch_profile_read(kernel_id, C.byref(st)))
    return dict(launches=st.launches, ms=st.ms, bytes=st.bytes, flops=st.flops)


def hch_profile_reset():
    _check(load_library().hch_profile_reset())


load_library()
