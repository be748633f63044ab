"""ctypes binding of libcsr5 (include/csr5.h).  Argument marshalling only: every
step of the conversion and of the SpMV runs in the library's HIP kernels.

Functions carry the C names.  Array arguments are torch tensors on the GPU (or
raw integer device addresses); PyTorch is used for device memory and streams
only.  A non-zero return code raises Csr5Error unless check=False.

The shared library must have been built (paper_1503_05032_amd/build.py); there
is no fallback of any kind.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcsr5.so")

CSR5_OK, CSR5_EINVAL, CSR5_ENOMEM, CSR5_EHIP, CSR5_ERANGE = 0, -1, -2, -3, -4
CSR5_OMEGA, CSR5_SIGMA_MIN, CSR5_SIGMA_MAX = 64, 1, 48
CSR5_STATIC_SCRATCH_BYTES = 4 << 20
CSR5_STATIC_MAX_TILES = CSR5_STATIC_SCRATCH_BYTES // 8 - 1
CSR5_FLAG_NONE, CSR5_FLAG_NO_HOST_CHECK = 0, 1
CSR5_FLAG_AUX_TWO_KERNELS, CSR5_FLAG_AUX_ONE_KERNEL = 2, 4
CSR5_STATUS_BAD_ROW_PTR, CSR5_STATUS_BAD_COL_IDX, CSR5_STATUS_HAS_DIRTY = 1, 2, 4
CSR5_STATUS_HAS_EMPTY_ROWS = 8
CSR5_ARRAY_TILE_PTR, CSR5_ARRAY_TILE_DESC, CSR5_ARRAY_EMPTY_OFFSET_PTR, CSR5_ARRAY_EMPTY_OFFSET = 0, 1, 2, 3
CSR5_DTYPE_F64, CSR5_DTYPE_F32, CSR5_DTYPE_BF16, CSR5_DTYPE_F16 = range(4)
CSR5_ROUTE_MAX_EXPERTS, CSR5_ROUTE_MAX_K, CSR5_NORM_MAX_N, CSR5_F8_BLOCK = 1024, 32, 32768, 128
CSR5_KERNEL_TILES, CSR5_KERNEL_PARTS, CSR5_KERNEL_WINDOW, CSR5_KERNEL_GATHERED, CSR5_KERNEL_PAIRS = range(5)

# every symbol include/csr5.h declares
SYMBOLS = [
    "csr5_sigma_auto", "csr5_workspace_bytes", "csr5_convert", "csr5_convert_ex", "csr5_spmv",
    "csr5_spmv_ex", "csr5_spmv_static", "csr5_spmv_profile", "csr5_stream_floor", "csr5_to_csr", "csr5_free", "csr5_status", "csr5_get_info",
    "csr5_get_shape", "csr5_get_form", "csr5_get_arrays",
    "csr5_read_array", "csr5_strerror", "csr5_baseline_csr_scalar", "csr5_baseline_csr_vector",
    "csr5s_convert_ex", "csr5s_spmv_ex", "csr5s_spmv_profile",
    "csr5l_workspace_bytes", "csr5l_convert_ex", "csr5l_get_arrays",
    "csr5_route_workspace_bytes", "csr5_route", "csr5_route_backward", "csr5_combine", "csr5_combine_backward",
    "csr5_grouped_gemm", "csr5_grouped_gemm_dx", "csr5_grouped_gemm_dw", "csr5_quantise", "csr5_gemm_f8",
    "csr5_grouped_gemm_f8", "csr5_rmsnorm", "csr5_rmsnorm_workspace_bytes", "csr5_rmsnorm_backward",
    "csr5_pages", "csr5_rotary", "csr5_attention", "csr5_attention_backward_workspace_bytes", "csr5_attention_backward",
    "csr5_attention_paged_workspace_bytes", "csr5_attention_paged",
]


class Csr5Error(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {csr5_strerror(code)} ({code})")


_lib = None


def load():
    """Loads libcsr5.so.  torch is imported first so that the library binds to
    the HIP runtime torch already brought into the process."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           f"`python {os.path.join(_PKG, 'build.py')}` (there is no fallback)")
    import torch  # noqa: F401
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, u32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_size_t
    lib.csr5_sigma_auto.restype = i32
    lib.csr5_sigma_auto.argtypes = [i64, i64]
    lib.csr5_workspace_bytes.restype = sz
    lib.csr5_workspace_bytes.argtypes = [i32, i32, i32]
    lib.csr5_convert.restype = C.c_int
    lib.csr5_convert.argtypes = [i32, i32, i32, vp, vp, vp, C.POINTER(vp)]
    lib.csr5_convert_ex.restype = C.c_int
    lib.csr5_convert_ex.argtypes = [i32, i32, i32, vp, vp, vp, i32, vp, sz, vp, u32, C.POINTER(vp)]
    lib.csr5s_convert_ex.restype = C.c_int
    lib.csr5s_convert_ex.argtypes = [i32, i32, i32, vp, vp, vp, i32, vp, sz, vp, u32, C.POINTER(vp)]
    lib.csr5l_workspace_bytes.restype = sz
    lib.csr5l_workspace_bytes.argtypes = [i32, i64, i32]
    lib.csr5l_convert_ex.restype = C.c_int
    lib.csr5l_convert_ex.argtypes = [i32, i32, i64, vp, vp, vp, i32, vp, sz, vp, u32, C.POINTER(vp)]
    lib.csr5l_get_arrays.restype = C.c_int
    lib.csr5l_get_arrays.argtypes = [vp] + [C.POINTER(vp)] * 4
    lib.csr5s_spmv_ex.restype = C.c_int
    lib.csr5s_spmv_ex.argtypes = [vp, vp, vp, vp]
    lib.csr5s_spmv_profile.restype = C.c_int
    lib.csr5s_spmv_profile.argtypes = [vp, vp, vp, vp, C.c_int, C.POINTER(C.c_float)]
    lib.csr5_spmv.restype = C.c_int
    lib.csr5_spmv.argtypes = [vp, vp, vp]
    lib.csr5_spmv_ex.restype = C.c_int
    lib.csr5_spmv_ex.argtypes = [vp, vp, vp, vp]
    lib.csr5_spmv_static.restype = C.c_int
    lib.csr5_spmv_static.argtypes = [vp, vp, vp, vp]
    lib.csr5_spmv_profile.restype = C.c_int
    lib.csr5_spmv_profile.argtypes = [vp, vp, vp, vp, C.c_int, C.POINTER(C.c_float)]
    lib.csr5_stream_floor.restype = C.c_int
    lib.csr5_stream_floor.argtypes = [vp, vp, C.c_size_t, vp, C.c_int, C.POINTER(C.c_float)]
    lib.csr5_to_csr.restype = C.c_int
    lib.csr5_to_csr.argtypes = [vp, vp]
    lib.csr5_free.restype = C.c_int
    lib.csr5_free.argtypes = [vp]
    lib.csr5_status.restype = C.c_int
    lib.csr5_status.argtypes = [vp, C.POINTER(u32)]
    lib.csr5_get_info.restype = C.c_int
    lib.csr5_get_info.argtypes = [vp] + [C.POINTER(i32)] * 6
    lib.csr5_get_shape.restype = C.c_int
    lib.csr5_get_shape.argtypes = [vp, C.POINTER(i32), C.POINTER(i32)]
    lib.csr5_get_form.restype = C.c_int
    lib.csr5_get_form.argtypes = [vp, vp] + [C.POINTER(i32)] * 3
    lib.csr5_get_arrays.restype = C.c_int
    lib.csr5_get_arrays.argtypes = [vp] + [C.POINTER(vp)] * 4
    lib.csr5_read_array.restype = C.c_int
    lib.csr5_read_array.argtypes = [vp, C.c_int, vp, sz]
    lib.csr5_baseline_csr_scalar.restype = C.c_int
    lib.csr5_baseline_csr_scalar.argtypes = [i32, vp, vp, vp, vp, vp, vp]
    lib.csr5_baseline_csr_vector.restype = C.c_int
    lib.csr5_baseline_csr_vector.argtypes = [i32, i32, vp, vp, vp, vp, vp, i32, vp]
    layer = {
        "csr5_route": [i32, i32, i32, C.c_int, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp],
        "csr5_route_backward": [i32, i32, i32, C.c_int, vp, vp, vp, vp, i64, vp],
        "csr5_combine": [i32, i32, i32, i32, C.c_int, vp, i64, vp, vp, vp, i64, vp, i64, vp],
        "csr5_combine_backward": [i32, i32, i32, i32, C.c_int, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp],
        "csr5_grouped_gemm": [i32, i32, i32, i32, C.c_int, vp, vp, i32, i64, vp, vp, i64, i64, vp, i64, vp],
        "csr5_grouped_gemm_dx": [i32, i32, i32, i32, C.c_int, vp, vp, i64, vp, i64, i64, vp, i64, vp],
        "csr5_grouped_gemm_dw": [i32, i32, i32, i32, C.c_int, vp, vp, i64, vp, i32, i64, vp, vp, i64, i64, vp],
        "csr5_quantise": [i32, i32, i32, C.c_int, vp, i64, vp, i64, vp, i64, i64, vp],
        "csr5_gemm_f8": [i32, i32, i32, C.c_int, vp, i64, vp, i64, i64, vp, i64, vp, i32, i64, i64, vp, i64, vp],
        "csr5_grouped_gemm_f8": [i32, i32, i32, i32, C.c_int, vp, vp, i32, i64, vp, i64, i64, vp, vp, i64, i64, vp, i32, i64, i64, i64, vp, i64, vp],
        "csr5_rmsnorm": [i32, i32, C.c_int, vp, i64, vp, i64, vp, C.c_float, vp, i64, vp, i64, vp, i64, vp, i64, i64, vp, vp],
        "csr5_rmsnorm_backward": [i32, i32, C.c_int, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp],
    }
    heads, cache = Heads, Cache
    layer.update({
        "csr5_pages": [i32, i32, i32, i32, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp],
        "csr5_rotary": [i32, i32, i32, i32, i32, C.c_int, i32, vp, i64, vp, vp, C.c_int, C.c_int, heads, heads, heads, heads, heads, vp, i32, i32, cache, cache, vp],
        "csr5_attention": [i32, i32, i32, i32, i32, i32, C.c_int, vp, vp, C.c_float, C.c_int, heads, heads, heads, heads, vp, vp],
        "csr5_attention_backward": [i32, i32, i32, i32, i32, i32, C.c_int, vp, vp, C.c_float, C.c_int, heads, heads, heads, heads, heads, vp, heads, heads, heads, vp, sz, vp],
        "csr5_attention_paged": [i32, i32, i32, i32, i32, C.c_int, vp, vp, vp, i32, i64, i32, i32, C.c_float, heads, cache, cache, heads, vp, vp, sz, vp],
    })
    for name, argtypes in layer.items():
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = argtypes
    lib.csr5_route_workspace_bytes.restype = sz
    lib.csr5_route_workspace_bytes.argtypes = [i32, i32, i32]
    lib.csr5_rmsnorm_workspace_bytes.restype = sz
    lib.csr5_rmsnorm_workspace_bytes.argtypes = [i32, i32]
    lib.csr5_attention_backward_workspace_bytes.restype = sz
    lib.csr5_attention_backward_workspace_bytes.argtypes = [i32, i32]
    lib.csr5_attention_paged_workspace_bytes.restype = sz
    lib.csr5_attention_paged_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i64]
    lib.csr5_strerror.restype = C.c_char_p
    lib.csr5_strerror.argtypes = [C.c_int]
    _lib = lib
    return lib


class Heads(C.Structure):
    """Rows of heads: csr5_heads_t."""
    _fields_ = [("p", C.c_void_p), ("row", C.c_int64), ("head", C.c_int64)]


class Cache(C.Structure):
    """Pages of rows of heads: csr5_cache_t."""
    _fields_ = [("p", C.c_void_p), ("page", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


def _ptr(t):
    """Device address of a torch tensor (or pass an int / None through)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t or None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous GPU tensor")
    return t.data_ptr() or None


_DTYPES: dict = {}      # filled on first use (torch is imported by load())


def _arr(t, dtypes, min_numel, name):
    """Device address of a torch tensor after checking what the library cannot
    check: element type and length.  A wrong one would make a kernel read or
    write outside the tensor, so it is refused here, on the host.  Integers
    (raw device addresses) and None pass through unchecked."""
    if t is None or isinstance(t, int):
        return _ptr(t)
    if not _DTYPES:
        import torch
        _DTYPES.update({"i32": torch.int32, "i64": torch.int64, "f64": torch.float64, "f32": torch.float32,
                        "u8": torch.uint8})
    if t.dtype is not _DTYPES[dtypes[0]] and not any(t.dtype is _DTYPES[d] for d in dtypes):
        raise ValueError(f"{name}: expected dtype {' or '.join(dtypes)}, got {t.dtype}")
    if t.numel() < min_numel:
        raise ValueError(f"{name}: needs at least {min_numel} elements, has {t.numel()}")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous GPU tensor")
    return t.data_ptr() or None


def _csr_args(m, n, nnz, row_ptr, col_idx, val, index, value):
    return (_arr(row_ptr, [index], m + 1, "row_ptr"), _arr(col_idx, ["i32"], nnz, "col_idx"),
            _arr(val, [value], nnz, "val"))


_current_stream = None      # returns torch's current stream on the current device, as an address


def _find_current_stream():
    """torch.cuda.current_stream() builds a Stream object, 2.9 us a call, as long as a small SpMV's kernel; torch's
    own launch code asks for the address only (0.3 us), and so does this where torch has that call."""
    import torch
    torch.cuda.current_stream()                          # initialises the device as before
    raw, device = (getattr(torch._C, f, None) for f in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(s):
    if s is None:
        global _current_stream
        if _current_stream is None:
            _current_stream = _find_current_stream()
        return _current_stream() or None
    if isinstance(s, int):
        return s or None
    return s.cuda_stream or None


def _chk(rc, where, check):
    if check and rc != CSR5_OK:
        raise Csr5Error(rc, where)
    return rc


def csr5_strerror(code):
    return load().csr5_strerror(int(code)).decode()


def csr5_sigma_auto(nnz, m):
    return int(load().csr5_sigma_auto(int(nnz), int(m)))


def csr5_workspace_bytes(m, nnz, sigma=0):
    return int(load().csr5_workspace_bytes(int(m), int(nnz), int(sigma)))


def csr5_convert(m, n, nnz, row_ptr, col_idx, val, check=True):
    """Returns the handle (an integer).  Uses the default stream and hipMalloc."""
    h = C.c_void_p()
    rc = load().csr5_convert(m, n, nnz, *_csr_args(m, n, nnz, row_ptr, col_idx, val, "i32", "f64"), C.byref(h))
    _chk(rc, "csr5_convert", check)
    return h.value if check else (rc, h.value)


def csr5_convert_ex(m, n, nnz, row_ptr, col_idx, val, sigma=0, workspace=None, stream=None,
                    flags=CSR5_FLAG_NONE, check=True):
    """`workspace` is a torch uint8 GPU tensor (or None -> hipMalloc inside)."""
    h = C.c_void_p()
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load().csr5_convert_ex(m, n, nnz, *_csr_args(m, n, nnz, row_ptr, col_idx, val, "i32", "f64"), int(sigma),
                                _arr(workspace, ["u8"], 0, "workspace"), wsb, _stream(stream), int(flags), C.byref(h))
    _chk(rc, "csr5_convert_ex", check)
    return h.value if check else (rc, h.value)


def csr5s_convert_ex(m, n, nnz, row_ptr, col_idx, val, sigma=0, workspace=None, stream=None,
                     flags=CSR5_FLAG_NONE, check=True):
    """Single precision: `val` is a float32 GPU tensor."""
    h = C.c_void_p()
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load().csr5s_convert_ex(m, n, nnz, *_csr_args(m, n, nnz, row_ptr, col_idx, val, "i32", "f32"), int(sigma),
                                 _arr(workspace, ["u8"], 0, "workspace"), wsb, _stream(stream), int(flags), C.byref(h))
    _chk(rc, "csr5s_convert_ex", check)
    return h.value if check else (rc, h.value)


def csr5l_workspace_bytes(m, nnz, sigma=0):
    return int(load().csr5l_workspace_bytes(int(m), int(nnz), int(sigma)))


def csr5l_convert_ex(m, n, nnz, row_ptr, col_idx, val, sigma=0, workspace=None, stream=None,
                     flags=CSR5_FLAG_NONE, check=True):
    """64-bit index variant: `row_ptr` is an int64 GPU tensor, nnz may exceed 2^31."""
    h = C.c_void_p()
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load().csr5l_convert_ex(m, n, int(nnz), *_csr_args(m, n, nnz, row_ptr, col_idx, val, "i64", "f64"), int(sigma),
                                 _arr(workspace, ["u8"], 0, "workspace"), wsb, _stream(stream), int(flags), C.byref(h))
    _chk(rc, "csr5l_convert_ex", check)
    return h.value if check else (rc, h.value)


def csr5l_get_arrays(h, check=True):
    """Device addresses of a 64-bit-index handle's arrays."""
    v = [C.c_void_p() for _ in range(4)]
    rc = _chk(load().csr5l_get_arrays(h, *[C.byref(a) for a in v]), "csr5l_get_arrays", check)
    if rc != CSR5_OK:
        return rc
    return dict(zip(["tile_ptr", "tile_desc", "empty_offset_ptr", "empty_offset"], [a.value for a in v]))


_shapes: dict = {}      # handle -> (m, n), so that an SpMV call costs no extra library call


def _xy(h, x, y, value):
    """x and y of an SpMV: element type of the entry point, at least n and m elements."""
    if not h:
        m, n = 0, 0
    else:
        mn = _shapes.get(h)
        if mn is None:
            mn = _shapes[h] = csr5_get_shape(h)
        m, n = mn
    return _arr(x, [value], n, "x"), _arr(y, [value], m, "y")


def csr5_get_shape(h):
    """(m, n) of the handle's matrix."""
    m, n = C.c_int32(), C.c_int32()
    _chk(load().csr5_get_shape(h, C.byref(m), C.byref(n)), "csr5_get_shape", True)
    return m.value, n.value


def csr5s_spmv_ex(h, x, y, stream=None, check=True):
    return _chk(load().csr5s_spmv_ex(h, *_xy(h, x, y, "f32"), _stream(stream)), "csr5s_spmv_ex", check)


def csr5s_spmv_profile(h, x, y, reps, stream=None):
    ms = (C.c_float * 2)()
    _chk(load().csr5s_spmv_profile(h, *_xy(h, x, y, "f32"), _stream(stream), int(reps), ms),
         "csr5s_spmv_profile", True)
    return float(ms[0]), float(ms[1])


def csr5_spmv(h, x, y, check=True):
    return _chk(load().csr5_spmv(h, *_xy(h, x, y, "f64")), "csr5_spmv", check)


def csr5_spmv_ex(h, x, y, stream=None, check=True):
    px, py = _xy(h, x, y, "f64")
    return _chk(load().csr5_spmv_ex(h, px, py, _stream(stream)), "csr5_spmv_ex", check)


def csr5_spmv_bound(h, x, y, stream=None):
    """csr5_spmv_ex (csr5s_spmv_ex for float32 tensors) with its arguments checked
    and marshalled once: returns a function of no arguments that makes the call,
    for loops that repeat one SpMV.  The tensors must stay alive and in place."""
    import torch
    f32 = not isinstance(x, int) and x is not None and x.dtype is torch.float32
    fn = load().csr5s_spmv_ex if f32 else load().csr5_spmv_ex
    where = "csr5s_spmv_ex" if f32 else "csr5_spmv_ex"
    args = (h,) + _xy(h, x, y, "f32" if f32 else "f64") + (_stream(stream),)

    def call():
        rc = fn(*args)
        if rc != CSR5_OK:
            raise Csr5Error(rc, where)
    return call


def csr5_spmv_static(h, x, y, stream=None, check=True):
    """csr5_spmv_ex without any allocation: the cross-tile array is the library's static one."""
    return _chk(load().csr5_spmv_static(h, *_xy(h, x, y, "f64"), _stream(stream)), "csr5_spmv_static", check)


def csr5_spmv_profile(h, x, y, reps, stream=None):
    """Mean kernel durations in ms: (tile kernel, carry fix-up)."""
    ms = (C.c_float * 2)()
    _chk(load().csr5_spmv_profile(h, *_xy(h, x, y, "f64"), _stream(stream), int(reps), ms),
         "csr5_spmv_profile", True)
    return float(ms[0]), float(ms[1])


def csr5_stream_floor(h, y, reps, stream=None):
    """Mean durations in ms of a bare read of the handle's tile streams: (reads only,
    reads plus the rows of y).  y (a handle-typed scratch vector) is overwritten."""
    ms = (C.c_float * 2)()
    _chk(load().csr5_stream_floor(h, _arr(y, ["f64", "f32"], 0, "y"), y.numel() * y.element_size(), _stream(stream),
                                  int(reps), ms), "csr5_stream_floor", True)
    return float(ms[0]), float(ms[1])


def csr5_to_csr(h, stream=None, check=True):
    return _chk(load().csr5_to_csr(h, _stream(stream)), "csr5_to_csr", check)


def csr5_free(h, check=True):
    _shapes.pop(h, None)
    return _chk(load().csr5_free(h), "csr5_free", check)


def csr5_status(h):
    st = C.c_uint32()
    _chk(load().csr5_status(h, C.byref(st)), "csr5_status", True)
    return st.value


def csr5_get_info(h):
    """dict(omega, sigma, p, p_complete, desc_words_per_lane, empty_offset_len)."""
    v = [C.c_int32() for _ in range(6)]
    _chk(load().csr5_get_info(h, *[C.byref(a) for a in v]), "csr5_get_info", True)
    keys = ["omega", "sigma", "p", "p_complete", "desc_words_per_lane", "empty_offset_len"]
    return {k: a.value for k, a in zip(keys, v)}


def csr5_get_form(h, stream=None):
    """dict(kernel, wave_tiles, plain): what the next SpMV of the handle on the stream would launch."""
    v = [C.c_int32() for _ in range(3)]
    _chk(load().csr5_get_form(h, _stream(stream), *[C.byref(a) for a in v]), "csr5_get_form", True)
    return {k: a.value for k, a in zip(["kernel", "wave_tiles", "plain"], v)}


def csr5_get_arrays(h, check=True):
    """Device addresses: dict(tile_ptr, tile_desc, empty_offset_ptr, empty_offset)."""
    v = [C.c_void_p() for _ in range(4)]
    rc = _chk(load().csr5_get_arrays(h, *[C.byref(a) for a in v]), "csr5_get_arrays", check)
    if rc != CSR5_OK:
        return rc
    return dict(zip(["tile_ptr", "tile_desc", "empty_offset_ptr", "empty_offset"], [a.value for a in v]))


def csr5_baseline_csr_scalar(m, row_ptr, col_idx, val, x, y, stream=None, check=True):
    nnz = 0
    return _chk(load().csr5_baseline_csr_scalar(m, _arr(row_ptr, ["i32"], m + 1, "row_ptr"), _arr(col_idx, ["i32"], nnz, "col_idx"),
                                                _arr(val, ["f64"], nnz, "val"), _arr(x, ["f64"], 0, "x"), _arr(y, ["f64"], m, "y"),
                                                _stream(stream)), "csr5_baseline_csr_scalar", check)


def csr5_baseline_csr_vector(m, nnz, row_ptr, col_idx, val, x, y, lanes_per_row=0, stream=None, check=True):
    return _chk(load().csr5_baseline_csr_vector(m, nnz, *_csr_args(m, 0, nnz, row_ptr, col_idx, val, "i32", "f64"),
                                                _arr(x, ["f64"], 0, "x"), _arr(y, ["f64"], m, "y"),
                                                int(lanes_per_row), _stream(stream)),
                "csr5_baseline_csr_vector", check)


def csr5_read_array(h, which, wide=False):
    """Host copy (NumPy) of one of the handle's arrays; wide=True for a handle
    made by csr5l_convert_ex (8-byte tile_ptr and empty_offset_ptr entries)."""
    info = csr5_get_info(h)
    count, dtype = {
        CSR5_ARRAY_TILE_PTR: (info["p"] + 1, np.uint64 if wide else np.uint32),
        CSR5_ARRAY_TILE_DESC: (info["p_complete"] * info["desc_words_per_lane"] * CSR5_OMEGA, np.uint32),
        CSR5_ARRAY_EMPTY_OFFSET_PTR: (info["p_complete"] + 1, np.int64 if wide else np.int32),
        CSR5_ARRAY_EMPTY_OFFSET: (info["empty_offset_len"], np.int32),
    }[which]
    out = np.empty(count, dtype=dtype)
    _chk(load().csr5_read_array(h, which, out.ctypes.data_as(C.c_void_p), out.nbytes),
         "csr5_read_array", True)
    return out


# ---------------------------------------------------------------------------------------------------------------------
# Products of a layer of experts (section 5 of the header).  Matrices are 2-D tensors whose rows are contiguous (views
# into wider ones are fine), weights of experts 3-D ones; sizes are taken from the tensors, and what the library cannot
# see (element types, lengths, that they are on one GPU) is checked here.  8-bit values are float8_e4m3fn or uint8 tensors.
# ---------------------------------------------------------------------------------------------------------------------
_TYPE_CODES: dict = {}      # 16- and 32-bit floating types -> dtype codes; filled on first use
_F8_TYPES: tuple = ()


def _code(t, name):
    if not _TYPE_CODES:
        import torch
        global _F8_TYPES
        load()
        _F8_TYPES = (torch.float8_e4m3fn, torch.uint8)
        _TYPE_CODES.update({torch.bfloat16: CSR5_DTYPE_BF16, torch.float16: CSR5_DTYPE_F16, torch.float32: CSR5_DTYPE_F32})
    code = _TYPE_CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: expected dtype bfloat16, float16 or float32, got {t.dtype}")
    return code


def _matrix(t, dtype, rows, cols, name):
    """Address and row stride of a matrix of `dtype` (None: 8-bit values) with exactly this shape."""
    if t.dtype is not dtype and not (dtype is None and t.dtype in _F8_TYPES):
        raise ValueError(f"{name}: expected dtype {dtype or 'float8_e4m3fn or uint8'}, got {t.dtype}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name}: expected shape {(rows, cols)}, got {tuple(t.shape)}")
    ld, step = t.stride()
    if not t.is_cuda or (step != 1 and cols > 1):
        raise ValueError(f"{name}: expected a GPU tensor with contiguous rows")
    return t.data_ptr() or None, ld if rows > 1 else max(ld, cols)


def _experts(t, dtype, groups, n, k, name):
    """Address, row stride and expert stride of weights [groups, n, k]."""
    if t.dtype is not dtype and not (dtype is None and t.dtype in _F8_TYPES):
        raise ValueError(f"{name}: expected dtype {dtype or 'float8_e4m3fn or uint8'}, got {t.dtype}")
    if t.shape != (groups, n, k):
        raise ValueError(f"{name}: expected shape {(groups, n, k)}, got {tuple(t.shape)}")
    group, ld, step = t.stride()
    if not t.is_cuda or (step != 1 and k > 1):
        raise ValueError(f"{name}: expected a GPU tensor with contiguous rows")
    return t.data_ptr() or None, ld if n > 1 else max(ld, k), group


def _stream_of(stream, *tensors):
    """The stream's address; refuses tensors of several GPUs, or of another one than the stream's (which an address does not say)."""
    gpus = {t.get_device() for t in tensors if t is not None and not isinstance(t, int)}
    if len(gpus) > 1:
        raise ValueError(f"expected tensors on one GPU, got some on GPUs {sorted(gpus)}")
    address, gpu = _stream(stream), getattr(stream, "device_index", None)
    if stream is None:
        import torch
        gpu = torch.cuda.current_device()
    if gpu is not None and gpus and gpu not in gpus:
        raise ValueError(f"the tensors are on GPU {gpus.pop()}, the stream is one of GPU {gpu}")
    return address


_marshal = None     # csrc/marshal.cpp: takes the tensors of a serving step's calls apart (and makes the same checks)


def _native():
    global _marshal
    if _marshal is None:
        load()
        path = os.path.join(_PKG, "_marshal.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python {os.path.join(_PKG, 'build.py')}` (there is no fallback)")
        from . import _marshal as module
        module.set_current_stream(lambda: _stream(None))
        _marshal = module
    return _marshal


def _space(t):
    """Address and bytes of a workspace (None: none)."""
    return (None, 0) if t is None else (_arr(t, ["u8"], 0, "workspace"), t.numel())


def csr5_route_workspace_bytes(tokens, experts, k):
    return int(load().csr5_route_workspace_bytes(int(tokens), int(experts), int(k)))


def csr5_route(logits, k, expert, weight, offset, source, place, workspace=None, stream=None, check=True):
    """The k experts of each row of `logits` [tokens, experts], their softmax, and the pairs grouped by expert.  Writes
    expert, place (int32) and weight (float32) [tokens * k], source (int32) [tokens * k] and offset (int32)
    [experts + 1]; `workspace` (uint8) has csr5_route_workspace_bytes bytes."""
    return _chk(_native().route(logits, k, expert, weight, offset, source, place, workspace, stream), "csr5_route", check)


def csr5_route_backward(expert, weight, dweight, dlogits, stream=None, check=True):
    """Writes dlogits [tokens, experts] from expert, weight and dweight [tokens, k]."""
    code = _code(dlogits, "dlogits")
    tokens, experts = dlogits.shape
    k = expert.shape[1]
    return _chk(load().csr5_route_backward(tokens, experts, k, code, _arr(expert, ["i32"], tokens * k, "expert"),
                                           _arr(weight, ["f32"], tokens * k, "weight"), _arr(dweight, ["f32"], tokens * k, "dweight"),
                                           *_matrix(dlogits, dlogits.dtype, tokens, experts, "dlogits"), _stream_of(stream, expert, weight, dweight, dlogits)),
                "csr5_route_backward", check)


def csr5_combine(z, place, y, weight=None, residual=None, stream=None, check=True):
    """y[t] = residual[t] + sum_j weight[t, j] * z[place[t, j]]; place and weight [tokens, k], z [rows, n]."""
    return _chk(_native().combine(z, place, y, weight, residual, stream), "csr5_combine", check)


def csr5_combine_backward(dy, z, place, weight, dz, dweight, stream=None, check=True):
    """Writes dz [rows, n] and dweight [tokens, k]."""
    code, dt = _code(z, "z"), z.dtype
    rows, n = z.shape
    tokens, k = place.shape
    return _chk(load().csr5_combine_backward(tokens, k, rows, n, code, *_matrix(dy, dt, tokens, n, "dy"), *_matrix(z, dt, rows, n, "z"),
                                             _arr(place, ["i32"], tokens * k, "place"), _arr(weight, ["f32"], tokens * k, "weight"),
                                             *_matrix(dz, dt, rows, n, "dz"), _arr(dweight, ["f32"], tokens * k, "dweight"),
                                             _stream_of(stream, dy, z, place, weight, dz, dweight)), "csr5_combine_backward", check)


def _source(source, rows, x_rows):
    if source is None:
        if x_rows < rows:
            raise ValueError(f"x: needs {rows} rows without source, has {x_rows}")
        return None
    return _arr(source, ["i32"], rows, "source")


def csr5_grouped_gemm(x, w, offset, y, source=None, stream=None, check=True):
    """y[r] = w[g] x[source[r]] for the rows r of each group g; x [x_rows, k], w [groups, n, k], y [rows, n]."""
    return _chk(_native().grouped_gemm(x, w, offset, y, source, stream), "csr5_grouped_gemm", check)


def csr5_grouped_gemm_dx(dy, w, offset, dx, stream=None, check=True):
    """dx[r] = w[g]^T dy[r] for the rows r of each group g; dy [rows, n], w [groups, n, k], dx [rows, k]."""
    code, dt = _code(dy, "dy"), dy.dtype
    rows, n = dy.shape
    groups, k = w.shape[0], w.shape[2]
    return _chk(load().csr5_grouped_gemm_dx(groups, rows, n, k, code, _arr(offset, ["i32"], groups + 1, "offset"), *_matrix(dy, dt, rows, n, "dy"),
                                            *_experts(w, dt, groups, n, k, "w"), *_matrix(dx, dt, rows, k, "dx"), _stream_of(stream, dy, w, offset, dx)),
                "csr5_grouped_gemm_dx", check)


def csr5_grouped_gemm_dw(dy, x, offset, dw, source=None, stream=None, check=True):
    """dw[g] = sum over the rows r of group g of dy[r] x[source[r]]^T; dy [rows, n], x [x_rows, k], dw [groups, n, k]."""
    code, dt = _code(dy, "dy"), dy.dtype
    rows, n = dy.shape
    x_rows, k = x.shape
    groups = dw.shape[0]
    px, ldx = _matrix(x, dt, x_rows, k, "x")
    return _chk(load().csr5_grouped_gemm_dw(groups, rows, n, k, code, _arr(offset, ["i32"], groups + 1, "offset"), *_matrix(dy, dt, rows, n, "dy"),
                                            px, x_rows, ldx, _source(source, rows, x_rows), *_experts(dw, dt, groups, n, k, "dw"),
                                            _stream_of(stream, dy, x, offset, dw, source)), "csr5_grouped_gemm_dw", check)


def csr5_quantise(x, q, scale, block_rows=1, stream=None, check=True):
    """q [rows, n] in 8 bits and scale [ceil(rows / block_rows), ceil(n / 128)] of x [rows, n]; block_rows 1 or 128."""
    return _chk(_native().quantise(x, q, scale, block_rows, stream), "csr5_quantise", check)


def csr5_gemm_f8(x, x_scale, w, w_scale, y, w_rows=CSR5_F8_BLOCK, stream=None, check=True):
    """y [m, n] = x [m, k] times w [n, k] transposed, both in 8 bits, with x_scale [m, ceil(k / 128)] and w_scale
    [ceil(n / w_rows), ceil(k / 128)]; w_rows 128 or 1."""
    return _chk(_native().gemm_f8(x, x_scale, w, w_scale, y, w_rows, stream), "csr5_gemm_f8", check)


def csr5_grouped_gemm_f8(x, x_scale, w, w_scale, offset, y, w_rows=CSR5_F8_BLOCK, source=None, stream=None, check=True):
    """csr5_grouped_gemm in 8 bits: x_scale [x_rows, ceil(k / 128)], w_scale [groups, ceil(n / w_rows), ceil(k / 128)]."""
    return _chk(_native().grouped_gemm_f8(x, x_scale, w, w_scale, offset, y, w_rows, source, stream), "csr5_grouped_gemm_f8", check)


def csr5_rmsnorm(x, gain, eps, residual=None, h=None, y=None, q=None, scale=None, rstd=None, stream=None, check=True):
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * gain by rows of x [rows, n]; writes those of h, y, q with scale
    [rows, ceil(n / 128)], and rstd [rows] that are given.  gain (or None: ones) [n]."""
    return _chk(_native().rmsnorm(x, gain, eps, residual, h, y, q, scale, rstd, stream), "csr5_rmsnorm", check)


def csr5_rmsnorm_workspace_bytes(rows, n):
    return int(load().csr5_rmsnorm_workspace_bytes(int(rows), int(n)))


def csr5_rmsnorm_backward(h, gain, rstd, dy, dh, dgain=None, workspace=None, residual_grad=None, stream=None, check=True):
    """dh [rows, n] (of x and the residual alike) and dgain [n] (float32) from dy and residual_grad [rows, n]; `workspace`
    (uint8, needed for dgain) has csr5_rmsnorm_workspace_bytes bytes."""
    code, dt = _code(h, "h"), h.dtype
    rows, n = h.shape
    if gain is not None and (gain.dtype is not dt or gain.shape != (n,) or not gain.is_cuda or not gain.is_contiguous()):
        raise ValueError(f"gain: expected a contiguous GPU tensor of {n} values of {dt}")
    return _chk(load().csr5_rmsnorm_backward(rows, n, code, *_matrix(h, dt, rows, n, "h"), None if gain is None else gain.data_ptr() or None,
                                             _arr(rstd, ["f32"], rows, "rstd"), *_matrix(dy, dt, rows, n, "dy"),
                                             *((None, 0) if residual_grad is None else _matrix(residual_grad, dt, rows, n, "residual_grad")),
                                             *_matrix(dh, dt, rows, n, "dh"), _arr(dgain, ["f32"], n, "dgain"), *_space(workspace),
                                             _stream_of(stream, h, gain, rstd, dy, dh, dgain, workspace, residual_grad)), "csr5_rmsnorm_backward", check)


# ---------------------------------------------------------------------------------------------------------------------
# The attention beside a layer of experts (section 6 of the header).  Queries, keys and values are 3-D tensors [rows, heads,
# d] at any strides whose heads are contiguous (views of one wide product, say), caches 4-D ones [pages, page, kv_heads, d].
# ---------------------------------------------------------------------------------------------------------------------
def csr5_pages(fresh, length, table, pool, state, page, offset, position, slot, length_out, state_out, stream=None, check=True):
    """The pages of a step of serving.  From fresh (new tokens; below 0: over) and length (cached ones) [requests], writes
    offset [requests + 1], position and slot [tokens], length_out [requests] and state_out [2], new pages into table
    [requests, width], and pages of requests that are over into the ring `pool`, whose free ones state [2] (first, count)
    names; all int32, and none that is written a part of another.  `page` tokens to a page, a power of two."""
    return _chk(_native().pages(fresh, length, table, pool, state, page, offset, position, slot, length_out, state_out, stream), "csr5_pages", check)


def csr5_rotary(q, k, position, frequency, q_out, k_out=None, axis=None, interleaved=False, inverse=False, v=None, slot=None, k_cache=None, v_cache=None, stream=None, check=True):
    """q [tokens, heads, d] and k [tokens, kv_heads, d] (or None) turned by position[axis[i]] * frequency[i] for pair i, backwards
    with `inverse` (the gradient), to q_out, and to k_out or, with v as it is, to slot[token] of k_cache and v_cache [pages, page, kv_heads, d].
    position int32 [tokens] or [axes, tokens], frequency float32 [rot / 2], axis int32 [rot / 2] (or None: all of axis 0), slot int32 [tokens]."""
    return _chk(_native().rotary(q, k, position, frequency, q_out, k_out, axis, interleaved, inverse, v, slot, k_cache, v_cache, stream), "csr5_rotary", check)


def csr5_attention(q, k, v, q_offset, k_offset, out, lse=None, scale=None, causal=True, stream=None, check=True):
    """Attention over packed sequences: q and out [rows, heads, d], k and v [k_rows, kv_heads, d], q_offset and k_offset int32
    [sequences + 1], lse float32 [heads, rows]; scale: d^-0.5 where it is None."""
    return _chk(_native().attention(q, k, v, q_offset, k_offset, out, lse, scale, causal, stream), "csr5_attention", check)


def csr5_attention_backward_workspace_bytes(rows, heads):
    return int(load().csr5_attention_backward_workspace_bytes(int(rows), int(heads)))


def csr5_attention_backward(dout, q, k, v, out, lse, q_offset, k_offset, dq, dk, dv, workspace, scale=None, causal=True, stream=None, check=True):
    """Gradients dq, dk and dv of csr5_attention from dout, out and lse; `workspace` (uint8) has
    csr5_attention_backward_workspace_bytes bytes."""
    return _chk(_native().attention_backward(dout, q, k, v, out, lse, q_offset, k_offset, dq, dk, dv, workspace, scale, causal, stream), "csr5_attention_backward", check)


def csr5_attention_paged_workspace_bytes(rows, heads, kv_heads, d, sequences, max_length):
    return int(load().csr5_attention_paged_workspace_bytes(int(rows), int(heads), int(kv_heads), int(d), int(sequences), int(max_length)))


def csr5_attention_paged(q, k_cache, v_cache, q_offset, length, table, out, workspace=None, lse=None, scale=None, stream=None, check=True):
    """Causal attention of each request's last tokens, q and out [rows, heads, d], over length[s] tokens in the pages table[s] of
    k_cache and v_cache [pages, page, kv_heads, d]; `workspace` (uint8) has csr5_attention_paged_workspace_bytes bytes, with
    max_length = table.shape[1] * page."""
    return _chk(_native().attention_paged(q, k_cache, v_cache, q_offset, length, table, out, workspace, lse, scale, stream), "csr5_attention_paged", check)
