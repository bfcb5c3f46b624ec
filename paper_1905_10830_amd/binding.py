"""ctypes binding of libfmtc.so: argument marshalling only.

Every function has the name of the C entry point without the `fmtc_` prefix
and passes torch device tensors as raw pointers on torch's current HIP
stream.  There is no CPU path: if the library is missing or has not been
built the first call raises.
"""
import ctypes
import operator
import os

NCHW, NHWC = 0, 1
OK, EINVAL, EBUFSIZE, ECORRUPT, ENOMEM, EHIP = range(6)
ERR_HEADER, ERR_TABLE, ERR_OFFSETS, ERR_CODE = 1, 2, 4, 8
F32, BF16, F16 = range(3)
E4M3, E5M2 = range(2)
SCALE_F32, SCALE_E8M0 = range(2)
F8_BLOCK = 128

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfmtc.so")

EXPORTS = [
    "fmtc_fit_basis", "fmtc_basis_import", "fmtc_basis_export", "fmtc_basis_channels", "fmtc_basis_destroy",
    "fmtc_delta", "fmtc_encode_bound", "fmtc_workspace_size", "fmtc_encode", "fmtc_encode_noalloc", "fmtc_decode",
    "fmtc_quantize",
    "fmtc_code_symbols", "fmtc_decode_symbols", "fmtc_stream_info", "fmtc_last_error",
    "fmtc_fit_table", "fmtc_table_import", "fmtc_table_export", "fmtc_table_destroy", "fmtc_encode_static_bound",
    "fmtc_encode_static", "fmtc_decode_static",
    "fmtc_fit_state_create", "fmtc_fit_state_update", "fmtc_fit_state_basis", "fmtc_fit_state_count",
    "fmtc_fit_state_destroy", "fmtc_basis_truncate",
    "fmtc_basis8_create", "fmtc_basis8_export", "fmtc_basis8_destroy", "fmtc_quantize_u8", "fmtc_reconstruct_u8",
    "fmtc_encode_u8", "fmtc_decode_u8",
    "fmtc_f8_quantize", "fmtc_f8_matmul_workspace_size", "fmtc_f8_matmul", "fmtc_f8_matmul_backward_workspace_size",
    "fmtc_f8_matmul_backward", "fmtc_block_norm", "fmtc_block_norm_workspace_size", "fmtc_block_norm_backward",
    "fmtc_profile_enable", "fmtc_profile_kernels", "fmtc_profile_name", "fmtc_profile_read", "fmtc_profile_copy",
    "fmtc_test_option", "fmtc_test_projection",
]

_lib = None


class _F8(ctypes.Structure):
    _fields_ = [("d_codes", ctypes.c_void_p), ("d_scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("depth", ctypes.c_int64), ("ld", ctypes.c_int64), ("ld_scales", ctypes.c_int64),
                ("format", ctypes.c_int32), ("scale", ctypes.c_int32), ("block_rows", ctypes.c_int32)]


class _Norm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("C", ctypes.c_int32), ("type", ctypes.c_int32),
                ("weight_type", ctypes.c_int32), ("reserved", ctypes.c_int32), ("d_y", ctypes.c_void_p),
                ("d_h", ctypes.c_void_p), ("ld_y", ctypes.c_int64), ("ld_h", ctypes.c_int64),
                ("d_w_post", ctypes.c_void_p), ("d_w_pre", ctypes.c_void_p), ("d_gate", ctypes.c_void_p),
                ("rows_per_gate", ctypes.c_int64), ("skip", ctypes.c_float), ("scale", ctypes.c_float),
                ("eps", ctypes.c_float)]


class FmtcError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"fmtc status {status}: {message}")
        self.status = status


def load_library():
    """Loads libfmtc.so (built by paper_1905_10830_amd.build).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build it with `python -m paper_1905_10830_amd.build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, sz, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
    lib.fmtc_fit_basis.argtypes = [vp, i64, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
    lib.fmtc_basis_import.argtypes = [i32, vp, vp, f32, ctypes.POINTER(vp)]
    lib.fmtc_basis_export.argtypes = [vp, vp, vp, vp, ctypes.POINTER(f32)]
    lib.fmtc_basis_channels.argtypes = [vp]
    lib.fmtc_basis_destroy.argtypes = [vp]
    lib.fmtc_basis_destroy.restype = None
    lib.fmtc_fit_state_create.argtypes = [i32, ctypes.POINTER(vp)]
    lib.fmtc_fit_state_update.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp]
    lib.fmtc_fit_state_basis.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
    lib.fmtc_fit_state_count.argtypes = [vp]
    lib.fmtc_fit_state_count.restype = i64
    lib.fmtc_fit_state_destroy.argtypes = [vp]
    lib.fmtc_fit_state_destroy.restype = None
    lib.fmtc_basis_truncate.argtypes = [vp, i32, ctypes.POINTER(vp)]
    lib.fmtc_basis8_create.argtypes = [vp, f32, ctypes.POINTER(vp)]
    lib.fmtc_basis8_export.argtypes = [vp, vp, ctypes.POINTER(f32), vp, ctypes.POINTER(f32), ctypes.POINTER(f32)]
    lib.fmtc_basis8_destroy.argtypes = [vp]
    lib.fmtc_basis8_destroy.restype = None
    lib.fmtc_quantize_u8.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, vp, vp]
    lib.fmtc_reconstruct_u8.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, vp, vp]
    lib.fmtc_encode_u8.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, i32, vp, sz, vp, vp, sz, vp]
    lib.fmtc_decode_u8.argtypes = [vp, vp, sz, vp, i64, i32, i32, i32, i32, i32, vp, vp, sz, vp]
    lib.fmtc_delta.argtypes = [f32, i32]
    lib.fmtc_delta.restype = f32
    lib.fmtc_encode_bound.argtypes = [i64, i32, i32, i32]
    lib.fmtc_encode_bound.restype = sz
    lib.fmtc_workspace_size.argtypes = [i64, i32, i32, i32]
    lib.fmtc_workspace_size.restype = sz
    lib.fmtc_encode.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, i32, vp, sz, vp, vp, sz, vp]
    lib.fmtc_encode_noalloc.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, i32, vp, sz, vp, vp]
    lib.fmtc_decode.argtypes = [vp, vp, sz, vp, i64, i32, i32, i32, i32, i32, vp, vp]
    lib.fmtc_fit_table.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
    lib.fmtc_table_import.argtypes = [vp, i32, ctypes.POINTER(vp)]
    lib.fmtc_table_export.argtypes = [vp, vp, ctypes.POINTER(i32)]
    lib.fmtc_table_destroy.argtypes = [vp]
    lib.fmtc_table_destroy.restype = None
    lib.fmtc_encode_static_bound.argtypes = [vp, i64, i32, i32]
    lib.fmtc_encode_static_bound.restype = sz
    lib.fmtc_encode_static.argtypes = [vp, vp, vp, i64, i32, i32, i32, i32, i32, vp, sz, vp, vp, sz, vp]
    lib.fmtc_decode_static.argtypes = [vp, vp, vp, sz, vp, i64, i32, i32, i32, i32, vp, vp]
    lib.fmtc_quantize.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.fmtc_code_symbols.argtypes = [vp, i64, i32, i32, i32, f32, vp, sz, vp, vp, sz, vp]
    lib.fmtc_decode_symbols.argtypes = [vp, sz, i64, i32, i32, vp, vp, vp]
    lib.fmtc_stream_info.argtypes = [vp, sz, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i64),
                                     ctypes.POINTER(i32), ctypes.POINTER(i64), ctypes.POINTER(f32),
                                     ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint64)]
    f8 = ctypes.POINTER(_F8)
    lib.fmtc_f8_quantize.argtypes = [vp, i32, i64, i64, i64, f8, f8, vp]
    lib.fmtc_f8_matmul_workspace_size.argtypes = [i64, i64, i64]
    lib.fmtc_f8_matmul_workspace_size.restype = sz
    lib.fmtc_f8_matmul.argtypes = [f8, f8, vp, vp, i32, i64, i32, vp, sz, vp]
    lib.fmtc_f8_matmul_backward_workspace_size.argtypes = [i64, i64, i64]
    lib.fmtc_f8_matmul_backward_workspace_size.restype = sz
    lib.fmtc_f8_matmul_backward.argtypes = [vp, i32, i64, i64, i64, f8, f8, i32, i32, vp, i32, i64, vp, i64, vp, i32, vp,
                                            sz, vp]
    lib.fmtc_block_norm.argtypes = [ctypes.POINTER(_Norm), vp, i64, vp, i64, f8, vp, vp]
    lib.fmtc_block_norm_workspace_size.argtypes = [i64, i32, i64]
    lib.fmtc_block_norm_workspace_size.restype = sz
    lib.fmtc_block_norm_backward.argtypes = [ctypes.POINTER(_Norm), vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp,
                                             sz, vp]
    lib.fmtc_last_error.restype = ctypes.c_char_p
    lib.fmtc_profile_enable.argtypes = [i32]
    lib.fmtc_profile_name.argtypes = [i32]
    lib.fmtc_profile_name.restype = ctypes.c_char_p
    lib.fmtc_profile_read.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                                      ctypes.POINTER(i32)]
    lib.fmtc_profile_copy.argtypes = [vp, vp, sz, vp]
    lib.fmtc_test_option.argtypes = [i32, i32]
    lib.fmtc_test_projection.argtypes = [i64, i32, i32, i32, i32, i32, i32, ctypes.c_char_p, sz]
    _lib = lib
    return lib


def _check(status):
    if status != OK:
        raise FmtcError(status, load_library().fmtc_last_error().decode())


def _stream():
    import torch

    try:  # the same stream as below, without the object around it (3 us of a call that launches one kernel)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream


def _dims(x, layout):
    if x.dim() != 4:
        raise ValueError("expected a 4-d tensor")
    if layout == NHWC:
        n, h, w, c = x.shape
    else:
        n, c, h, w = x.shape
    return n, c, h, w


def _dev(t, dtype):
    import torch

    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise ValueError(f"expected a contiguous device tensor of {dtype}")
    return ctypes.c_void_p(t.data_ptr())


class Basis:
    """Owns an fmtc_basis handle."""

    def __init__(self, handle):
        self._h = handle

    @property
    def C(self):
        return load_library().fmtc_basis_channels(self._h)

    def export(self):
        """-> T (C,C) fp32, mu (C) fp32, eigenvalues (C) fp64, range A (numpy / float)."""
        import numpy as np

        c = self.C
        T = np.empty((c, c), np.float32)
        mu = np.empty(c, np.float32)
        eig = np.empty(c, np.float64)
        A = ctypes.c_float(0)
        _check(load_library().fmtc_basis_export(self._h, T.ctypes.data, mu.ctypes.data, eig.ctypes.data,
                                                ctypes.byref(A)))
        return T, mu, eig, np.float32(A.value)

    def truncate(self, keep):
        """-> a new Basis that keeps the `keep` leading components (the other rows of T are zero)."""
        out = ctypes.c_void_p()
        _check(load_library().fmtc_basis_truncate(self._h, int(keep), ctypes.byref(out)))
        return Basis(out)

    def close(self):
        if self._h:
            load_library().fmtc_basis_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def fit_basis(x, layout=NHWC):
    import torch

    n, c, h, w = _dims(x, layout)
    out = ctypes.c_void_p()
    _check(load_library().fmtc_fit_basis(_dev(x, torch.float32), n, c, h, w, layout, _stream(), ctypes.byref(out)))
    return Basis(out)


class Basis8:
    """Owns an fmtc_basis8 handle: the 8-bit basis for unsigned 8-bit activations x = act_scale * xq."""

    def __init__(self, basis, act_scale):
        self._h = ctypes.c_void_p()
        _check(load_library().fmtc_basis8_create(basis._h, float(act_scale), ctypes.byref(self._h)))
        self.C = basis.C

    def export(self):
        """-> Tq int8 (C,C), s_T, mean_fix int32 (C), act_scale, range A."""
        import numpy as np

        Tq = np.empty((self.C, self.C), np.int8)
        mf = np.empty(self.C, np.int32)
        sT, sx, A = ctypes.c_float(0), ctypes.c_float(0), ctypes.c_float(0)
        _check(load_library().fmtc_basis8_export(self._h, Tq.ctypes.data, ctypes.byref(sT), mf.ctypes.data,
                                                 ctypes.byref(sx), ctypes.byref(A)))
        return Tq, np.float32(sT.value), mf, np.float32(sx.value), np.float32(A.value)

    def close(self):
        if self._h:
            load_library().fmtc_basis8_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def quantize_u8(basis8, xq, bits, layout=NHWC, syms=None):
    """Asynchronous.  xq: uint8 device tensor (4-d).  -> symbols uint8 [P, C]."""
    import torch

    n, c, h, w = _dims(xq, layout)
    if syms is None:
        syms = torch.empty((n * h * w, c), dtype=torch.uint8, device=xq.device)
    _check(load_library().fmtc_quantize_u8(basis8._h, _dev(xq, torch.uint8), n, c, h, w, layout, bits,
                                           _dev(syms, torch.uint8), _stream()))
    return syms


def reconstruct_u8(basis8, syms, shape, bits, layout=NHWC, out=None):
    """Asynchronous.  symbols [P, C] -> uint8 activations of the 4-d `shape`."""
    import torch

    if out is None:
        out = torch.empty(tuple(shape), dtype=torch.uint8, device=syms.device)
    n, c, h, w = _dims(out, layout)
    _check(load_library().fmtc_reconstruct_u8(basis8._h, _dev(syms, torch.uint8), n, c, h, w, layout, bits,
                                              _dev(out, torch.uint8), _stream()))
    return out


def encode_u8(basis8, xq, bits, layout=NHWC, chunk_syms=4096, stream_out=None, out_bytes=None, workspace=None):
    """Asynchronous.  -> (stream_out uint8 tensor of capacity encode_bound, out_bytes int64[1] device tensor)."""
    import torch

    n, c, h, w = _dims(xq, layout)
    P = n * h * w
    if stream_out is None:
        stream_out = torch.empty(encode_bound(P, c, bits, chunk_syms), dtype=torch.uint8, device=xq.device)
    if out_bytes is None:
        out_bytes = torch.zeros(1, dtype=torch.int64, device=xq.device)
    if workspace is None:
        workspace = torch.empty(workspace_size(P, c, bits, chunk_syms), dtype=torch.uint8, device=xq.device)
    _check(load_library().fmtc_encode_u8(basis8._h, _dev(xq, torch.uint8), n, c, h, w, layout, bits, chunk_syms,
                                         _dev(stream_out, torch.uint8), stream_out.numel(),
                                         ctypes.c_void_p(out_bytes.data_ptr()), _dev(workspace, torch.uint8),
                                         workspace.numel(), _stream()))
    return stream_out, out_bytes


def decode_u8(basis8, stream_in, shape, bits, layout=NHWC, out=None, err_flag=None, nbytes=None, workspace=None):
    """Asynchronous.  -> (uint8 activations of `shape`, err_flag int32[1] device tensor)."""
    import torch

    if out is None:
        out = torch.empty(tuple(shape), dtype=torch.uint8, device=stream_in.device)
    if err_flag is None:
        err_flag = torch.zeros(1, dtype=torch.int32, device=stream_in.device)
    n, c, h, w = _dims(out, layout)
    if workspace is None and c > 128:  # narrower tensors are decoded and reconstructed by one kernel
        workspace = torch.empty(n * h * w * c, dtype=torch.uint8, device=stream_in.device)
    _check(load_library().fmtc_decode_u8(basis8._h, _dev(stream_in, torch.uint8),
                                         stream_in.numel() if nbytes is None else int(nbytes),
                                         _dev(out, torch.uint8), n, c, h, w, layout, bits,
                                         ctypes.c_void_p(err_flag.data_ptr()),
                                         None if workspace is None else _dev(workspace, torch.uint8),
                                         0 if workspace is None else workspace.numel(), _stream()))
    return out, err_flag


class FitState:
    """Owns an fmtc_fit_state handle: calibration statistics accumulated over several tensors."""

    def __init__(self, C):
        self._h = ctypes.c_void_p()
        _check(load_library().fmtc_fit_state_create(int(C), ctypes.byref(self._h)))

    @property
    def count(self):
        return load_library().fmtc_fit_state_count(self._h)

    def update(self, x, layout=NHWC):
        import torch

        n, c, h, w = _dims(x, layout)
        _check(load_library().fmtc_fit_state_update(self._h, _dev(x, torch.float32), n, c, h, w, layout, _stream()))

    def basis(self, x, layout=NHWC):
        """Basis of everything seen so far; the dynamic range is measured on x."""
        import torch

        n, c, h, w = _dims(x, layout)
        out = ctypes.c_void_p()
        _check(load_library().fmtc_fit_state_basis(self._h, _dev(x, torch.float32), n, c, h, w, layout, _stream(),
                                                   ctypes.byref(out)))
        return Basis(out)

    def close(self):
        if self._h:
            load_library().fmtc_fit_state_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def basis_import(T, mu, range_A):
    import numpy as np

    T = np.ascontiguousarray(T, dtype=np.float32)
    mu = np.ascontiguousarray(mu, dtype=np.float32)
    out = ctypes.c_void_p()
    _check(load_library().fmtc_basis_import(T.shape[0], T.ctypes.data, mu.ctypes.data, float(range_A),
                                            ctypes.byref(out)))
    return Basis(out)


def delta(range_A, bits):
    return load_library().fmtc_delta(float(range_A), int(bits))


def encode_bound(P, C, bits, chunk_syms=4096):
    return load_library().fmtc_encode_bound(P, C, bits, chunk_syms)


def workspace_size(P, C, bits, chunk_syms=4096):
    return load_library().fmtc_workspace_size(P, C, bits, chunk_syms)


def encode(basis, x, bits, layout=NHWC, chunk_syms=4096, stream_out=None, out_bytes=None, workspace=None):
    """Asynchronous.  -> (stream_out uint8 tensor of capacity encode_bound, out_bytes int64[1] device tensor)."""
    import torch

    n, c, h, w = _dims(x, layout)
    P = n * h * w
    if stream_out is None:
        stream_out = torch.empty(encode_bound(P, c, bits, chunk_syms), dtype=torch.uint8, device=x.device)
    if out_bytes is None:
        out_bytes = torch.zeros(1, dtype=torch.int64, device=x.device)
    if workspace is None:
        workspace = torch.empty(workspace_size(P, c, bits, chunk_syms), dtype=torch.uint8, device=x.device)
    _check(load_library().fmtc_encode(basis._h, _dev(x, torch.float32), n, c, h, w, layout, bits, chunk_syms,
                                      _dev(stream_out, torch.uint8), stream_out.numel(),
                                      _dev(out_bytes, torch.int64), _dev(workspace, torch.uint8),
                                      workspace.numel(), _stream()))
    return stream_out, out_bytes


NOALLOC_SCRATCH_BYTES = 6 << 20


def encode_noalloc(basis, x, bits, stream_out, out_bytes, layout=NHWC, chunk_syms=4096):
    """Asynchronous.  fmtc_encode with the workspace in the library's own device array; the caller brings the
    outputs (nothing is allocated here either)."""
    import torch

    n, c, h, w = _dims(x, layout)
    _check(load_library().fmtc_encode_noalloc(basis._h, _dev(x, torch.float32), n, c, h, w, layout, bits, chunk_syms,
                                              _dev(stream_out, torch.uint8), stream_out.numel(),
                                              _dev(out_bytes, torch.int64), _stream()))
    return stream_out, out_bytes


class Table:
    """Owns an fmtc_table handle (a code table fixed at calibration time)."""

    def __init__(self, handle):
        self._h = handle

    def export(self):
        """-> (code lengths uint8[2^bits] numpy, bits)."""
        import numpy as np

        ln = np.zeros(256, np.uint8)
        bits = ctypes.c_int32(0)
        _check(load_library().fmtc_table_export(self._h, ln.ctypes.data, ctypes.byref(bits)))
        return ln[: 1 << bits.value].copy(), bits.value

    @property
    def bits(self):
        return self.export()[1]

    def close(self):
        if self._h:
            load_library().fmtc_table_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def fit_table(basis, x, bits, layout=NHWC):
    import torch

    n, c, h, w = _dims(x, layout)
    out = ctypes.c_void_p()
    _check(load_library().fmtc_fit_table(basis._h, _dev(x, torch.float32), n, c, h, w, layout, bits, _stream(),
                                         ctypes.byref(out)))
    return Table(out)


def table_import(lengths, bits):
    import numpy as np

    ln = np.ascontiguousarray(lengths, dtype=np.uint8)
    if ln.size != 1 << bits:
        raise ValueError("one length per symbol of the alphabet")
    out = ctypes.c_void_p()
    _check(load_library().fmtc_table_import(ln.ctypes.data, bits, ctypes.byref(out)))
    return Table(out)


def encode_static_bound(table, P, C, chunk_syms=4096):
    return load_library().fmtc_encode_static_bound(table._h, P, C, chunk_syms)


def encode_static(basis, table, x, layout=NHWC, chunk_syms=4096, stream_out=None, out_bytes=None, workspace=None):
    """Asynchronous.  -> (stream_out uint8 tensor, out_bytes int64[1] device tensor)."""
    import torch

    n, c, h, w = _dims(x, layout)
    P = n * h * w
    bits = table.bits
    if stream_out is None:
        stream_out = torch.empty(encode_static_bound(table, P, c, chunk_syms), dtype=torch.uint8, device=x.device)
    if out_bytes is None:
        out_bytes = torch.zeros(1, dtype=torch.int64, device=x.device)
    if workspace is None:
        workspace = torch.empty(workspace_size(P, c, bits, chunk_syms), dtype=torch.uint8, device=x.device)
    _check(load_library().fmtc_encode_static(basis._h, table._h, _dev(x, torch.float32), n, c, h, w, layout,
                                             chunk_syms, _dev(stream_out, torch.uint8), stream_out.numel(),
                                             _dev(out_bytes, torch.int64), _dev(workspace, torch.uint8),
                                             workspace.numel(), _stream()))
    return stream_out, out_bytes


def decode_static(basis, table, stream_in, shape, layout=NHWC, xhat=None, err_flag=None, nbytes=None):
    """Asynchronous.  -> (xhat fp32 tensor of `shape`, err_flag int32[1] device tensor)."""
    import torch

    if xhat is None:
        xhat = torch.empty(shape, dtype=torch.float32, device=stream_in.device)
    if err_flag is None:
        err_flag = torch.zeros(1, dtype=torch.int32, device=stream_in.device)
    n, c, h, w = _dims(xhat, layout)
    _check(load_library().fmtc_decode_static(basis._h, table._h, _dev(stream_in, torch.uint8),
                                             stream_in.numel() if nbytes is None else nbytes,
                                             _dev(xhat, torch.float32), n, c, h, w, layout,
                                             _dev(err_flag, torch.int32), _stream()))
    return xhat, err_flag


def decode(basis, stream_in, shape, bits, layout=NHWC, xhat=None, err_flag=None, nbytes=None):
    """Asynchronous.  -> (xhat fp32 tensor of `shape`, err_flag int32[1] device tensor).
    A caller-supplied err_flag must be zero on entry: the decoder only ORs bits into it."""
    import torch

    if xhat is None:
        xhat = torch.empty(shape, dtype=torch.float32, device=stream_in.device)
    if err_flag is None:
        err_flag = torch.zeros(1, dtype=torch.int32, device=stream_in.device)
    n, c, h, w = _dims(xhat, layout)
    _check(load_library().fmtc_decode(basis._h, _dev(stream_in, torch.uint8),
                                      stream_in.numel() if nbytes is None else int(nbytes),
                                      _dev(xhat, torch.float32), n, c, h, w, layout, bits,
                                      _dev(err_flag, torch.int32), _stream()))
    return xhat, err_flag


def quantize(basis, x, bits, layout=NHWC, syms=None, hist=None, workspace=None):
    """Asynchronous.  -> (symbols uint8 [P, C], histogram int32 [256])."""
    import torch

    n, c, h, w = _dims(x, layout)
    P = n * h * w
    if syms is None:
        syms = torch.empty((P, c), dtype=torch.uint8, device=x.device)
    if hist is None:
        hist = torch.zeros(256, dtype=torch.int32, device=x.device)
    if workspace is None:
        workspace = torch.empty(workspace_size(P, c, bits, 4096), dtype=torch.uint8, device=x.device)
    _check(load_library().fmtc_quantize(basis._h, _dev(x, torch.float32), n, c, h, w, layout, bits,
                                        _dev(syms, torch.uint8), _dev(hist, torch.int32),
                                        _dev(workspace, torch.uint8), workspace.numel(), _stream()))
    return syms, hist


def code_symbols(syms, C, bits, delta_value, chunk_syms=4096, stream_out=None, out_bytes=None, workspace=None):
    """Asynchronous.  syms: uint8 device tensor with P*C elements.  -> (stream_out, out_bytes)."""
    import torch

    P = syms.numel() // C
    if stream_out is None:
        stream_out = torch.empty(encode_bound(P, C, bits, chunk_syms), dtype=torch.uint8, device=syms.device)
    if out_bytes is None:
        out_bytes = torch.zeros(1, dtype=torch.int64, device=syms.device)
    if workspace is None:
        workspace = torch.empty(workspace_size(P, C, bits, chunk_syms), dtype=torch.uint8, device=syms.device)
    _check(load_library().fmtc_code_symbols(_dev(syms, torch.uint8), P, C, bits, chunk_syms, float(delta_value),
                                            _dev(stream_out, torch.uint8), stream_out.numel(),
                                            _dev(out_bytes, torch.int64), _dev(workspace, torch.uint8),
                                            workspace.numel(), _stream()))
    return stream_out, out_bytes


def decode_symbols(stream_in, P, C, bits, syms=None, err_flag=None, nbytes=None):
    """Asynchronous.  -> (symbols uint8 [P, C], err_flag int32[1])."""
    import torch

    if syms is None:
        syms = torch.empty((P, C), dtype=torch.uint8, device=stream_in.device)
    if err_flag is None:
        err_flag = torch.zeros(1, dtype=torch.int32, device=stream_in.device)
    _check(load_library().fmtc_decode_symbols(_dev(stream_in, torch.uint8),
                                              stream_in.numel() if nbytes is None else int(nbytes), P, C, bits,
                                              _dev(syms, torch.uint8), _dev(err_flag, torch.int32), _stream()))
    return syms, err_flag


def stream_info(header_bytes):
    """header_bytes: the first 64 bytes of a stream on the host (bytes / numpy uint8)."""
    buf = bytes(bytearray(header_bytes))[:64]
    bits, C, ppc = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    P, nch = ctypes.c_int64(), ctypes.c_int64()
    dlt = ctypes.c_float()
    pbits, sbytes = ctypes.c_uint64(), ctypes.c_uint64()
    _check(load_library().fmtc_stream_info(buf, len(buf), ctypes.byref(bits), ctypes.byref(C), ctypes.byref(P),
                                           ctypes.byref(ppc), ctypes.byref(nch), ctypes.byref(dlt),
                                           ctypes.byref(pbits), ctypes.byref(sbytes)))
    return dict(bits=bits.value, C=C.value, P=P.value, px_per_chunk=ppc.value, n_chunks=nch.value,
                delta=dlt.value, payload_bits=pbits.value, stream_bytes=sbytes.value)


# ---- a block of a network in 8-bit floating point ----
# Like every call of this module these are not recorded by torch's autograd: what they return has no history, whatever their
# inputs require.  The gradients are f8_matmul_backward and block_norm_backward.

_KINDS = {}    # torch type -> F32, BF16, F16; filled with torch's first use
_FORMATS = {}  # torch type -> E4M3, E5M2
_SCALES = {}   # torch type -> SCALE_F32, SCALE_E8M0


def _types():
    import torch

    _KINDS.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    _FORMATS.update({torch.float8_e4m3fn: E4M3, torch.float8_e5m2: E5M2})
    _SCALES.update({torch.float32: SCALE_F32, torch.float8_e8m0fnu: SCALE_E8M0})


def _dtype(t):
    if not _KINDS:
        _types()
    try:
        return _KINDS[t]
    except KeyError:
        raise ValueError(f"expected float32, bfloat16 or float16, got {t}") from None


def _rows(t, what, cols=None, rows=None, dtype=None):
    """A device matrix whose rows are contiguous -> (pointer, type, row stride)."""
    try:
        (r, c), (step_r, step_c), ok = t.shape, t.stride(), t.is_cuda
    except (AttributeError, ValueError):
        ok = False
    if not ok:
        raise ValueError(f"{what}: expected a 2-d device tensor")
    if (cols is not None and c != cols) or (rows is not None and r != rows):
        raise ValueError(f"{what}: expected {rows} x {cols} values, got {r} x {c}")
    if c > 1 and step_c != 1:
        raise ValueError(f"{what}: the values of a row have to be adjacent")
    kind = t.dtype
    if dtype is not None and kind != dtype:
        raise ValueError(f"{what}: expected {dtype}, got {kind}")
    return t.data_ptr(), _dtype(kind), step_r if r > 1 else c


def _vector(t, what, n, dtype=None):
    """A contiguous device vector of n values -> pointer (None: None)."""
    if t is None:
        return None
    try:
        if t.is_cuda and t.is_contiguous() and t.numel() == n and (dtype is None or t.dtype == dtype):
            return t.data_ptr()
    except AttributeError:
        pass
    raise ValueError(f"{what}: expected {n} contiguous device values" + (f" of {dtype}" if dtype else ""))


def _matrix(rows, cols, dtype, device):
    """A new tensor [rows, cols] (the cheapest of torch's ways to make one)."""
    import torch

    return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)


def _workspace(workspace, size, device):
    """-> (the tensor, its address, its bytes); a new one of `size` bytes if there is none"""
    import torch

    if workspace is None:
        if not size:
            return None, None, 0
        workspace = torch.empty(size, dtype=torch.uint8, device=device)
        return workspace, workspace.data_ptr(), size
    return workspace, _dev(workspace, torch.uint8), workspace.numel()


class F8:
    """A matrix [rows, depth] in 8-bit floating point with a scale per block (fmtc_f8): codes, a tensor [rows, ld] of
    torch.float8_e4m3fn or torch.float8_e5m2 (ld: depth rounded up to 128 or more, zeros behind the depth), and scales
    [ceil(depth / 128), ceil(rows / block_rows)] of torch.float32 or torch.float8_e8m0fnu."""

    __slots__ = ("_codes", "_scales", "_rows", "_depth", "_block_rows", "_at_codes", "_at_scales", "_ref")

    def __init__(self, codes, scales, depth, block_rows=1):
        if not _FORMATS:
            _types()
        try:
            (rows, width), (n_blocks, n_rows) = codes.shape, scales.shape
            fmt, kind = _FORMATS[codes.dtype], _SCALES[scales.dtype]
            (ld, step), (ld_scales, step_scales) = codes.stride(), scales.stride()
            ok = codes.is_cuda and scales.is_cuda
        except (AttributeError, KeyError, ValueError):
            ok = False
        if not ok:
            raise ValueError("F8: expected 2-d device tensors, codes in an 8-bit format, scales f32 or e8m0")
        blocks = -(-depth // F8_BLOCK)
        if depth < 1 or block_rows not in (1, F8_BLOCK) or width < blocks * F8_BLOCK or n_blocks != blocks or \
                n_rows != -(-rows // block_rows):
            raise ValueError(f"F8: codes {tuple(codes.shape)} and scales {tuple(scales.shape)} do not hold {rows} x {depth} "
                             f"values in blocks of {block_rows} x {F8_BLOCK}")
        if step != 1 or (n_rows > 1 and step_scales != 1):
            raise ValueError("F8: the codes of a row and the scales of a block of the depth have to be adjacent")
        self._set(codes, scales, rows, depth, block_rows, ld if rows > 1 else width, ld_scales if blocks > 1 else n_rows, fmt, kind)

    def _set(self, codes, scales, rows, depth, block_rows, ld, ld_scales, fmt, kind):
        self._codes, self._scales = codes, scales
        self._rows, self._depth, self._block_rows = rows, depth, block_rows
        self._at_codes = at_codes = codes.data_ptr()
        self._at_scales = at_scales = scales.data_ptr()
        self._ref = ctypes.byref(_F8(at_codes, at_scales, rows, depth, ld, ld_scales, fmt, kind, block_rows))
        return self

    # What the library reads and writes was checked when the object was made: nothing of it is assigned anew.
    codes = property(operator.attrgetter("_codes"))
    scales = property(operator.attrgetter("_scales"))
    rows = property(operator.attrgetter("_rows"))
    depth = property(operator.attrgetter("_depth"))
    block_rows = property(operator.attrgetter("_block_rows"))


def f8_empty(rows, depth, fmt=E4M3, scales=SCALE_F32, block_rows=1, device="cuda"):
    """An F8 to be written by f8_quantize or block_norm."""
    import torch

    if rows < 0 or depth < 1 or block_rows not in (1, F8_BLOCK):
        raise ValueError(f"f8_empty: {rows} x {depth} values in blocks of {block_rows} rows")
    blocks = -(-depth // F8_BLOCK)
    ld, ld_scales = blocks * F8_BLOCK, -(-rows // block_rows)
    return F8.__new__(F8)._set(
        _matrix(rows, ld, torch.float8_e5m2 if fmt == E5M2 else torch.float8_e4m3fn, device),
        _matrix(blocks, ld_scales, torch.float8_e8m0fnu if scales == SCALE_E8M0 else torch.float32, device),
        rows, depth, block_rows, ld, ld_scales, fmt, scales)


def _f8(q):
    if q is None:
        return None
    if q._codes.data_ptr() != q._at_codes or q._scales.data_ptr() != q._at_scales:
        which = "codes" if q._codes.data_ptr() != q._at_codes else "scales"
        raise ValueError(f"F8: {which} are not in the memory that they had when it was made")
    return q._ref


def f8_quantize(x, by_rows=True, by_cols=False, fmt=E4M3, scales=SCALE_F32, block_rows=1):
    """Asynchronous.  x: device matrix [rows, cols].  -> (F8 [rows, cols] or None, F8 [cols, rows] or None); by_rows and
    by_cols say which are wanted, or are the F8 to be written."""
    ptr, kind, ld = _rows(x, "x")
    rows, cols = x.shape
    if by_rows is True:
        by_rows = f8_empty(rows, cols, fmt, scales, block_rows, x.device)
    if by_cols is True:
        by_cols = f8_empty(cols, rows, fmt, scales, block_rows, x.device) if rows else None
    by_rows, by_cols = by_rows or None, by_cols or None
    _check(load_library().fmtc_f8_quantize(ptr, kind, rows, cols, ld, _f8(by_rows), _f8(by_cols), _stream()))
    return by_rows, by_cols


def f8_matmul_workspace_size(M, N, K):
    return load_library().fmtc_f8_matmul_workspace_size(M, N, K)


def f8_matmul(a, b, bias=None, out=None, dtype=None, accumulate=False, workspace=None):
    """Asynchronous.  a: F8 [M, K], b: F8 [N, K] -> a b^T + bias [M, N] in `dtype` (bf16 unless given, or out's)."""
    import torch

    M, N = a._rows, b._rows
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the output that is added to")
        kind, ld = _dtype(dtype or torch.bfloat16), N
        out = _matrix(M, N, dtype or torch.bfloat16, a._codes.device)
        ptr = out.data_ptr()
    else:
        ptr, kind, ld = _rows(out, "out", N, M, dtype)
    lib = load_library()
    workspace, ws, size = _workspace(workspace, lib.fmtc_f8_matmul_workspace_size(M, N, a._depth), out.device)
    _check(lib.fmtc_f8_matmul(_f8(a), _f8(b), _vector(bias, "bias", N, torch.float32), ptr, kind, ld, int(accumulate), ws, size,
                              _stream()))
    return out


def f8_matmul_backward_workspace_size(P, K, O):
    return load_library().fmtc_f8_matmul_backward_workspace_size(P, K, O)


def f8_matmul_backward(dy, w_t, x_t, fmt=E4M3, scales=SCALE_F32, bias=False, dx=None, dw=None, dbias=None, accumulate=False,
                       workspace=None):
    """Asynchronous.  Gradients of y = x w^T + bias: dy [P, O]; w_t: the weights as F8 [K, O] in 128 x 128 blocks (None: no
    dx); x_t: x by columns as F8 [K, P] (None: no dw).  -> (dx [P, K] in dy's type, dw [O, K] f32, dbias [O] f32), None
    where not wanted (dbias: wanted with bias=True or where given).  accumulate: dw and dbias are added to.  Without rows
    (P = 0: f8_quantize gives no x by columns) x_t may be None all the same: dw is 0, as wide as the weights or as given."""
    import torch

    ptr, kind, ld = _rows(dy, "dy")
    P, O = dy.shape
    if accumulate and ((x_t is not None and dw is None) or (bias and dbias is None)):
        raise ValueError("accumulate needs the outputs that are added to")
    x_c, x_rows = (None, 0) if x_t is None else (_f8(x_t), x_t.rows)
    if P == 0 and x_t is None:
        if dw is not None:
            _rows(dw, "dw", dtype=torch.float32)
            x_rows = dw.shape[1]
        elif w_t is not None and not accumulate:
            x_rows = w_t.rows
        x_c = _F8(rows=x_rows) if x_rows else None
    if w_t is not None and dx is None:
        dx = _matrix(P, w_t.rows, dy.dtype, dy.device)
    if x_c is not None and dw is None:
        dw = _matrix(O, x_rows, torch.float32, dy.device)
    if bias and dbias is None:
        dbias = torch.empty(O, dtype=torch.float32, device=dy.device)
    if (dx is not None and w_t is None) or (dw is not None and x_c is None):
        raise ValueError("dx needs w_t, dw needs x_t")
    dx_ptr, dx_kind, dx_ld = _rows(dx, "dx", w_t.rows, P) if dx is not None else (None, F32, 0)
    dw_ptr, _, dw_ld = _rows(dw, "dw", x_rows, O, torch.float32) if dw is not None else (None, F32, 0)
    K = w_t.rows if w_t is not None else x_rows or 1
    lib = load_library()
    workspace, ws, size = _workspace(workspace, lib.fmtc_f8_matmul_backward_workspace_size(P, K, O), dy.device)
    _check(lib.fmtc_f8_matmul_backward(ptr, kind, P, O, ld, _f8(w_t), x_c, fmt, scales, dx_ptr, dx_kind, dx_ld, dw_ptr, dw_ld,
                                       _vector(dbias, "dbias", O, torch.float32), int(accumulate), ws, size, _stream()))
    return dx, dw, dbias


def _norm_args(y, h, w_post, w_pre, gate, rows_per_gate, skip, scale, eps):
    P, C = h.shape
    h_ptr, kind, ld_h = _rows(h, "h")
    y_ptr, _, ld_y = _rows(y, "y", C, P, h.dtype) if y is not None else (None, 0, 0)
    like = w_pre if w_pre is not None else w_post if w_post is not None else gate
    weights = None if like is None else like.dtype
    if (w_post is not None and w_post.dtype != weights) or (gate is not None and gate.dtype != weights):
        raise ValueError("w_post, w_pre and gate have different types")
    if gate is None:
        rows_per_gate, gate_ptr = 0, None
    else:
        rows_per_gate = int(rows_per_gate)
        if rows_per_gate < 0:
            rows_per_gate = -1  # (refused)
        elif rows_per_gate == 0 or rows_per_gate > P:
            rows_per_gate = P or 1  # (one row for all, however many more it says)
        gate_ptr = _vector(gate, "gate", -(-P // rows_per_gate) * C if P and rows_per_gate > 0 else gate.numel())
    return _Norm(P, C, kind, F32 if like is None else _dtype(weights), 0, y_ptr, h_ptr, ld_y, ld_h, _vector(w_post, "w_post", C),
                 _vector(w_pre, "w_pre", C), gate_ptr, rows_per_gate, skip, scale, eps)


def block_norm(y, h, w_post, w_pre, gate=None, rows_per_gate=0, skip=1.0, scale=1.0, eps=1e-6, h_out=None, n_out=None,
               stats=None):
    """Asynchronous.  u = w_post y / rms(y); h' = skip h + scale gate u; n = w_pre h' / rms(h').  y (or None), h: [P, C];
    gate: [ceil(P / rows_per_gate), C] (rows_per_gate 0: one row for all).  h_out: the tensor to write h' to (None: a new
    one, False: not stored); n_out: a tensor or an F8 to write n to (None: a new tensor).  stats: the f32 tensor [2, P]
    that the backward pass needs, or True for a new one.  -> (h', n, stats), None where there is none."""
    import torch

    a = _norm_args(y, h, w_post, w_pre, gate, rows_per_gate, skip, scale, eps)
    P, C = h.shape
    kind, device = h.dtype, h.device
    h_ptr, h_ld = None, C
    if h_out is None:
        h_out = _matrix(P, C, kind, device)
        h_ptr = h_out.data_ptr()
    elif h_out is False:
        h_out = None
    else:
        h_ptr, _, h_ld = _rows(h_out, "h_out", C, P, kind)
    n_ptr, n_ld, n_codes = None, C, None
    if isinstance(n_out, F8):
        n_codes = n_out
    elif n_out is not None:
        n_ptr, _, n_ld = _rows(n_out, "n_out", C, P, kind)
    elif w_pre is not None:
        n_out = _matrix(P, C, kind, device)
        n_ptr = n_out.data_ptr()
    if stats is True:
        stats = _matrix(2, P, torch.float32, device)
        s_ptr = stats.data_ptr()
    else:
        s_ptr = _vector(stats, "stats", 2 * P, torch.float32)
    _check(load_library().fmtc_block_norm(ctypes.byref(a), h_ptr, h_ld, n_ptr, n_ld, _f8(n_codes), s_ptr, _stream()))
    return h_out, n_out, stats


def block_norm_workspace_size(P, C, rows_per_gate=0):
    """Bytes for block_norm_backward; rows_per_gate: 0 without a gate, P with one row for all."""
    return load_library().fmtc_block_norm_workspace_size(P, C, rows_per_gate)


def block_norm_backward(dn, dh, y, h_out, stats, w_post, w_pre, gate=None, rows_per_gate=0, skip=1.0, scale=1.0, dy=None,
                        dh_in=None, workspace=None):
    """Asynchronous.  dn, dh: gradients of n and of h' (either may be None); h_out: h' as block_norm stored it, stats as it
    left them.  dy, dh_in: tensors to write to (None: new ones).  -> (dy, dh_in, dw_post, dw_pre, dgate), the last three in
    f32 (0 where there are no rows), None where there is no such input."""
    import torch

    a = _norm_args(y, h_out, w_post, w_pre, gate, rows_per_gate, skip, scale, 0.0)
    P, C = h_out.shape
    kind, device = h_out.dtype, h_out.device
    new = lambda like: torch.empty_like(like, dtype=torch.float32) if like is not None else None  # noqa: E731
    dw_post, dw_pre, dgate = new(w_post), new(w_pre), new(gate)
    if dgate is not None and P == 0:  # (the library sees a gate of no rows then)
        dgate.zero_()
    of = lambda t, what: _rows(t, what, C, P, kind) if t is not None else (None, 0, 0)  # noqa: E731
    (dn_p, _, dn_ld), (dh_p, _, dh_ld) = of(dn, "dn"), of(dh, "dh")
    if dy is None and y is not None:
        dy = _matrix(P, C, kind, device)
        dy_p, dy_ld = dy.data_ptr(), C
    else:
        dy_p, _, dy_ld = of(dy, "dy")
    if dh_in is None:
        dh_in = _matrix(P, C, kind, device)
        di_p, di_ld = dh_in.data_ptr(), C
    else:
        di_p, _, di_ld = of(dh_in, "dh_in")
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    lib = load_library()
    workspace, ws, size = _workspace(workspace, lib.fmtc_block_norm_workspace_size(P, C, a.rows_per_gate), h_out.device)
    _check(lib.fmtc_block_norm_backward(ctypes.byref(a), _vector(stats, "stats", 2 * P, torch.float32), dn_p, dn_ld, dh_p, dh_ld,
                                        dy_p, dy_ld, di_p, di_ld, ptr(dw_post), ptr(dw_pre), ptr(dgate), ws, size, _stream()))
    return dy, dh_in, dw_post, dw_pre, dgate


TEST_STATIC_TWO_KERNELS, TEST_DECODE_ONE_ROW, TEST_SHORT_WAITS = 0, 1, 2


def test_option(option, value):
    """Forces a path or the end of a wait (tests only); value 0 restores the library's own choice."""
    _check(load_library().fmtc_test_option(int(option), int(value)))


test_option.__test__ = False  # (not a test, whatever a collector makes of the name)


def test_projection(shape, layout=NHWC, bits=4, keep=None):
    """-> the form of the projection kernel that a tensor of the 4-d `shape` takes, as a text (tests only)."""
    n, h, w, c = shape if layout == NHWC else (shape[0], shape[2], shape[3], shape[1])
    text = ctypes.create_string_buffer(64)
    _check(load_library().fmtc_test_projection(n, c, h, w, layout, bits, c if keep is None else keep, text, len(text)))
    return text.value.decode()


test_projection.__test__ = False


def profile_enable(max_launches_per_kernel):
    _check(load_library().fmtc_profile_enable(int(max_launches_per_kernel)))


def profile_copy(dst, src):
    """Yardstick copy of src into dst (uint8 device tensors of equal size, a multiple of 16 bytes)."""
    import torch

    _check(load_library().fmtc_profile_copy(_dev(dst, torch.uint8), _dev(src, torch.uint8), src.numel(), _stream()))


def profile_read():
    """-> {kernel name: (avg_ms, min_ms, launches)} for the kernels launched since profile_enable."""
    lib = load_library()
    out = {}
    for k in range(lib.fmtc_profile_kernels()):
        avg, mn, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_int()
        _check(lib.fmtc_profile_read(k, ctypes.byref(avg), ctypes.byref(mn), ctypes.byref(n)))
        if n.value:
            out[lib.fmtc_profile_name(k).decode()] = (avg.value, mn.value, n.value)
    return out
