"""Thin ctypes binding of libco3.so (include/co3.h): argument marshalling only.

torch is used for device memory and streams; every step of the codec runs in the HIP
kernels of the library.  There is no CPU fallback: loading fails loudly when the library has
not been built (python -m paper_2204_08211_amd.build).
"""
import ctypes as C
import functools
import os
import struct

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libco3.so")

CHUNK = 4096
SUB = 64
SUBS_PER_CHUNK = 64
STATUS_WORDS = 8
(STAT_NONFINITE, STAT_CLAMPED, STAT_NOCODE, STAT_CAPACITY, STAT_CODELEN, STAT_CORRUPT, STAT_STALLED) = range(7)
BOOK_FIXED, BOOK_EMPIRICAL = 0, 1
OK, ERR_ARG, ERR_FORMAT, ERR_CAPACITY, ERR_CODELEN, ERR_CORRUPT, ERR_HIP = 0, -1, -2, -3, -4, -5, -6

EXPORTS = [
    "co3_plan_create", "co3_plan_set_bias", "co3_plan_destroy", "co3_plan_num_chunks", "co3_plan_num_books",
    "co3_plan_alphabet", "co3_plan_symbols_bytes", "co3_plan_workspace_bytes", "co3_plan_stream_words",
    "co3_build_codebook", "co3_build_codebook_device", "co3_codebook_export", "co3_codebook_num_books",
    "co3_codebook_destroy", "co3_encode", "co3_decode", "co3_ps_aggregate", "co3_status_string",
    "co3_profile_begin", "co3_profile_end", "co3_gennorm_weights", "co3_plan_fit_workspace_bytes", "co3_gennorm_fit",
    "co3_model_weights_device", "co3_model_bias_device", "co3_plan_set_bias_device", "co3_bias_from_model", "co3_scale_from_model",
    "co3_plan_scale_workspace_bytes", "co3_model_scale_device", "co3_plan_set_gain_device",
    "co3_plan_bias_workspace_bytes", "co3_set_lookback_polls", "co3_encode_static", "co3_plan_set_gain",
    "co3_matrix_plan_create", "co3_matrix_plan_destroy", "co3_matrix_plan_workspace_bytes", "co3_matrix_plan_elements",
    "co3_orthogonalize", "co3_muon_update", "co3_layernorm", "co3_layernorm_backward_workspace_bytes", "co3_layernorm_backward",
]


class Format(C.Structure):
    _fields_ = [("exp_bits", C.c_int32), ("mant_bits", C.c_int32)]


class GennormParams(C.Structure):
    _fields_ = [("mu", C.c_double), ("alpha", C.c_double), ("beta", C.c_double), ("kurtosis", C.c_double)]


class Segment(C.Structure):
    _fields_ = [("offset", C.c_uint64), ("length", C.c_uint64), ("codebook", C.c_int32), ("reserved", C.c_int32)]


class EncodeArgs(C.Structure):
    _fields_ = [("g", C.c_void_p), ("m", C.c_void_p), ("m_out", C.c_void_p), ("row_stride", C.c_uint64),
                ("gamma", C.c_float), ("mode", C.c_int32), ("books", C.c_void_p), ("symbols", C.c_void_p),
                ("hist", C.c_void_p), ("words", C.c_void_p), ("words_stride", C.c_uint64),
                ("chunk_offset", C.c_void_p), ("sub_bits", C.c_void_p), ("payload_bits", C.c_void_p),
                ("status", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("rounding", C.c_int32), ("reserved", C.c_int32), ("seed", C.c_uint64)]


class DecodeArgs(C.Structure):
    _fields_ = [("words", C.c_void_p), ("words_stride", C.c_uint64), ("chunk_offset", C.c_void_p),
                ("sub_bits", C.c_void_p), ("books", C.c_void_p), ("symbols", C.c_void_p), ("q", C.c_void_p),
                ("q_stride", C.c_uint64), ("status", C.c_void_p)]


class AggregateArgs(C.Structure):
    _fields_ = [("words", C.c_void_p), ("words_stride", C.c_uint64), ("chunk_offset", C.c_void_p),
                ("sub_bits", C.c_void_p), ("books", C.c_void_p), ("out", C.c_void_p), ("status", C.c_void_p),
                ("model", C.c_void_p), ("eta", C.c_float), ("reserved", C.c_int32)]


class Matrix(C.Structure):
    _fields_ = [("offset", C.c_uint64), ("ld", C.c_uint64), ("rows", C.c_uint32), ("cols", C.c_uint32), ("scale", C.c_float),
                ("reserved", C.c_int32)]


class OrthogonalizeArgs(C.Structure):
    _fields_ = [("g", C.c_void_p), ("out", C.c_void_p), ("coefficients", C.c_void_p), ("steps", C.c_uint32), ("eps", C.c_float),
                ("status", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class MuonArgs(C.Structure):
    _fields_ = [("g", C.c_void_p), ("momentum", C.c_void_p), ("model", C.c_void_p), ("coefficients", C.c_void_p),
                ("steps", C.c_uint32), ("eps", C.c_float), ("eta", C.c_float), ("beta", C.c_float), ("weight_decay", C.c_float),
                ("nesterov", C.c_int32), ("status", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class LayernormArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("weight", C.c_void_p), ("bias", C.c_void_p), ("mean", C.c_void_p),
                ("rstd", C.c_void_p), ("rows", C.c_uint64), ("x_stride", C.c_uint64), ("y_stride", C.c_uint64),
                ("cols", C.c_uint32), ("type", C.c_int32), ("eps", C.c_float), ("reserved", C.c_int32)]


class LayernormBackwardArgs(C.Structure):
    _fields_ = [("dy", C.c_void_p), ("x", C.c_void_p), ("dx", C.c_void_p), ("weight", C.c_void_p), ("mean", C.c_void_p),
                ("rstd", C.c_void_p), ("dweight", C.c_void_p), ("dbias", C.c_void_p), ("grad_stride", C.c_uint64),
                ("rows_per_user", C.c_uint64), ("dy_stride", C.c_uint64), ("x_stride", C.c_uint64), ("dx_stride", C.c_uint64),
                ("U", C.c_uint32), ("cols", C.c_uint32), ("type", C.c_int32), ("accumulate", C.c_int32),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


_CODES = {C.c_void_p: "P", C.c_uint64: "Q", C.c_uint32: "I", C.c_int32: "i", C.c_float: "f", C.c_size_t: "N"}


def _packer(struct_type):
    """struct.Struct.pack of a structure's fields in their order (0 for a null pointer): the same bytes as the ctypes
    structure, in a third of the time; calls of a few microseconds are made with it."""
    p = struct.Struct("@" + "".join(_CODES[t] for _, t in struct_type._fields_) + "0Q")
    assert p.size == C.sizeof(struct_type)
    return p.pack


_pack_orthogonalize, _pack_muon = _packer(OrthogonalizeArgs), _packer(MuonArgs)
_pack_layernorm, _pack_layernorm_backward = _packer(LayernormArgs), _packer(LayernormBackwardArgs)


class KernelTime(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("total_ms", C.c_double), ("launches", C.c_uint64)]


class Co3Error(RuntimeError):
    def __init__(self, where, code):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


_lib = None


def lib():
    """The loaded library.  Raises if it has not been built: there is no fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2204_08211_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.co3_plan_create.argtypes = [Format, C.c_uint32, C.c_uint64, C.c_uint32, C.c_void_p, C.c_void_p,
                                      C.c_int32, C.POINTER(C.c_void_p)]
        L.co3_plan_set_bias.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_plan_set_gain.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_plan_destroy.argtypes = [C.c_void_p]
        L.co3_plan_destroy.restype = None
        for name, rt in [("co3_plan_num_chunks", C.c_uint64), ("co3_plan_num_books", C.c_uint32),
                         ("co3_plan_alphabet", C.c_uint32), ("co3_plan_symbols_bytes", C.c_size_t),
                         ("co3_plan_workspace_bytes", C.c_size_t), ("co3_plan_fit_workspace_bytes", C.c_size_t),
                         ("co3_plan_bias_workspace_bytes", C.c_size_t)]:
            getattr(L, name).argtypes = [C.c_void_p]
            getattr(L, name).restype = rt
        L.co3_plan_stream_words.argtypes = [C.c_void_p, C.c_uint32]
        L.co3_plan_stream_words.restype = C.c_uint64
        L.co3_build_codebook.argtypes = [Format, C.c_uint32, C.c_void_p, C.POINTER(C.c_void_p)]
        L.co3_build_codebook_device.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_codebook_export.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_codebook_num_books.argtypes = [C.c_void_p]
        L.co3_codebook_num_books.restype = C.c_uint32
        L.co3_codebook_destroy.argtypes = [C.c_void_p]
        L.co3_codebook_destroy.restype = None
        L.co3_encode.argtypes = [C.c_void_p, C.POINTER(EncodeArgs), C.c_void_p]
        L.co3_encode_static.argtypes = [C.c_void_p, C.POINTER(EncodeArgs), C.c_void_p]
        L.co3_decode.argtypes = [C.c_void_p, C.POINTER(DecodeArgs), C.c_void_p]
        L.co3_ps_aggregate.argtypes = [C.c_void_p, C.POINTER(AggregateArgs), C.c_void_p]
        L.co3_profile_end.argtypes = [C.POINTER(KernelTime), C.c_uint32, C.POINTER(C.c_uint32)]
        L.co3_gennorm_weights.argtypes = [Format, C.c_int32, C.c_double, C.c_double, C.c_double, C.c_void_p]
        L.co3_gennorm_fit.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint64, C.c_float, C.c_void_p, C.c_void_p,
                                      C.c_size_t, C.c_void_p]
        L.co3_model_weights_device.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_model_bias_device.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                            C.c_void_p]
        L.co3_plan_set_bias_device.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_plan_scale_workspace_bytes.argtypes = [C.c_void_p]
        L.co3_plan_scale_workspace_bytes.restype = C.c_size_t
        L.co3_model_scale_device.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_size_t, C.c_void_p]
        L.co3_plan_set_gain_device.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_bias_from_model.argtypes = [Format, C.c_double, C.c_double, C.c_double, C.POINTER(C.c_int32),
                                          C.POINTER(C.c_double)]
        L.co3_scale_from_model.argtypes = [Format, C.c_double, C.c_double, C.c_double, C.POINTER(C.c_int32),
                                           C.POINTER(C.c_float), C.POINTER(C.c_float), C.POINTER(C.c_double)]
        L.co3_set_lookback_polls.argtypes = [C.c_uint32]
        L.co3_set_lookback_polls.restype = None
        L.co3_matrix_plan_create.argtypes = [C.c_uint32, C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_void_p)]
        L.co3_matrix_plan_destroy.argtypes = [C.c_void_p]
        L.co3_matrix_plan_destroy.restype = None
        L.co3_matrix_plan_workspace_bytes.argtypes = [C.c_void_p]
        L.co3_matrix_plan_workspace_bytes.restype = C.c_size_t
        L.co3_matrix_plan_elements.argtypes = [C.c_void_p]
        L.co3_matrix_plan_elements.restype = C.c_uint64
        L.co3_orthogonalize.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]   # arguments: by reference, or packed
        L.co3_muon_update.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.co3_layernorm.argtypes = [C.c_void_p, C.c_void_p]
        L.co3_layernorm_backward_workspace_bytes.argtypes = [C.c_uint32, C.c_uint64, C.c_uint32]
        L.co3_layernorm_backward_workspace_bytes.restype = C.c_size_t
        L.co3_layernorm_backward.argtypes = [C.c_void_p, C.c_void_p]
        L.co3_status_string.argtypes = [C.c_int]
        L.co3_status_string.restype = C.c_char_p
        _lib = L
    return _lib


def profile_begin():
    _check("co3_profile_begin", lib().co3_profile_begin())


def profile_end():
    """{kernel name: (total ms, launches)} for the launches since profile_begin()."""
    arr = (KernelTime * 32)()
    n = C.c_uint32(0)
    _check("co3_profile_end", lib().co3_profile_end(arr, 32, C.byref(n)))
    return {arr[i].name.decode(): (arr[i].total_ms, int(arr[i].launches)) for i in range(n.value)}


LOOKBACK_POLLS_DEFAULT = 1 << 20


def set_lookback_polls(polls):
    """Bound of the single-sweep encoder's wait for the chunks ahead (re-reads per entry); 0 gives up at once."""
    lib().co3_set_lookback_polls(int(polls))


def status_string(code):
    return lib().co3_status_string(int(code)).decode()


def _check(where, rc):
    if rc != OK:
        raise Co3Error(where, rc)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


_torch_c = None


def _stream(stream=None):
    if stream is not None:
        return C.c_void_p(stream.cuda_stream)
    global _torch_c
    if _torch_c is None:
        import torch
        torch.cuda.current_stream()   # torch's own set-up of the device
        _torch_c = torch._C
    # torch.cuda.current_stream() makes a Stream object of this number, which takes longer than some kernels here
    return C.c_void_p(_torch_c._cuda_getCurrentRawStream(_torch_c._cuda_getDevice()))


class Plan:
    """co3_plan: U users, d elements, [sgn,exp,mant] format, layers and per-(user, layer) bias."""

    def __init__(self, E, M, U, d, bias, seg_len=None, seg_book=None, per_user_books=False):
        self.E, self.M, self.U, self.d = int(E), int(M), int(U), int(d)
        self.seg_len = [int(d)] if seg_len is None else [int(x) for x in seg_len]
        self.nseg = len(self.seg_len)
        self.seg_book = [0] * self.nseg if seg_book is None else [int(x) for x in seg_book]
        self.per_user_books = bool(per_user_books)
        bias = np.ascontiguousarray(np.broadcast_to(np.asarray(bias, dtype=np.int32), (self.U, self.nseg)))
        segs = (Segment * self.nseg)()
        off = 0
        for k, (n, b) in enumerate(zip(self.seg_len, self.seg_book)):
            segs[k] = Segment(off, n, b, 0)
            off += n
        h = C.c_void_p()
        _check("co3_plan_create", lib().co3_plan_create(Format(self.E, self.M), self.U, self.d, self.nseg,
                                                        C.cast(segs, C.c_void_p), bias.ctypes.data_as(C.c_void_p),
                                                        int(self.per_user_books), C.byref(h)))
        self.handle = h
        self.bias = bias
        self.num_chunks = int(lib().co3_plan_num_chunks(h))
        self.num_books = int(lib().co3_plan_num_books(h))
        self.A = int(lib().co3_plan_alphabet(h))
        self.symbols_bytes = int(lib().co3_plan_symbols_bytes(h))
        self.workspace_bytes = int(lib().co3_plan_workspace_bytes(h))
        self.sym_stride = (self.d + 127) // 128 * 128
        self.wide = self.A > 256          # alphabets above 8 bits: 16-bit symbols

    def set_bias(self, bias, stream=None):
        bias = np.ascontiguousarray(np.broadcast_to(np.asarray(bias, dtype=np.int32), (self.U, self.nseg)))
        _check("co3_plan_set_bias", lib().co3_plan_set_bias(self.handle, bias.ctypes.data_as(C.c_void_p), _stream(stream)))
        self.bias = bias

    def set_gain(self, gain, inv_gain, stream=None):
        """Real-valued scale on top of the integer bias: float32 [U][nseg] pairs (None, None: back to 1)."""
        if gain is None:
            _check("co3_plan_set_gain", lib().co3_plan_set_gain(self.handle, None, None, _stream(stream)))
            return
        gain = np.ascontiguousarray(np.broadcast_to(np.asarray(gain, dtype=np.float32), (self.U, self.nseg)))
        inv_gain = np.ascontiguousarray(np.broadcast_to(np.asarray(inv_gain, dtype=np.float32), (self.U, self.nseg)))
        _check("co3_plan_set_gain", lib().co3_plan_set_gain(self.handle, gain.ctypes.data_as(C.c_void_p),
                                                          inv_gain.ctypes.data_as(C.c_void_p), _stream(stream)))

    def stream_words(self, max_code_len=64):
        return int(lib().co3_plan_stream_words(self.handle, int(max_code_len)))

    def close(self):
        if getattr(self, "handle", None):
            lib().co3_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Codebook:
    """co3_codebook: a set of Huffman code tables living on the device."""

    def __init__(self, handle, E, M, nbooks):
        self.handle, self.E, self.M, self.nbooks = handle, E, M, nbooks
        self.A = 1 << (1 + E + M)

    def export(self, book=0, stream=None):
        length = np.zeros(self.A, np.uint8)
        code = np.zeros(self.A, np.uint64)
        _check("co3_codebook_export", lib().co3_codebook_export(self.handle, int(book), length.ctypes.data_as(C.c_void_p),
                                                                code.ctypes.data_as(C.c_void_p), _stream(stream)))
        return length, code

    def close(self):
        if getattr(self, "handle", None):
            lib().co3_codebook_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def co3_build_codebook(E, M, nbooks, weights=None):
    """Huffman tables from host integer weights [nbooks][A] (None: empty set for device builds)."""
    h = C.c_void_p()
    wp = None
    if weights is not None:
        weights = np.ascontiguousarray(weights, dtype=np.uint64).reshape(nbooks, 1 << (1 + E + M))
        wp = weights.ctypes.data_as(C.c_void_p)
    _check("co3_build_codebook", lib().co3_build_codebook(Format(E, M), int(nbooks), wp, C.byref(h)))
    return Codebook(h, E, M, nbooks)


def co3_gennorm_weights(E, M, bias, mu, alpha, beta):
    """uint64[A] Huffman weights of the symbols when g + gamma m is GenNorm(mu, alpha, beta)."""
    w = np.zeros(1 << (1 + E + M), dtype=np.uint64)
    _check("co3_gennorm_weights", lib().co3_gennorm_weights(Format(E, M), int(bias), float(mu), float(alpha),
                                                            float(beta), w.ctypes.data_as(C.c_void_p)))
    return w


def co3_build_codebook_device(books, weights, status, stream=None):
    """Rebuild the set from device weights (uint64 viewed as an int64 tensor [nbooks][A])."""
    _check("co3_build_codebook_device",
           lib().co3_build_codebook_device(books.handle, _ptr(weights), _ptr(status), _stream(stream)))


def co3_gennorm_fit(plan, g, m, gamma, params=None, workspace=None, stream=None):
    """GenNorm(mu, alpha, beta) of v = g + gamma m per user and layer by matching mean, variance and
    kurtosis (Sec. III eq. (kurtosis)).  Returns a float64 device tensor [U][nseg][4] = (mu, alpha, beta,
    kurtosis); g, m are float32 device tensors [U][row_stride]."""
    import torch
    assert g.dim() == 2 and g.shape == m.shape and g.stride(1) == 1 and g.stride(0) == m.stride(0)
    if params is None:
        params = torch.zeros((plan.U, plan.nseg, 4), dtype=torch.float64, device=g.device)
    if workspace is None:
        workspace = torch.empty(int(lib().co3_plan_fit_workspace_bytes(plan.handle)), dtype=torch.uint8, device=g.device)
    _check("co3_gennorm_fit", lib().co3_gennorm_fit(plan.handle, g.data_ptr(), m.data_ptr(), g.stride(0),
                                                      float(np.float32(gamma)), params.data_ptr(), workspace.data_ptr(),
                                                      workspace.numel(), _stream(stream)))
    return params


def co3_model_weights_device(plan, params, weights=None, stream=None):
    """Integer weights [num_books][A] (uint64 viewed as an int64 device tensor) of the model code for fitted
    parameters; feed them to co3_build_codebook_device."""
    import torch
    if weights is None:
        weights = torch.zeros((plan.num_books, plan.A), dtype=torch.int64, device=params.device)
    _check("co3_model_weights_device",
           lib().co3_model_weights_device(plan.handle, params.data_ptr(), weights.data_ptr(), _stream(stream)))
    return weights


def co3_model_bias_device(plan, params, install=True, stream=None):
    """Exponent bias per user and layer from fitted parameters (eq. (exp bias) with integer b): returns
    (int32 device tensor [U][nseg], float64 device tensor [U][nseg] of expected squared errors) and, with
    install, makes it the plan's bias table."""
    import torch
    bias = torch.zeros((plan.U, plan.nseg), dtype=torch.int32, device=params.device)
    err = torch.zeros((plan.U, plan.nseg), dtype=torch.float64, device=params.device)
    ws = torch.empty(int(lib().co3_plan_bias_workspace_bytes(plan.handle)), dtype=torch.uint8, device=params.device)
    _check("co3_model_bias_device",
           lib().co3_model_bias_device(plan.handle, params.data_ptr(), bias.data_ptr(), err.data_ptr(), ws.data_ptr(),
                                       ws.numel(), _stream(stream)))
    if install:
        _check("co3_plan_set_bias_device", lib().co3_plan_set_bias_device(plan.handle, bias.data_ptr(), _stream(stream)))
    return bias, err


def co3_model_scale_device(plan, params, install=True, stream=None):
    """Exponent bias and real-valued scale per user and layer from fitted parameters (eq. (exp bias) with real b):
    returns (int32 device tensor [U][nseg], float32 device tensor [U][nseg][2] of (gain, inv_gain), float64 device
    tensor [U][nseg] of expected squared errors) and, with install, makes them the plan's bias and scale."""
    import torch
    bias = torch.zeros((plan.U, plan.nseg), dtype=torch.int32, device=params.device)
    pairs = torch.ones((plan.U, plan.nseg, 2), dtype=torch.float32, device=params.device)
    err = torch.zeros((plan.U, plan.nseg), dtype=torch.float64, device=params.device)
    ws = torch.empty(int(lib().co3_plan_scale_workspace_bytes(plan.handle)), dtype=torch.uint8, device=params.device)
    _check("co3_model_scale_device",
           lib().co3_model_scale_device(plan.handle, params.data_ptr(), bias.data_ptr(), pairs.data_ptr(), err.data_ptr(),
                                        ws.data_ptr(), ws.numel(), _stream(stream)))
    if install:
        _check("co3_plan_set_bias_device", lib().co3_plan_set_bias_device(plan.handle, bias.data_ptr(), _stream(stream)))
        _check("co3_plan_set_gain_device", lib().co3_plan_set_gain_device(plan.handle, pairs.data_ptr(), _stream(stream)))
    return bias, pairs, err


def co3_scale_from_model(E, M, mu, alpha, beta):
    """eq. (exp bias) with real b on the host: (bias, gain, inv_gain, expected squared error); the pair is what
    Plan.set_gain takes."""
    b = C.c_int32(0)
    gn, ig = C.c_float(1.0), C.c_float(1.0)
    e = C.c_double(0.0)
    _check("co3_scale_from_model", lib().co3_scale_from_model(Format(E, M), float(mu), float(alpha), float(beta),
                                                            C.byref(b), C.byref(gn), C.byref(ig), C.byref(e)))
    return int(b.value), float(gn.value), float(ig.value), float(e.value)


def co3_bias_from_model(E, M, mu, alpha, beta):
    """(bias, expected squared error) of eq. (exp bias) with integer b for GenNorm(mu, alpha, beta); host."""
    b = C.c_int32(0)
    e = C.c_double(0.0)
    _check("co3_bias_from_model", lib().co3_bias_from_model(Format(E, M), float(mu), float(alpha), float(beta),
                                                          C.byref(b), C.byref(e)))
    return int(b.value), float(e.value)


class RoundBuffers:
    """Device buffers of one round, allocated with torch (plumbing only)."""

    def __init__(self, plan, device="cuda:0", words_stride=None, max_code_len=32):
        import torch
        self.plan = plan
        U, nch = plan.U, plan.num_chunks
        self.words_stride = int(words_stride) if words_stride is not None else plan.stream_words(max_code_len)
        dev = torch.device(device)
        self.symbols = torch.zeros(plan.symbols_bytes, dtype=torch.uint8, device=dev)
        self.hist = torch.zeros((plan.num_books, plan.A), dtype=torch.int64, device=dev)
        self.words = torch.zeros((U, self.words_stride), dtype=torch.int32, device=dev)
        self.chunk_offset = torch.zeros((U, nch + 1), dtype=torch.int64, device=dev)
        self.sub_bits = torch.zeros((U, nch * SUBS_PER_CHUNK), dtype=torch.int16, device=dev)
        self.payload_bits = torch.zeros(U, dtype=torch.int64, device=dev)
        self.status = torch.zeros(STATUS_WORDS, dtype=torch.int64, device=dev)
        self.workspace = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device=dev)

    def symbols_2d(self):
        return symbols_2d(self.plan, self.symbols)


def symbols_2d(plan, buf):
    """[U][d] view of a symbols buffer (uint8 tensor of plan.symbols_bytes): bytes, or 16-bit words for wide alphabets."""
    import torch
    if plan.wide:
        return buf[:2 * plan.U * plan.sym_stride].view(torch.int16).view(plan.U, plan.sym_stride)[:, :plan.d]
    return buf[:plan.U * plan.sym_stride].view(plan.U, plan.sym_stride)[:, :plan.d]


ROUND_NEAREST, ROUND_STOCHASTIC = 0, 1


STATIC_SCRATCH_BYTES = 8 << 20


def co3_encode(plan, books, g, m, m_out, gamma, buf, mode=BOOK_EMPIRICAL, stream=None, single_sweep=False,
               stochastic_seed=None, static=False, single_sweep_hist=False):
    """User side of one round for all U users (Algorithm 1 lines 8-10).  g, m, m_out are float32
    device tensors [U][row_stride]; outputs land in `buf` (RoundBuffers).  single_sweep (fixed code
    only) passes no symbols and no hist buffer, which selects the library's single-sweep encoder;
    single_sweep_hist passes the hist buffer all the same (the sweep then also counts the symbols).
    stochastic_seed: None = closest representative, else the stochastic conversion keyed by that seed.
    static: call co3_encode_static (the library's own static workspace, no allocation; buf.workspace is not passed)."""
    assert not single_sweep or mode == BOOK_FIXED
    assert g.dim() == 2 and g.shape == m.shape == m_out.shape and g.stride(1) == 1
    assert g.stride(0) == m.stride(0) == m_out.stride(0)
    a = EncodeArgs(g.data_ptr(), m.data_ptr(), m_out.data_ptr(), g.stride(0), float(np.float32(gamma)), int(mode),
                   books.handle, None if single_sweep else buf.symbols.data_ptr(),
                   None if (single_sweep and not single_sweep_hist) else buf.hist.data_ptr(), buf.words.data_ptr(),
                   buf.words_stride, buf.chunk_offset.data_ptr(), buf.sub_bits.data_ptr(),
                   buf.payload_bits.data_ptr(), buf.status.data_ptr(), None if static else buf.workspace.data_ptr(),
                   0 if static else buf.workspace.numel(), ROUND_NEAREST if stochastic_seed is None else ROUND_STOCHASTIC, 0,
                   0 if stochastic_seed is None else int(stochastic_seed) & 0xffffffffffffffff)
    if static:
        _check("co3_encode_static", lib().co3_encode_static(plan.handle, C.byref(a), _stream(stream)))
    else:
        _check("co3_encode", lib().co3_encode(plan.handle, C.byref(a), _stream(stream)))


def co3_decode(plan, books, buf, symbols=None, q=None, stream=None):
    """Invert the streams in `buf` into symbols (uint8, plan.symbols_bytes) and/or values q [U][stride]."""
    a = DecodeArgs(buf.words.data_ptr(), buf.words_stride, buf.chunk_offset.data_ptr(), buf.sub_bits.data_ptr(),
                   books.handle, None if symbols is None else symbols.data_ptr(),
                   None if q is None else q.data_ptr(), 0 if q is None else q.stride(0), buf.status.data_ptr())
    _check("co3_decode", lib().co3_decode(plan.handle, C.byref(a), _stream(stream)))


def co3_ps_aggregate(plan, books, buf, out, stream=None, model=None, eta=0.0):
    """PS side: out[d] = (1/U) sum_u ghat^(u) decoded from the streams in `buf`; with `model` (float32
    device tensor [d]) also model -= eta * that average (Algorithm 1 line 14), in the same pass.  `out`
    may be None when `model` is given."""
    assert out is not None or model is not None
    assert out is None or out.numel() >= plan.d
    assert model is None or (model.numel() >= plan.d and model.is_contiguous())
    a = AggregateArgs(buf.words.data_ptr(), buf.words_stride, buf.chunk_offset.data_ptr(), buf.sub_bits.data_ptr(),
                      books.handle, None if out is None else out.data_ptr(), buf.status.data_ptr(),
                      None if model is None else model.data_ptr(), float(np.float32(eta)), 0)
    _check("co3_ps_aggregate", lib().co3_ps_aggregate(plan.handle, C.byref(a), _stream(stream)))


# ---- training around the codec: layer norm, the orthogonalised update ----

F32, BF16, F16 = 0, 1, 2
PRODUCTS_PAIR, PRODUCTS_HIGH = 0, 1
MAX_NS_STEPS = 32
MAX_NORM_COLS = 32768
MUON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


@functools.lru_cache(maxsize=1)
def _tensor_types():
    import torch
    return {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def tensor_type(dtype):
    """CO3_F32, CO3_BF16 or CO3_F16 of a torch dtype."""
    t = _tensor_types().get(dtype)
    if t is None:
        raise TypeError(f"float32, bfloat16 or float16 tensors are taken, not {dtype}")
    return t


def _allocate_on(stream):
    """For what a call allocates: memory of the stream that it runs on, which is not given to another before it is done there."""
    import torch
    return torch.cuda.stream(stream)   # None: the current one


def _stream_of(gpu, stream):
    """The stream of a call with tensors of this GPU (as Tensor.get_device() says it: -1 is the host)."""
    if gpu < 0:
        raise ValueError("tensors on a GPU are taken")
    if _torch_c is None:
        _stream()
    on = _torch_c._cuda_getDevice() if stream is None else stream.device.index
    if on != gpu:
        raise ValueError(f"tensors on GPU {on}, which the stream is of, are taken, not on {gpu}")
    return _torch_c._cuda_getCurrentRawStream(gpu) if stream is None else stream.cuda_stream


def _call_on(gpu, call, *args):
    """call(*args) with this GPU current: the handle of a GPU's default stream is 0, which means that of the current one."""
    if _torch_c._cuda_getDevice() == gpu:
        return call(*args)
    import torch
    with torch.cuda.device(gpu):
        return call(*args)


class MatrixPlan:
    """co3_matrix_plan: matrices (offset, rows, cols[, ld]) of a flat vector of `dtype`, and the factor of each one's
    orthogonalised form (scales; None: 1).  products: PRODUCTS_PAIR, about fp32's precision, or PRODUCTS_HIGH, a third of
    the matrix instructions at errors of about bfloat16's rounding."""

    def __init__(self, matrices, dtype=None, scales=None, products=PRODUCTS_PAIR):
        import torch
        dtype = torch.float32 if dtype is None else dtype
        self.dtype, self.count = dtype, len(matrices)
        self.products = PRODUCTS_PAIR if products is None else int(products)
        scales = [1.0] * self.count if scales is None else [float(x) for x in scales]
        assert len(scales) == self.count
        table = (Matrix * self.count)()
        for k, (m, scale) in enumerate(zip(matrices, scales)):
            offset, rows, cols = (int(x) for x in m[:3])
            table[k] = Matrix(offset, int(m[3]) if len(m) > 3 else cols, rows, cols, scale, 0)
        h = C.c_void_p()
        _check("co3_matrix_plan_create", lib().co3_matrix_plan_create(self.count, C.cast(table, C.c_void_p), tensor_type(dtype),
                                                                      self.products, C.byref(h)))
        self.handle = h
        self.workspace_bytes = int(lib().co3_matrix_plan_workspace_bytes(h))
        self.elements = int(lib().co3_matrix_plan_elements(h))
        self.gpu = torch.cuda.current_device()

    def close(self):
        if getattr(self, "handle", None):
            lib().co3_matrix_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


@functools.lru_cache(maxsize=64)
def _ns_triples(triples, steps):
    c = np.asarray(triples, dtype=np.float32)
    return np.ascontiguousarray(np.broadcast_to(c, (steps, 3)))


def _ns_coefficients(coefficients, steps):
    """float32 [steps][3]: one triple for all steps, or one of each."""
    if type(coefficients) is not tuple or not all(type(x) is float for x in coefficients):
        coefficients = tuple(map(tuple, np.broadcast_to(np.asarray(coefficients, dtype=np.float32), (int(steps), 3)).tolist()))
    return _ns_triples(coefficients, int(steps))


def _matrix_vector(plan, t, name):
    if t.dtype != plan.dtype or t.dim() != 1 or not t.is_contiguous() or t.numel() < plan.elements or t.get_device() != plan.gpu:
        raise ValueError(f"{name}: a contiguous vector of at least {plan.elements} {plan.dtype} elements on the plan's GPU is taken")


def _matrix_workspace(plan, workspace, status, stream):
    if status is not None and (status.get_device() != plan.gpu or status.numel() < STATUS_WORDS or status.element_size() != 8 or
                               not status.is_contiguous()):
        raise ValueError(f"status: {STATUS_WORDS} contiguous int64 elements on the plan's GPU are taken")
    if workspace is None:
        import torch
        with _allocate_on(stream):
            workspace = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device=f"cuda:{plan.gpu}")
    elif workspace.get_device() != plan.gpu or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous memory of the plan's GPU is taken")
    return workspace


def co3_orthogonalize(plan, g, out=None, steps=5, coefficients=MUON_COEFFICIENTS, eps=1e-7, workspace=None, status=None,
                      stream=None):
    """out = scale * Newton-Schulz iterate of every matrix of the flat vector g (out may be g; None: a new vector, with
    zeros outside the matrices).  coefficients: (a, b, c) of every step, or `steps` triples.  status (int64
    [STATUS_WORDS], or None): matrices whose norm is not finite are added to status[STAT_NONFINITE]."""
    _matrix_vector(plan, g, "g")
    on = _stream_of(plan.gpu, stream)
    if out is None:
        import torch
        with _allocate_on(stream):
            out = torch.zeros_like(g)
    _matrix_vector(plan, out, "out")
    workspace = _matrix_workspace(plan, workspace, status, stream)
    c = _ns_coefficients(coefficients, steps)
    a = _pack_orthogonalize(g.data_ptr(), out.data_ptr(), c.ctypes.data, int(steps), float(eps),
                          0 if status is None else status.data_ptr(), workspace.data_ptr(), workspace.nbytes)
    _check("co3_orthogonalize", lib().co3_orthogonalize(plan.handle, a, on))
    return out


def co3_muon_update(plan, g, momentum, model, eta, beta=0.95, nesterov=True, weight_decay=0.0, steps=5,
                    coefficients=MUON_COEFFICIENTS, eps=1e-7, workspace=None, status=None, stream=None):
    """momentum = beta momentum + g, u = g + beta momentum (nesterov) or momentum, model = model (1 - eta weight_decay) -
    eta scale NS(u), for every matrix of the float32 vectors; the elements outside the matrices stay."""
    for t, name in ((g, "g"), (momentum, "momentum"), (model, "model")):
        _matrix_vector(plan, t, name)
    on = _stream_of(plan.gpu, stream)
    workspace = _matrix_workspace(plan, workspace, status, stream)
    c = _ns_coefficients(coefficients, steps)
    a = _pack_muon(g.data_ptr(), momentum.data_ptr(), model.data_ptr(), c.ctypes.data, int(steps), float(eps), float(eta), float(beta),
                 float(weight_decay), int(bool(nesterov)), 0 if status is None else status.data_ptr(), workspace.data_ptr(),
                 workspace.nbytes)
    _check("co3_muon_update", lib().co3_muon_update(plan.handle, a, on))


def _norm_rows(t, name):
    """(users, rows per user, columns, elements between rows) of a [rows, cols] or [users, rows, cols] tensor."""
    shape = t.shape
    if len(shape) == 3:
        users, rows, cols = shape
    elif len(shape) == 2:
        users, (rows, cols) = 1, shape
    else:
        raise ValueError(f"{name}: [rows, cols] or [users, rows, cols] is taken")
    if t.is_contiguous():
        return users, rows, cols, cols
    stride = t.stride(-2) if rows > 1 else t.stride(0) if len(shape) == 3 and users > 1 else cols
    if t.stride(-1) != 1 and cols > 1:
        raise ValueError(f"{name}: rows have to be contiguous")
    if len(shape) == 3 and users > 1 and rows > 1 and t.stride(0) != rows * stride:
        raise ValueError(f"{name}: all rows have to lie the same distance apart")
    return users, rows, cols, stride


def _norm_vector(t, n, name, gpu, f32):
    if t is None:
        return 0
    if t.dtype is not f32 or t.numel() != n or t.get_device() != gpu or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous float32 elements on x's device are taken")
    return t.data_ptr()


@functools.lru_cache(maxsize=1)
def _float32():
    import torch
    return torch.float32


def _rows_like(t, shape, dtype, name, gpu):
    """Elements between the rows of a tensor of x's shape and type."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != gpu:
        raise ValueError(f"{name}: the shape, type and device of x are taken")
    return shape[-1] if t.is_contiguous() else _norm_rows(t, name)[3]


def co3_layernorm(x, weight=None, bias=None, eps=1e-5, y=None, mean=None, rstd=None, stream=None):
    """(y, mean, rstd) of x [rows, cols] or [users, rows, cols] (float32, bfloat16, float16; rows may lie apart): y of x's
    type, mean and rstd float32 without the last dimension.  weight, bias: float32 [cols] or None.  y may be x."""
    users, rows, cols, stride = _norm_rows(x, "x")
    shape, dtype, gpu, f32 = x.shape, x.dtype, x.get_device(), _float32()
    kind = tensor_type(dtype)
    if y is None or mean is None or rstd is None:
        import torch
        with _allocate_on(stream):
            y = torch.empty(shape, dtype=dtype, device=x.device) if y is None else y
            mean = torch.empty(shape[:-1], dtype=f32, device=x.device) if mean is None else mean
            rstd = torch.empty(shape[:-1], dtype=f32, device=x.device) if rstd is None else rstd
    a = _pack_layernorm(x.data_ptr(), y.data_ptr(), _norm_vector(weight, cols, "weight", gpu, f32), _norm_vector(bias, cols, "bias", gpu, f32),
                      _norm_vector(mean, users * rows, "mean", gpu, f32), _norm_vector(rstd, users * rows, "rstd", gpu, f32), users * rows, stride,
                      _rows_like(y, shape, dtype, "y", gpu), cols, kind, float(eps), 0)
    on = _stream_of(gpu, stream)
    _check("co3_layernorm", _call_on(gpu, lib().co3_layernorm, a, on))
    return y, mean, rstd


def co3_layernorm_backward_workspace_bytes(users, rows, cols):
    return int(lib().co3_layernorm_backward_workspace_bytes(int(users), int(rows), int(cols)))


def _grad_rows(t, users, cols, name, gpu, f32):
    """Elements between two users' gradients."""
    shape = t.shape
    if t.dtype is not f32 or t.get_device() != gpu or shape[-1] != cols or (shape[0] if len(shape) == 2 else 1) != users or \
            len(shape) > 2 or (cols > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: float32 [users, cols] on x's device with contiguous rows is taken ([cols] for one user)")
    return t.stride(0) if users > 1 else cols


def co3_layernorm_backward(dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, accumulate=False, workspace=None,
                           stream=None):
    """dx of co3_layernorm, and where dweight / dbias are given (float32 [users, cols], rows may lie apart: a layer's part of
    the users' gradients that co3_encode reads) the weight's gradients of every user: written, or added with accumulate."""
    users, rows, cols, x_stride = _norm_rows(x, "x")
    stride = cols
    shape, dtype, gpu, f32 = x.shape, x.dtype, x.get_device(), _float32()
    kind = tensor_type(dtype)
    if dweight is not None:
        stride = _grad_rows(dweight, users, cols, "dweight", gpu, f32)
    if dbias is not None:
        other = _grad_rows(dbias, users, cols, "dbias", gpu, f32)
        if dweight is not None and other != stride:
            raise ValueError("dweight and dbias: the same distance between users is taken")
        stride = other
    if dx is None or workspace is None:
        import torch
        with _allocate_on(stream):
            dx = torch.empty(shape, dtype=dtype, device=x.device) if dx is None else dx
            if workspace is None and (dweight is not None or dbias is not None):
                workspace = torch.empty(co3_layernorm_backward_workspace_bytes(users, rows, cols), dtype=torch.uint8, device=x.device)
    if workspace is not None and (workspace.get_device() != gpu or not workspace.is_contiguous()):
        raise ValueError("workspace: contiguous memory of x's GPU is taken")
    a = _pack_layernorm_backward(dy.data_ptr(), x.data_ptr(), dx.data_ptr(), _norm_vector(weight, cols, "weight", gpu, f32),
                              _norm_vector(mean, users * rows, "mean", gpu, f32), _norm_vector(rstd, users * rows, "rstd", gpu, f32),
                              0 if dweight is None else dweight.data_ptr(), 0 if dbias is None else dbias.data_ptr(),
                              stride, rows, _rows_like(dy, shape, dtype, "dy", gpu), x_stride, _rows_like(dx, shape, dtype, "dx", gpu), users, cols,
                              kind, 1 if accumulate else 0, 0 if workspace is None else workspace.data_ptr(),
                              0 if workspace is None else workspace.nbytes)
    on = _stream_of(gpu, stream)
    _check("co3_layernorm_backward", _call_on(gpu, lib().co3_layernorm_backward, a, on))
    return dx
