"""ctypes binding of libtahq.so: same names as the C ABI, marshalling only."""
import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
# TAHQ_LIBRARY lets an experiment load another build of the same library
_LIB_PATH = os.environ.get("TAHQ_LIBRARY") or os.path.join(HERE, "libtahq.so")

F32, BF16 = 0, 1


class TahqError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {tahq_status_string(status)} (status {status})")


class tahq_config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("batch", C.c_uint32), ("seq", C.c_uint32), ("hidden", C.c_uint32),
        ("tile", C.c_uint32), ("dtype", C.c_uint32), ("scope", C.c_uint32),
        ("budget_bits", C.c_float), ("tau", C.c_float),
        ("eps_l1", C.c_float), ("eps_log", C.c_float), ("eps_ratio", C.c_float),
        ("alloc_tile", C.c_uint32), ("low_bits", C.c_uint32),
    ]


class tahq_naive_config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("batch", C.c_uint32), ("seq", C.c_uint32), ("hidden", C.c_uint32),
        ("dtype", C.c_uint32), ("bits", C.c_uint32), ("scale", C.c_float),
    ]


class tahq_mx4_config(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "rows", "cols", "ld", "dtype", "transform", "scale_rule")]


class tahq_mx4_matmul_config(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "m", "n", "k", "ldc", "out_dtype", "accumulate")]


class tahq_norm_config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("rows", C.c_uint32), ("cols", C.c_uint32), ("dtype", C.c_uint32), ("gate_rows", C.c_uint32),
        ("eps", C.c_float), ("residual_scale", C.c_float),
        ("accumulate", C.c_uint32), ("transform", C.c_uint32), ("scale_rule", C.c_uint32),
    ]


_lib = None


def library_path():
    return _LIB_PATH


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2506_01352_amd.build` "
            "(there is no fallback path)")
    L = C.CDLL(_LIB_PATH)
    P = C.POINTER(tahq_config)
    L.tahq_config_default.restype = None
    L.tahq_config_default.argtypes = [P]
    L.tahq_k_per_unit.restype = C.c_uint64
    L.tahq_k_per_unit.argtypes = [P]
    L.tahq_packed_size.restype = C.c_size_t
    L.tahq_packed_size.argtypes = [P]
    L.tahq_workspace_size.restype = C.c_size_t
    L.tahq_workspace_size.argtypes = [P]
    L.tahq_encode.restype = C.c_int
    L.tahq_encode.argtypes = [P, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_void_p]
    L.tahq_encode_noalloc.restype = C.c_int
    L.tahq_encode_noalloc.argtypes = [P, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.tahq_encode_phases.restype = C.c_int
    L.tahq_encode_phases.argtypes = [P, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_uint32,
                                     C.c_void_p]
    L.tahq_samples_packed_size.restype = C.c_size_t
    L.tahq_samples_packed_size.argtypes = [P, C.c_uint32]
    L.tahq_samples_workspace_size.restype = C.c_size_t
    L.tahq_samples_workspace_size.argtypes = [P, C.c_uint32]
    L.tahq_encode_samples.restype = C.c_int
    L.tahq_encode_samples.argtypes = [P, C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p,
                                      C.c_size_t, C.c_void_p]
    L.tahq_decode_samples.restype = C.c_int
    L.tahq_decode_samples.argtypes = [P, C.c_uint32, C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint32,
                                      C.c_void_p]
    L.tahq_decode.restype = C.c_int
    L.tahq_decode.argtypes = [P, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p]
    L.tahq_tile_entropy.restype = C.c_int
    L.tahq_tile_entropy.argtypes = [P, C.c_void_p, C.c_void_p, C.c_void_p]
    L.tahq_alloc_tile_entropy.restype = C.c_int
    L.tahq_alloc_tile_entropy.argtypes = [P, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.tahq_parse_header.restype = C.c_int
    L.tahq_parse_header.argtypes = [C.c_void_p, P]
    L.tahq_status_string.restype = C.c_char_p
    L.tahq_status_string.argtypes = [C.c_int]
    L.tahq_version.restype = C.c_uint32
    L.tahq_version.argtypes = []
    PN = C.POINTER(tahq_naive_config)
    L.tahq_naive_config_default.restype = None
    L.tahq_naive_config_default.argtypes = [PN]
    L.tahq_naive_packed_size.restype = C.c_size_t
    L.tahq_naive_packed_size.argtypes = [PN]
    L.tahq_naive_encode.restype = C.c_int
    L.tahq_naive_encode.argtypes = [PN, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.tahq_naive_decode.restype = C.c_int
    L.tahq_naive_decode.argtypes = [PN, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint32, C.c_void_p]
    V, Z, PX, PM, PB = C.c_void_p, C.c_size_t, C.POINTER(tahq_mx4_config), C.POINTER(tahq_mx4_matmul_config), C.POINTER(tahq_norm_config)
    for name, result, arguments in (
            ("tahq_mx4_config_default", None, [PX]),
            ("tahq_mx4_packed_size", Z, [C.c_uint32, C.c_uint32]),
            ("tahq_mx4_quantize", C.c_int, [PX, V, V, Z, V, Z, V]),
            ("tahq_mx4_dequantize", C.c_int, [PX, V, Z, V, V]),
            ("tahq_mx4_matmul_config_default", None, [PM]),
            ("tahq_mx4_matmul_workspace_size", Z, [PM]),
            ("tahq_mx4_matmul", C.c_int, [PM, V, Z, V, Z, V, V, Z, V]),
            ("tahq_mx4_linear_workspace_size", Z, [PX, PM]),
            ("tahq_mx4_linear", C.c_int, [PX, PM, V, V, Z, V, V, Z, V]),
            ("tahq_norm_config_default", None, [PB]),
            ("tahq_norm_forward", C.c_int, [PB, V, V, V, V, V, V, V, V, Z, V, V]),
            ("tahq_norm_workspace_size", Z, [PB]),
            ("tahq_norm_backward", C.c_int, [PB] + [V] * 14 + [Z, V])):
        f = getattr(L, name)
        f.restype, f.argtypes = result, arguments
    _lib = L
    return L


def tahq_config_default():
    cfg = tahq_config()
    _load().tahq_config_default(C.byref(cfg))
    return cfg


def make_config(batch, seq, hidden, tile, dtype, budget_bits, tau=2.0, eps_l1=1e-8, eps_log=1e-8,
                eps_ratio=1e-8, scope=0, alloc_tile=0, low_bits=0):
    cfg = tahq_config_default()
    cfg.alloc_tile = alloc_tile
    cfg.low_bits = low_bits
    cfg.batch, cfg.seq, cfg.hidden, cfg.tile = batch, seq, hidden, tile
    cfg.dtype, cfg.scope = dtype, scope
    cfg.budget_bits, cfg.tau = budget_bits, tau
    cfg.eps_l1, cfg.eps_log, cfg.eps_ratio = eps_l1, eps_log, eps_ratio
    return cfg


def tahq_k_per_unit(cfg):
    return int(_load().tahq_k_per_unit(C.byref(cfg)))


def tahq_packed_size(cfg):
    return int(_load().tahq_packed_size(C.byref(cfg)))


def tahq_workspace_size(cfg):
    return int(_load().tahq_workspace_size(C.byref(cfg)))


def tahq_status_string(status):
    return _load().tahq_status_string(int(status)).decode()


def tahq_version():
    return int(_load().tahq_version())


def _dev_ptr(t):
    """Device address of a torch tensor (None -> NULL); ctypes converts it."""
    if t is None or isinstance(t, int):
        return t
    assert t.is_cuda and t.is_contiguous(), "device tensor, contiguous"
    return t.data_ptr()


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


_ESIZE = {F32: 4, BF16: 2}


def _check_tensor(where, name, t, elements, dtype):
    """The C ABI carries no capacity for the activation tensors: refuse, on the host, a tensor that is shorter than
    batch*seq*hidden elements of `dtype`, or whose elements have another size (byte buffers are taken as they are)."""
    if t is None or isinstance(t, int):
        return
    esize = _ESIZE.get(dtype)
    if esize is None:
        return                                   # the library rejects the dtype itself
    size = t.element_size()
    if size != esize and size != 1:
        raise ValueError(f"{where}: {name} has {size}-byte elements, the configuration says {esize}")
    if t.numel() * size < elements * esize:
        raise ValueError(f"{where}: {name} holds {_nbytes(t)} bytes, the configuration needs {elements * esize}")


def _elements(cfg):
    return cfg.batch * cfg.seq * cfg.hidden


_current_raw_stream = None


def _stream_handle(stream):
    """Address of a stream; of torch's current stream on the current device if there is none.  The calls on small tensors are
    bound by what they cost the host, and the stream object torch.cuda.current_stream() builds was a fifth of that."""
    global _current_raw_stream
    if stream is None:
        if _current_raw_stream is None:
            import torch
            handle = torch.cuda.current_stream().cuda_stream         # initialises torch.cuda if nothing has yet
            raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
            if raw is None or device is None:
                return handle
            _current_raw_stream = lambda: raw(device())
        return _current_raw_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def tahq_encode(cfg, d_in, d_packed, d_workspace, stream=None, packed_capacity=None, workspace_capacity=None):
    """Enqueue the encoder.  All tensors are device tensors owned by the caller."""
    cap = _nbytes(d_packed) if packed_capacity is None else packed_capacity
    wcap = _nbytes(d_workspace) if workspace_capacity is None else workspace_capacity
    _check_tensor("tahq_encode", "d_in", d_in, _elements(cfg), cfg.dtype)
    rc = (_lib or _load()).tahq_encode(C.byref(cfg), _dev_ptr(d_in), _dev_ptr(d_packed), cap, _dev_ptr(d_workspace), wcap,
                             _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_encode")


NOALLOC_MAX_WORKSPACE = 32 << 20     # TAHQ_NOALLOC_MAX_WORKSPACE of include/tahq.h


def tahq_encode_noalloc(cfg, d_in, d_packed, stream=None, packed_capacity=None):
    """tahq_encode on the library's built-in scratch: no workspace argument, nothing allocated."""
    cap = _nbytes(d_packed) if packed_capacity is None else packed_capacity
    _check_tensor("tahq_encode_noalloc", "d_in", d_in, _elements(cfg), cfg.dtype)
    rc = (_lib or _load()).tahq_encode_noalloc(C.byref(cfg), _dev_ptr(d_in), _dev_ptr(d_packed), cap, _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_encode_noalloc")


PHASE_PROLOGUE, PHASE_ENTROPY, PHASE_SELECT, PHASE_QUANT, PHASE_ALL = 1, 2, 4, 8, 15
SELECT_MULTI_LAUNCH = 16      # option bit for tahq_encode_phases: see include/tahq.h


def tahq_encode_phases(cfg, d_in, d_packed, d_workspace, phases, stream=None):
    _check_tensor("tahq_encode_phases", "d_in", d_in, _elements(cfg), cfg.dtype)
    rc = (_lib or _load()).tahq_encode_phases(C.byref(cfg), _dev_ptr(d_in), _dev_ptr(d_packed), _nbytes(d_packed),
                                    _dev_ptr(d_workspace), _nbytes(d_workspace), phases, _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_encode_phases")


def tahq_decode(cfg, d_packed, d_out, out_dtype, stream=None, packed_bytes=None):
    nbytes = _nbytes(d_packed) if packed_bytes is None else packed_bytes
    _check_tensor("tahq_decode", "d_out", d_out, _elements(cfg), out_dtype)
    rc = (_lib or _load()).tahq_decode(C.byref(cfg), _dev_ptr(d_packed), nbytes, _dev_ptr(d_out), out_dtype, None, 0,
                             _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_decode")


def tahq_samples_packed_size(cfg, count):
    return int(_load().tahq_samples_packed_size(C.byref(cfg), count))


def tahq_samples_workspace_size(cfg, count):
    return int(_load().tahq_samples_workspace_size(C.byref(cfg), count))


def tahq_encode_samples(cfg, first, count, d_in, d_packed, d_workspace, stream=None):
    """Samples [first, first + count) of the whole tensor d_in -> a self-contained stream in d_packed."""
    _check_tensor("tahq_encode_samples", "d_in", d_in, _elements(cfg), cfg.dtype)
    rc = (_lib or _load()).tahq_encode_samples(C.byref(cfg), first, count, _dev_ptr(d_in), _dev_ptr(d_packed), _nbytes(d_packed),
                                     _dev_ptr(d_workspace), _nbytes(d_workspace), _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_encode_samples")


def tahq_decode_samples(cfg, first, count, d_packed, d_out, out_dtype, stream=None):
    """A stream of tahq_encode_samples -> samples [first, first + count) of the whole tensor d_out."""
    _check_tensor("tahq_decode_samples", "d_out", d_out, _elements(cfg), out_dtype)
    rc = (_lib or _load()).tahq_decode_samples(C.byref(cfg), first, count, _dev_ptr(d_packed), _nbytes(d_packed), _dev_ptr(d_out),
                                     out_dtype, _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_decode_samples")


def tahq_tile_entropy(cfg, d_in, d_entropy, stream=None):
    _check_tensor("tahq_tile_entropy", "d_in", d_in, _elements(cfg), cfg.dtype)
    _check_tensor("tahq_tile_entropy", "d_entropy", d_entropy, _elements(cfg) // max(cfg.tile, 1), F32)
    rc = (_lib or _load()).tahq_tile_entropy(C.byref(cfg), _dev_ptr(d_in), _dev_ptr(d_entropy), _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_tile_entropy")


def tahq_alloc_tile_entropy(cfg, d_in, d_entropy, d_workspace, stream=None):
    _check_tensor("tahq_alloc_tile_entropy", "d_in", d_in, _elements(cfg), cfg.dtype)
    _check_tensor("tahq_alloc_tile_entropy", "d_entropy", d_entropy,
                  _elements(cfg) // max(cfg.alloc_tile or cfg.tile, 1), F32)
    rc = (_lib or _load()).tahq_alloc_tile_entropy(C.byref(cfg), _dev_ptr(d_in), _dev_ptr(d_entropy), _dev_ptr(d_workspace),
                                         _nbytes(d_workspace), _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_alloc_tile_entropy")


def tahq_parse_header(header_bytes):
    buf = C.create_string_buffer(bytes(header_bytes[:64]), 64)
    cfg = tahq_config()
    rc = _load().tahq_parse_header(buf, C.byref(cfg))
    if rc != 0:
        raise TahqError(rc, "tahq_parse_header")
    return cfg


# ---- backward-pass fixed-point compressor (include/tahq_naive.h)

def tahq_naive_config_default():
    cfg = tahq_naive_config()
    _load().tahq_naive_config_default(C.byref(cfg))
    return cfg


def make_naive_config(batch, seq, hidden, dtype, bits, scale=1.0):
    cfg = tahq_naive_config_default()
    cfg.batch, cfg.seq, cfg.hidden, cfg.dtype, cfg.bits, cfg.scale = batch, seq, hidden, dtype, bits, scale
    return cfg


def tahq_naive_packed_size(cfg):
    return int(_load().tahq_naive_packed_size(C.byref(cfg)))


def tahq_naive_encode(cfg, d_in, d_packed, stream=None, packed_capacity=None):
    cap = _nbytes(d_packed) if packed_capacity is None else packed_capacity
    _check_tensor("tahq_naive_encode", "d_in", d_in, _elements(cfg), cfg.dtype)
    rc = (_lib or _load()).tahq_naive_encode(C.byref(cfg), _dev_ptr(d_in), _dev_ptr(d_packed), cap, _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_naive_encode")


def tahq_naive_decode(cfg, d_packed, d_out, out_dtype, stream=None, packed_bytes=None):
    nbytes = _nbytes(d_packed) if packed_bytes is None else packed_bytes
    _check_tensor("tahq_naive_decode", "d_out", d_out, _elements(cfg), out_dtype)
    rc = (_lib or _load()).tahq_naive_decode(C.byref(cfg), _dev_ptr(d_packed), nbytes, _dev_ptr(d_out), out_dtype,
                                   _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_naive_decode")


class Codec:
    """Buffers for one configuration, allocated once through torch, and the two calls on them."""

    def __init__(self, cfg, device="cuda:0", out_dtype=None):
        import torch
        self.cfg = cfg
        self.out_dtype = cfg.dtype if out_dtype is None else out_dtype
        size = tahq_packed_size(cfg)
        if size == 0:
            raise TahqError(2, "tahq_packed_size")
        n = cfg.batch * cfg.seq * cfg.hidden
        self.packed = torch.empty(size, dtype=torch.uint8, device=device)
        self.workspace = torch.empty(max(tahq_workspace_size(cfg), 16), dtype=torch.uint8, device=device)
        self.out = torch.empty(n, dtype=torch.float32 if self.out_dtype == F32 else torch.bfloat16, device=device)

    def encode(self, d_in, stream=None):
        tahq_encode(self.cfg, d_in, self.packed, self.workspace, stream)
        return self.packed

    def decode(self, stream=None):
        tahq_decode(self.cfg, self.packed, self.out, self.out_dtype, stream)
        return self.out


# ---- microscaled 4-bit matrices (include/tahq_mx4.h)

MX4_FLOOR, MX4_COVER = 0, 1


def tahq_mx4_config_default():
    cfg = tahq_mx4_config()
    _load().tahq_mx4_config_default(C.byref(cfg))
    return cfg


def make_mx4_config(rows, cols, dtype, ld=0, transform=0, scale_rule=MX4_FLOOR):
    cfg = tahq_mx4_config_default()
    cfg.rows, cfg.cols, cfg.dtype, cfg.ld, cfg.transform, cfg.scale_rule = rows, cols, dtype, ld, transform, scale_rule
    return cfg


def tahq_mx4_packed_size(rows, cols):
    return int(_load().tahq_mx4_packed_size(rows, cols))


def _strided_elements(rows, cols, ld):
    """Elements from the first to the last one of a [rows, cols] tensor of row stride ld."""
    return (rows - 1) * (ld or cols) + cols if rows and cols else 0


def _rows_ptr(t, cols, ld):
    """Device address of a row-major tensor whose rows may lie `ld` elements apart (0: `cols`): contiguous, or a two-dimensional view that
    says so.  A broadcast view, whose rows are one row, is neither."""
    if t is None or isinstance(t, int):
        return t
    if not t.is_contiguous():
        apart = t.is_cuda and t.dim() == 2 and t.stride(1) == 1 and t.stride(0) == (ld or cols)
        assert apart, "device tensor, rows of unit stride, ld apart"
        return t.data_ptr()
    return _dev_ptr(t)


_half = None


def _check_not_half(where, name, t, dtype):
    """float16 is no bf16, though its elements have the size that _check_tensor asks for (integers and bytes are taken for bf16's bits)."""
    global _half
    if _half is None:
        import torch
        _half = torch.float16
    if dtype == BF16 and getattr(t, "dtype", None) is _half:
        raise ValueError(f"{where}: {name} is a tensor of {t.dtype}, the configuration says torch.bfloat16")


def _check_rows(where, name, t, rows, cols, ld, dtype):
    """_check_tensor for a tensor of rows that lie `ld` elements apart; a view is checked by its own shape."""
    if t is None or isinstance(t, int):
        return
    _check_not_half(where, name, t, dtype)
    if t.is_contiguous():
        _check_tensor(where, name, t, _strided_elements(rows, cols, ld), dtype)
    elif dtype in _ESIZE and (t.element_size() != _ESIZE[dtype] or t.dim() != 2 or t.shape[0] < rows or t.shape[1] < cols):
        raise ValueError(f"{where}: {name} is a {tuple(t.shape)} view of {t.element_size()}-byte elements, the configuration needs "
                         f"[{rows}, {cols}] of {_ESIZE[dtype]}")


def tahq_mx4_quantize(cfg, d_in, d_packed=None, d_packed_t=None, stream=None):
    """[rows, cols] -> packed along rows (d_packed) and / or along columns (d_packed_t), read once."""
    _check_rows("tahq_mx4_quantize", "d_in", d_in, cfg.rows, cfg.cols, cfg.ld, cfg.dtype)
    rc = (_lib or _load()).tahq_mx4_quantize(C.byref(cfg), _rows_ptr(d_in, cfg.cols, cfg.ld), _dev_ptr(d_packed), _nbytes(d_packed),
                                             _dev_ptr(d_packed_t), _nbytes(d_packed_t), _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_mx4_quantize")


def tahq_mx4_dequantize(cfg, d_packed, d_out, stream=None):
    _check_rows("tahq_mx4_dequantize", "d_out", d_out, cfg.rows, cfg.cols, cfg.ld, cfg.dtype)
    rc = (_lib or _load()).tahq_mx4_dequantize(C.byref(cfg), _dev_ptr(d_packed), _nbytes(d_packed), _rows_ptr(d_out, cfg.cols, cfg.ld),
                                               _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_mx4_dequantize")


def tahq_mx4_matmul_config_default():
    cfg = tahq_mx4_matmul_config()
    _load().tahq_mx4_matmul_config_default(C.byref(cfg))
    return cfg


def make_mx4_matmul_config(m, n, k, out_dtype, ldc=0, accumulate=0):
    cfg = tahq_mx4_matmul_config_default()
    cfg.m, cfg.n, cfg.k, cfg.out_dtype, cfg.ldc, cfg.accumulate = m, n, k, out_dtype, ldc, accumulate
    return cfg


def tahq_mx4_matmul_workspace_size(cfg):
    return int(_load().tahq_mx4_matmul_workspace_size(C.byref(cfg)))


def tahq_mx4_matmul(cfg, d_a, d_b, d_c, d_workspace=None, stream=None):
    """C[m, n] (+)= A[m, k] B[n, k]^T of packed matrices."""
    _check_rows("tahq_mx4_matmul", "d_c", d_c, cfg.m, cfg.n, cfg.ldc, cfg.out_dtype)
    rc = (_lib or _load()).tahq_mx4_matmul(C.byref(cfg), _dev_ptr(d_a), _nbytes(d_a), _dev_ptr(d_b), _nbytes(d_b), _rows_ptr(d_c, cfg.n, cfg.ldc),
                                           _dev_ptr(d_workspace), _nbytes(d_workspace), _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_mx4_matmul")


def tahq_mx4_linear_workspace_size(x, cfg):
    return int(_load().tahq_mx4_linear_workspace_size(C.byref(x), C.byref(cfg)))


def tahq_mx4_linear(x, cfg, d_x, d_b, d_y, d_workspace, stream=None):
    """y[m, n] (+)= quantized(x)[m, k] B[n, k]^T, x in fp32 or bf16."""
    _check_rows("tahq_mx4_linear", "d_x", d_x, x.rows, x.cols, x.ld, x.dtype)
    _check_rows("tahq_mx4_linear", "d_y", d_y, cfg.m, cfg.n, cfg.ldc, cfg.out_dtype)
    rc = (_lib or _load()).tahq_mx4_linear(C.byref(x), C.byref(cfg), _rows_ptr(d_x, x.cols, x.ld), _dev_ptr(d_b), _nbytes(d_b),
                                           _rows_ptr(d_y, cfg.n, cfg.ldc), _dev_ptr(d_workspace), _nbytes(d_workspace), _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_mx4_linear")


def _bytes_on(device, size):
    import torch
    return torch.empty(max(size, 16), dtype=torch.uint8, device=device)


def _packed_on(device, rows, cols, transform):
    """A buffer for a packed matrix, which carries what its bytes do not tell: rows, columns and whether blocks are rotated."""
    t = _bytes_on(device, tahq_mx4_packed_size(rows, cols))
    t.mx4_form = (rows, cols, transform)
    return t


def _check_packed(where, name, t, form, size):
    """A packed matrix that a class is given: of the form that the buffer carries, if it does, and bytes enough."""
    if getattr(t, "mx4_form", None) != form or t.numel() < size:
        _check_bytes(where, name, t, form, size)


def _check_bytes(where, name, t, form, size):
    if t.element_size() != 1 or t.numel() < size or not t.is_contiguous() or getattr(t, "mx4_form", form) != form:
        raise ValueError(f"{where}: {name} is a {tuple(t.shape)} tensor of {t.dtype}{', packed as ' + str(t.mx4_form) if hasattr(t, 'mx4_form') else ''}: "
                         f"{size} bytes of a packed matrix of (rows, cols, transform) = {form} are needed")


def _check_slot(where, slot, in_flight):
    if not 0 <= slot < in_flight:
        raise ValueError(f"{where}: slot {slot} of {in_flight} micro-batches in flight")


def _torch_dtype(dtype):
    import torch
    return torch.float32 if dtype == F32 else torch.bfloat16


def _holds(t, rows, cols):
    return t.numel() == rows * cols and (t.dim() < 2 or t.shape[-1] == cols)


def _input_of(where, name, t, rows, cols, dtype):
    """Device address of a class's input: a contiguous device tensor of `dtype`, [.., cols] with `rows` rows in all, or flat.  What a call on a
    few tokens takes is mostly what it costs the host, so the classes look at an input once and keep their own buffers' addresses at hand;
    a single row is the same in any shape."""
    if (t.dtype is not dtype or not t.is_contiguous() or not t.is_cuda
            or (t.numel() != cols if rows == 1 else t.shape != (rows, cols) and not _holds(t, rows, cols))):
        raise ValueError(f"{where}: {name} is a {tuple(t.shape)} tensor of {t.dtype} on {t.device}"
                         f"{'' if t.is_contiguous() else ', not contiguous'}: [{rows}, {cols}] contiguous elements of {dtype} on the GPU are needed")
    return t.data_ptr()


class Mx4Tensor:
    """Buffers of one tensor's packed form, along its rows and if asked along its columns, and of its values back."""

    def __init__(self, cfg, transposed=False, device="cuda:0"):
        import torch
        if tahq_mx4_packed_size(cfg.rows, cfg.cols) == 0:
            raise TahqError(2, "tahq_mx4_packed_size")
        self.cfg = cfg
        self.packed = _packed_on(device, cfg.rows, cfg.cols, cfg.transform)
        self.packed_t = _packed_on(device, cfg.cols, cfg.rows, cfg.transform) if transposed else None
        self._values = make_mx4_config(cfg.rows, cfg.cols, cfg.dtype, 0, cfg.transform, cfg.scale_rule)
        self._values_t = make_mx4_config(cfg.cols, cfg.rows, cfg.dtype, 0, cfg.transform, cfg.scale_rule)
        kind = _torch_dtype(cfg.dtype)
        self.out = torch.empty(cfg.rows, cfg.cols, dtype=kind, device=device)
        self.out_t = torch.empty(cfg.cols, cfg.rows, dtype=kind, device=device) if transposed else None

    def quantize(self, d_in, stream=None):
        """Packs a [rows, cols] tensor, one with its rows in several dimensions, or the whole buffer that they lie in, ld elements apart; flat
        buffers and bytes are taken as they are."""
        cfg = self.cfg
        if not isinstance(d_in, int) and d_in.shape != self.out.shape and d_in.dim() > 1 and d_in.element_size() > 1:
            cols = d_in.shape[-1]
            if cols not in (cfg.cols, cfg.ld) or d_in.numel() != cfg.rows * cols:
                raise ValueError(f"Mx4Tensor.quantize: d_in is a {tuple(d_in.shape)} tensor, the configuration says [{cfg.rows}, {cfg.cols}]")
        tahq_mx4_quantize(self.cfg, d_in, self.packed, self.packed_t, stream)
        return (self.packed,) if self.packed_t is None else (self.packed, self.packed_t)

    def dequantize(self, stream=None):
        """The values of the packed forms: (x,), or (x, x transposed)."""
        tahq_mx4_dequantize(self._values, self.packed, self.out, stream)
        if self.packed_t is None:
            return (self.out,)
        tahq_mx4_dequantize(self._values_t, self.packed_t, self.out_t, stream)
        return self.out, self.out_t


class Mx4Linear:
    """A linear layer y = x W^T in mx4 for a fixed number of tokens: W packed once, buffers for x, y and, for training, for the
    backward pass.  `weight`: [n, k], fp32 or bf16, which is also the dtype of x, y and their gradients; grad_w is fp32.
    in_flight: micro-batches that go forward before the first of them comes back.  Each has a slot: its own y, and in training its own x
    along its tokens, until the slot's next forward pass.  The other buffers (gradients among them) are the next call's: calls of one layer follow
    each other, on one stream or ordered by the caller, as they do the constructor's packing of W on torch's current stream."""

    def __init__(self, weight, tokens, transform=0, scale_rule=MX4_FLOOR, training=False, accumulate=0, in_flight=1):
        import torch
        if weight.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"Mx4Linear: the weight is a tensor of {weight.dtype}, float32 or bfloat16 is needed")
        _check_slot("Mx4Linear", 0, in_flight)
        n, k = weight.shape
        device, dtype = weight.device, F32 if weight.dtype == torch.float32 else BF16
        self.training = training
        self._x = make_mx4_config(tokens, k, dtype, 0, transform, scale_rule)
        self._dy = make_mx4_config(tokens, n, dtype, 0, transform, scale_rule)
        self._w = make_mx4_config(n, k, dtype, 0, transform, scale_rule)
        self._forward = make_mx4_matmul_config(tokens, n, k, dtype)
        self._dx = make_mx4_matmul_config(tokens, k, n, dtype)
        self._dw = make_mx4_matmul_config(n, k, tokens, F32, 0, accumulate)
        if not tahq_mx4_linear_workspace_size(self._x, self._forward):
            raise TahqError(2, "tahq_mx4_linear_workspace_size")
        self.weight = _bytes_on(device, tahq_mx4_packed_size(n, k))
        self._in_flight = in_flight
        self._ys = [torch.empty(tokens, n, dtype=weight.dtype, device=device) for _ in range(in_flight)]
        self.y = self._ys[0]
        need = tahq_mx4_linear_workspace_size(self._x, self._forward)
        self.weight_t = self.x_t = None
        if training:
            self.weight_t = _bytes_on(device, tahq_mx4_packed_size(k, n))
            self.x = _packed_on(device, tokens, k, transform)
            self._x_ts = [_packed_on(device, k, tokens, transform) for _ in range(in_flight)]
            self.x_t = self._x_ts[0]
            self.dy, self.dy_t = _bytes_on(device, tahq_mx4_packed_size(tokens, n)), _bytes_on(device, tahq_mx4_packed_size(n, tokens))
            self.grad_x = torch.empty(tokens, k, dtype=weight.dtype, device=device)
            self.grad_w = torch.zeros(n, k, dtype=torch.float32, device=device)
            need = max([need] + [tahq_mx4_matmul_workspace_size(c) for c in (self._forward, self._dx, self._dw)])
        self.workspace = _bytes_on(device, need)
        self._kind = weight.dtype
        self._x_form, self._x_t_form = (((r, c, transform), tahq_mx4_packed_size(r, c)) for r, c in ((tokens, k), (k, tokens)))
        self._forward_x_t = [None] * in_flight    # what a slot's last forward pass was of, along its tokens
        self._linear = (C.byref(self._x), C.byref(self._forward))
        self._own = [(self.weight.data_ptr(), self.weight.numel(), y.data_ptr(), self.workspace.data_ptr(), self.workspace.numel())
                     for y in self._ys]
        if training:
            self._dy_by_ref, self._dx_by_ref, self._dw_by_ref = C.byref(self._dy), C.byref(self._dx), C.byref(self._dw)
            self._own_backward = (*((t.data_ptr(), t.numel()) for t in (self.dy, self.dy_t, self.weight_t, self.workspace)),
                                  self.grad_x.data_ptr(), self.grad_w.data_ptr())
            self._own_x = [(self.x.data_ptr(), self.x.numel(), x_t.data_ptr(), x_t.numel()) for x_t in self._x_ts]
        self.update(weight)

    def update(self, weight, stream=None):
        """Pack W, e.g. after an optimizer's step."""
        _input_of("Mx4Linear.update", "weight", weight, self._w.rows, self._w.cols, self._kind)
        tahq_mx4_quantize(self._w, weight, self.weight, self.weight_t, stream)

    def forward(self, x, stream=None, slot=0):
        """y; in training x is kept along its tokens for the weight's gradient."""
        d_x = _input_of("Mx4Linear.forward", "x", x, self._x.rows, self._x.cols, self._kind)
        if slot:
            _check_slot("Mx4Linear.forward", slot, self._in_flight)
        if not self.training:
            rc = _lib.tahq_mx4_linear(*self._linear, d_x, *self._own[slot], _stream_handle(stream))
            if rc != 0:
                raise TahqError(rc, "tahq_mx4_linear")
            return self._ys[slot]
        self._forward_x_t[slot] = None
        handle = _stream_handle(stream)
        rc = _lib.tahq_mx4_quantize(self._linear[0], d_x, *self._own_x[slot], handle)
        if rc != 0:
            raise TahqError(rc, "tahq_mx4_quantize")
        return self._multiply(self._own_x[0][:2], self._x_ts[slot], handle, slot)

    def product(self, x_packed, stream=None, x_packed_t=None, slot=0):
        """y of an x that is packed already, e.g. by BlockNorm.  The backward pass reads the same x packed along its tokens: x_packed_t, which
        stays the caller's; without it there is no backward pass of this y."""
        _check_packed("Mx4Linear.product", "x_packed", x_packed, *self._x_form)
        if x_packed_t is not None:
            _check_packed("Mx4Linear.product", "x_packed_t", x_packed_t, *self._x_t_form)
        if slot:
            _check_slot("Mx4Linear.product", slot, self._in_flight)
        return self._multiply((_dev_ptr(x_packed), x_packed.numel()), x_packed_t, _stream_handle(stream), slot)

    def _multiply(self, x_packed, x_packed_t, handle, slot):
        self._forward_x_t[slot] = None
        weight, weight_size, *y_and_workspace = self._own[slot]
        rc = _lib.tahq_mx4_matmul(self._linear[1], *x_packed, weight, weight_size, *y_and_workspace, handle)
        if rc != 0:
            raise TahqError(rc, "tahq_mx4_matmul")
        self._forward_x_t[slot] = x_packed_t
        return self._ys[slot]

    def backward(self, grad_y, stream=None, slot=0):
        """(gradient of x, gradient of W) of the slot's last forward pass; the latter is added to with accumulate = 1."""
        if not self.training:
            raise ValueError("Mx4Linear.backward: the layer was not made with training=True")
        if slot:
            _check_slot("Mx4Linear.backward", slot, self._in_flight)
        x_t = self._forward_x_t[slot]
        if x_t is None:
            raise ValueError("Mx4Linear.backward: there is no x along its tokens: no forward pass, or a product without x_packed_t")
        d_dy = _input_of("Mx4Linear.backward", "grad_y", grad_y, self._dy.rows, self._dy.cols, self._kind)
        dy, dy_t, weight_t, workspace, grad_x, grad_w = self._own_backward
        handle = _stream_handle(stream)
        for name, call in (
                ("tahq_mx4_quantize", (self._dy_by_ref, d_dy, *dy, *dy_t)),
                ("tahq_mx4_matmul", (self._dx_by_ref, *dy, *weight_t, grad_x, *workspace)),
                ("tahq_mx4_matmul", (self._dw_by_ref, *dy_t, _dev_ptr(x_t), x_t.numel(), grad_w, *workspace))):
            rc = getattr(_lib, name)(*call, handle)
            if rc != 0:
                raise TahqError(rc, name)
        return self.grad_x, self.grad_w


# ---- norms before and after a block (include/tahq_norm.h)

NORM_MAX_COLS = 8192


def tahq_norm_config_default():
    cfg = tahq_norm_config()
    _load().tahq_norm_config_default(C.byref(cfg))
    return cfg


def make_norm_config(rows, cols, dtype, gate_rows=0, eps=1e-6, residual_scale=1.0, accumulate=0, transform=0, scale_rule=MX4_FLOOR):
    cfg = tahq_norm_config_default()
    cfg.rows, cfg.cols, cfg.dtype, cfg.gate_rows, cfg.eps, cfg.residual_scale = rows, cols, dtype, gate_rows, eps, residual_scale
    cfg.accumulate, cfg.transform, cfg.scale_rule = accumulate, transform, scale_rule
    return cfg


def _gate_groups(cfg):
    return -(-cfg.rows // cfg.gate_rows) if cfg.gate_rows else 0


def _check_norm(where, cfg, tensors, weights, gate):
    for name, t in (*tensors.items(), *weights.items(), ("d_gate", gate)):
        _check_not_half(where, name, t, cfg.dtype)
    for name, t in tensors.items():
        _check_tensor(where, name, t, cfg.rows * cfg.cols, cfg.dtype)
    for name, t in weights.items():
        _check_tensor(where, name, t, cfg.cols, cfg.dtype)
    _check_tensor(where, "d_gate", gate, _gate_groups(cfg) * cfg.cols, cfg.dtype)


def tahq_norm_forward(cfg, d_residual, d_block, d_w_post, d_gate, d_w_pre, d_residual_out, d_h=None, d_h_mx4=None, d_stats=None,
                      stream=None):
    """r' = residual_scale r + gate RMSNorm(block) w_post and h = RMSNorm(r') w_pre; halves may be None, see include/tahq_norm.h."""
    _check_norm("tahq_norm_forward", cfg, {"d_residual": d_residual, "d_block": d_block, "d_residual_out": d_residual_out, "d_h": d_h},
                {"d_w_post": d_w_post, "d_w_pre": d_w_pre}, d_gate)
    _check_tensor("tahq_norm_forward", "d_stats", d_stats, 2 * cfg.rows, F32)
    rc = (_lib or _load()).tahq_norm_forward(
        C.byref(cfg), _dev_ptr(d_residual), _dev_ptr(d_block), _dev_ptr(d_w_post), _dev_ptr(d_gate), _dev_ptr(d_w_pre),
        _dev_ptr(d_residual_out), _dev_ptr(d_h), _dev_ptr(d_h_mx4), _nbytes(d_h_mx4), _dev_ptr(d_stats), _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_norm_forward")


def tahq_norm_workspace_size(cfg):
    return int(_load().tahq_norm_workspace_size(C.byref(cfg)))


def tahq_norm_backward(cfg, d_grad_residual_out, d_grad_h, d_block, d_w_post, d_gate, d_residual_out, d_w_pre, d_stats,
                       d_grad_residual, d_grad_block, d_grad_w_post, d_grad_gate, d_grad_w_pre, d_workspace, stream=None):
    _check_norm("tahq_norm_backward", cfg,
                {"d_grad_residual_out": d_grad_residual_out, "d_grad_h": d_grad_h, "d_block": d_block, "d_residual_out": d_residual_out,
                 "d_grad_residual": d_grad_residual, "d_grad_block": d_grad_block}, {"d_w_post": d_w_post, "d_w_pre": d_w_pre}, d_gate)
    for name, t, n in (("d_stats", d_stats, 2 * cfg.rows), ("d_grad_w_post", d_grad_w_post, cfg.cols),
                       ("d_grad_w_pre", d_grad_w_pre, cfg.cols), ("d_grad_gate", d_grad_gate, _gate_groups(cfg) * cfg.cols)):
        _check_tensor("tahq_norm_backward", name, t, n, F32)
    rc = (_lib or _load()).tahq_norm_backward(
        C.byref(cfg), _dev_ptr(d_grad_residual_out), _dev_ptr(d_grad_h), _dev_ptr(d_block), _dev_ptr(d_w_post), _dev_ptr(d_gate),
        _dev_ptr(d_residual_out), _dev_ptr(d_w_pre), _dev_ptr(d_stats), _dev_ptr(d_grad_residual), _dev_ptr(d_grad_block),
        _dev_ptr(d_grad_w_post), _dev_ptr(d_grad_gate), _dev_ptr(d_grad_w_pre), _dev_ptr(d_workspace), _nbytes(d_workspace),
        _stream_handle(stream))
    if rc != 0:
        raise TahqError(rc, "tahq_norm_backward")


class BlockNorm:
    """Buffers of one configuration's norms.  mx4: h leaves as a packed matrix; otherwise in the configuration's dtype.  training: with the
    buffers of the backward pass.  All are made, and gradients that are added to cleared, on torch's current stream: a call on another
    stream comes after that stream has waited for it.
    in_flight: micro-batches that go forward before the first of them comes back.  Each has a slot: its own r', h and statistics, until the
    slot's next forward pass; backward is given a slot's r' and stats_of(slot).  Gradients are the next backward call's."""

    def __init__(self, cfg, mx4=False, device="cuda:0", training=True, in_flight=1):
        import torch
        need = tahq_norm_workspace_size(cfg)
        if need == 0:
            raise TahqError(2, "tahq_norm_workspace_size")
        self.cfg, self.mx4, kind = cfg, mx4, _torch_dtype(cfg.dtype)
        shape = (cfg.rows, cfg.cols)
        _check_slot("BlockNorm", 0, in_flight)

        def plain():
            return torch.empty(shape, dtype=kind, device=device)

        # (r', h, statistics) of each slot, and where a call finds them
        self._slots = [(plain(), _packed_on(device, *shape, cfg.transform) if mx4 else plain(),
                        torch.empty(2, cfg.rows, dtype=torch.float32, device=device)) for _ in range(in_flight)]
        self._results = [(out, h) for out, h, _ in self._slots]
        self.residual_out, self.h, self.stats = self._slots[0]
        self.training = training
        if training:
            self.workspace = _bytes_on(device, need)
            self.grad_residual, self.grad_block = (plain() for _ in range(2))
            sums = torch.zeros if cfg.accumulate else torch.empty
            self.grad_w_post, self.grad_w_pre = (sums(cfg.cols, dtype=torch.float32, device=device) for _ in range(2))
            self.grad_gate = sums(_gate_groups(cfg), cfg.cols, dtype=torch.float32, device=device) if cfg.gate_rows else None
        self._kind, self._sizes = kind, (cfg.rows, cfg.cols, _gate_groups(cfg))
        self._cfg, self._own, self._own_post = C.byref(cfg), [], []
        for out, h, stats in self._slots:
            own = out.data_ptr(), h.data_ptr(), stats.data_ptr()
            self._own.append((own[0], None, own[1], h.numel(), own[2]) if mx4 else (own[0], own[1], None, 0, own[2]))
            self._own_post.append((own[0], None, None, 0, own[2]))

    def stats_of(self, slot):
        _check_slot("BlockNorm.stats_of", slot, len(self._slots))
        return self._slots[slot][2]

    def forward(self, residual, block, w_post, gate, w_pre, stream=None, slot=0):
        """(r', h); block, w_post and gate may be None, or w_pre."""
        if slot:
            _check_slot("BlockNorm.forward", slot, len(self._slots))
        where, kind, (rows, cols, groups) = "BlockNorm.forward", self._kind, self._sizes
        rc = _lib.tahq_norm_forward(
            self._cfg, _input_of(where, "residual", residual, rows, cols, kind),
            None if block is None else _input_of(where, "block", block, rows, cols, kind),
            None if w_post is None else _input_of(where, "w_post", w_post, 1, cols, kind),
            None if gate is None else _input_of(where, "gate", gate, groups, cols, kind),
            None if w_pre is None else _input_of(where, "w_pre", w_pre, 1, cols, kind),
            *(self._own if w_pre is not None else self._own_post)[slot], _stream_handle(stream))
        if rc != 0:
            raise TahqError(rc, "tahq_norm_forward")
        return self._results[slot] if w_pre is not None else (self._slots[slot][0], None)

    def backward(self, grad_residual_out, grad_h, block, w_post, gate, residual_out, w_pre, stats, stream=None):
        """Gradients of residual, block, w_post, gate and w_pre by name; None for what there is not."""
        if not self.training:
            raise ValueError("BlockNorm.backward: the norm was not made with training=True")
        # in the order of the call's arguments
        got = {"grad_residual": self.grad_residual, "grad_block": None, "grad_w_post": None, "grad_gate": None, "grad_w_pre": None}
        if block is not None:
            got.update(grad_block=self.grad_block, grad_w_post=self.grad_w_post, grad_gate=self.grad_gate)
        if grad_h is not None:
            got["grad_w_pre"] = self.grad_w_pre
        where, kind, (rows, cols, groups) = "BlockNorm.backward", self._kind, self._sizes

        def at(name, t, count=rows, width=cols, dtype=kind):
            return None if t is None else _input_of(where, name, t, count, width, dtype)

        rc = _lib.tahq_norm_backward(
            self._cfg, at("grad_residual_out", grad_residual_out), at("grad_h", grad_h), at("block", block), at("w_post", w_post, 1),
            at("gate", gate, groups), at("residual_out", residual_out), at("w_pre", w_pre, 1),
            at("stats", stats, 2, rows, self.stats.dtype), *(None if t is None else t.data_ptr() for t in got.values()),
            self.workspace.data_ptr(), self.workspace.numel(), _stream_handle(stream))
        if rc != 0:
            raise TahqError(rc, "tahq_norm_backward")
        return got
