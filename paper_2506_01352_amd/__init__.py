"""tahq: TAH-Quant stage-boundary activation codec for MI355X (gfx950).

The work is done by hand-written HIP kernels in libtahq.so behind a C ABI
(include/tahq.h; include/tahq_naive.h for the backward-pass fixed-point compressor;
include/tahq_mx4.h and include/tahq_norm.h for what a stage runs next to the codec: microscaled 4-bit
matrices and their products, and the norms around a block).  This package is argument marshalling only: it hands device
pointers of torch tensors and the current HIP stream to the library.  There is
no CPU or PyTorch fallback: if the library is missing, importing the binding's
functions raises.
"""
from .binding import (  # noqa: F401
    F32, BF16, TahqError, make_config, tahq_config,
    tahq_config_default, tahq_k_per_unit, tahq_packed_size, tahq_workspace_size,
    tahq_encode, tahq_encode_phases, tahq_decode, tahq_encode_noalloc, NOALLOC_MAX_WORKSPACE,
    tahq_samples_packed_size, tahq_samples_workspace_size, tahq_encode_samples, tahq_decode_samples,
    PHASE_PROLOGUE, PHASE_ENTROPY, PHASE_SELECT, PHASE_QUANT, PHASE_ALL, SELECT_MULTI_LAUNCH,
    tahq_tile_entropy, tahq_alloc_tile_entropy, tahq_parse_header,
    tahq_status_string, tahq_version, library_path, Codec,
    tahq_naive_config, make_naive_config, tahq_naive_config_default, tahq_naive_packed_size,
    tahq_naive_encode, tahq_naive_decode,
    MX4_FLOOR, MX4_COVER, tahq_mx4_config, make_mx4_config, tahq_mx4_config_default, tahq_mx4_packed_size,
    tahq_mx4_quantize, tahq_mx4_dequantize, tahq_mx4_matmul_config, make_mx4_matmul_config,
    tahq_mx4_matmul_config_default, tahq_mx4_matmul_workspace_size, tahq_mx4_matmul,
    tahq_mx4_linear_workspace_size, tahq_mx4_linear, Mx4Tensor, Mx4Linear,
    NORM_MAX_COLS, tahq_norm_config, make_norm_config, tahq_norm_config_default, tahq_norm_workspace_size,
    tahq_norm_forward, tahq_norm_backward, BlockNorm,
)
