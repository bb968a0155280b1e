"""FluxBin LUT-GEMV hot path for AMD Instinct MI355X (gfx950).

The product is the C-ABI library ``libfluxbin.so`` (``include/fluxbin.h``; ``include/fluxbin_quant.h`` for 4-bit linears and
the 8-bit key/value cache); ``fluxbin`` is its thin ctypes binding.
"""
from . import fluxbin  # noqa: F401
from .fluxbin import (  # noqa: F401
    FluxbinError,
    Kv8Cache,
    PackedLayer,
    PackedW4,
    fluxbin_debug_indices,
    fluxbin_kv8_append,
    fluxbin_kv8_attention,
    fluxbin_kv8_cache_query,
    fluxbin_kv8_read,
    fluxbin_kv8_workspace_query,
    fluxbin_layer_from_header,
    fluxbin_lut_gemm_smallbatch,
    fluxbin_lut_gemv,
    fluxbin_pack,
    fluxbin_pack_query,
    fluxbin_unpack_canonical,
    fluxbin_w4_gemm,
    fluxbin_w4_pack,
    fluxbin_w4_pack_query,
    fluxbin_w4_quantize,
    fluxbin_w4_workspace_query,
    fluxbin_workspace_init,
    fluxbin_workspace_query,
    make_kv8_cache,
    make_kv8_workspace,
    make_shape,
    make_w4_workspace,
    make_workspace,
)
