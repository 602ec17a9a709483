"""B200-native relay-boundary prompt-KV compression (headwise eviction + Orthogonal BackFill).

The product is the C-ABI CUDA library declared in ``include/obf.h``; this package
holds its sources (``csrc/``), the in-tree build step, a ctypes binding with the
same entry-point names, and the seeded synthetic input generator.
"""
from . import synth  # noqa: F401
from .binding import (  # noqa: F401
    OBF_BF16, OBF_F32, OBF_OK, ObfAttend, ObfCache, ObfDiag, ObfError, ObfEvict, ObfParams, ObfPrefix, ObfQuantized, ObfQuantizedRead,
    ObfQuantizedWrite, QuantizedCache, attend, attend_quantized, attend_quantized_workspace, attend_shared, attend_workspace, compress_caches,
    evict_by_mass, evict_only, evict_only_static, load, make_cache, make_params, obf_attend_workspace_bytes, obf_compress, obf_compress_host,
    obf_compress_profiled, obf_host_arena_bytes, obf_last_device_status, obf_last_launch_count, obf_static_scratch_status, obf_status_string,
    obf_workspace_bytes, parse_diag, quantized_cache, read_quantized, write_quantized)
