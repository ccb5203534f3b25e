"""SPHQuant decode path for MI355X (gfx950): C-ABI library libsph.so and its Python binding."""
from .sph import (EXPORTS, FORMATS, LIB_PATH, SphError, SphLibraryMissing, SphWeights,  # noqa: F401
                  codes_to_host, encode, format_supported, gemm, gemm_small, gemm_small_noalloc, gemv,
                  kmeans_codebook, kmeans_workspace_bytes, load_library, pack, packed_bytes, status_str,
                  unpack, workspace_bytes)
from .attn import (KVCache, attention, attention_shared, attention_shared_workspace_bytes,  # noqa: F401
                   attention_weights, attention_weights_workspace_bytes, attention_workspace_bytes, kv_append, kv_evict,
                   kv_read, rope, rope_axes, rope_frequencies, rope_table)
from .block import AttentionBlock  # noqa: F401
