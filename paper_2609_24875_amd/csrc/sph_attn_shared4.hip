// sph_attention_shared's kernels for pages of 4 bits: files of their own, so that they build beside each other.
#include "sph_attn_shared.h"

const void* sph_attn_shared_kernel4(int dim, SharedKind kind, int nb, bool uni) { return shared_kernel<4>(dim, kind, nb, uni); }
