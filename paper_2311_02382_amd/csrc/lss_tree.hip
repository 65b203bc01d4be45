// Attention of drafted tokens over a paged cache (lss_paged_attn_tree): which kernel a call takes.
#include "lss_serve.h"

namespace lss {

size_t paged_tree_workspace_bytes(int64_t rows, int B, int H, int H_kv, int d, int max_len, int) { return tree_narrow_workspace_bytes(rows, B, H, H_kv, d, max_len); }

template <typename T>
hipError_t launch_paged_tree(const TreeArgs &a, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    return launch_tree_narrow<T>(a, q, k_cache, v_cache, out, lse, scratch, st);
}

template hipError_t launch_paged_tree<bf16_t>(const TreeArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_paged_tree<float>(const TreeArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
