// Instances of the attention for drafted tokens on caches of kind MOE_CACHE_FP8.
#include "tree_attn_kernel.h"

namespace moe {

int launch_tree_fp8(const TreeArgs& a, const TreeParts& p, int head_dim, int mt, int wr, hipStream_t s) {
    return launch_tree_kind<MOE_CACHE_FP8>(a, p, head_dim, mt, wr, s);
}

}  // namespace moe
