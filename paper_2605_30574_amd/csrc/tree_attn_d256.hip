// Instantiates the tree attention kernels for head_dim 256.
#include "tree_attn.hpp"

namespace splice_dev {
bool launch_tree_d256(const TreeArgs &a, const splice::TreePlan &p, int kv_format, hipStream_t stream) {
    return launch_tree<256>(a, p, kv_format, stream);
}
}  // namespace splice_dev
