// Instantiates the tree attention kernels for head_dim 64.
#include "tree_attn.hpp"

namespace splice_dev {
bool launch_tree_d64(const TreeArgs &a, const splice::TreePlan &p, int kv_format, hipStream_t stream) {
    return launch_tree<64>(a, p, kv_format, stream);
}
}  // namespace splice_dev
