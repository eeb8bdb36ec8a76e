// Instantiates the tree attention kernels for head_dim 128.
#include "tree_attn.hpp"

namespace splice_dev {
bool launch_tree_d128(const TreeArgs &a, const splice::TreePlan &p, int kv_format, hipStream_t stream) {
    return launch_tree<128>(a, p, kv_format, stream);
}
}  // namespace splice_dev
