// Kernels of the attention over 4-bit pages with heads of 64 (page_attn.hpp).
#include "page_attn.hpp"

namespace splice_dev {
bool launch_page_attn_d64(const PageArgs &args, const splice::PagePlan &p, int most_count, hipStream_t stream) {
    return launch_page_attn<64>(args, p, most_count, stream);
}
}  // namespace splice_dev
