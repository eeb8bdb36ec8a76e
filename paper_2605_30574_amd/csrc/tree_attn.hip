// tree_attn.hip -- host side of splice_tree_attn (splice_tree.h): checks, plan,
// launch.  The kernels are in tree_attn.hpp, one unit per head_dim.

#include "tree_attn.hpp"

using splice_dev::TreeArgs;

namespace {

// Compute units of the current device (256 when HIP cannot tell: the plan then still holds, it only
// balances for that many).
int compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) {
        (void)hipGetLastError();
        return 256;
    }
    if (dev < 64 && (n = known[dev].load()) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) {
        (void)hipGetLastError();
        return 256;
    }
    if (dev < 64) known[dev].store(n);
    return n;
}

}  // namespace

extern "C" {

int64_t splice_tree_attn_workspace_bytes(const splice_shape *shape, const splice_call *call, const splice_tree *tree) {
    int32_t rc = splice::validate_tree_shape(shape, tree);
    if (rc != SPLICE_OK) return rc;
    if (!call) return SPLICE_EINVAL;
    splice_call checked = *call;
    checked.step = 0;
    rc = splice::validate_call(*shape, &checked);
    if (rc != SPLICE_OK) return rc;
    return (int64_t)splice::tree_most_bytes(*shape, checked, tree->n_nodes, compute_units());
}

int32_t splice_tree_attn(const splice_shape *shape, const splice_call *call, const splice_tree *tree,
                         const int32_t *cell_LW, const int32_t *cell_step, const int32_t *depth,
                         const uint64_t *visible, const void *q, const void *clean_k, const void *clean_v,
                         const void *donor_k, const void *donor_v, const void *gen_k, const void *gen_v,
                         const uint8_t *gen_k_exp, const uint8_t *gen_v_exp, void *out, float *lse, void *workspace,
                         size_t workspace_bytes, void *stream) {
    int32_t rc = splice::validate_tree(shape, tree, cell_step);
    if (rc != SPLICE_OK) return rc;
    const splice_shape &sh = *shape;
    if (!call) return SPLICE_EINVAL;
    splice_call checked = *call;
    checked.step = 0;   // every node takes its own step
    rc = splice::validate_call(sh, &checked);
    if (rc != SPLICE_OK) return rc;
    if (!isfinite(call->scale * splice_dev::kLog2e)) return SPLICE_EINVAL;
    rc = splice::validate_cells(sh, cell_LW);
    if (rc != SPLICE_OK) return rc;
    if (sh.n_cells == 0) return SPLICE_OK;
    const bool zero = sh.donor_kind == SPLICE_DONOR_ZERO, has_prompt = sh.prompt_len > 0;
    const bool f8 = tree->kv_format == SPLICE_KV_E4M3;
    if (!depth || !visible || !q || !gen_k || !gen_v || !out || !lse) return SPLICE_EINVAL;
    if (has_prompt && (!clean_k || !clean_v)) return SPLICE_EINVAL;
    if (zero ? (donor_k || donor_v) : (has_prompt && (!donor_k || !donor_v))) return SPLICE_EINVAL;
    if (f8 ? (!gen_k_exp || !gen_v_exp) : (gen_k_exp || gen_v_exp)) return SPLICE_EINVAL;
    const void *ptrs[] = {q, clean_k, clean_v, donor_k, donor_v, gen_k, gen_v, out};
    for (const void *p : ptrs)
        if (!splice::aligned(p, 16)) return SPLICE_EINVAL;
    if (!splice::aligned(depth, 4) || !splice::aligned(visible, 8) || !splice::aligned(lse, 4)) return SPLICE_EINVAL;

    const int T = tree->n_nodes;
    TreeArgs args;
    int n = 0;
    const splice::TreePlan p = splice::tree_prepare(sh, checked, *tree, cell_LW, cell_step, compute_units(), n, args.step, args.slots);
    if (n == 0) return SPLICE_OK;
    if (p.bytes > 0 && (!workspace || !splice::aligned(workspace, 256) || workspace_bytes < p.bytes)) return SPLICE_EWORKSPACE;
    splice_dev::TreeCall &a = args.call;
    a.q = (const char *)q;
    a.ck = (const char *)clean_k;
    a.cv = (const char *)clean_v;
    a.dk = (const char *)donor_k;
    a.dv = (const char *)donor_v;
    a.gk = (const char *)gen_k;
    a.gv = (const char *)gen_v;
    a.gke = gen_k_exp;
    a.gve = gen_v_exp;
    a.depth = depth;
    a.visible = visible;
    a.out = (__bf16 *)out;
    a.lse = lse;
    a.part = (_Float16 *)workspace;
    a.record = (float4 *)((char *)workspace + (size_t)p.n_slots * T * sh.n_q_heads * sh.head_dim * 2);
    a.T = T;
    a.G = splice::group_of(sh);
    a.lgG = a.G == 1 ? 0 : (a.G == 2 ? 1 : (a.G == 4 ? 2 : 3));
    a.Hkv = sh.n_kv_heads;
    a.Tp = sh.prompt_len;
    a.cap = sh.gen_capacity;
    a.span_lo = sh.span_lo;
    a.span_hi = sh.span_hi;
    a.window = call->window;
    a.zero_donor = zero ? 1 : 0;
    a.n_active = n;
    a.row_tiles = p.row_tiles;
    a.per = p.per;
    a.n_p = p.n_p;
    a.p_tiles = p.p_tiles;
    a.p_heavy0 = p.p_heavy0;
    a.p_heavy = p.p_heavy;
    a.split = p.split;
    a.qk_scale = call->scale * splice_dev::kLog2e;
    hipStream_t st = (hipStream_t)stream;
    const bool ok = sh.head_dim == 64    ? splice_dev::launch_tree_d64(args, p, tree->kv_format, st)
                    : sh.head_dim == 128 ? splice_dev::launch_tree_d128(args, p, tree->kv_format, st)
                                         : splice_dev::launch_tree_d256(args, p, tree->kv_format, st);
    return ok ? SPLICE_OK : SPLICE_EHIP;
}

}  // extern "C"
