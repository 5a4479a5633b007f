// Entry points of the launch code's rules for products, built with the host compiler alone.
#include "hxt_product_rules.h"

extern "C" {

// out: tile, parts, steps of a part, half-tile columns, direct, copies of p and q, bytes of the workspace in use
void product_way(int64_t m, int64_t n, int64_t depth, int64_t es, int p_across, int q_across, int p_direct, int q_direct, uint64_t work_bytes, uint64_t *out)
{
    const hxt::Way w = hxt::way_for(m, n, depth, es, p_across, q_across, p_direct, q_direct, work_bytes);
    uint64_t used = hxt::parts_bytes(w.shape, m, n);
    if (w.copy_p) used = std::max(used, w.p_at + (p_across ? hxt::copy_bytes(depth, m, es) : hxt::copy_bytes(m, depth, es)));
    if (w.copy_q) used = std::max(used, w.q_at + (q_across ? hxt::copy_bytes(depth, n, es) : hxt::copy_bytes(n, depth, es)));
    const uint64_t all[] = {w.shape.tile, w.shape.splits, w.shape.split_steps, w.shape.half, w.direct, w.copy_p, w.copy_q, used};
    for (int i = 0; i < 8; ++i) out[i] = all[i];
}

uint64_t product_work(int64_t m, int64_t n, int64_t depth, int64_t es, int p_across, int q_across)
{
    return hxt::work_for(m, n, depth, es, p_across, q_across);
}

}  // extern "C"
