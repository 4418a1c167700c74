// Attention on the host: what a call was given, checked, and how it is cut into workgroups.
#pragma once
#include <algorithm>

#include "rkb_attn.h"

namespace rkb {

struct attn_plan {
    bool few;        // up to 32 rows of one key head a workgroup, each wave with keys of its own
    int64_t blocks;  // workgroups of one split
    int splits;      // parts of the keys
};

struct attn_results {
    rkb_heads o;
    float *o32, *lse;
};

template <class F>
int with_attn_type(int dtype, F go)
{
    return dtype == RKB_F16 ? go((f16 *)nullptr) : go((bf16 *)nullptr);
}

template <class F>
int with_width(int64_t dim, F go)
{
    if (dim <= 64) return go(std::integral_constant<int, 64>());
    if (dim <= 128) return go(std::integral_constant<int, 128>());
    return go(std::integral_constant<int, 256>());
}

inline heads_at at_of(const rkb_heads &h) { return {(char *)h.p, h.batch, h.row, h.head}; }

attn_plan plan_fwd(const rkb_attn &a);
size_t attn_fwd_parts_bytes(const attn_plan &plan, const rkb_attn &a);
int run_attn_fwd(const attn_in &p, const rkb_attn &a, const attn_plan &plan, const attn_results &res, char *parts, hipStream_t st);

// The backward's launches and the memory they need besides aligned copies and a forward made again.
struct attn_bwd_plan {
    int64_t q_blocks, k_blocks;
    int q_splits, k_splits;
    int64_t stats_rows;  // of a [batch, heads] row sums array, padded
};
attn_bwd_plan plan_bwd(const rkb_attn &a);
size_t attn_bwd_bytes(const attn_bwd_plan &plan, const rkb_attn &a);
struct attn_grads {
    rkb_heads d_o, o;
    const float *o32, *lse;
    rkb_heads dq, dk, dv;
    void *dtable;
};
int run_attn_bwd(const attn_in &p, const rkb_attn &a, const attn_bwd_plan &plan, const attn_grads &g, char *ws, hipStream_t st);

}  // namespace rkb
