// Attention's C entry points (rk_block.h): arguments checked, operands that are not aligned copied, launches cut.
#include <cmath>
#include <cstring>

#include "rkb_attn.h"
#include "rkb_attn_args.h"
#include "rkb_attn_cut.h"
#include "rkb_buckets.h"

namespace rkb {
namespace {

constexpr int64_t MOST_BLOCKS = (int64_t)1 << 21;  // workgroups of a launch
constexpr size_t WS_ALIGN_ATTN = 256;

// ------------------------------------------------------------------ checks

bool good_attn(const rkb_attn *a)
{
    if (!a || !good_dtype16(a->dtype)) return false;
    if (a->batch < 0 || a->q_rows < 0 || a->k_rows < 0 || a->batch > RKB_MAX_TOKENS || a->q_rows > RKB_MAX_TOKENS || a->k_rows > RKB_MAX_TOKENS)
        return false;
    if (a->kv_heads < 1 || a->heads < 1 || a->heads > 65536 || a->heads % a->kv_heads || a->dim < 1 || a->dim > RKB_MAX_DIM) return false;
    if (!(a->scale > 0.0f) || !std::isfinite(a->scale * LOG2E)) return false;  // else a score of 0 is NaN in steps of log2
    if (a->first < -((int64_t)1 << 40) || a->first > (int64_t)1 << 40) return false;
    if ((uintptr_t)a->firsts % 4 || (uintptr_t)a->lens % 4) return false;
    if (a->mask && a->batch > 1 && (a->mask_stride < 0 || a->mask_stride > (int64_t)1 << 40)) return false;
    if (!a->table) return true;
    const int sides = a->two_sided ? 2 : 1, count = a->buckets / sides;
    if (a->table_dtype != a->dtype && a->table_dtype != RKB_F32) return false;
    return (uintptr_t)a->table % dtype_size(a->table_dtype) == 0 && a->buckets <= RKB_MAX_BUCKETS && a->buckets % sides == 0 && count >= 2 &&
           a->max_distance > count / 2 && a->max_distance <= RKB_MAX_DISTANCE;
}

// A copy of a tensor argument whose strides that no element needs are 0.
rkb_heads settled_heads(const rkb_heads *h, int64_t batch, int64_t rows, int64_t heads)
{
    if (!h) return rkb_heads{nullptr, 0, 0, 0};
    return rkb_heads{h->p, batch > 1 ? h->batch : 0, rows > 1 ? h->row : 0, heads > 1 ? h->head : 0};
}

bool good_heads_in(const rkb_heads &h, int64_t elements, int size)
{
    auto good = [](int64_t s) { return s >= 0 && s <= (int64_t)1 << 40; };
    return elements == 0 || (h.p && (uintptr_t)h.p % size == 0 && good(h.batch) && good(h.row) && good(h.head));
}

bool good_heads_out(const rkb_heads &h, int64_t batch, int64_t rows, int64_t heads, int64_t dim, int size)
{
    return batch * rows == 0 || (good_heads_in(h, 1, size) && elements_apart(h, batch, rows, heads, dim));
}

bool aligned_heads(const rkb_heads &h, int64_t dim)
{
    return dim % 8 == 0 && (uintptr_t)h.p % 16 == 0 && h.batch % 8 == 0 && h.row % 8 == 0 && h.head % 8 == 0 && h.row <= (int64_t)1 << 22;
}

attn_in make_in(const rkb_attn &a)
{
    attn_in p;
    std::memset((void *)&p, 0, sizeof p);
    p.B = (int)a.batch;
    p.Q = (int)a.q_rows;
    p.T = (int)a.k_rows;
    p.H = (int)a.heads;
    p.K = (int)a.kv_heads;
    p.G = (int)(a.heads / a.kv_heads);
    p.D = (int)a.dim;
    p.causal = a.causal != 0;
    p.scale = a.scale;
    p.c = a.scale * LOG2E;
    p.first = a.first;
    p.firsts = a.firsts;
    p.lens = a.lens;
    p.mask = a.mask;
    p.mask_stride = a.batch > 1 ? a.mask_stride : 0;
    p.bias.table = a.table;
    if (a.table) {
        p.bias.f32 = a.table_dtype == RKB_F32;
        p.bias.sides = a.two_sided ? 2 : 1;
        p.bias.count = a.buckets / p.bias.sides;
        set_borders(p.bias.border, MAX_BUCKETS, p.bias.count, a.max_distance);
        p.bias.far = p.bias.border[p.bias.count - 2];
    }
    return p;
}

// ------------------------------------------------------------------ aligned copies

struct heads_job {
    heads_at from;
    uint16_t *to;  // [batch, rows, heads, ld]
    int64_t chunks_all;
    int rows, heads, dim, chunks;
};
struct heads_jobs {
    heads_job job[4];
};

__global__ __launch_bounds__(256) void k_pad_heads(heads_jobs jobs)
{
    const heads_job j = jobs.job[blockIdx.y];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < j.chunks_all; i += (int64_t)gridDim.x * 256) {
        int64_t r = i / j.chunks;
        const int c = (int)(i - r * j.chunks) * 8, left = j.dim - c;
        const int64_t h = r % j.heads;
        r /= j.heads;
        const uint16_t *from = j.from.at<uint16_t>(r / j.rows, r % j.rows, h) + c;
        vec<uint16_t, 8> v;
        if (left >= 8) {
            __builtin_memcpy(&v, from, 16);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < left ? from[e] : (uint16_t)0;
        }
        *(vec<uint16_t, 8> *)(j.to + i * 8) = v;
    }
}

size_t copy_bytes(int64_t batch, int64_t rows, int64_t heads, int64_t dim)
{
    return (size_t)round_up(batch * rows * heads * round_up(dim, 8) * 2, WS_ALIGN_ATTN);
}

struct attn_workspace {
    char *at, *end;
    heads_jobs jobs;
    int n = 0;
    attn_workspace(void *ws, size_t bytes) : at((char *)ws), end((char *)ws + bytes) {}
    char *take(size_t bytes)
    {
        char *p = at;
        at += bytes;
        return p;
    }
    void align(rkb_heads &h, int64_t batch, int64_t rows, int64_t heads, int64_t dim)
    {
        if (batch * rows == 0 || aligned_heads(h, dim)) return;
        const int64_t ld = round_up(dim, 8), chunks = ld / 8;
        char *to = take(copy_bytes(batch, rows, heads, dim));
        jobs.job[n++] = heads_job{at_of(h), (uint16_t *)to, batch * rows * heads * chunks, (int)rows, (int)heads, (int)dim, (int)chunks};
        h = rkb_heads{to, batch > 1 ? rows * heads * ld : 0, rows > 1 ? heads * ld : 0, heads > 1 ? ld : 0};
    }
    int run(hipStream_t st)
    {
        if (!n) return RKB_OK;
        int64_t most = 0;
        for (int i = 0; i < n; ++i) most = std::max(most, jobs.job[i].chunks_all);
        return launch(k_pad_heads, dim3((uint32_t)std::min<int64_t>((most + 255) / 256, 4096), n), dim3(256), st, jobs);
    }
};


size_t again_bytes(const rkb_attn &a, const attn_plan &plan)
{
    return round_up(a.batch * a.q_rows * a.heads * a.dim * 4, WS_ALIGN_ATTN) + round_up(a.batch * a.q_rows * a.heads * 4, WS_ALIGN_ATTN) +
           attn_fwd_parts_bytes(plan, a);
}

// So that no launch has 2^32 lanes, which take at least 128 rows of a head for a workgroup of 256, but two such workgroups of heads of more than 128
// columns, and one for 64 rows of queries and keys in the norms' kernel.
bool fits_launches(const rkb_attn &a, bool backward)
{
    auto good = [&](int64_t heads, int64_t rows) {
        const int64_t units = a.batch * heads;
        return units <= MOST_BLOCKS && units * ((rows + 127) / 128) <= MOST_BLOCKS;
    };
    return good(a.heads, a.q_rows) && (!backward || good(a.kv_heads, a.k_rows));
}

}  // namespace

// ------------------------------------------------------------------ how a call is cut

static int split_of(int64_t blocks, int64_t want, int64_t most)
{
    return blocks == 0 ? 1 : (int)std::max<int64_t>(1, std::min({want / blocks, most, (int64_t)64}));
}

// Keys are split, for 512 workgroups, into parts of at least 256: one token over 1024 cached ones takes 20 us so, 22 by 128, 25 without
// splits; 6 x 199 queries over 777 keys, forward and backward, 131 by 256 and 142 by 1024.
attn_plan plan_fwd(const rkb_attn &a)
{
    const int64_t rows = a.q_rows * (a.heads / a.kv_heads);
    attn_plan plan{};
    plan.few = few_queries_win(a.q_rows, a.dim, a.table != nullptr);
    plan.blocks = plan.few ? a.batch * a.kv_heads * ((rows + 31) / 32) : a.batch * a.heads * ((a.q_rows + 127) / 128);
    plan.splits = split_of(plan.blocks, 512, a.k_rows / 256);
    return plan;
}

// Splits as above, and of the queries for dk and dv, whose workgroups of wider heads fill a compute unit each.
attn_bwd_plan plan_bwd(const rkb_attn &a)
{
    attn_bwd_plan plan;
    const int64_t group = a.heads / a.kv_heads;
    plan.stats_rows = round_up(a.q_rows, 64);
    plan.q_blocks = a.batch * a.heads * ((a.q_rows + 127) / 128);
    plan.k_blocks = a.batch * a.kv_heads * ((a.k_rows + 127) / 128);
    plan.q_splits = split_of(plan.q_blocks, 512, a.k_rows / 256);
    plan.k_splits = split_of(plan.k_blocks, a.dim <= 64 ? 512 : 256, group * a.q_rows / 256);
    return plan;
}

}  // namespace rkb

using namespace rkb;

extern "C" int rkb_attn_fwd_workspace(const rkb_attn *a, int cache, int aligned, size_t *bytes)
{
    if (!bytes || !good_attn(a) || !fits_launches(*a, false)) return RKB_E_INVAL;
    *bytes = attn_fwd_parts_bytes(plan_fwd(*a), *a);
    if (!aligned || a->dim % 8)
        *bytes += copy_bytes(a->batch, a->q_rows, a->heads, a->dim) + (cache ? 0 : 2 * copy_bytes(a->batch, a->k_rows, a->kv_heads, a->dim));
    return RKB_OK;
}

extern "C" int rkb_attn_fwd(const rkb_attn *a, const rkb_heads *q, const rkb_heads *k, const rkb_heads *v, const rkb_kv8 *cache,
                            const rkb_heads *o, float *o32, float *lse, void *workspace, size_t ws_bytes, void *stream)
{
    if (!good_attn(a) || !fits_launches(*a, false) || (cache ? k || v : !k || !v) || !q || !o) return RKB_E_INVAL;
    const int64_t B = a->batch, Q = a->q_rows, T = a->k_rows, H = a->heads, K = a->kv_heads, D = a->dim;
    rkb_heads qs = settled_heads(q, B, Q, H), ks = settled_heads(k, B, T, K), vs = settled_heads(v, B, T, K), os = settled_heads(o, B, Q, H);
    if (!good_heads_in(qs, B * Q, 2) || !good_heads_out(os, B, Q, H, D, 2) || (uintptr_t)o32 % 16 || (uintptr_t)lse % 4) return RKB_E_INVAL;
    if (cache ? (cache->tokens < T || cache->tokens > RKB_MAX_TOKENS || (B * T && (!cache->codes || !cache->exps || (uintptr_t)cache->codes % 16)))
              : (!good_heads_in(ks, B * T, 2) || !good_heads_in(vs, B * T, 2)))
        return RKB_E_INVAL;
    if (B * Q == 0) return RKB_OK;
    const attn_plan plan = plan_fwd(*a);
    attn_workspace ws(workspace, ws_bytes);
    ws.align(qs, B, Q, H, D);
    if (!cache) {
        ws.align(ks, B, T, K, D);
        ws.align(vs, B, T, K, D);
    }
    char *const parts = ws.take(attn_fwd_parts_bytes(plan, *a));
    if (ws.at != workspace && (!workspace || (uintptr_t)workspace % WS_ALIGN_ATTN)) return RKB_E_INVAL;
    if (ws.at > ws.end) return RKB_E_NOMEM;
    const hipStream_t st = (hipStream_t)stream;
    const int rc = ws.run(st);
    if (rc != RKB_OK) return rc;
    attn_in p = make_in(*a);
    p.q = at_of(qs);
    p.k = at_of(ks);
    p.v = at_of(vs);
    if (cache) {
        p.codes = cache->codes;
        p.exps = cache->exps;
        p.room = round_up(cache->tokens, RKB_GROUP);
        p.ld = round_up(D, 16);
    }
    return run_attn_fwd(p, *a, plan, attn_results{os, o32, lse}, parts, st);
}

extern "C" int rkb_attn_bwd_workspace(const rkb_attn *a, int again, int aligned, size_t *bytes)
{
    if (!bytes || !good_attn(a) || !fits_launches(*a, true)) return RKB_E_INVAL;
    *bytes = attn_bwd_bytes(plan_bwd(*a), *a) + (again ? again_bytes(*a, plan_fwd(*a)) : 0);
    if (!aligned || a->dim % 8) *bytes += 2 * copy_bytes(a->batch, a->q_rows, a->heads, a->dim) + 2 * copy_bytes(a->batch, a->k_rows, a->kv_heads, a->dim);
    return RKB_OK;
}

extern "C" int rkb_attn_bwd(const rkb_attn *a, const rkb_heads *d_o, const rkb_heads *q, const rkb_heads *k, const rkb_heads *v,
                            const rkb_heads *o, const float *o32, const float *lse, const rkb_heads *dq, const rkb_heads *dk,
                            const rkb_heads *dv, void *dtable, void *workspace, size_t ws_bytes, void *stream)
{
    if (!good_attn(a) || !fits_launches(*a, true) || !d_o || !q || !k || !v || !dq || !dk || !dv) return RKB_E_INVAL;
    const int64_t B = a->batch, Q = a->q_rows, T = a->k_rows, H = a->heads, K = a->kv_heads, D = a->dim;
    rkb_heads ds = settled_heads(d_o, B, Q, H), qs = settled_heads(q, B, Q, H), ks = settled_heads(k, B, T, K), vs = settled_heads(v, B, T, K);
    rkb_heads os = settled_heads(o, B, Q, H), dqs = settled_heads(dq, B, Q, H), dks = settled_heads(dk, B, T, K), dvs = settled_heads(dv, B, T, K);
    const bool again = !lse;
    if (!good_heads_in(ds, B * Q, 2) || !good_heads_in(qs, B * Q, 2) || !good_heads_in(ks, B * T, 2) || !good_heads_in(vs, B * T, 2) ||
        (dq->p && !good_heads_out(dqs, B, Q, H, D, 2)) || !dk->p != !dv->p ||
        (dk->p && (!good_heads_out(dks, B, T, K, D, 2) || !good_heads_out(dvs, B, T, K, D, 2))))
        return RKB_E_INVAL;
    if (again ? (o32 || os.p) : (B * Q > 0 && (o32 ? os.p != nullptr : !good_heads_in(os, 1, 2)))) return RKB_E_INVAL;
    if ((uintptr_t)o32 % 16 || (uintptr_t)lse % 4 || (dtable && (!a->table || (uintptr_t)dtable % dtype_size(a->table_dtype)))) return RKB_E_INVAL;
    const attn_bwd_plan plan = plan_bwd(*a);
    attn_workspace ws(workspace, ws_bytes);
    ws.align(ds, B, Q, H, D);
    ws.align(qs, B, Q, H, D);
    ws.align(ks, B, T, K, D);
    ws.align(vs, B, T, K, D);
    attn_grads g{ds, os, o32, lse, dqs, dks, dvs, dtable};
    const attn_plan forward = plan_fwd(*a);
    char *parts = nullptr;
    if (again) {
        g.o32 = (float *)ws.take(round_up(B * Q * H * D * 4, WS_ALIGN_ATTN));
        g.lse = (float *)ws.take(round_up(B * Q * H * 4, WS_ALIGN_ATTN));
        parts = ws.take(attn_fwd_parts_bytes(forward, *a));
    }
    char *const rest = ws.take(attn_bwd_bytes(plan, *a));
    if (ws.at != workspace && (!workspace || (uintptr_t)workspace % WS_ALIGN_ATTN)) return RKB_E_INVAL;
    if (ws.at > ws.end) return RKB_E_NOMEM;
    const hipStream_t st = (hipStream_t)stream;
    int rc = ws.run(st);
    attn_in p = make_in(*a);
    p.q = at_of(qs);
    p.k = at_of(ks);
    p.v = at_of(vs);
    if (rc == RKB_OK && again && B * Q > 0)
        rc = run_attn_fwd(p, *a, forward, attn_results{rkb_heads{nullptr, 0, 0, 0}, (float *)g.o32, (float *)g.lse}, parts, st);
    return rc == RKB_OK ? run_attn_bwd(p, *a, plan, g, rest, st) : rc;
}
