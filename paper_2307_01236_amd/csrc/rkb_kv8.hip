// A cache of keys and values in 8 bits: tokens written and loaded (rk_block.h).
//
// A block of 32 tokens of a head is a workgroup's.  Writing, it loads the block's new tokens once, takes their maximum, brings the codes
// that were there to the new step and stores the block whole, so that no two workgroups touch the same block and the
// result does not depend on their order.
//
// Both are bound by memory and, when small, by a launch: 100 rows into 8 caches of 8 heads of 128 take 6 us, all 8 x 1024 tokens out again 14 us
// (50 MB; about 4 of it are the launch).
#include <algorithm>

#include "rkb_common.h"

namespace rkb {
namespace {

constexpr int SPAN = 16, LANES = 256;  // columns of a lane

struct kv_side {
    const char *p;
    int64_t b, t, h;  // in elements
};

struct kv_write {
    kv_side in[2];
    int64_t first;
    const int32_t *firsts, *counts;
    int8_t *codes;
    uint8_t *exps;
    int64_t rows, tokens, room;
    int B, K, D, ld, blocks;  // blocks of a head that a write may touch
};

__device__ inline uint32_t max_of_block(uint32_t v, uint32_t *shared)
{
#pragma unroll
    for (int i = 1; i < WAVE; i *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, i));
    if (threadIdx.x % WAVE == 0) shared[threadIdx.x / WAVE] = v;
    __syncthreads();
    return max(max(shared[0], shared[1]), max(shared[2], shared[3]));
}

// A lane has 16 columns of a token: 32 tokens of up to 256 columns are two passes of 256 lanes.
template <class T>
__global__ __launch_bounds__(LANES) void k_kv8_write(kv_write w)
{
    __shared__ uint32_t shared[4];
    constexpr int N = CHUNK<T>, PASSES = RKB_GROUP * RKB_MAX_DIM / SPAN / LANES;
    int n = blockIdx.x;
    const int which = n % w.blocks;
    n /= w.blocks;
    const int kv = n % w.K, b = n / w.K, side = blockIdx.y;
    const int64_t start = w.first + (w.firsts ? w.firsts[b] : 0), count = w.counts ? min(max((int64_t)w.counts[b], (int64_t)0), w.rows) : w.rows;
    const int64_t lo = max(start, (int64_t)0), hi = min(start + count, w.tokens);  // tokens written
    if (lo >= hi) return;
    const int64_t block = lo / RKB_GROUP + which, t0 = block * RKB_GROUP;
    if (t0 >= hi) return;
    const int64_t head = ((int64_t)side * w.B + b) * w.K + kv;
    int8_t *const codes = w.codes + (head * w.room + t0) * w.ld;
    uint8_t *const exp = w.exps + head * (w.room / RKB_GROUP) + block;
    const int keep = (int)max(lo - t0, (int64_t)0), spans = w.ld / SPAN;  // tokens of the block that stay
    const uint8_t old = *exp;

    float v[PASSES][SPAN];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
        const int at = k * LANES + threadIdx.x, r = at / spans, col = (at - r * spans) * SPAN;
        const int64_t t = t0 + r;
        const bool fresh = r < RKB_GROUP && t >= lo && t < hi;
        const kv_side &in = w.in[side];
        const T *from = (const T *)in.p + b * in.b + (fresh ? t - start : 0) * in.t + kv * in.h + col;
#pragma unroll
        for (int c = 0; c < SPAN; c += N) {
            float x[N];
            load_chunk<T>(from + c, fresh ? w.D - col - c : 0, x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[k][c + e] = x[e];
                top = max_bits(top, x[e]);
            }
        }
    }
    top = max_of_block(top, shared);
    const float most = __uint_as_float(top);
    const bool bad = !finite(most) || (keep > 0 && old == 255);
    int e = bad ? 0 : step_exp(most);
    if (!bad && keep > 0) e = max(e, (int)old - 127);
    const float inv = bad ? 0.0f : two_to(-e), shift = keep > 0 && !bad && old > 0 ? two_to(max((int)old - 127 - e, -126)) : 0.0f;
    const bool high = e > CODE_TOP_EXP<T>;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
        const int at = k * LANES + threadIdx.x, r = at / spans, col = (at - r * spans) * SPAN;
        if (r >= RKB_GROUP) continue;
        vec<uint32_t, 4> *const to = (vec<uint32_t, 4> *)(codes + (int64_t)r * w.ld + col);
        float x[SPAN];
        if (r < keep) {
            if (!bad && shift == 1.0f && !high) continue;
            const vec<int8_t, 16> q = *(const vec<int8_t, 16> *)to;
            // codes of codes: whole numbers times the ratio of the steps
#pragma unroll
            for (int c = 0; c < SPAN; ++c) x[c] = (float)q[c] * shift;
            *to = codes_of<SPAN>(x, 1.0f, high);
        } else {
#pragma unroll
            for (int c = 0; c < SPAN; ++c) x[c] = bad ? 0.0f : v[k][c];
            *to = codes_of<SPAN>(x, inv, high);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *exp = bad ? (uint8_t)255 : (uint8_t)(e + 127);
}

struct kv_load {
    char *p[2];
    int64_t b[2], t[2], h[2];
    const int8_t *codes;
    const uint8_t *exps;
    int64_t tokens, room, chunks_all;
    int B, K, D, ld, chunks;
};

// A lane has 8 columns of a token.  Neighbouring lanes go on in the columns, then the heads and then the tokens, as k and v lie in most programs:
// stores are contiguous and a token's codes whole pieces of 64 to 256 bytes.
template <class T>
__global__ __launch_bounds__(LANES) void k_kv8_load(kv_load w)
{
    const int side = blockIdx.y;
    if (!w.p[side]) return;
    const bool small = w.chunks_all >> 31 == 0;  // 64-bit division is slow
    for (int64_t i = (int64_t)blockIdx.x * LANES + threadIdx.x; i < w.chunks_all; i += (int64_t)gridDim.x * LANES) {
        const int64_t n = small ? (uint32_t)i / (uint32_t)w.chunks : i / w.chunks;
        const int col = (int)(i - n * w.chunks) * 8;
        const int64_t bt = small ? (uint32_t)n / (uint32_t)w.K : n / w.K;
        const int kv = (int)(n - bt * w.K), b = (int)(small ? (uint32_t)bt / (uint32_t)w.tokens : bt / w.tokens);
        const int64_t t = bt - b * w.tokens, at = ((int64_t)side * w.B + b) * w.K + kv;
        const vec<int8_t, 8> q = *(const vec<int8_t, 8> *)(w.codes + (at * w.room + t) * w.ld + col);
        const uint8_t e = w.exps[at * (w.room / RKB_GROUP) + t / RKB_GROUP];
        const float step = e == 0 ? 0.0f : step_of(e);
        float v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = (float)q[c] * step;
        store8<T>((T *)w.p[side] + b * w.b[side] + t * w.t[side] + kv * w.h[side] + col, w.D - col, v);
    }
}

bool good_kv(int dtype, int64_t batch, int64_t kv_heads, int64_t dim, const rkb_kv8 *c)
{
    return good_dtype16(dtype) && batch >= 0 && batch <= RKB_MAX_TOKENS && kv_heads >= 1 && kv_heads <= 65536 && dim >= 1 && dim <= RKB_MAX_DIM && c &&
           c->tokens >= 0 && c->tokens <= RKB_MAX_TOKENS &&
           (double)batch * (double)kv_heads * (double)c->tokens <= (double)((int64_t)1 << 48) &&  // more than any memory holds
           (batch * c->tokens == 0 || (c->codes && c->exps && (uintptr_t)c->codes % 16 == 0));
}

bool good_strides(const rkb_heads &h, int64_t batch, int64_t rows, int64_t heads)
{
    auto good = [](int64_t s, int64_t n) { return n <= 1 || (s >= 0 && s <= (int64_t)1 << 40); };
    return h.p && (uintptr_t)h.p % 2 == 0 && good(h.batch, batch) && good(h.row, rows) && good(h.head, heads);
}

}  // namespace
}  // namespace rkb

using namespace rkb;

extern "C" int rkb_kv8_write(int dtype, int64_t batch, int64_t rows, int64_t kv_heads, int64_t dim, const rkb_heads *k, const rkb_heads *v,
                             int64_t first, const int32_t *firsts, const int32_t *counts, const rkb_kv8 *cache, void *stream)
{
    if (!good_kv(dtype, batch, kv_heads, dim, cache) || rows < 0 || rows > RKB_MAX_TOKENS || !k || !v || first < -((int64_t)1 << 40) ||
        first > (int64_t)1 << 40 || (uintptr_t)firsts % 4 || (uintptr_t)counts % 4)
        return RKB_E_INVAL;
    if (batch * rows == 0 || cache->tokens == 0) return RKB_OK;
    if (!good_strides(*k, batch, rows, kv_heads) || !good_strides(*v, batch, rows, kv_heads)) return RKB_E_INVAL;
    kv_write w{};
    w.B = (int)batch;
    w.K = (int)kv_heads;
    w.D = (int)dim;
    w.ld = (int)round_up(dim, 16);
    w.rows = rows;
    w.tokens = cache->tokens;
    w.room = round_up(cache->tokens, RKB_GROUP);
    // rows tokens from anywhere in a block touch at most this many
    w.blocks = (int)std::min<int64_t>((rows + 2 * RKB_GROUP - 2) / RKB_GROUP, w.room / RKB_GROUP);
    const int64_t blocks = w.blocks * kv_heads;
    if (batch > ((int64_t)1 << 22) / blocks) return RKB_E_INVAL;
    const rkb_heads *in[2] = {k, v};
    for (int i = 0; i < 2; ++i)
        w.in[i] = kv_side{(const char *)in[i]->p, batch > 1 ? in[i]->batch : 0, rows > 1 ? in[i]->row : 0, kv_heads > 1 ? in[i]->head : 0};
    w.first = first;
    w.firsts = firsts;
    w.counts = counts;
    w.codes = cache->codes;
    w.exps = cache->exps;
    const dim3 grid((uint32_t)(blocks * batch), 2);
    return dtype == RKB_F16 ? launch(k_kv8_write<f16>, grid, dim3(LANES), (hipStream_t)stream, w)
                            : launch(k_kv8_write<bf16>, grid, dim3(LANES), (hipStream_t)stream, w);
}

extern "C" int rkb_kv8_load(int dtype, int64_t batch, int64_t kv_heads, int64_t dim, const rkb_kv8 *cache, const rkb_heads *k,
                            const rkb_heads *v, void *stream)
{
    if (!good_kv(dtype, batch, kv_heads, dim, cache) || !k || !v) return RKB_E_INVAL;
    const int64_t tokens = cache->tokens;
    if (batch * tokens == 0 || (!k->p && !v->p)) return RKB_OK;
    kv_load w{};
    const rkb_heads *out[2] = {k, v};
    for (int i = 0; i < 2; ++i) {
        if (!out[i]->p) continue;
        if (!good_strides(*out[i], batch, tokens, kv_heads) || !elements_apart(*out[i], batch, tokens, kv_heads, dim)) return RKB_E_INVAL;
        w.p[i] = (char *)out[i]->p;
        w.b[i] = batch > 1 ? out[i]->batch : 0;
        w.t[i] = tokens > 1 ? out[i]->row : 0;
        w.h[i] = kv_heads > 1 ? out[i]->head : 0;
    }
    w.codes = cache->codes;
    w.exps = cache->exps;
    w.tokens = tokens;
    w.room = round_up(tokens, RKB_GROUP);
    w.B = (int)batch;
    w.K = (int)kv_heads;
    w.D = (int)dim;
    w.ld = (int)round_up(dim, 16);
    w.chunks = (int)((dim + 7) / 8);
    w.chunks_all = batch * kv_heads * tokens * w.chunks;
    const dim3 grid((uint32_t)std::min<int64_t>((w.chunks_all + LANES - 1) / LANES, 1 << 16), 2);
    return dtype == RKB_F16 ? launch(k_kv8_load<f16>, grid, dim3(LANES), (hipStream_t)stream, w)
                            : launch(k_kv8_load<bf16>, grid, dim3(LANES), (hipStream_t)stream, w);
}
