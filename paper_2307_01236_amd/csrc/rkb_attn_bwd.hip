// Attention backward (rk_block.h).  Probabilities are made again from the row sums that the forward left: dq by a kernel like the
// forward, with queries stationary, dk and dv by one with keys stationary, so that every sum has one owner and a
// fixed order.  That makes the scores and dp twice and, with dq's correction, 8 products instead of 5; it needs no atomics and no [queries, keys] matrix.
#include <algorithm>
#include <climits>

#include "rkb_attn.h"
#include "rkb_attn_args.h"

namespace rkb {
namespace {

constexpr int ROWS = 128, WAVES = 4;  // stationary rows and waves of a workgroup
constexpr int NORM_ROWS = 64;         // rows whose largest norm is kept

struct bwd_in {
    heads_at d_o, o;
    const float *o32, *lse;
    float *delta, *lse2;     // [B, H, stats_rows]: do . o, and -lse in steps of log2 (-inf: a row without keys, or none)
    uint32_t *do_norms, *v_norms;  // f16: bits of the largest |do|^2 and |v|^2 of NORM_ROWS rows: [B, H, stats_rows / NORM_ROWS] and [B, K, ..]
    uint32_t *seen;          // [B, H, stats_rows / 32]: bit r: row r has keys
    int64_t stats_rows;
    heads_at dq, dk, dv;
    float *dq_part, *pk_part, *dk_part, *dv_part;  // [splits, rows, D] each, where there are several; pk: of sum p k
    float *row_part;         // [splits, B, H, stats_rows]: parts of the sums of ds, where there are several
    float *table_part;       // [H, B key tiles splits, buckets]
    int wide;                // bit 0: dq, 1: dk and dv take 8-byte stores
};

// ds enters the products in T.  In f16 a ds of many keys falls below the range (1/4096 of a gradient of 1e-2 is 2e-6), so it is
// scaled by a power of two from |ds| <= 2 |do| |v|, whose largest values of a key head a pass over both finds.
template <class T>
__device__ inline float ds_scale(const bwd_in &g, const attn_in &p, int b, int kv)
{
    if constexpr (!std::is_same_v<T, f16>) return 1.0f;
    const int64_t rows = g.stats_rows / NORM_ROWS * p.G, keys = (p.T + NORM_ROWS - 1) / NORM_ROWS, at = (int64_t)b * p.K + kv;
    uint32_t most[2] = {0, 0};
    for (int64_t n = threadIdx.x % WAVE; n < rows; n += WAVE) most[0] = max(most[0], g.do_norms[at * rows + n]);
    for (int64_t n = threadIdx.x % WAVE; n < keys; n += WAVE) most[1] = max(most[1], g.v_norms[at * keys + n]);
#pragma unroll
    for (int i = 1; i < WAVE; i *= 2) {
        most[0] = max(most[0], (uint32_t)__shfl_xor((int)most[0], i));
        most[1] = max(most[1], (uint32_t)__shfl_xor((int)most[1], i));
    }
    const float x = __uint_as_float(most[0]), y = __uint_as_float(most[1]);
    if (!(x > 0.0f && y > 0.0f && finite(x) && finite(y))) return 1.0f;
    const float e = 12.0f - ceilf(0.5f * (__builtin_amdgcn_logf(x) + __builtin_amdgcn_logf(y)));
    return two_to((int)fminf(fmaxf(e, -100.0f), 100.0f));
}
// p <= 1 likewise, by a fixed power of two.
template <class T>
constexpr float P_LIFT = std::is_same_v<T, f16> ? 14.0f : 0.0f;

// ------------------------------------------------------------------ norms (f16)

// Bound by latency: 6 us for 6 x 199 queries and 777 keys, whose 4 MB are 1 us at the memory's rate.
// The largest |do|^2 of those of NORM_ROWS queries of a head that have keys, or |v|^2 of the live ones among as many keys of a key head; 16 lanes a row.
template <class T>
__global__ __launch_bounds__(256) void k_attn_norms(attn_in p, bwd_in g)
{
    __shared__ uint32_t shared[4];
    const int q_chunks = (int)(g.stats_rows / NORM_ROWS), k_chunks = (p.T + NORM_ROWS - 1) / NORM_ROWS, of_q = p.B * p.H * q_chunks;
    const bool keys = (int)blockIdx.x >= of_q;
    const int n = (int)blockIdx.x - (keys ? of_q : 0), chunks = keys ? k_chunks : q_chunks, heads = keys ? p.K : p.H;
    const int bh = n / chunks, r0 = (n - bh * chunks) * NORM_ROWS, b = bh / heads, h = bh - b * heads, lane = threadIdx.x % 16;
    const int rows = keys ? len_of(p, b) : p.Q;
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < NORM_ROWS / 16; ++k) {
        const int r = r0 + k * 16 + threadIdx.x / 16;
        float norm = 0.0f;
        if (r < rows && (keys ? mask_byte(p, b, r, rows) != 0 : g.lse[(int64_t)bh * p.Q + r] != NEG_INF)) {
            const T *row = keys ? p.v.at<T>(b, r, h) : g.d_o.at<T>(b, r, h);
            for (int c = lane * 8; c < p.D; c += 128) {
                float x[8];
                load8<T>(row + c, p.D - c, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) norm = __builtin_fmaf(x[e], x[e], norm);
            }
        }
        most = max(most, __float_as_uint(lane_sum<16>(norm)) & 0x7fffffffu);
    }
#pragma unroll
    for (int i = 1; i < WAVE; i *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, i));
    if (threadIdx.x % WAVE == 0) shared[threadIdx.x / WAVE] = most;
    __syncthreads();
    if (threadIdx.x == 0) (keys ? g.v_norms : g.do_norms)[n] = max(max(shared[0], shared[1]), max(shared[2], shared[3]));
}

// ------------------------------------------------------------------ what a lane stores of a row

template <class T, int A>
__device__ inline void store_grad(T *to, float *part, bool wide, int width, const f32x16 (&acc)[A], float times, bool zero, int lane)
{
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = a * 32 + q * 8 + half_row(lane);
            f32x4 w;
            vec<T, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = zero ? 0.0f : acc[a][q * 4 + e] * times;
                v[e] = (T)settled<T>(w[e]);
            }
            if (part) {
                if (col + 4 <= width && width % 4 == 0) {
                    *(f32x4 *)(part + col) = w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + e < width) part[col + e] = w[e];
                }
            } else if (col + 4 <= width && wide) {
                *(vec<T, 4> *)(to + col) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < width) to[col + e] = v[e];
            }
        }
}

// ------------------------------------------------------------------ dq
//
// A row's delta = do . o and -lse are formed here, where its do is in registers, and left for dk and dv.  delta comes from an o that
// was summed from rounded probabilities (and may be rounded itself), so ds of a row adds up to some r
// instead of 0.  Then delta + r is what delta should have been, to 32 bits: it is left for dk, dv and the bias's gradient, which
// are formed from it afterwards.  dq itself is sum ds k - r sum p k, whose second product shares the keys' fragments with the first.
// Heads of more than 128 columns are two workgroups', each with half of dq's columns.
//
// 4 x 2048 queries of 32 heads of 128 over 4096 keys of 8 (some padded): 670 to 730 us, 1.0 to 1.1 PFLOP/s with four products; without sum p k 527 to 540.  Two
// waves of a unit hide part of each other's waits: each waits 41 % of its time, and the matrix units are busy 53 %.  One wave with twice the registers,
// which then need not keep do in LDS, took 800.
template <class T, int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_attn_dq(attn_in p, bwd_in g, int splits)
{
    using L = lay<DP>;
    constexpr bool DO_LDS = DP == 128;  // a wave's do lies in LDS: two waves of a unit leave it 256 registers, of which the sums take 128
    constexpr int TILE = DP >= 128 ? 32 : 64, N = TILE / 32, BYTES = TILE * DP * 2, C = DP / 16, HALVES = DP == 256 ? 2 : 1, A = DP / 32 / HALVES;
    __shared__ __align__(16) char k0[BYTES], k1[BYTES], v0[BYTES], v1[BYTES];
    __shared__ __align__(16) char own_do[DO_LDS ? WAVES * 32 * DP * 2 : 16];
    __shared__ float by_distance[2 * (MAX_FAR + PAD) + 1];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int q_tiles = (p.Q + ROWS - 1) / ROWS;
    int w = unit_order(blockIdx.x, p.B * p.K, p.G * splits * q_tiles * HALVES);
    const int a0 = w % HALVES * A;  // the first of this workgroup's column blocks of 32
    w /= HALVES;
    const int qt = q_tiles - 1 - w % q_tiles;
    w /= q_tiles;
    const int split = w % splits, bh = w / splits, b = bh / p.H, h = bh - b * p.H, kv = h / p.G;
    const int len = len_of(p, b), first = first_of(p, b);
    const int q0 = qt * ROWS, q1 = min(q0 + ROWS, p.Q);
    const int end = p.causal ? min(len, max(first + q1 - 1, -1) + 1) : len;
    const int tiles = (end + TILE - 1) / TILE, each = (tiles + splits - 1) / splits;
    const int t0 = split * each, t1 = min(tiles, t0 + each);

    const int i = q0 + wave * 32 + lane % 32;
    const bool there = i < p.Q;
    const int pos_lo = first + q0 + wave * 32, pos_hi = pos_lo + 31;
    frag<T> q[C], d[C];
    load_stationary<T, DP>(q, p.q.at<T>(b, min(i, p.Q - 1), h), lane, p.D, there);
    load_stationary<T, DP>(d, g.d_o.at<T>(b, min(i, p.Q - 1), h), lane, p.D, there);
    const bool counted = i < g.stats_rows && a0 == 0;  // rows past the last query are left as rows without keys, for tiles that reach there
    const int64_t stat = (int64_t)bh * g.stats_rows + i;
    float lse = NEG_INF, delta = 0.0f;
    if (there) {
        const float l = g.lse[(int64_t)bh * p.Q + i];
        const T *o = g.o32 ? nullptr : g.o.at<T>(b, i, h);
        const float *o32 = g.o32 ? g.o32 + (((int64_t)b * p.Q + i) * p.H + h) * p.D : nullptr;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = c * 16 + lane / 32 * 8;
            float v[8];
            if (o32)
                load8<float>(o32 + col, p.D - col, v);
            else
                load8<T>(o + col, p.D - col, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = __builtin_fmaf((float)d[c][e], v[e], delta);
        }
        lse = l == NEG_INF ? NEG_INF : -l * LOG2E;
    }
    delta = half_sum(delta);
    if (lse == NEG_INF) delta = 0.0f;
    if (counted && lane < 32 && split == 0) {
        const uint32_t seen = (uint32_t)__ballot(lse != NEG_INF);
        if (lane == 0) g.seen[stat / 32] = seen;
        g.lse2[stat] = lse;
        if (g.row_part) g.delta[stat] = delta;
    }
    const float lift = ds_scale<T>(g, p, b, kv);
    const int far = p.bias.far;
    lds_byte *const my_do = (lds_byte *)own_do + wave * 32 * L::PITCH;
    if constexpr (DO_LDS) {
#pragma unroll
        for (int c = 0; c < C; ++c) *(__attribute__((address_space(3))) frag<T> *)(my_do + (L::rows_place(lane) ^ c * 32)) = d[c];
        asm volatile("" ::: "memory");
    }
    if (p.bias.table) fill_bias<T>(by_distance, p, h, threadIdx.x, 256);

    tile_copy<DP, TILE, WAVES> kc, vc;
    const T *const kp = p.k.at<T>(b, 0, kv), *const vp = p.v.at<T>(b, 0, kv);
    kc.set(wave, lane, p.k.t, p.D);
    vc.set(wave, lane, p.v.t, p.D);
    constexpr uint64_t ALL = N == 2 ? ~(uint64_t)0 : 0xffffffffu;
    auto fetch = [&](int t, uint64_t live, lds_byte *kto, lds_byte *vto) __attribute__((always_inline)) {
        const int64_t key = (int64_t)t * TILE;
        const bool all = (live & ALL) == ALL && p.D == DP;
        kc.copy(wave, lane, (const char *)(kp + key * p.k.t), live, all, kto);
        vc.copy(wave, lane, (const char *)(vp + key * p.v.t), live, all, vto);
    };

    f32x16 acc[A] = {}, pk[A] = {};
    const int place = L::rows_place(lane), cols[2] = {L::cols_place(lane, 0), L::cols_place(lane, 1)};
    float row_sum[2] = {0.0f, 0.0f};
    const float lifted = lse + P_LIFT<T>, drop = __builtin_amdgcn_exp2f(-P_LIFT<T>), ds_times = lift * drop;
    auto compute = [&](int t, uint64_t live, lds_byte *kt, lds_byte *vt) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int key0 = t * TILE + n * 32;
            f32x16 s = {}, dp = {};
            int own = place;
            asm volatile("" : "+v"(own));  // places in do are worked out each time, too
#pragma unroll
            for (int c = 0; c < C; ++c) {
                s = mma32(L::template rows<T>(kt, place, c, n * 32), q[c], s);
                if constexpr (DO_LDS)
                    dp = mma32(L::template rows<T>(vt, place, c, n * 32), L::template rows<T>(my_do, own, c, 0), dp);
                else
                    dp = mma32(L::template rows<T>(vt, place, c, n * 32), d[c], dp);
            }
            float by = p.c;
            int me = lane;
            asm volatile("" : "+v"(me));  // nothing of this is worked out ahead of the loop: it would hold registers in every turn
            if (p.bias.table) {
                by = 1.0f;
                add_bias(s, p.c, by_distance, far, key0, pos_lo + me % 32, pos_lo, pos_hi, me);
            }
            kill_dead(s, (uint32_t)(live >> n * 32), p.causal ? pos_lo + me % 32 - key0 : INT_MAX, me, NEG_INF);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                frag<T> fp, fd;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = half * 8 + e;
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], by, lifted)), ds = x * (dp[r] - delta);
                    row_sum[r % 2] += ds;
                    fp[e] = (T)x;
                    fd[e] = (T)(std::is_same_v<T, f16> ? ds * ds_times : ds);
                }
#pragma unroll
                for (int a = 0; a < A; ++a) {
                    const frag<T> keys = L::template cols<T>(kt, cols, a0 + a, n * 32 + half * 16);
                    acc[a] = mma32(keys, fd, acc[a]);
                    pk[a] = mma32(keys, fp, pk[a]);
                }
            }
        }
    };

    if (t0 < t1) {
        uint8_t byte = mask_byte(p, b, t0 * TILE + lane, len);
        uint64_t live = keys_alive(p, t0 * TILE, len, byte);
        fetch(t0, live, (lds_byte *)k0, (lds_byte *)v0);
        byte = mask_byte(p, b, (t0 + 1) * TILE + lane, len);
        auto step = [&](int t, char *kh, char *vh, char *kn, char *vn) __attribute__((always_inline)) {
            wait_all();
            uint64_t next = 0;
            if (t + 1 < t1) {
                next = keys_alive(p, (t + 1) * TILE, len, byte);
                byte = mask_byte(p, b, (t + 2) * TILE + lane, len);
                fetch(t + 1, next, (lds_byte *)kn, (lds_byte *)vn);
            }
            compute(t, live, (lds_byte *)kh, (lds_byte *)vh);
            live = next;
        };
        for (int t = t0; t < t1; t += 2) {
            step(t, k0, v0, k1, v1);
            if (t + 1 < t1) step(t + 1, k1, v1, k0, v0);
        }
    }
    // places are worked out again, so that they hold no registers in the loop
    int me = threadIdx.x % WAVE;
    asm volatile("" : "+v"(me));
    const int row_i = q0 + wave * 32 + me % 32;
    const bool none = lifted == NEG_INF, stored = row_i < p.Q;
    const float r = half_sum(row_sum[0] + row_sum[1]) * drop;
    if (stored && g.dq.p) {
        const int64_t row = ((int64_t)b * p.Q + row_i) * p.H + h, rows = (int64_t)p.B * p.Q * p.H, part = (split * rows + row) * p.D + a0 * 32;
        const float times = p.scale / lift;
        if (g.dq_part) {
            store_grad<T, A>(nullptr, g.pk_part + part, false, p.D - a0 * 32, pk, p.scale * drop, none, me);
        } else {
            const float less = r * lift * drop;
#pragma unroll
            for (int a = 0; a < A; ++a)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[a][e] = __builtin_fmaf(-less, pk[a][e], acc[a][e]);
        }
        store_grad<T, A>(g.dq.at<T>(b, row_i, h) + a0 * 32, g.dq_part ? g.dq_part + part : nullptr, g.wide & 1, p.D - a0 * 32, acc, times, none, me);
    }
    if (row_i < g.stats_rows && a0 == 0 && me < 32) {
        const int64_t at = (int64_t)bh * g.stats_rows + row_i;
        if (g.row_part)
            g.row_part[(int64_t)split * p.B * p.H * g.stats_rows + at] = none ? 0.0f : r;
        else
            g.delta[at] = none ? 0.0f : delta + r;
    }
}

// delta + r where splits of the keys left parts of r, and no dq is asked for (else k_attn_grads does it).
__global__ __launch_bounds__(256) void k_attn_delta_join(attn_in p, bwd_in g, int splits)
{
    const int64_t rows = (int64_t)p.B * p.H * g.stats_rows;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < rows; at += (int64_t)gridDim.x * 256) {
        float r = 0.0f;
        for (int s = 0; s < splits; ++s) r += g.row_part[s * rows + at];
        g.delta[at] += r;
    }
}

// dtable[c, h]: a wave adds up what a head's workgroups found of a bucket.
template <class T>
__global__ __launch_bounds__(WAVE) void k_attn_dtable(attn_in p, const float *part, int64_t of_head, void *dtable)
{
    const int buckets = p.bias.count * p.bias.sides, h = blockIdx.x / buckets, c = blockIdx.x - h * buckets;
    float sum = 0.0f;
    for (int64_t n = threadIdx.x; n < of_head; n += WAVE) sum += part[(h * of_head + n) * buckets + c];
    sum = lane_sum<64>(sum);
    if (threadIdx.x) return;
    const int64_t at = (int64_t)c * p.H + h;
    if (p.bias.f32)
        ((float *)dtable)[at] = sum;
    else
        ((T *)dtable)[at] = (T)settled<T>(sum);
}

// ------------------------------------------------------------------ dk and dv
//
// A workgroup has 128 keys of one key head, 32 a wave, and passes over the queries of all heads that share it in tiles of 32 (of q and do), RING of
// them in LDS in turn.  While the matrix units form the next tile's scores and dp, the vector units make this tile's probabilities and ds, which
// then enter dv and dk.  Heads of more than 128 columns are two workgroups', each with half of dk's and dv's columns: all of them do not fit
// into registers.
//
// 4 x 2048 queries of 32 heads of 128 over 4096 keys of 8 (some padded): 880 to 910 us, 0.8 PFLOP/s with four products.  A wave has a unit's registers to
// itself, so nothing but its own order hides what it waits for: it waits 30 % of its time and issues in half of it, while the matrix units are busy
// 42 % and LDS 26 %.  With a bias, 16 x 512 x 512, 12 heads of 64: 82 us; its two waves of a unit wait 45 % of their time
// each, and the issue is busy 60 %.
//
// FAR: the largest distance that the bias looks up (0: no bias).  Its gradient, ds by buckets, is summed over diagonals: a wave lays the
// queries x 32 keys of some registers into LDS at (query, key - query), whose columns are diagonals, and a lane adds up a column.  What no
// register ever writes there stays 0.  Tiles that lie beyond FAR whole are added up in registers.
template <class T, int DP, int FAR>
__global__ __launch_bounds__(256, DP == 64 && FAR <= 128 ? 2 : 1) void k_attn_dkv(attn_in p, bwd_in g, int splits)
{
    using L = lay<DP>;
    constexpr int TILE = 32, BYTES = TILE * DP * 2, C = DP / 16, HALVES = DP / 128 > 1 ? 2 : 1, A = DP / 32 / HALVES;
    // DIAG queries are laid out at a time, in AREAS places in turn (the fewer where little LDS is left); the pitch keeps a wave's writes in different banks
    constexpr int DIAG = DP == 256 && FAR > 128 ? 8 : 16, AREAS = DIAG == 16 ? 2 : 1, PITCH = DIAG == 16 ? 57 : 41;
    // CARRY: the first fragments of the next turn are read at this one's end, so that its products need not wait for them.
    constexpr bool CARRY = DP == 128 && FAR <= 128;
    // Tiles that LDS holds; of them a turn copies the one AHEAD further on, and finds that of NEED further on landed.
    constexpr int RING = DP == 256 ? 3 : CARRY ? 6 : 4, AHEAD = DP == 256 ? 2 : CARRY ? 4 : 3, NEED = CARRY ? 2 : 1;
    constexpr int FLYING = (AHEAD - 1 - NEED) * (2 * tile_copy<DP, TILE, WAVES>::MINE + 1);  // copies that may be on their way beyond those
    constexpr int B3 = RING > 3 ? BYTES : 16, B5 = RING > 5 ? BYTES : 16;
    __shared__ __align__(16) char q0[BYTES], q1[BYTES], q2[BYTES], q3[B3], q4[B5], q5[B5], d0[BYTES], d1[BYTES], d2[BYTES], d3[B3], d4[B5], d5[B5];
    char *const qs[6] = {q0, q1, q2, q3, q4, q5}, *const ds[6] = {d0, d1, d2, d3, d4, d5};
    __shared__ __align__(16) float stats[RING][WAVES][64];  // of each wave: 32 rows' -lse2, then their delta
    __shared__ float by_distance[2][FAR ? 2 * (FAR + PAD) + 1 : 1], sums[FAR ? WAVES : 1][2 * FAR + 1], diag[FAR ? WAVES : 1][FAR ? AREAS : 1][FAR ? DIAG * PITCH : 1];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int k_tiles = (p.T + ROWS - 1) / ROWS;
    int w = unit_order(blockIdx.x, p.B * p.K, splits * k_tiles * HALVES);
    const int a0 = w % HALVES * A;  // the first of this workgroup's column blocks of 32
    w /= HALVES;
    const int kt = w % k_tiles;
    w /= k_tiles;
    const int split = w % splits, bk = w / splits, b = bk / p.K, kv = bk - b * p.K;
    const int len = len_of(p, b), first = first_of(p, b);
    const int wave_key = kt * ROWS + wave * 32, key = wave_key + lane % 32;
    const bool alive = key < len && mask_byte(p, b, key, len), all_alive = __all(alive);

    // queries that see any of the workgroup's keys: those from `from` on
    const int from = p.causal ? (int)min((int64_t)p.Q, max((int64_t)0, (int64_t)kt * ROWS - first)) : 0;
    const int tile0 = from / TILE, q_tiles = (p.Q + TILE - 1) / TILE, of_head = kt * ROWS < len ? max(0, q_tiles - tile0) : 0;
    const int64_t all = (int64_t)of_head * p.G, each = (all + splits - 1) / splits;
    const int64_t t0 = split * each, t1 = min(all, t0 + each);

    frag<T> k[C], v[C];
    load_stationary<T, DP>(k, p.k.at<T>(b, min(key, p.T - 1), kv), lane, p.D, alive);
    load_stationary<T, DP>(v, p.v.at<T>(b, min(key, p.T - 1), kv), lane, p.D, alive);
    const float lift = ds_scale<T>(g, p, b, kv);
    const float ds_times = std::is_same_v<T, f16> ? lift * __builtin_amdgcn_exp2f(-P_LIFT<T>) : 1.0f;
    const int far = p.bias.far;

    tile_copy<DP, TILE, WAVES> qc, dc;
    qc.set(wave, lane, p.q.t, p.D);
    dc.set(wave, lane, g.d_o.t, p.D);
    // the next tile to be copied: its tile, and where its rows and row sums are
    int copy_t = 0, copy_h = 0;
    const char *copy_q = nullptr, *copy_d = nullptr;
    const float *copy_s = nullptr;
    const int64_t q_step = TILE * p.q.t * 2, d_step = TILE * g.d_o.t * 2;
    auto copy_from = [&](int h, int t) __attribute__((always_inline)) {
        copy_t = t;
        copy_q = (const char *)p.q.at<T>(b, (int64_t)t * TILE, h);
        copy_d = (const char *)g.d_o.at<T>(b, (int64_t)t * TILE, h);
        copy_s = (lane < 32 ? g.lse2 : g.delta) + ((int64_t)b * p.H + h) * g.stats_rows + t * TILE + lane % 32;  // rows are padded
    };
    // Queries without keys become zeros: 0 times whatever lies there would not be 0.  Only order, masks and bias leave such queries; whether any
    // did is looked up once.
    bool gaps = false;
    if (of_head && (p.causal || p.mask || FAR > 0)) {
        const uint32_t *const seen = g.seen + ((int64_t)b * p.H + kv * p.G) * (g.stats_rows / TILE);
        const int words = (int)(g.stats_rows / TILE), last = p.Q % TILE;
        const uint32_t of_last = last ? (1u << last) - 1 : ~0u;
        for (int64_t n = threadIdx.x % WAVE; n < (int64_t)words * p.G; n += WAVE) {
            const int at = (int)(n % words);
            gaps |= seen[n] != (at < q_tiles - 1 ? ~0u : at == q_tiles - 1 ? of_last : 0u);
        }
        gaps = __any(gaps);
    }
    auto fetch = [&](char *qto, char *dto, float *sto) __attribute__((always_inline)) {
        const int n = p.Q - copy_t * TILE;
        uint64_t live = n >= TILE ? 0xffffffffu : ((uint64_t)1 << n) - 1;
        if (gaps) live = g.seen[((int64_t)b * p.H + copy_h) * (g.stats_rows / TILE) + copy_t];
        const bool whole = (uint32_t)live == ~0u && p.D == DP;
        qc.copy(wave, lane, copy_q, live, whole, (lds_byte *)qto);
        dc.copy(wave, lane, copy_d, live, whole, (lds_byte *)dto);
        __builtin_amdgcn_global_load_lds((global_void *)copy_s, (lds_void *)(lds_byte *)(sto + wave * 64), 4, 0, 0);
        copy_q += q_step;
        copy_d += d_step;
        copy_s += TILE;
        if (++copy_t == q_tiles) copy_from(++copy_h, tile0);
    };

    f32x16 dk[A] = {}, dv[A] = {}, sa, sb, pa, pb;  // scores and dp of two tiles
    float by = p.c, add = 0.0f;                     // of the tile that waits: its scores are x by + add in steps of log2
    const int place = L::rows_place(lane), cols[2] = {L::cols_place(lane, 0), L::cols_place(lane, 1)};
    float far_sum[2] = {0.0f, 0.0f};  // of keys far behind, far ahead
    auto add_up = [&](const f32x16 &ds, int pos0) __attribute__((always_inline)) {
        if constexpr (FAR > 0) {
            if (wave_key - pos0 - 31 >= far || wave_key + 31 - pos0 <= -far) {
                float sum[2] = {0.0f, 0.0f};
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[r % 2] += ds[r];
                if (wave_key > pos0)
                    far_sum[1] += sum[0] + sum[1];
                else
                    far_sum[0] += sum[0] + sum[1];
                return;
            }
            int me = lane;
            asm volatile("" : "+v"(me));  // nothing of this is worked out ahead of the loop
            constexpr int PARTS = 32 / DIAG;
            auto lay_out = [&](int part) __attribute__((always_inline)) {
                float *const to = diag[wave][part % AREAS] + half_row(me) * (PITCH - 1) + me % 32 + DIAG - 1;
#pragma unroll
                for (int r = 0; r < DIAG / 2; ++r) to[(r / 4 * 8 + r % 4) * (PITCH - 1)] = ds[part * (DIAG / 2) + r];
            };
            auto collect = [&](int part) __attribute__((always_inline)) {
                if (me < 31 + DIAG) {
                    const float *const from = diag[wave][part % AREAS] + me;
                    float sum[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int row = 0; row < DIAG; ++row) sum[row % 2] += from[row * PITCH];
                    const int rel = wave_key - pos0 - part * DIAG + me - (DIAG - 1);
                    if (rel >= far)
                        far_sum[1] += sum[0] + sum[1];
                    else if (rel <= -far)
                        far_sum[0] += sum[0] + sum[1];
                    else
                        sums[wave][rel + far] += sum[0] + sum[1];
                }
            };
            // what one lane writes others read: in this order
            if constexpr (AREAS == PARTS) {
#pragma unroll
                for (int part = 0; part < PARTS; ++part) lay_out(part);
                asm volatile("" ::: "memory");
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    collect(part);
                    asm volatile("" ::: "memory");
                }
            } else {
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    lay_out(part);
                    asm volatile("" ::: "memory");
                    collect(part);
                    asm volatile("" ::: "memory");
                }
            }
        }
    };
    // What this workgroup found of a head's buckets goes to its place; the sums start again.
    auto flush = [&](int h) {
        if constexpr (FAR > 0) {
            if (!g.table_part) return;
            const float behind = lane_sum<64>(far_sum[0]), ahead = lane_sum<64>(far_sum[1]);
            far_sum[0] = far_sum[1] = 0.0f;
            if (lane == 0) {
                sums[wave][0] = behind;
                sums[wave][2 * far] = ahead;
            }
            __syncthreads();
            // a wave adds up a bucket, 64 distances at a time
            const int count = p.bias.count, buckets = count * p.bias.sides;
            const int64_t of_head = (int64_t)p.B * k_tiles * splits, me = ((int64_t)b * k_tiles + kt) * splits + split;
            for (int c = wave; c < buckets && a0 == 0; c += WAVES) {
                const int side = c / count, n = c - side * count;
                const int lo = n == 0 ? side : p.bias.border[n - 1], hi = n == count - 1 ? far : p.bias.border[n] - 1;
                // the positions in sums; of a one-sided bias, keys ahead count as distance 0
                const int from = side ? far + lo : far - hi, to = side ? far + hi : p.bias.sides == 1 && n == 0 ? 2 * far : far - lo;
                float sum = 0.0f;
                for (int at = from + lane; at <= to; at += WAVE) sum += (sums[0][at] + sums[1][at]) + (sums[2][at] + sums[3][at]);
                sum = lane_sum<64>(sum);
                if (lane == 0) g.table_part[(h * of_head + me) * buckets + c] = sum * __builtin_amdgcn_exp2f(-P_LIFT<T>);
            }
            __syncthreads();
            for (int n = lane; n <= 2 * far; n += WAVE) sums[wave][n] = 0.0f;
        }
    };
    // Scores of a tile that its lanes do not see alike: bias by distance, keys behind the query, dead keys (whose own sums are not stored, but the
    // bias's would have them).  Then x are steps of log2 themselves.
    auto adjust = [&](int hg, int t, f32x16 &s) __attribute__((always_inline)) {
        const int pos0 = first + t * TILE;
        by = p.c;
        add = 0.0f;
        bool near = false;
        if constexpr (FAR > 0) {
            const bool ahead = wave_key - pos0 - 31 >= far, behind = wave_key + 31 - pos0 <= -far;
            near = !ahead && !behind;
            if (!near) add = by_distance[hg & 1][ahead ? 2 * (far + PAD) : 0];
        }
        const bool hidden = p.causal && pos0 < wave_key + 31;
        if (!near && !hidden && (FAR == 0 || all_alive)) return;
        int me = lane;
        asm volatile("" : "+v"(me));  // nothing of this is worked out ahead of the loop
        const int rel = wave_key + me % 32 - pos0 - half_row(me);  // of register 0
        if (FAR > 0 && near) {
            const float *const at = by_distance[hg & 1] + rel + far + PAD;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], p.c, at[-(r / 4 * 8 + r % 4)]);
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], p.c, add);
        }
        if (hidden || (FAR > 0 && !all_alive)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = (hidden && rel > r / 4 * 8 + r % 4) || (FAR > 0 && !alive) ? NEG_INF : s[r];
        }
        by = 1.0f;
        add = 0.0f;
    };
    constexpr int READS = CARRY ? 4 : DP == 256 ? 2 : 3;  // fragments that are read ahead of their products
    frag<T> rf[READS + 1];
    f32x4 off[4], delta[4];
    auto read_rows = [&](char *qn, char *dn, int n) __attribute__((always_inline)) {  // fragments of q and do in turn
        return L::template rows<T>((lds_byte *)(n % 2 ? dn : qn), place, n / 2, 0);
    };
    // What a turn starts with: its tile's row sums, the next tile's first fragments.
    auto start = [&](const float *stat, char *qn, char *dn) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < READS; ++n) rf[n] = read_rows(qn, dn, n);
#pragma unroll
        for (int r8 = 0; r8 < 4; ++r8) {
            off[r8] = *(const f32x4 *)(stat + r8 * 8 + half_row(lane));
            delta[r8] = *(const f32x4 *)(stat + 32 + r8 * 8 + half_row(lane));
        }
    };
    // One turn, started.  s and dp: this tile's, which lies in qh and dh; s2, dp2: the next one's, in qn and dn.  What the vector units do is
    // dealt out between the matrix instructions: the first 16 queries' during the next tile's products, the others' during the first
    // 16 queries' own.
    auto turn = [&](char *qh, char *dh, char *qn, char *dn, f32x16 &s, f32x16 &dp, f32x16 &s2, f32x16 &dp2) __attribute__((always_inline)) {
        constexpr int SKEW = 2, EARLY = 2, N = 2 * C - EARLY;  // EARLY: products that run before the row sums are there
        auto pin = [] { __builtin_amdgcn_sched_barrier(0); };
        auto here = [&](int n) __attribute__((always_inline)) {  // fragments of do and q in turn, of both halves
            return L::template cols<T>((lds_byte *)(n % 2 ? qh : dh), cols, a0 + n / 2 % A, n / 2 / A * 16);
        };
        frag<T> cf[READS + 1], fp[2], fd[2];
        float x[16];
        auto scale = [&](int e) __attribute__((always_inline)) {
            x[e] = __builtin_fmaf(s[e], by, FAR > 0 || P_LIFT<T> != 0.0f ? off[e / 4][e % 4] + (add + P_LIFT<T>) : off[e / 4][e % 4]);
            dp[e] -= delta[e / 4][e % 4];
        };
        auto power = [&](int e) __attribute__((always_inline)) { x[e] = __builtin_amdgcn_exp2f(x[e]); };
        auto soften = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
            for (int e = from; e < to; ++e) {
                if (e + 2 * SKEW < 16) scale(e + 2 * SKEW);
                if (e + SKEW < 16) power(e + SKEW);
                dp[e] *= x[e];
                fp[e / 8][e % 8] = (T)x[e];
                fd[e / 8][e % 8] = (T)(std::is_same_v<T, f16> ? dp[e] * ds_times : dp[e]);
            }
        };
#pragma unroll
        for (int n = 0; n < 2 * C; ++n) {
            if (n + READS < 2 * C)
                rf[(n + READS) % (READS + 1)] = read_rows(qn, dn, n + READS);
            else
                cf[n + READS - 2 * C] = here(n + READS - 2 * C);
            if (n % 2)
                dp2 = mma32(rf[n % (READS + 1)], v[n / 2], n == 1 ? f32x16{} : dp2);
            else
                s2 = mma32(rf[n % (READS + 1)], k[n / 2], n == 0 ? f32x16{} : s2);
            if (n == EARLY - 1) {
#pragma unroll
                for (int e = 0; e < 2 * SKEW; ++e) scale(e);
#pragma unroll
                for (int e = 0; e < SKEW; ++e) power(e);
            }
            if (n >= EARLY) soften((n - EARLY) * 8 / N, (n - EARLY + 1) * 8 / N);
            pin();
        }
#pragma unroll
        for (int n = 0; n < 4 * A; ++n) {
            if (n + READS < 4 * A) cf[(n + READS) % (READS + 1)] = here(n + READS);
            if (n % 2)
                dk[n / 2 % A] = mma32(cf[n % (READS + 1)], fd[n / 2 / A], dk[n / 2 % A]);
            else
                dv[n / 2 % A] = mma32(cf[n % (READS + 1)], fp[n / 2 / A], dv[n / 2 % A]);
            if (n < 2 * A) soften(8 + n * 8 / (2 * A), 8 + (n + 1) * 8 / (2 * A));
            pin();
        }
    };

    int heads_done[2] = {0, 0};  // heads that this workgroup left sums of
    if constexpr (FAR > 0) {
        for (int n = lane; n <= 2 * far; n += WAVE) sums[wave][n] = 0.0f;
        for (int n = lane; n < AREAS * DIAG * PITCH; n += WAVE) diag[wave][0][n] = 0.0f;
    }
    if (t0 < t1) {
        int hg = (int)(t0 / of_head), t = (int)(t0 - (int64_t)hg * of_head) + tile0, filled = hg;
        copy_h = kv * p.G + hg;
        copy_from(copy_h, t);
        heads_done[0] = hg;
        heads_done[1] = (int)((t1 - 1) / of_head) + 1;
        if constexpr (FAR > 0) {
            fill_bias<T>(by_distance[hg & 1], p, kv * p.G + hg, threadIdx.x, 256);
            if (hg + 1 < heads_done[1]) fill_bias<T>(by_distance[hg + 1 & 1], p, kv * p.G + hg + 1, threadIdx.x, 256);
        }
#pragma unroll
        for (int n = 0; n < AHEAD; ++n)
            if (t0 + n < t1) fetch(qs[n], ds[n], stats[n][0]);
        wait_all();
        sa = pa = f32x16{};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            sa = mma32(L::template rows<T>((lds_byte *)q0, place, c, 0), k[c], sa);
            pa = mma32(L::template rows<T>((lds_byte *)d0, place, c, 0), v[c], pa);
        }
        adjust(hg, t, sa);
        if constexpr (CARRY) start(stats[0][wave], q1, d1);
        // Tile `at`, the ring's n-th.  The one AHEAD further on goes where one was that all waves have read when they pass the barrier.  Copies land in
        // order, so those of later tiles need not be waited for.
        auto step = [&](int64_t at, auto place_in_ring) __attribute__((always_inline)) {
            constexpr int n = place_in_ring(), HERE = n % RING, NEXT = (n + 1) % RING, THEN = (n + 2) % RING, COPY = (n + AHEAD) % RING;
            f32x16 &s = n % 2 ? sb : sa, &dp = n % 2 ? pb : pa, &s2 = n % 2 ? sa : sb, &dp2 = n % 2 ? pa : pb;
            if constexpr (FAR > 0)
                if (filled != hg) {
                    flush(kv * p.G + filled);
                    filled = hg;
                    if (hg + 1 < heads_done[1]) fill_bias<T>(by_distance[hg + 1 & 1], p, kv * p.G + hg + 1, threadIdx.x, 256);
                }
            if (FLYING > 0 && at + AHEAD - 1 < t1)
                __builtin_amdgcn_s_waitcnt(wait_copies(FLYING));
            else
                __builtin_amdgcn_s_waitcnt(wait_copies(0));
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (at + AHEAD < t1) fetch(qs[COPY], ds[COPY], stats[COPY][0]);
            if constexpr (!CARRY) start(stats[HERE][wave], qs[NEXT], ds[NEXT]);
            turn(qs[HERE], ds[HERE], qs[NEXT], ds[NEXT], s, dp, s2, dp2);
            // behind the last tile: whatever lies there, not used
            if constexpr (CARRY) start(stats[NEXT][wave], qs[THEN], ds[THEN]);
            add_up(dp, first + t * TILE);
            if (++t == q_tiles) {
                t = tile0;
                ++hg;
            }
            if (at + 1 < t1) adjust(hg, t, s2);
        };
        for (int64_t at = t0; at < t1; at += RING == 4 ? 4 : 6) {
            step(at, std::integral_constant<int, 0>());
            if (at + 1 < t1) step(at + 1, std::integral_constant<int, 1>());
            if (at + 2 < t1) step(at + 2, std::integral_constant<int, 2>());
            if (at + 3 < t1) step(at + 3, std::integral_constant<int, 3>());
            if constexpr (RING != 4) {
                if (at + 4 < t1) step(at + 4, std::integral_constant<int, 4>());
                if (at + 5 < t1) step(at + 5, std::integral_constant<int, 5>());
            }
        }
        flush(kv * p.G + filled);
    }
    if constexpr (FAR > 0)
        if (g.table_part && a0 == 0) {
            const int buckets = p.bias.count * p.bias.sides;
            const int64_t of_head = (int64_t)p.B * k_tiles * splits, me = ((int64_t)b * k_tiles + kt) * splits + split;
            for (int hg = 0; hg < p.G; ++hg)
                if ((hg < heads_done[0] || hg >= heads_done[1]) && threadIdx.x < buckets)
                    g.table_part[((kv * p.G + hg) * of_head + me) * buckets + threadIdx.x] = 0.0f;
        }
    if (key >= p.T || !g.dk.p) return;
    const int64_t row = ((int64_t)b * p.T + key) * p.K + kv, rows = (int64_t)p.B * p.T * p.K, at = (split * rows + row) * p.D + a0 * 32;
    store_grad<T, A>(g.dk.at<T>(b, key, kv) + a0 * 32, g.dk_part ? g.dk_part + at : nullptr, g.wide >> 1 & 1, p.D - a0 * 32, dk, p.scale / lift, !alive, lane);
    store_grad<T, A>(g.dv.at<T>(b, key, kv) + a0 * 32, g.dv_part ? g.dv_part + at : nullptr, g.wide >> 1 & 1, p.D - a0 * 32, dv,
                     __builtin_amdgcn_exp2f(-P_LIFT<T>), !alive, lane);
}

// ------------------------------------------------------------------ splits joined

struct grad_join {
    const float *part;
    heads_at to;
    int64_t rows;  // batch * n * heads
    int n, heads;
    // dq: parts of sum p k, taken r times, whose parts are [splits, batch, heads, stats_rows] and which is added to delta; else NULL
    const float *less, *by;
    float *delta;
    int64_t stats_rows, by_size;
};

// A lane has 4 columns of a row (with `wide` as one piece); splits are added in order.  Mostly a launch's latency: 5 to 6 us.
template <class T>
__global__ __launch_bounds__(256) void k_attn_grads(grad_join j0, grad_join j1, int D, int splits, int wide)
{
    const grad_join &j = blockIdx.y ? j1 : j0;
    const uint32_t quads = (D + 3) / 4;
    const int64_t size = j.rows * D, all = j.rows * quads;
    const bool small = all >> 31 == 0;  // 64-bit division is slow
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t row = small ? (uint32_t)at / quads : at / quads, t = small ? (uint32_t)row / (uint32_t)j.heads : row / j.heads;
        const int64_t b = small ? (uint32_t)t / (uint32_t)j.n : t / j.n;
        const int col = (int)(at - row * quads) * 4;
        const float *const from = j.part + row * D + col, *const less = j.less + row * D + col;
        float r = 0.0f;
        if (j.less) {
            const int64_t stat = (b * j.heads + (row - t * j.heads)) * j.stats_rows + (t - b * j.n);
            for (int s = 0; s < splits; ++s) r += j.by[s * j.by_size + stat];
            if (col == 0) j.delta[stat] += r;
            r = -r;
        }
        T *const to = j.to.at<T>(b, t - b * j.n, row - t * j.heads) + col;
        if (wide) {
            f32x4 sum = {};
#pragma unroll 4
            for (int s = 0; s < splits; ++s) sum += *(const f32x4 *)(from + s * size);
            if (j.less) {
                f32x4 pk = {};
#pragma unroll 4
                for (int s = 0; s < splits; ++s) pk += *(const f32x4 *)(less + s * size);
                sum += pk * r;
            }
            vec<T, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (T)settled<T>(sum[e]);
            *(vec<T, 4> *)to = v;
        } else {
            for (int e = 0; e < 4 && col + e < D; ++e) {
                float sum = 0.0f;
                for (int s = 0; s < splits; ++s) sum += from[s * size + e];
                if (j.less) {
                    float pk = 0.0f;
                    for (int s = 0; s < splits; ++s) pk += less[s * size + e];
                    sum = __builtin_fmaf(pk, r, sum);
                }
                to[e] = (T)settled<T>(sum);
            }
        }
    }
}

bool takes_8_bytes(const rkb_heads &h, int64_t dim)
{
    return dim % 4 == 0 && (uintptr_t)h.p % 8 == 0 && h.batch % 4 == 0 && h.row % 4 == 0 && h.head % 4 == 0;
}

struct bwd_memory {
    size_t stats, seen, norms[2], dq, rows, dkv, table;
    bwd_memory(const attn_bwd_plan &plan, const rkb_attn &a)
    {
        auto up = [](size_t n) { return (size_t)round_up((int64_t)n, 256); };
        stats = up((size_t)a.batch * a.heads * plan.stats_rows * 4);
        seen = up(stats / 32);
        norms[0] = a.dtype == RKB_F16 ? up((size_t)a.batch * a.heads * (plan.stats_rows / NORM_ROWS) * 4) : 0;
        norms[1] = a.dtype == RKB_F16 ? up((size_t)a.batch * a.kv_heads * ((a.k_rows + NORM_ROWS - 1) / NORM_ROWS) * 4) : 0;
        dq = plan.q_splits > 1 ? up((size_t)plan.q_splits * a.batch * a.q_rows * a.heads * a.dim * 4) : 0;
        dkv = plan.k_splits > 1 ? up((size_t)plan.k_splits * a.batch * a.k_rows * a.kv_heads * a.dim * 4) : 0;
        rows = plan.q_splits > 1 ? plan.q_splits * stats : 0;
        table = a.table ? up((size_t)plan.k_blocks * plan.k_splits * (a.heads / a.kv_heads) * a.buckets * 4) : 0;
    }
    size_t all() const { return 2 * stats + seen + norms[0] + norms[1] + 2 * dq + rows + 2 * dkv + table; }
};

}  // namespace

size_t attn_bwd_bytes(const attn_bwd_plan &plan, const rkb_attn &a) { return bwd_memory(plan, a).all(); }

int run_attn_bwd(const attn_in &p, const rkb_attn &a, const attn_bwd_plan &plan, const attn_grads &gr, char *ws, hipStream_t st)
{
    const bwd_memory mem(plan, a);
    bwd_in g{at_of(gr.d_o), at_of(gr.o), gr.o32, gr.lse};
    g.stats_rows = plan.stats_rows;
    auto take = [&](size_t n) {
        char *const at = ws;
        ws += n;
        return n ? at : nullptr;
    };
    g.delta = (float *)take(mem.stats);
    g.lse2 = (float *)take(mem.stats);
    g.seen = (uint32_t *)take(mem.seen);
    g.do_norms = (uint32_t *)take(mem.norms[0]);
    g.v_norms = (uint32_t *)take(mem.norms[1]);
    g.dq = at_of(gr.dq);
    g.dk = at_of(gr.dk);
    g.dv = at_of(gr.dv);
    g.dq_part = (float *)take(mem.dq);
    g.pk_part = (float *)take(mem.dq);
    g.row_part = (float *)take(mem.rows);
    g.dk_part = (float *)take(mem.dkv);
    g.dv_part = (float *)take(mem.dkv);
    g.table_part = gr.dtable ? (float *)take(mem.table) : nullptr;
    g.wide = takes_8_bytes(gr.dq, a.dim) | (takes_8_bytes(gr.dk, a.dim) && takes_8_bytes(gr.dv, a.dim)) << 1;
    return with_attn_type(a.dtype, [&](auto *tp) {
        using T = std::remove_pointer_t<decltype(tp)>;
        int rc = RKB_OK;
        const int64_t rows = a.batch * a.heads, keys = a.batch * a.kv_heads;
        const int64_t chunks = rows * (plan.stats_rows / NORM_ROWS) + keys * ((a.k_rows + NORM_ROWS - 1) / NORM_ROWS);
        if (std::is_same_v<T, f16> && chunks > 0) rc = launch(k_attn_norms<T>, dim3((uint32_t)chunks), dim3(256), st, p, g);
        if (rc != RKB_OK) return rc;
        return with_width(a.dim, [&](auto dp) {
            constexpr int DP = dp();
            const dim3 q_grid((uint32_t)(plan.q_blocks * plan.q_splits * (DP == 256 ? 2 : 1))), k_grid((uint32_t)(plan.k_blocks * plan.k_splits * (DP == 256 ? 2 : 1)));
            int rc = RKB_OK;
            auto join = [&](const grad_join &x, const grad_join &y, int splits, int jobs, int wide) {
                const int64_t blocks = std::min<int64_t>((x.rows * ((a.dim + 3) / 4) + 255) / 256, 1 << 16);
                return launch(k_attn_grads<T>, dim3((uint32_t)blocks, jobs), dim3(256), st, x, y, (int)a.dim, splits, wide);
            };
            if (plan.q_blocks) rc = launch(k_attn_dq<T, DP>, q_grid, dim3(256), st, p, g, plan.q_splits);
            if (rc == RKB_OK && g.row_part && plan.q_blocks && !gr.dq.p)
                rc = launch(k_attn_delta_join, dim3((uint32_t)std::min<int64_t>((rows * plan.stats_rows + 255) / 256, 1 << 16)), dim3(256), st, p, g,
                            plan.q_splits);
            if (rc == RKB_OK && plan.q_splits > 1 && gr.dq.p) {
                const grad_join j{g.dq_part, g.dq, a.batch * a.q_rows * a.heads, (int)a.q_rows, (int)a.heads,
                                  g.pk_part, g.row_part, g.delta, g.stats_rows, rows * g.stats_rows};
                rc = join(j, j, plan.q_splits, 1, g.wide & 1);
            }
            if (rc == RKB_OK && plan.k_blocks && (gr.dk.p || gr.dtable)) {
                if (!p.bias.table)
                    rc = launch(k_attn_dkv<T, DP, 0>, k_grid, dim3(256), st, p, g, plan.k_splits);
                else if (p.bias.far <= 128)
                    rc = launch(k_attn_dkv<T, DP, 128>, k_grid, dim3(256), st, p, g, plan.k_splits);
                else
                    rc = launch(k_attn_dkv<T, DP, MAX_FAR>, k_grid, dim3(256), st, p, g, plan.k_splits);
            }
            if (rc == RKB_OK && gr.dtable)
                rc = launch(k_attn_dtable<T>, dim3((uint32_t)(a.heads * a.buckets)), dim3(WAVE), st, p, (const float *)g.table_part,
                            a.batch * ((a.k_rows + ROWS - 1) / ROWS) * plan.k_splits, gr.dtable);
            if (rc == RKB_OK && plan.k_splits > 1 && gr.dk.p) {
                const int64_t n = a.batch * a.k_rows * a.kv_heads;
                rc = join({g.dk_part, g.dk, n, (int)a.k_rows, (int)a.kv_heads}, {g.dv_part, g.dv, n, (int)a.k_rows, (int)a.kv_heads}, plan.k_splits, 2, g.wide >> 1);
            }
            return rc;
        });
    });
}

}  // namespace rkb
