// Attention forward (rk_block.h): softmax(scale q k^T + bias) v in one pass over the keys, with the
// running maximum and sum of each row.
#include <algorithm>
#include <climits>

#include "rkb_attn.h"
#include "rkb_attn_args.h"

namespace rkb {
namespace {

constexpr int ROWS = 128, TILE = 64, WAVES = 4;  // queries of a workgroup, keys of a tile
// How far a row's maximum may pass what its sums are relative to before they are scaled down (a power of two).
constexpr float SLACK = 8.0f;
// Probabilities are kept times 2^this: they enter a product rounded to T, and f16 loses bits below 2^-14.
template <class T>
constexpr float LIFT = std::is_same_v<T, f16> ? 7.0f : 0.0f;

// Where a kernel's results go: finished rows, or a split's part.
struct attn_out {
    heads_at o;        // 16 bits, may be NULL
    float *o32;        // [B, Q, H, D], may be NULL
    float *lse;        // [B, H, Q], may be NULL
    float *part, *part_ml;  // [splits, B H Q, D] and [splits, B H Q, 2], where there are several
    int wide;          // o's rows take 8-byte stores
};

// A row's softmax so far: its sums are relative to 2^(base - LIFT).
struct running {
    float m = NEG_INF, l = 0.0f;
    __device__ float base() const { return m == NEG_INF ? 0.0f : m; }
};

// Scores of N 32-key pieces, in steps of log2 (times c where raw), become probabilities; acc and the sum follow the maximum.
template <class T, int N, int A>
__device__ inline void soften(f32x16 (&s)[N], float c, running &run, f32x16 (&acc)[A])
{
    float top = s[0][0];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][r]);
    top = half_max(top) * c;
    if (__any(top > run.m + SLACK || (run.m == NEG_INF && top > NEG_INF))) {
        const float m = fmaxf(run.m, top), f = __builtin_amdgcn_exp2f(run.m - (m == NEG_INF ? 0.0f : m));
        run.m = m;
        run.l *= f;
#pragma unroll
        for (int a = 0; a < A; ++a) acc[a] *= f;
    }
    const float off = LIFT<T> - run.base();
    float sum[4] = {};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[i][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][r], c, off));
            sum[r % 4] += s[i][r];
        }
    run.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// Stores a lane's part of a row's 32 columns from 32 d on: groups of 4.
template <class T, int A>
__device__ inline void store_row(const attn_in &p, const attn_out &out, int b, int i, int h, const f32x16 (&acc)[A], float times, int lane)
{
    T *to = out.o.p ? out.o.at<T>(b, i, h) : nullptr;
    float *to32 = out.o32 ? out.o32 + (((int64_t)b * p.Q + i) * p.H + h) * p.D : nullptr;
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = a * 32 + g * 8 + half_row(lane);
            vec<T, 4> v;
            f32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = acc[a][g * 4 + e] * times;
                if (times == 0.0f) w[e] = 0.0f;
                v[e] = (T)settled<T>(w[e]);
            }
            if (col + 4 <= p.D && out.wide) {
                if (to) *(vec<T, 4> *)(to + col) = v;
                if (to32) *(f32x4 *)(to32 + col) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < p.D) {
                        if (to) to[col + e] = v[e];
                        if (to32) to32[col + e] = w[e];
                    }
            }
        }
}

// Finishes a row (there: it exists), or leaves a split's part of it.
template <class T, int A>
__device__ inline void finish(const attn_in &p, const attn_out &out, int split, int b, int i, int h, bool there, const running &run, float l,
                              const f32x16 (&acc)[A], int lane)
{
    if (!there) return;
    const int64_t row = ((int64_t)b * p.H + h) * p.Q + i;
    if (!out.part) {
        store_row<T, A>(p, out, b, i, h, acc, l == 0.0f ? 0.0f : 1.0f / l, lane);
        if (out.lse && lane < 32) out.lse[row] = l == 0.0f ? NEG_INF : (run.base() - LIFT<T> + __builtin_amdgcn_logf(l)) * LN2;
        return;
    }
    const int64_t at = (int64_t)split * p.B * p.H * p.Q + row;
    if (lane < 32) {
        out.part_ml[2 * at] = run.base() - LIFT<T>;
        out.part_ml[2 * at + 1] = l;
    }
    float *to = out.part + at * p.D;
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = a * 32 + g * 8 + half_row(lane);
            if (col + 4 <= p.D && p.D % 4 == 0) {
                f32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = acc[a][g * 4 + e];
                *(f32x4 *)(to + col) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < p.D) to[col + e] = acc[a][g * 4 + e];
            }
        }
}

// The end of the keys that a workgroup's queries see.
__device__ inline int keys_end(const attn_in &p, int len, int last_pos)
{
    return p.causal ? min(len, max(last_pos, -1) + 1) : len;
}

// ------------------------------------------------------------------ many rows
//
// A wave has 32 queries of one head, a workgroup 128, and passes over the keys in tiles of 64 that its four waves
// share, two tiles of keys and values in LDS in turn.  While the matrix units form the scores of the next 32 keys and add
// these ones' values, the vector units make probabilities of these keys' scores.
//
// 4 x 2048 queries of 32 heads of 128 over 4096 keys of 8 (some padded): 360 to 390 us, 0.9 to 1.0 PFLOP/s (a large product by the library 1.4 to 1.6).  Between two
// barriers each wave has 64 matrix instructions, which take 16 ns each by themselves; exponentials and conversions beside them keep the issue
// busy 87 % of the time, the matrix units 53 %.  64 columns: 0.79 PFLOP/s, half the products per probability, the issue busy 90 %.
template <class T, int DP, bool CACHE>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_attn(attn_in p, attn_out out, int splits)
{
    using L = lay<DP>;
    constexpr int BYTES = TILE * DP * 2, C = DP / 16, A = DP / 32;
    __shared__ __align__(16) char k0[BYTES], k1[BYTES], v0[BYTES], v1[BYTES];
    __shared__ float by_distance[2 * (MAX_FAR + PAD) + 1];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int q_tiles = (p.Q + ROWS - 1) / ROWS;
    int w = unit_order(blockIdx.x, p.B * p.K, p.G * splits * q_tiles);
    const int qt = q_tiles - 1 - w % q_tiles;  // the longest first, where queries see the keys before them
    w /= q_tiles;
    const int split = w % splits, bh = w / splits, b = bh / p.H, h = bh - b * p.H, kv = h / p.G;
    const int len = len_of(p, b), first = first_of(p, b);
    const int q0 = qt * ROWS, q1 = min(q0 + ROWS, p.Q), row0 = q0 + wave * 32;
    const int tiles = (keys_end(p, len, first + q1 - 1) + TILE - 1) / TILE, each = (tiles + splits - 1) / splits;
    const int t0 = split * each, t1 = min(tiles, t0 + each);
    const int pos_lo = first + row0, pos_hi = pos_lo + 31;

    const int i = row0 + lane % 32;
    frag<T> q[C];
    load_stationary<T, DP>(q, p.q.at<T>(b, min(i, p.Q - 1), h), lane, p.D, i < p.Q);
    const int far = p.bias.far;
    float far_behind = 0.0f, far_ahead = 0.0f;
    if (p.bias.table) {
        fill_bias<T>(by_distance, p, h, threadIdx.x, 256);
        __syncthreads();
        far_behind = by_distance[0];
        far_ahead = by_distance[2 * (far + PAD)];
    }

    tile_copy<DP, TILE, WAVES> kc, vc;
    tile_codes<T, DP, TILE, 256> kq, vq;
    const T *kp = nullptr, *vp = nullptr;
    const int8_t *ck = nullptr, *cv = nullptr;
    const uint8_t *ek = nullptr, *ev = nullptr;
    if constexpr (CACHE) {
        const int64_t head = (int64_t)b * p.K + kv, all = (int64_t)p.B * p.K;
        ck = p.codes + head * p.room * p.ld;
        cv = p.codes + (all + head) * p.room * p.ld;
        ek = p.exps + head * (p.room / RKB_GROUP);
        ev = p.exps + (all + head) * (p.room / RKB_GROUP);
    } else {
        kp = p.k.at<T>(b, 0, kv);
        vp = p.v.at<T>(b, 0, kv);
        kc.set(wave, lane, p.k.t, p.D);
        vc.set(wave, lane, p.v.t, p.D);
    }
    // Keys come to LDS in tiles that start 32 keys after the tiles of values: the 64 from `key` on, which is no key before the first.
    auto fetch_k = [&](int key, lds_byte *to) __attribute__((always_inline)) {
        const int n = len - key;
        if (n <= 0) return;
        const uint64_t live = n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1;
        if constexpr (CACHE)
            kq.load(threadIdx.x, ck + (int64_t)key * p.ld, ek + key / RKB_GROUP, p.ld, live, n);
        else
            kc.copy(wave, lane, (const char *)(kp + (int64_t)key * p.k.t), live, n >= 64 && p.D == DP, to);
    };
    auto fetch_v = [&](int t, uint64_t live, lds_byte *to) __attribute__((always_inline)) {
        const int64_t key = (int64_t)t * TILE;
        if constexpr (CACHE)
            vq.load(threadIdx.x, cv + key * p.ld, ev + key / RKB_GROUP, p.ld, live, len - (int)key);
        else
            vc.copy(wave, lane, (const char *)(vp + key * p.v.t), live, live == ~(uint64_t)0 && p.D == DP, to);
    };

    f32x16 acc[A] = {}, sa, sb;
    running run;
    float top = NEG_INF, by = p.c, add = 0.0f;  // of the piece that waits: x by + add are its scores in steps of log2, top the largest x
    const int k_place = L::rows_place(lane), v_place[2] = {L::cols_place(lane, 0), L::cols_place(lane, 1)};
    // A piece that not all queries see alike: bias by distance, dead keys.  Then x are steps of log2 themselves.
    // Before simple_end all queries see all keys of a piece, from as far as the bias tells apart.
    const float add_simple = p.bias.table ? far_behind : 0.0f;
    const int simple_end = p.mask ? INT_MIN : min(min(len, p.causal ? pos_lo + 1 : INT_MAX), p.bias.table ? pos_lo - far + 1 : INT_MAX) - 31;
    auto adjust = [&](int key0, uint32_t live, f32x16 &s) __attribute__((always_inline)) {
        if (key0 < simple_end) {
            by = p.c;
            add = add_simple;
            return;
        }
        const bool behind = key0 + 31 - pos_lo <= -far, ahead = key0 - pos_hi >= far, near = p.bias.table && !behind && !ahead;
        by = p.c;
        add = !p.bias.table || near ? 0.0f : behind ? far_behind : far_ahead;
        if (!near && live == ~0u && !(p.causal && key0 + 31 > pos_lo)) return;
        int me = lane;
        asm volatile("" : "+v"(me));  // nothing of this is worked out ahead of the loop: it would hold registers in every turn
        const int pos = pos_lo + me % 32;
        if (near)
            add_bias(s, p.c, by_distance, far, key0, pos, pos_lo, pos_hi, me);
        else
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], p.c, add);
        kill_dead(s, live, p.causal ? pos - key0 : INT_MAX, me, NEG_INF);
        top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        by = 1.0f;
        add = 0.0f;
    };
    // One turn: softens the piece `now`, adds its values (rows vn.. of vt), and forms the next piece's scores (rows kn.. of kt).
    // What the vector units do is dealt out between the matrix instructions, in this order and no other.
    auto turn = [&](lds_byte *kt, int kn, lds_byte *vt, int vn, f32x16 &now, f32x16 &then) __attribute__((always_inline)) {
        constexpr int AHEAD = 4, EARLY = C / 4, N = C - EARLY, SKEW = 2;
        auto pin = [] { __builtin_amdgcn_sched_barrier(0); };
        frag<T> kf[AHEAD + 1], vf[AHEAD + 1], f[2];
#pragma unroll
        for (int c = 0; c < AHEAD; ++c) kf[c] = L::template rows<T>(kt, k_place, c, kn);
        auto values = [&](int n) __attribute__((always_inline)) {  // the n-th fragment of both halves
            return L::template cols<T>(vt, v_place, n % A, vn + n / A * 16);
        };
        auto read_ahead = [&](int c) __attribute__((always_inline)) {
            if (c + AHEAD < C)
                kf[(c + AHEAD) % (AHEAD + 1)] = L::template rows<T>(kt, k_place, c + AHEAD, kn);
            else
                vf[c + AHEAD - C] = values(c + AHEAD - C);
        };
        // the first products run while the maximum is looked at
#pragma unroll
        for (int c = 0; c < EARLY; ++c) {
            read_ahead(c);
            then = mma32(kf[c], q[c], c == 0 ? f32x16{} : then);
        }
        pin();
        top = __builtin_fmaf(half_max(top), by, add);
        if (__any(top > run.m + SLACK)) {
            const float m = fmaxf(run.m, top), x = __builtin_amdgcn_exp2f(run.m - (m == NEG_INF ? 0.0f : m));
            run.m = m;
            run.l *= x;
#pragma unroll
            for (int a = 0; a < A; ++a) acc[a] *= x;
        }
        const float off = LIFT<T> + add - run.base();
        // The 16 probabilities, in three steps that run SKEW of them apart, so that no instruction waits for the one before it.
        float x[16], sum[2] = {};
        auto scale = [&](int e) __attribute__((always_inline)) { x[e] = __builtin_fmaf(now[e], by, off); };
        auto power = [&](int e) __attribute__((always_inline)) { x[e] = __builtin_amdgcn_exp2f(x[e]); };
        auto soften = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
            for (int e = from; e < to; ++e) {
                if (e + 2 * SKEW < 16) scale(e + 2 * SKEW);
                if (e + SKEW < 16) power(e + SKEW);
                sum[e % 2] += x[e];
                asm volatile("" : "+v"(sum[e % 2]));  // here, and not behind all products
                f[e / 8][e % 8] = (T)x[e];
            }
        };
#pragma unroll
        for (int e = 0; e < 2 * SKEW; ++e) scale(e);
#pragma unroll
        for (int e = 0; e < SKEW; ++e) power(e);
        pin();
#pragma unroll
        for (int c = EARLY; c < C; ++c) {
            read_ahead(c);
            then = mma32(kf[c % (AHEAD + 1)], q[c], then);
            soften((c - EARLY) * 8 / N, (c - EARLY + 1) * 8 / N);
            pin();
        }
        float big[2];  // largest scores of the next piece
        auto largest = [&](int from, int to) __attribute__((always_inline)) {
            if (from == 0) big[0] = then[0], big[1] = then[1];
#pragma unroll
            for (int r = max(from, 2); r < to; ++r) {
                big[r / 2 % 2] = fmaxf(big[r / 2 % 2], then[r]);
                if (r % 4 == 3) asm volatile("" : "+v"(big[r / 2 % 2]));
            }
        };
#pragma unroll
        for (int n = 0; n < 2 * A; ++n) {
            if (n + AHEAD < 2 * A) vf[(n + AHEAD) % (AHEAD + 1)] = values(n + AHEAD);
            acc[n % A] = mma32(vf[n % (AHEAD + 1)], f[n / A], acc[n % A]);
            if (n < A)
                soften(8 + n * 8 / A, 8 + (n + 1) * 8 / A);
            else
                largest((n - A) * 16 / A, (n - A + 1) * 16 / A);
            pin();
        }
        run.l += sum[0] + sum[1];
        top = fmaxf(big[0], big[1]);
        asm volatile("" : "+v"(run.l), "+v"(top));
    };

    if (t0 < t1) {
        uint8_t byte = mask_byte(p, b, t0 * TILE + lane, len);
        uint64_t live = keys_alive(p, t0 * TILE, len, byte), next = 0;
        byte = mask_byte(p, b, (t0 + 1) * TILE + lane, len);
        fetch_k(t0 * TILE, (lds_byte *)k1);  // whose first half is the first piece
        if constexpr (CACHE) kq.put(threadIdx.x, (lds_byte *)k1);
        fetch_k(t0 * TILE + 32, (lds_byte *)k0);
        fetch_v(t0, live, (lds_byte *)v0);
        if constexpr (CACHE) {
            if (t0 * TILE + 32 < len) kq.put(threadIdx.x, (lds_byte *)k0);
            vq.put(threadIdx.x, (lds_byte *)v0);
        }
        wait_all();
        sa = f32x16{};
#pragma unroll
        for (int c = 0; c < C; ++c) sa = mma32(L::template rows<T>((lds_byte *)k1, k_place, c, 0), q[c], sa);
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, sa[r]);
        adjust(t0 * TILE, (uint32_t)live, sa);
        // One tile of values, kh: the keys of its second piece and the next tile's first.  The next tiles go where the last ones
        // were, which all waves have read when they pass the barrier.
        auto step = [&](int t, char *kh, char *vh, char *kn, char *vn) __attribute__((always_inline)) {
            wait_all();
            const bool more = t + 1 < t1;
            next = 0;
            if (more) {
                next = keys_alive(p, (t + 1) * TILE, len, byte);
                byte = mask_byte(p, b, (t + 2) * TILE + lane, len);
                fetch_k((t + 1) * TILE + 32, (lds_byte *)kn);
                fetch_v(t + 1, next, (lds_byte *)vn);
            }
            turn((lds_byte *)kh, 0, (lds_byte *)vh, 0, sa, sb);
            adjust(t * TILE + 32, (uint32_t)(live >> 32), sb);
            turn((lds_byte *)kh, 32, (lds_byte *)vh, 32, sb, sa);  // behind the last tile: scores of whatever lies there, not used
            adjust((t + 1) * TILE, (uint32_t)next, sa);
            if constexpr (CACHE)
                if (more) {
                    if ((t + 1) * TILE + 32 < len) kq.put(threadIdx.x, (lds_byte *)kn);
                    vq.put(threadIdx.x, (lds_byte *)vn);
                }
            live = next;
        };
        for (int t = t0; t < t1; t += 2) {
            step(t, k0, v0, k1, v1);
            if (t + 1 < t1) step(t + 1, k1, v1, k0, v0);
        }
    }
    finish<T, A>(p, out, split, b, i, h, i < p.Q, run, half_sum(run.l), acc, lane);
}

// ------------------------------------------------------------------ few rows
//
// Up to 32 or 64 queries (rkb_attn_cut.h).  A workgroup has up to 32 rows of one key head: queries and the heads that share it, queries first.  Each wave takes keys of its
// own, in tiles of 32 that no other wave waits for, and the waves' sums are joined at the end.  A cache's keys go from
// memory to the matrix units' registers (a lane has 16 neighbouring columns of a key, and all keys' and queries' columns are taken in that
// order), its values through LDS, to be read by columns; two tiles of both wait in registers until they are due.
//
// Bound by memory: 64 sequences of up to 1500 keys of 16 heads of 64 take 55 to 57 us (5.2 to 5.4 TB/s), 16 caches of up to 32768 tokens, 64 heads on 8
// of 128, 159 to 162 us (4.9 TB/s; through LDS both ways and one tile ahead it was 457).  One token over 1024 cached ones takes 13 to 15 us, all latency.
template <int DP, bool CACHE, bool BIAS>
constexpr int FEW_BLOCKS = (DP == 256 ? 2 : 4) * 32 * DP * 2 * (CACHE ? 2 : 4) + (BIAS ? 32 * (MAX_BUCKETS + 1) * 4 + 2 * MAX_FAR + 1 : 0) + 2048 <=
                                   80 * 1024 && DP < 256 ? 2 : 1;  // workgroups of a compute unit, by LDS

template <class T, int DP, bool CACHE, bool BIAS>
__global__ __launch_bounds__((DP == 256 ? 2 : 4) * WAVE, (FEW_BLOCKS<DP, CACHE, BIAS>)) void k_attn_few(attn_in p, attn_out out, int splits)
{
    using L = lay<DP>;
    constexpr int W = DP == 256 ? 2 : 4, KEYS = 32, BYTES = KEYS * DP * 2, C = DP / 16, A = DP / 32;
    // what a wave copies ahead of its work; a cache's tiles wait in registers instead.  (k0 takes part in the join of the waves.)
    constexpr int SPARE = CACHE ? 16 : W * BYTES;
    __shared__ __align__(16) char k0[W * BYTES], v0[W * BYTES], k1[SPARE], v1[SPARE];
    __shared__ float table[BIAS ? 32 * (MAX_BUCKETS + 1) : 1];
    __shared__ uint8_t bucket[BIAS ? 2 * MAX_FAR + 1 : 1];
    __shared__ float ml[W][2][32];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int rows = p.Q * p.G, row_tiles = (rows + 31) / 32;
    int w = unit_order(blockIdx.x, p.B * p.K, splits * row_tiles);
    const int rt = w % row_tiles;
    w /= row_tiles;
    const int split = w % splits, bk = w / splits, b = bk / p.K, kv = bk - b * p.K;
    const int len = len_of(p, b), first = first_of(p, b);
    const int r0 = rt * 32, r = r0 + lane % 32;
    const bool there = r < rows;
    const int i = min(r, rows - 1) / p.G, h = kv * p.G + min(r, rows - 1) % p.G;
    const int pos = first + i, pos_lo = first + r0 / p.G, pos_hi = first + min(r0 + 31, rows - 1) / p.G;
    const int tiles = (keys_end(p, len, pos_hi) + KEYS - 1) / KEYS, parts = splits * W, each = (tiles + parts - 1) / parts;
    const int t0 = (split * W + wave) * each, t1 = min(tiles, t0 + each);

    frag<T> q[C];
    const T *const row = p.q.at<T>(b, i, h);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = c / 2 * 32 + lane / 32 * 16 + c % 2 * 8;
        frag<T> z = {};
        if (there && col < p.D) z = *(const frag<T> *)(row + col);
        q[c] = z;
    }
    const int buckets = p.bias.sides * p.bias.count, far = p.bias.far;
    if constexpr (BIAS) {
        for (int n = threadIdx.x; n <= 2 * far; n += W * WAVE) bucket[n] = (uint8_t)bucket_of(p.bias, n - far);
        // A row that does not exist sees no key: its maximum would else move when the others' sums are scaled, and with that their bits.
        for (int n = threadIdx.x; n < 32 * buckets; n += W * WAVE) {
            const int row = r0 + n % 32;
            table[n % 32 * (buckets + 1) + n / 32] = row < rows ? table_value<T>(p, n / 32, kv * p.G + row % p.G) : NEG_INF;
        }
        __syncthreads();
    }
    const float *mine = table + lane % 32 * (buckets + 1);

    tile_copy<DP, KEYS, 1> kc, vc;
    struct waiting {  // a cache's tile: this lane's codes of its key, and the values'
        u32x4 k[C / 2];
        uint8_t exp;
        tile_codes<T, DP, KEYS, WAVE> v;
        uint32_t live;
    } first_tile, second_tile;
    const T *kp = nullptr, *vp = nullptr;
    const int8_t *ck = nullptr, *cv = nullptr;
    const uint8_t *ek = nullptr, *ev = nullptr;
    if constexpr (CACHE) {
        const int64_t head = (int64_t)b * p.K + kv, all = (int64_t)p.B * p.K;
        ck = p.codes + head * p.room * p.ld;
        cv = p.codes + (all + head) * p.room * p.ld;
        ek = p.exps + head * (p.room / RKB_GROUP);
        ev = p.exps + (all + head) * (p.room / RKB_GROUP);
    } else {
        kp = p.k.at<T>(b, 0, kv);
        vp = p.v.at<T>(b, 0, kv);
        kc.set(0, lane, p.k.t, p.D);
        vc.set(0, lane, p.v.t, p.D);
    }
    // A tile on its way: copied to LDS, or a cache's to registers.  Of rows and columns that do not exist the last ones that do are
    // read instead: such scores are replaced, such columns meet zeros of the query.
    auto fetch = [&](int t, uint32_t live, waiting &to, lds_byte *kto, lds_byte *vto) __attribute__((always_inline)) {
        const int64_t key = (int64_t)t * KEYS;
        if constexpr (CACHE) {
            const int rows = len - (int)key, spans = (int)p.ld / 16;
            const int8_t *const from = ck + (key + min(lane % 32, rows - 1)) * p.ld;
#pragma unroll
            for (int c = 0; c < C / 2; ++c) to.k[c] = *(const u32x4 *)(from + min(c * 2 + lane / 32, spans - 1) * 16);
            to.exp = ek[t];
            to.live = live;
            to.v.load(lane, cv + key * p.ld, ev + t, p.ld, live, rows);
        } else {
            const bool all = live == ~0u && p.D == DP;
            kc.copy(0, lane, (const char *)(kp + key * p.k.t), live, all, kto);
            vc.copy(0, lane, (const char *)(vp + key * p.v.t), live, all, vto);
        }
    };

    f32x16 acc[A] = {};
    running run;
    const int k_place = L::at(lane % 32, lane / 32 * 2), v_place[2] = {L::cols_place(lane, 0), L::cols_place(lane, 1)};
    auto score = [&](const waiting &w, lds_byte *kt) __attribute__((always_inline)) {
        f32x16 s = {};
        const float step = !CACHE || w.exp == 0 ? 0.0f : step_of(w.exp);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            frag<T> f;
            if constexpr (CACHE)
                f = code_values<T>(w.k[c / 2][c % 2 * 2], w.k[c / 2][c % 2 * 2 + 1], step);
            else
                f = *(__attribute__((address_space(3))) frag<T> *)(kt + (k_place ^ (c / 2 * 64 + c % 2 * 16)));
            s = mma32(f, q[c], s);
        }
        return s;
    };
    auto compute = [&](int t, uint32_t live, const f32x16 &raw, lds_byte *vt) __attribute__((always_inline)) {
        const int key0 = t * KEYS;
        f32x16 s[1] = {raw};
        float by = p.c;
        if constexpr (BIAS) {
            by = 1.0f;
            if (key0 - pos_hi >= far || key0 + 31 - pos_lo <= -far) {
                const float add = mine[bucket[key0 - pos_hi >= far ? 2 * far : 0]];
#pragma unroll
                for (int n = 0; n < 16; ++n) s[0][n] = __builtin_fmaf(s[0][n], p.c, add);
            } else {
                const int d = key0 + half_row(lane) - pos + far;
#pragma unroll
                for (int n = 0; n < 16; ++n) s[0][n] = __builtin_fmaf(s[0][n], p.c, mine[bucket[min(max(d + n / 4 * 8 + n % 4, 0), 2 * far)]]);
            }
        }
        kill_dead(s[0], live, p.causal ? pos - key0 : INT_MAX, lane, NEG_INF);
        soften<T>(s, by, run, acc);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const frag<T> f = to_frag<T>(s[0], half);
#pragma unroll
            for (int a = 0; a < A; ++a) acc[a] = mma32(L::template cols<T>(vt, v_place, a, half * 16), f, acc[a]);
        }
    };

    auto alive = [&](int t, uint8_t byte) { return (uint32_t)keys_alive(p, t * KEYS, len, byte); };
    auto byte_of = [&](int t) { return mask_byte(p, b, t * KEYS + lane % 32, len); };
    if (t0 < t1) {
        lds_byte *const kh0 = (lds_byte *)k0 + wave * BYTES, *const vh0 = (lds_byte *)v0 + wave * BYTES;
        if constexpr (CACHE) {
            uint8_t byte = byte_of(t0);
            auto ahead = [&](int t, waiting &w) __attribute__((always_inline)) {
                const uint32_t live = alive(t, byte);
                byte = byte_of(min(t + 1, t1 - 1));
                fetch(t, live, w, kh0, vh0);
            };
            // Behind the end the last tile is loaded again: how many loads are on their way is always the same, so that the older ones can be
            // waited for alone.
            auto step = [&](int t, waiting &w) __attribute__((always_inline)) {
                const f32x16 s = score(w, kh0);
                w.v.put(lane, vh0);
                const uint32_t live = w.live;
                asm volatile("" ::: "memory");  // other lanes read what this one wrote
                ahead(min(t + 2, t1 - 1), w);
                compute(t, live, s, vh0);
                asm volatile("" ::: "memory");
            };
            ahead(t0, first_tile);
            ahead(min(t0 + 1, t1 - 1), second_tile);
            for (int t = t0;;) {
                step(t, first_tile);
                if (++t == t1) break;
                step(t, second_tile);
                if (++t == t1) break;
            }
        } else {
            lds_byte *const kh1 = (lds_byte *)k1 + wave * BYTES, *const vh1 = (lds_byte *)v1 + wave * BYTES;
            uint32_t live = alive(t0, byte_of(t0));
            uint8_t byte = byte_of(t0 + 1);
            fetch(t0, live, first_tile, kh0, vh0);
            auto step = [&](int t, lds_byte *kh, lds_byte *vh, lds_byte *kn, lds_byte *vn) __attribute__((always_inline)) {
                uint32_t next = 0;
                if (t + 1 < t1) {
                    next = alive(t + 1, byte);
                    byte = byte_of(t + 2);
                    fetch(t + 1, next, first_tile, kn, vn);
                    // copies land in order: all but the next tile's have
                    __builtin_amdgcn_s_waitcnt(wait_copies(2 * tile_copy<DP, KEYS, 1>::MINE));
                } else {
                    __builtin_amdgcn_s_waitcnt(wait_copies(0));
                }
                asm volatile("" ::: "memory");
                compute(t, live, score(first_tile, kh), vh);
                asm volatile("" ::: "memory");
                live = next;
            };
            for (int t = t0; t < t1; t += 2) {
                step(t, kh0, vh0, kh1, vh1);
                if (t + 1 < t1) step(t + 1, kh1, vh1, kh0, vh0);
            }
        }
    }

    // Join the waves: each brings its sums to the common maximum; then wave 0 adds them, in order.  A wave's sums are BYTES * 2 bytes, as
    // its tiles of keys and values were.
    float l = half_sum(run.l);
    if (lane < 32) {
        ml[wave][0][lane] = l == 0.0f ? NEG_INF : run.base();
        ml[wave][1][lane] = l;
    }
    wait_all();
    float top = NEG_INF;
#pragma unroll
    for (int n = 0; n < W; ++n) top = fmaxf(top, ml[n][0][lane % 32]);
    const float base = top == NEG_INF ? 0.0f : top;
    float total = 0.0f;
#pragma unroll
    for (int n = 0; n < W; ++n) {
        const float f = ml[n][0][lane % 32];
        total += f == NEG_INF ? 0.0f : ml[n][1][lane % 32] * __builtin_amdgcn_exp2f(f - base);
    }
    const float scale = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(run.base() - base);
    // one half of the columns in the keys' memory, the other in the values'
    auto slot = [&](int from, int a, int g) {
        char *const at = a < A / 2 ? k0 : v0;
        return (f32x4 *)(at + from * BYTES + (((a % (A / 2)) * 4 + g) * WAVE + lane) * 16);
    };
    if (wave > 0) {
#pragma unroll
        for (int a = 0; a < A; ++a)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = scale == 0.0f ? 0.0f : acc[a][g * 4 + e] * scale;
                *slot(wave, a, g) = x;
            }
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[a][g * 4 + e] = scale == 0.0f ? 0.0f : acc[a][g * 4 + e] * scale;
    for (int n = 1; n < W; ++n)
#pragma unroll
        for (int a = 0; a < A; ++a)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 x = *slot(n, a, g);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[a][g * 4 + e] += x[e];
            }
    run.m = top;
    finish<T, A>(p, out, split, b, i, h, there, run, total, acc, lane);
}

// ------------------------------------------------------------------ splits joined
//
// A lane has four columns of a row; splits are added in order.  A launch's latency (4 to 8 us) is most of it.
template <class T>
__global__ __launch_bounds__(256) void k_attn_join(attn_in p, attn_out out, int splits)
{
    // keys are split for up to 256 workgroups, of up to 128 rows each: all of this fits 32 bits
    const uint32_t quads = (p.D + 3) / 4, rows = (uint32_t)p.B * p.H * p.Q, at = blockIdx.x * 256 + threadIdx.x, row = at / quads;
    const int col = (int)(at - row * quads) * 4;
    if (row >= rows) return;
    using f32x2 = vec<float, 2>;
    const f32x2 *const ml = (const f32x2 *)out.part_ml + row;
    const float *const from = out.part + (int64_t)row * p.D + col;
    const int64_t size = (int64_t)rows * p.D;
    float top = NEG_INF;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const f32x2 x = ml[(int64_t)s * rows];
        top = x[1] != 0.0f ? fmaxf(top, x[0]) : top;
    }
    const float base = top == NEG_INF ? 0.0f : top;
    float l = 0.0f;
    f32x4 v = {};
    const bool whole = p.D % 4 == 0;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const f32x2 x = ml[(int64_t)s * rows];
        f32x4 part = {};
        if (whole) {
            part = *(const f32x4 *)(from + s * size);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < p.D) part[e] = from[s * size + e];
        }
        const bool any = x[1] != 0.0f;
        const float f = any ? __builtin_amdgcn_exp2f(x[0] - base) : 0.0f;
        l += x[1] * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = any ? __builtin_fmaf(part[e], f, v[e]) : v[e];
    }
    const float times = l == 0.0f ? 0.0f : 1.0f / l;
    const uint32_t bh = row / p.Q, i = row - bh * p.Q, b = bh / p.H, h = bh - b * p.H;
    T *to = out.o.p ? out.o.at<T>(b, i, h) : nullptr;
    float *to32 = out.o32 ? out.o32 + (((int64_t)b * p.Q + i) * p.H + h) * p.D : nullptr;
    v *= times;
    if (out.wide) {
        vec<T, 4> x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (T)settled<T>(v[e]);
        if (to) *(vec<T, 4> *)(to + col) = x;
        if (to32) *(f32x4 *)(to32 + col) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < p.D) {
                if (to) to[col + e] = (T)settled<T>(v[e]);
                if (to32) to32[col + e] = v[e];
            }
    }
    if (out.lse && col == 0) out.lse[row] = l == 0.0f ? NEG_INF : (base + __builtin_amdgcn_logf(l)) * LN2;
}

}  // namespace

// ------------------------------------------------------------------ launches

size_t attn_fwd_parts_bytes(const attn_plan &plan, const rkb_attn &a)
{
    if (plan.splits == 1) return 0;
    const size_t rows = (size_t)a.batch * a.heads * a.q_rows * plan.splits;
    return round_up(rows * a.dim * 4, 256) + round_up(rows * 8, 256);
}

int run_attn_fwd(const attn_in &p, const rkb_attn &a, const attn_plan &plan, const attn_results &res, char *parts, hipStream_t st)
{
    attn_out out{{(char *)res.o.p, res.o.batch, res.o.row, res.o.head}, res.o32, res.lse, nullptr, nullptr, 0};
    out.wide = a.dim % 4 == 0 && (uintptr_t)res.o.p % 8 == 0 && res.o.batch % 4 == 0 && res.o.row % 4 == 0 && res.o.head % 4 == 0;
    if (plan.splits > 1) {
        const size_t rows = (size_t)a.batch * a.heads * a.q_rows * plan.splits;
        out.part = (float *)parts;
        out.part_ml = (float *)(parts + round_up(rows * a.dim * 4, 256));
    }
    const dim3 grid((uint32_t)(plan.blocks * plan.splits));
    const int rc = with_attn_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return with_width(a.dim, [&](auto dp) {
            constexpr int DP = dp();
            if (!plan.few)
                return p.codes ? launch(k_attn<T, DP, true>, grid, dim3(256), st, p, out, plan.splits)
                               : launch(k_attn<T, DP, false>, grid, dim3(256), st, p, out, plan.splits);
            const dim3 block((DP == 256 ? 2 : 4) * WAVE);
            if (p.bias.table)
                return p.codes ? launch(k_attn_few<T, DP, true, true>, grid, block, st, p, out, plan.splits)
                               : launch(k_attn_few<T, DP, false, true>, grid, block, st, p, out, plan.splits);
            return p.codes ? launch(k_attn_few<T, DP, true, false>, grid, block, st, p, out, plan.splits)
                           : launch(k_attn_few<T, DP, false, false>, grid, block, st, p, out, plan.splits);
        });
    });
    if (rc != RKB_OK || plan.splits == 1) return rc;
    const int64_t lanes = (int64_t)a.batch * a.heads * a.q_rows * ((a.dim + 3) / 4);
    return with_attn_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return launch(k_attn_join<T>, dim3((uint32_t)((lanes + 255) / 256)), dim3(256), st, p, out, plan.splits);
    });
}

}  // namespace rkb
