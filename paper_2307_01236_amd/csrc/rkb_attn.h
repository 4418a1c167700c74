// What the attention kernels share (rkb_attn.hip, rkb_attn_bwd.hip): the layout of tiles in LDS, how they are
// filled, the matrix instructions' fragments, which keys live, and the bias by relative position.
//
// Every kernel has a stationary side, whose 32 rows a wave holds as columns of 32 x 32 x 16 matrix instructions, and
// a streamed side that passes through LDS in tiles of rows.  A product "streamed x stationary" (scores, dp) leaves a
// lane with one stationary row and 16 of 32 streamed ones, so that softmax sums are sums within a
// lane and one exchange; its registers are, converted, the right operand of the next product (o, dq, dk, dv: sums over streamed
// rows), whose left operand is the tile read through LDS's transposing read.  That operand's k order is the
// one the registers have: lanes 0 to 31 hold the rows 0-3 and 8-11 of each 16, lanes 32 to 63 the rows 4-7 and 12-15.
#pragma once
#include "rkb_common.h"
#include "rkb_tile.h"

namespace rkb {

using f32x16 = vec<float, 16>;

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
constexpr float NEG_INF = -__builtin_inff();
constexpr int MAX_BUCKETS = RKB_MAX_BUCKETS, MAX_FAR = RKB_MAX_DISTANCE;

__device__ inline f32x16 mma32(frag<bf16> a, frag<bf16> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mma32(frag<f16> a, frag<f16> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Row (of 32) that a lane's register r of a product holds: 8 (r / 4) + r % 4 + this.
__device__ inline int half_row(int lane) { return lane / 32 * 4; }

// Sum, or maximum, of the two halves' values of one column.
__device__ inline float half_sum(float v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ inline float half_max(float v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// ------------------------------------------------------------------ arguments

struct heads_at {  // a [batch, rows, heads, width] tensor; strides in elements
    char *p;
    int64_t b, t, h;
    template <class T>
    __device__ T *at(int64_t bi, int64_t ti, int64_t hi) const
    {
        return (T *)p + bi * b + ti * t + hi * h;
    }
};

struct bias_table {
    const void *table;  // [buckets, heads], NULL: no bias
    int f32;            // 32-bit, else of the operands' type
    int sides, count;   // buckets of a side
    int far;            // the least distance of a side's last bucket
    int border[MAX_BUCKETS];  // the least distance of buckets 1 .., then INT_MAX
};

struct attn_in {
    int B, Q, T, H, K, G, D;
    int causal;
    float scale, c;  // c = scale log2(e)
    int64_t first;
    const int32_t *firsts, *lens;
    const uint8_t *mask;
    int64_t mask_stride;
    heads_at q, k, v;
    const int8_t *codes;  // [2, B, K, room, ld], or NULL
    const uint8_t *exps;  // [2, B, K, room / 32]
    int64_t room, ld;
    bias_table bias;
};

constexpr int FAR_POSITION = 1 << 30;

__device__ inline int len_of(const attn_in &p, int b) { return p.lens ? min(max(p.lens[b], 0), p.T) : p.T; }

// The position of a sequence's first query: past 2^30 either way, all keys are as far.
__device__ inline int first_of(const attn_in &p, int b)
{
    const int64_t at = p.first + (p.firsts ? p.firsts[b] : 0);
    return (int)min(max(at, (int64_t)-FAR_POSITION), (int64_t)FAR_POSITION);
}

// Which of units x each workgroups a block is.  Workgroups go to the 8 dies in turn.  A unit (a key head of a sequence) is one die's, so that its
// L2 holds what they share, and units are dealt out in turn, so that sequences of different lengths are, too; those left over
// when every die has as many are cut into runs.
__device__ inline int unit_order(int block, int units, int each)
{
    const int dealt = units / 8 * 8 * each;
    if (block < dealt) {
        const int i = block / 8, round = i / each;
        return (round * 8 + block % 8) * each + (i - round * each);
    }
    const int left = units * each - dealt, share = left / 8, rest = left % 8, die = block % 8;
    return dealt + die * share + min(die, rest) + (block - dealt) / 8;
}

// ------------------------------------------------------------------ tiles in LDS
//
// A tile has rows of DP (64, 128 or 256) 16-bit columns without gaps.  The 16-byte chunks of row r are permuted
// by fold(r) (xor): the 16 rows that a fragment's lanes read at one chunk fall into different banks, and so do
// the 64-byte pieces of the 4 rows that a transposing read takes together.

template <int DP>
struct lay {
    static_assert(DP == 64 || DP == 128 || DP == 256);
    static constexpr int PITCH = DP * 2, CHUNKS = DP / 8;
    static __device__ int fold(int r)
    {
        return DP == 64 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
    }
    static __device__ int at(int r, int chunk) { return r * PITCH + (chunk ^ fold(r)) * 16; }

    // Where a lane's part of a fragment of rows lies: row lane % 32, columns 16 c + 8 (lane / 32).. are at this ^ 32 c.
    static __device__ int rows_place(int lane) { return at(lane % 32, lane / 32); }
    // Where a lane's part of a transposed fragment lies: columns 32 d.. of rows 16 s.. are at (this ^ 64 d) + 16 s PITCH; `up`: the second read, of rows 8 further on.
    static __device__ int cols_place(int lane, int up)
    {
        const int r = lane / 32 * 4 + lane % 16 / 4 + up * 8;
        return at(r, lane / 16 % 2 * 2 + lane % 4 / 2) + lane % 2 * 8;
    }
    template <class T>
    static __device__ frag<T> rows(lds_byte *tile, int place, int c, int r0)
    {
        return *(__attribute__((address_space(3))) frag<T> *)(tile + (place ^ c * 32) + r0 * PITCH);
    }
    template <class T>
    static __device__ frag<T> cols(lds_byte *tile, const int (&place)[2], int d, int r0)
    {
        using half_frag = vec<short, 4>;
        using lds_half = __attribute__((address_space(3))) half_frag;
        const half_frag lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_half *)(tile + (place[0] ^ d * 64) + r0 * PITCH));
        const half_frag hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_half *)(tile + (place[1] ^ d * 64) + r0 * PITCH));
        return __builtin_bit_cast(frag<T>, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// A tile of ROWS rows filled by WAVES waves with direct copies, 16 bytes a lane.  Rows start at multiples of 16 bytes;
// their columns past `width` (a multiple of 8) and rows that are not live become zeros.
template <int DP, int ROWS, int WAVES>
struct tile_copy {
    static constexpr int PIECES = ROWS * DP * 2 / PIECE, MINE = PIECES / WAVES, ROWS_EACH = PIECE / (DP * 2);
    static_assert(PIECES % WAVES == 0);
    uint32_t off[MINE], wide;  // wide: bit i: piece i's columns exist

    static __device__ int row(int piece, int lane) { return piece * ROWS_EACH + lane / (DP / 8); }
    __device__ void set(int wave, int lane, int64_t stride, int width)
    {
        wide = 0;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int r = row(wave * MINE + i, lane), chunk = lane % (DP / 8) ^ lay<DP>::fold(r);
            off[i] = (uint32_t)(r * stride * 2 + chunk * 16);
            wide |= (uint32_t)(chunk * 8 < width) << i;
        }
    }
    // from: the tile's first row; live: bit r: row r exists; all: every row and column does.
    __device__ void copy(int wave, int lane, const char *from, uint64_t live, bool all, lds_byte *to) const
    {
        if (all) {
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                uint32_t o = off[i];
                asm volatile("" : "+v"(o));  // stays 32 bits wide: the copy adds it to a scalar address
                copy_piece(from + o, to + (wave * MINE + i) * PIECE);
            }
        } else {
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                const bool there = (wide >> i & 1) && (live >> row(wave * MINE + i, lane) & 1);
                copy_piece(there ? from + off[i] : (const char *)&zero_chunk, to + (wave * MINE + i) * PIECE);
            }
        }
    }
};

// A word's n-th byte as a signed whole number.  (One instruction; written out it becomes two or three, which the compiler also
// moves ahead of a loop's turn, where four words wait instead of one.)
template <int n>
__device__ inline float code_of(uint32_t word)
{
    float v;
    if constexpr (n == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(v) : "v"(word));
    if constexpr (n == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(v) : "v"(word));
    if constexpr (n == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(v) : "v"(word));
    if constexpr (n == 3) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(v) : "v"(word));
    return v;
}

// Eight codes as values of T: whole numbers of up to 8 bits times a power of two, exact.
template <class T>
__device__ inline frag<T> code_values(uint32_t lo, uint32_t hi, float step)
{
    const float v[8] = {code_of<0>(lo), code_of<1>(lo), code_of<2>(lo), code_of<3>(lo), code_of<0>(hi), code_of<1>(hi), code_of<2>(hi), code_of<3>(hi)};
    frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (T)(v[i] * step);
    return f;
}

// The same tile from a cache's codes, through registers: load, then (later) put.  Nothing is decided between the loads: rows and
// columns that do not exist are read from where the last ones that do lie, and become zeros when they are put.
template <class T, int DP, int ROWS, int LANES>
struct tile_codes {
    static constexpr int EACH = ROWS * DP / 16 / LANES, SPANS = DP / 16, BLOCKS = ROWS / RKB_GROUP;
    static_assert(ROWS * DP / 16 % LANES == 0 && BLOCKS <= 2);
    u32x4 q[EACH];
    uint8_t exp[BLOCKS];
    uint64_t live;
    int spans;

    // from: the codes of the tile's first row, exps: those of its blocks; rows: how many exist (at least one).
    __device__ void load(int t, const int8_t *from, const uint8_t *exps, int64_t ld, uint64_t alive, int rows)
    {
        live = alive;
        spans = (int)ld / 16;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int n = t + i * LANES, r = min(n / SPANS, rows - 1), span = min(n % SPANS, spans - 1);
            q[i] = *(const u32x4 *)(from + r * (int)ld + span * 16);
        }
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) exp[k] = exps[min(k, (rows - 1) / RKB_GROUP)];
    }
    __device__ void put(int t, lds_byte *to) const
    {
        float step[BLOCKS];
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) step[k] = exp[k] == 0 ? 0.0f : step_of(exp[k]);
        constexpr uint64_t ALL = ROWS == 64 ? ~(uint64_t)0 : ((uint64_t)1 << ROWS % 64) - 1;
        const bool all = (live & ALL) == ALL && spans == SPANS;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int n = t + i * LANES, r = n / SPANS, span = n % SPANS;
            const bool there = all || ((live >> r & 1) && span < spans);
            const float by = !there ? 0.0f : BLOCKS == 1 || r < RKB_GROUP ? step[0] : step[BLOCKS - 1];
            using lds_frag = __attribute__((address_space(3))) frag<T>;
            *(lds_frag *)(to + lay<DP>::at(r, span * 2)) = code_values<T>(there ? q[i][0] : 0u, there ? q[i][1] : 0u, by);
            *(lds_frag *)(to + lay<DP>::at(r, span * 2 + 1)) = code_values<T>(there ? q[i][2] : 0u, there ? q[i][3] : 0u, by);
        }
    }
};

// All copies and LDS accesses of this wave, and then of the workgroup, are done.
__device__ inline void wait_all()
{
    __builtin_amdgcn_s_waitcnt(wait_copies(0));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A stationary row's fragments: columns 16 c + 8 (lane / 32).. of the row.  Rows are 16-byte aligned, width a multiple of 8.
template <class T, int DP>
__device__ inline void load_stationary(frag<T> (&f)[DP / 16], const T *row, int lane, int width, bool there)
{
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const int col = c * 16 + lane / 32 * 8;
        frag<T> z = {};
        if (there && col < width) z = *(const frag<T> *)(row + col);
        f[c] = z;
    }
}

// Two of a product's register groups as a fragment of 16 rows of the next product.
template <class T>
__device__ inline frag<T> to_frag(const f32x16 &s, int half)
{
    frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (T)s[half * 8 + i];
    return f;
}

// ------------------------------------------------------------------ which keys live

// Bits of the 64 keys from k0 on, for the whole workgroup: those before len whose mask byte (of this lane's key) is set.
__device__ inline uint64_t keys_alive(const attn_in &p, int k0, int len, uint8_t mask_byte)
{
    const int n = len - k0;
    uint64_t bits = n >= 64 ? ~(uint64_t)0 : n <= 0 ? 0 : ((uint64_t)1 << n) - 1;
    if (p.mask) bits &= __ballot(mask_byte != 0);
    return bits;
}
__device__ inline uint8_t mask_byte(const attn_in &p, int b, int k, int len)
{
    return p.mask && k >= 0 && k < len ? p.mask[b * p.mask_stride + k] : (uint8_t)1;
}

// Registers of a 32-key piece whose key does not live, or lies behind the lane's query, become `to`.  bits: of the 32 keys;
// ahead: the query's position less the piece's first key, or INT_MAX where order does not matter.
__device__ inline void kill_dead(f32x16 &s, uint32_t bits, int ahead, int lane, float to)
{
    const int h = half_row(lane);
    if (bits != ~0u) {
        const uint32_t w = bits >> h;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = w >> (r / 4 * 8 + r % 4) & 1 ? s[r] : to;
    }
    if (__any(ahead < 31)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = r / 4 * 8 + r % 4 <= ahead - h ? s[r] : to;
    }
}

// ------------------------------------------------------------------ bias by relative position

// Borders are counted 16 at a time, so that a wave waits for one wide scalar load instead of 16.
__device__ inline int bucket_of(const bias_table &t, int rel)
{
    const int d = t.sides == 2 ? abs(rel) : max(-rel, 0);
    int n = 0;
    for (int i = 0; i < t.count - 1; i += 16) {
#pragma unroll
        for (int k = 0; k < 16; ++k) n += d >= t.border[i + k];
    }
    return n + (t.sides == 2 && rel > 0 ? t.count : 0);
}

// A table entry times log2(e).  One that is meant to hide its keys does: next to it a score, and the logarithm of a
// row's sum, would be lost in 32 bits.
template <class T>
__device__ inline float table_value(const attn_in &p, int bucket, int h)
{
    const int64_t i = (int64_t)bucket * p.H + h;
    const float v = p.bias.f32 ? ((const float *)p.bias.table)[i] : (float)((const T *)p.bias.table)[i];
    return v <= -1e30f ? NEG_INF : v * LOG2E;
}

// One head's bias by distance: entry n is that of relative position n - far - PAD.  Beyond far the last buckets go on for as
// much as 32 queries x 32 keys that reach nearer than far can pass it, so that nothing is clamped.
constexpr int PAD = 64;

template <class T>
__device__ inline void fill_bias(float *by_distance, const attn_in &p, int h, int t, int lanes)
{
    for (int n = t; n <= 2 * (p.bias.far + PAD); n += lanes) by_distance[n] = table_value<T>(p, bucket_of(p.bias, n - p.bias.far - PAD), h);
}

// Adds a head's bias to a 32-key piece of scores: key0 the piece's first key, pos the lane's query; pos_lo and pos_hi
// bound the wave's.  s = s c + bias.
__device__ inline void add_bias(f32x16 &s, float c, const float *by_distance, int far, int key0, int pos, int pos_lo, int pos_hi, int lane)
{
    if (key0 - pos_hi >= far || key0 + 31 - pos_lo <= -far) {
        const float b = by_distance[key0 - pos_hi >= far ? 2 * (far + PAD) : 0];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], c, b);
    } else {
        const float *const at = by_distance + key0 + half_row(lane) - pos + far + PAD;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], c, at[r / 4 * 8 + r % 4]);
    }
}

}  // namespace rkb
