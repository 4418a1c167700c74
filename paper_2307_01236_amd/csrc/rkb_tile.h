// A tile of a product on the matrix units, staged through LDS (used by rkb_gemm.hip).
//
// C[m, n] = sum over k of A(m, k) B(n, k) in tiles of TM x TN, depth 64.  A workgroup of WM x WN
// waves keeps its tile of C in registers; the operands' next 64 columns are copied from memory
// straight into LDS (16 bytes a lane, no registers in between) while the waves work on the present
// ones, in two or four buffers.  An operand lies in memory either with k adjacent (a row per m or n)
// or with m or n adjacent (a row per k); the matrix units want 8 neighbouring k of one row in a
// lane, which LDS reads as they lie in the first form, and by its transposing read in the second.
//
// LDS layout of an operand's stage, in 1-KiB pieces that one wave copies with one instruction:
//   k adjacent: 8 rows of 128 bytes; the 16-byte chunks of row r are permuted by r / 2 (xor), so that the 16
//     rows that a fragment's lanes read at one k fall into different banks;
//   a row per k: rows that a transposing read takes together (k, k+1, k+2, k+3 and the
//     same 8 further on) lie in different pieces, each 32 bytes longer than it is full, which puts them
//     into different banks and leaves every fragment's place a constant offset.
//
// Bound by the matrix units, whose clock falls with the operands' bits: 256 x 256 tiles reach 1.45 PFLOP/s at
// 8192 x 4096 x 8192 (bf16, random operands; 1.83 on zeros), 1.36 at 4096 x 4096 x 4096, and 1.26 and 1.35 at 8192 x 11264 x
// 4096 and 11264 x 4096 x 8192, whose tiles fill 5.5 rounds of workgroups.  A tile's start and end cost about 5 us.
#pragma once
#include <type_traits>

#include "rkb_common.h"
#include "rkb_cut.h"

namespace rkb {

template <class T>
using frag = vec<T, 8>;

__device__ inline f32x4 mma(frag<bf16> a, frag<bf16> b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mma(frag<f16> a, frag<f16> b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// s_waitcnt for all LDS reads and all but the last n copies
constexpr int wait_copies(int n) { return (n & 15) | 0x70 | n >> 4 << 14; }
constexpr int PIECE = 1024;              // bytes that one wave's copy instruction brings
constexpr int PIECE_APART = PIECE + 32;  // distance of pieces of the row-per-k form

// What the copy instructions read for k past the end: zeros.
__device__ const u32x4 zero_chunk = {0, 0, 0, 0};

using lds_byte = __attribute__((address_space(3))) char;
using lds_void = __attribute__((address_space(3))) void;
using global_void = const __attribute__((address_space(1))) void;

__device__ inline void copy_piece(const void *from, lds_byte *to)
{
    __builtin_amdgcn_global_load_lds((global_void *)from, (lds_void *)to, 16, 0, 0);
}

// ROWS rows (of m or n) of an operand, staged by WAVES waves.  NEAR: k adjacent.  PAIR: rows of two matrices,
// 32 of one and 32 of the other in turn, so that a wave's 64 rows are the same 32 of both.
template <class T, int ROWS, int WAVES, bool NEAR, bool PAIR>
struct stager {
    static constexpr int PIECES = ROWS * DEPTH * 2 / PIECE, MINE = PIECES / WAVES;
    static constexpr int APART = NEAR ? PIECE : PIECE_APART, BYTES = PIECES * APART;
    static_assert(PIECES % WAVES == 0 && sizeof(T) == 2 && (NEAR || !PAIR));

    uint32_t off[MINE];  // this lane's bytes from the stage's start, by piece

    static __device__ int k_of(int piece, int lane)  // row per k: which k of the stage
    {
        if constexpr (ROWS == 256) return piece / 4 * 8 + piece % 4 + lane / 32 * 4;
        static_assert(ROWS == 256 || ROWS == 128);
        return piece / 4 * 8 + piece % 4 + (lane / 16 & 1) * 4 + lane / 32 * 32;
    }
    static __device__ int chunk_of(int piece, int lane)  // k adjacent: which 8 k
    {
        const int row = piece * 8 + lane / 8;
        return lane % 8 ^ (row / 2 & 7);
    }

    static __device__ bool exists(int piece, int lane, int left)  // whether this lane's k does
    {
        if constexpr (NEAR)
            return chunk_of(piece, lane) * 8 < left;
        else
            return k_of(piece, lane) < left;
    }

    // r0: the tile's first row, rows: those that exist (the last one stands in for the others: what it gives there is
    // never stored).  For a row per k, rows is a multiple of 8.
    __device__ void set(int wave, int lane, int64_t r0, int64_t rows, int64_t stride)
    {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int piece = wave * MINE + i;
            if constexpr (NEAR) {
                const int at = piece * 8 + lane / 8, row = PAIR ? at / 64 * 32 + at % 32 : at;
                const int64_t r = min(r0 + row, rows - 1) - r0;
                off[i] = (uint32_t)(r * stride * 2 + chunk_of(piece, lane) * 16);
            } else {
                const int64_t c = min(r0 + lane % (ROWS / 8) * 8, rows - 8) - r0;
                off[i] = (uint32_t)(k_of(piece, lane) * stride * 2 + c * 2);
            }
        }
    }

    // base(piece): the address of the stage's start (uniform).  FULL: all its k exist; else `left` of them do.
    template <bool FULL, class B>
    __device__ void copy(int wave, int lane, B base, int left, lds_byte *to) const
    {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int piece = wave * MINE + i;
            uint32_t o = off[i];
            asm volatile("" : "+v"(o));  // stays 32 bits wide: the copy adds it to a scalar address
            const char *from = base(piece) + o;
            if (!FULL && !exists(piece, lane, left)) from = (const char *)&zero_chunk;
            copy_piece(from, to + piece * APART);
        }
    }

    // Where a lane's part of fragment 0 (rows from r0 on) of a stage lies; `half`: the first or second 32 k.
    static __device__ int place(int r0, int lane, int half)
    {
        if constexpr (NEAR) {
            const int row = r0 + lane % 16, chunk = half * 4 + lane / 16;
            return row * 128 + (chunk ^ (row / 2 & 7)) * 16;
        } else {
            const int g = lane / 16, j = lane % 16 / 4;
            if constexpr (ROWS == 256)
                return ((half * 4 + g) * 4 + j) * PIECE_APART + r0 * 2 + lane % 4 * 8;
            else
                return (g * 4 + j) * PIECE_APART + half * 512 + r0 * 2 + lane % 4 * 8;
        }
    }

    // Fragment f: rows 16 f .. 16 f + 15 from the place's first.
    static __device__ frag<T> read(lds_byte *at, int f)
    {
        if constexpr (NEAR) {
            return *(__attribute__((address_space(3))) frag<T> *)(at + f * 16 * 128);
        } else {
            using half_frag = vec<short, 4>;
            using lds_half = __attribute__((address_space(3))) half_frag;
            const half_frag lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_half *)(at + f * 32));
            const half_frag hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_half *)(at + f * 32 + ROWS * 2));
            return __builtin_bit_cast(frag<T>, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// One launch: `problems` products of the same sizes, each a sum over PARTS operand pairs.  Part p of problem i is
//   a[PARTS i + p] b[0]   where weights' gradients are formed (B a row per k, as is A),
//   a[p] b[p % 2]         where dx is (one problem),
//   a[0] b[0] and a[0] b[1] side by side for an epilogue of two sums.
// The operands of one kind share their stride.
struct product {
    const char *a[4], *b[2];
    int64_t sa, sb, sb2;  // sb2: of b[1], where it differs (few rows only)
    int64_t M, N, K;
    int problems;
    int tiles_m, tiles_n;
    int splits, split_stages;  // stages (of all parts) that one workgroup takes
};

// Which tile a workgroup takes.  Workgroups go to the 8 dies in turn; each die gets a run of
// neighbouring tiles, in bands of 8 tile rows, so that its L2 holds what they share.
struct tile_at {
    int m, n, problem, split;
};

__device__ inline tile_at find_tile(const product &pr, int block)
{
    const int tiles = pr.tiles_m * pr.tiles_n, total = tiles * pr.problems * pr.splits;
    const int die = block % 8, share = total / 8, rest = total % 8;
    int w = die * share + min(die, rest) + block / 8;
    tile_at t;
    t.problem = w / (tiles * pr.splits);
    w -= t.problem * tiles * pr.splits;
    t.split = w / tiles;
    w -= t.split * tiles;
    const int band = 8 * pr.tiles_n, first = w / band * 8, high = min(pr.tiles_m - first, 8);
    w %= band;
    t.m = first + w % high;
    t.n = w / high;
    return t;
}

// Bytes of a stage of both operands in LDS.
template <class T, int TM, int TN, int WAVES, bool ANEAR, bool BNEAR, bool PAIR>
constexpr int STAGE_BYTES = stager<T, TM, WAVES, ANEAR, false>::BYTES + stager<T, TN, WAVES, BNEAR, PAIR>::BYTES;

// The workgroup's tile of a launch's `block`th workgroup.  BUFS: stages that LDS holds, one in each of `lds`.
template <class T, class EPI, int TM, int TN, int WM, int WN, int BUFS, bool ANEAR, bool BNEAR, int PARTS>
__device__ __forceinline__ void product_tile(const product &pr, const EPI &epi, int block, lds_byte *const (&lds)[4])
{
    constexpr int WAVES = WM * WN, SUMS = EPI::SUMS;
    constexpr int FM = TM / WM / 16, FN = TN / WN / 16;  // fragments of a wave
    static_assert(FN == 4 && (BUFS == 2 || BUFS == 4));
    using SA = stager<T, TM, WAVES, ANEAR, false>;
    using SB = stager<T, TN, WAVES, BNEAR, SUMS == 2>;
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int wm = wave / WN, wn = wave % WN;
    const tile_at t = find_tile(pr, block);
    const int64_t m0 = (int64_t)t.m * TM, n0 = (int64_t)t.n * (TN / SUMS);
    const int stages_k = (int)((pr.K + DEPTH - 1) / DEPTH);
    const int first = t.split * pr.split_stages, last = min(stages_k * PARTS, first + pr.split_stages);

    SA sa;
    SB sb;
    sa.set(wave, lane, m0, pr.M, pr.sa);
    sb.set(wave, lane, n0, pr.N, pr.sb);
    const int64_t a_row0 = (ANEAR ? m0 * pr.sa : m0) * 2, b_row0 = (BNEAR ? n0 * pr.sb : n0) * 2;
    const int64_t a_step = ANEAR ? 2 : pr.sa * 2, b_step = BNEAR ? 2 : pr.sb * 2;

    auto copy = [&](auto full, int s, lds_byte *to) {
        const int part = PARTS == 1 ? 0 : PARTS == 2 ? s >= stages_k : s / stages_k;
        const int k0 = (s - part * stages_k) * DEPTH, left = (int)pr.K - k0;
        const char *pa = pr.a[0], *pb = pr.b[0], *pu = pr.b[1] + b_row0 + k0 * b_step;
#pragma unroll
        for (int i = 1; i < 4; ++i)  // by selection: a place in an array that is only known at run time would be loaded again
            if (i < (ANEAR ? PARTS : 2 * PARTS) && i == (ANEAR ? part : PARTS * t.problem + part)) pa = pr.a[i];
        if (ANEAR && !BNEAR && part % 2) pb = pr.b[1];
        pa += a_row0 + k0 * a_step;
        pb += b_row0 + k0 * b_step;
        sa.template copy<full()>(wave, lane, [&](int) { return pa; }, left, to);
        sb.template copy<full()>(wave, lane, [&](int piece) { return SUMS == 2 && piece / 4 % 2 ? pu : pb; }, left, to + SA::BYTES);
    };
    constexpr std::true_type full{};
    constexpr std::false_type any{};
    const int a_at[2] = {SA::place(wm * FM * 16, lane, 0), SA::place(wm * FM * 16, lane, 1)};
    const int b_at[2] = {SB::place(wn * FN * 16, lane, 0), SB::place(wn * FN * 16, lane, 1)};

    f32x4 acc[FM][FN] = {};
    frag<T> fa[2][FM], fb[2][FN];
    auto fetch = [&](int half, lds_byte *from) {
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[half][j] = SB::read(from + SA::BYTES + b_at[half], j);
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[half][i] = SA::read(from + a_at[half], i);
    };
    auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mma(fb[half][j], fa[half][i], acc[i][j]);
    };
    // The reads of the next fragments, and `copies` of a later stage, are spread over the products of the
    // present fragments: first B's, of which all are needed at once, then A's, each when about as
    // many of the present ones have been used up, so that few registers hold both.
    auto mix = [&](auto copies) {
        constexpr int RA = ANEAR ? 1 : 2, RB = BNEAR ? 1 : 2, EACH = (FM * FN - 2 * FN) / FM;
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // matrix instructions
            __builtin_amdgcn_sched_group_barrier(0x100, RB, 0);  // LDS reads
            if (i < copies()) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            if constexpr (EACH > 0) __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, RA, 0);
            if (FN + i < copies()) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, FM * FN - FN - FM * EACH, 0);
    };
    // Stage s from buffer `at` while the next ones lie in, or are on their way to, the others.  All waves have read
    // this buffer when they pass the barrier, and all copies of the next stage have landed (copies land in
    // order: those of BUFS - 2 later stages may still be on their way); so stage s + BUFS may be copied over
    // this one while its second half is multiplied.  AHEAD: that stage exists and is full.
    constexpr int FLYING = (BUFS - 2) * (SA::MINE + SB::MINE);
    auto stage = [&](auto ahead, int s, auto at) {
        lds_byte *here = lds[at()], *next = lds[(at() + 1) % BUFS];
        fetch(1, here);
        multiply(0);
        mix(std::integral_constant<int, 0>());
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(ahead() ? wait_copies(FLYING) : wait_copies(0));
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (ahead()) {
            copy(full, s + BUFS, here);
            fetch(0, next);
            multiply(1);
            mix(std::integral_constant<int, SA::MINE + SB::MINE>());
            __builtin_amdgcn_sched_barrier(0);
        } else {
            if (s + BUFS < last) copy(any, s + BUFS, here);
            fetch(0, next);  // past the last stage: whatever lies there, not used
            multiply(1);
            mix(std::integral_constant<int, 0>());
        }
    };
    constexpr std::integral_constant<int, 0> at0{};
    constexpr std::integral_constant<int, 1> at1{};
    constexpr std::integral_constant<int, BUFS == 4 ? 2 : 0> at2{};
    constexpr std::integral_constant<int, BUFS == 4 ? 3 : 1> at3{};
    if (first < last) {
        if (BUFS == 4 && first + 3 < last) copy(any, first + 3, lds[3]);
        if (BUFS == 4 && first + 2 < last) copy(any, first + 2, lds[2]);
        if (first + 1 < last) copy(any, first + 1, lds[1]);
        copy(any, first, lds[0]);
        __builtin_amdgcn_s_waitcnt(wait_copies(0));
        __builtin_amdgcn_s_barrier();
        fetch(0, lds[0]);
        const bool ragged = pr.K % DEPTH != 0;
        for (int s = first; s < last;) {
            // the next stage that is not full, or the end
            const int stop = !ragged ? last : min(last, ((PARTS == 1 ? 0 : (s + BUFS) / stages_k) + 1) * stages_k - 1);
            for (; s + 2 * BUFS - 1 < stop; s += BUFS) {
                stage(full, s, at0);
                stage(full, s + 1, at1);
                if constexpr (BUFS == 4) {
                    stage(full, s + 2, at2);
                    stage(full, s + 3, at3);
                }
            }
            stage(any, s, at0);
            if (s + 1 < last) stage(any, s + 1, at1);
            if constexpr (BUFS == 4) {
                if (s + 2 < last) stage(any, s + 2, at2);
                if (s + 3 < last) stage(any, s + 3, at3);
            }
            s += BUFS;
        }
    }

    // Hand out units of 16 rows by 32 columns.  A lane holds columns 4 q + i of a fragment's 16 (q =
    // lane / 16); swapping between neighbouring q of a unit's two fragments leaves it 8 neighbours.
    const int q = lane / 16, col8 = (q & 1) * 16 + q / 2 * 8;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t row = m0 + wm * FM * 16 + i * 16 + lane % 16;
        float v[FN / 2][8];
#pragma unroll
        for (int unit = 0; unit < FN / 2; ++unit)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][unit * 2][e]),
                                                                  __float_as_uint(acc[i][unit * 2 + 1][e]), false, false);
                v[unit][e] = __uint_as_float(two[0]);
                v[unit][4 + e] = __uint_as_float(two[1]);
            }
        if constexpr (SUMS == 2) {
            epi(t.split, row, n0 + wn * 32 + col8, v[0], v[1]);
        } else {
#pragma unroll
            for (int unit = 0; unit < FN / 2; ++unit)
                epi(t.problem * pr.splits + t.split, row, n0 + wn * 64 + unit * 32 + col8, v[unit]);
        }
    }
}

// The stages' buffers, as separate arrays: the compiler must see that reads of one do not wait for copies into another.
#define RKB_STAGE_BUFFERS(BYTES, BUFS)                                                                                   \
    __shared__ __align__(16) char s0[BYTES], s1[BYTES], s2[BUFS > 2 ? BYTES : 16], s3[BUFS > 2 ? BYTES : 16];            \
    lds_byte *const lds[4] = {(lds_byte *)s0, (lds_byte *)s1, (lds_byte *)s2, (lds_byte *)s3}

template <class T, class EPI, int TM, int TN, int WM, int WN, int BUFS, bool ANEAR, bool BNEAR, int PARTS>
__global__ __launch_bounds__(WM *WN *WAVE) void k_product(product pr, EPI epi)
{
    constexpr int BYTES = STAGE_BYTES<T, TM, TN, WM * WN, ANEAR, BNEAR, EPI::SUMS == 2>;
    RKB_STAGE_BUFFERS(BYTES, BUFS);
    product_tile<T, EPI, TM, TN, WM, WN, BUFS, ANEAR, BNEAR, PARTS>(pr, epi, blockIdx.x, lds);
}

}  // namespace rkb
