// How the products of librkblock are cut: which tile, how many workgroups share a long sum, which launches
// (used by rkb_gemm.hip).  Plain C++ on sizes alone, so that a host without a GPU can ask what a size takes.
#pragma once
#include <algorithm>
#include <cstdint>

#include "rk_block.h"

namespace rkb {

constexpr int DEPTH = 64;                        // k of a tile's stage
constexpr int64_t MAX_TILES = (int64_t)1 << 22;  // workgroups of a launch: 512 threads of each in 32 bits

// Whether a lane's place in a stage of `tile_rows` rows that run along k, `stride` elements apart, is a 32-bit number of
// bytes from the tile's first row.  Callers' strides are at most STRIDE_LIMIT (others' rows are copied into the
// workspace); copies, and dg and du, have rows as long as their columns rounded up to 8, up to RKB_MAX_COLS.
constexpr int64_t STRIDE_LIMIT = (int64_t)1 << 22;
constexpr bool rows_in_reach(int tile_rows, int64_t stride) { return (tile_rows - 1) * stride * 2 + (DEPTH - 8) * 2 <= UINT32_MAX; }
static_assert(rows_in_reach(256, STRIDE_LIMIT) && rows_in_reach(128, RKB_MAX_COLS));

// How a product is cut: the tile, its buffers, and how many workgroups share the stages of one tile (splits).
struct cut {
    int tm, tn, bufs, splits;
    double us;  // what the choice expects it to take
};

// The tiles, with the microseconds of one stage in a workgroup that runs nearly alone and on a full chip
// (where the clock is lower and L2 shared), and of a tile's start and end, fitted to measured products
// of 64 to 8192 rows (bf16).  Small tiles pay more per product and fill the chip sooner: at 8192 x 4096 x 11264 the
// gated forward takes 1140 us by 256 x 256, 1237 by 192 x 256 and 1368 by 128 x 128; at 1024 x 1280 x 5120 it takes
// 36.7, 30.7 and 36.4; at 512 x 1024 x 4096, 27.3, 22.0 and 12.2.  Four buffers hide the latency of copies where a compute
// unit has one workgroup: 128 x 4096 x 4096 takes 26.8 us with them and 40.0 with two, 1024 x 1280 x 5120
// 36.7 and 36.4.  `ends` is that of a plain epilogue: what the gated forward's does more is in no figure here.  At
// 1999 x 1024 x 2730 it takes 25 us with silu (bf16) and nothing kept, 31 where it keeps codes; 31 and 34 with gelu (f16).
struct tile_kind {
    int tm, tn, bufs, slots;  // slots: workgroups that 256 compute units hold at once
    double alone, busy, ends;
};
constexpr tile_kind TILES[] = {
    {256, 256, 2, 256, 1.05, 1.68, 5.0},
    {192, 256, 2, 256, 0.82, 1.29, 4.5},
    {128, 128, 2, 512, 0.49, 0.95, 2.5},
    {128, 128, 4, 256, 0.36, 0.48, 3.5},
};
constexpr double JOIN_FIXED = 4.0, JOIN_BYTES = 4.5e6;  // microseconds, bytes a microsecond
constexpr double LAUNCH = 6.0;                          // a launch more, from the end of the work before it

// The cut that these figures expect to be fastest.  Splits share a long K among workgroups where the tiles alone do
// not fill the chip, at the price of 32-bit partial sums written and read once: dw of 512 x 512 over 16384
// rows takes 174 us whole and 25 in 16 splits, of 2048 x 2048 over 2048 rows 28 whole and 34 in 2.  near: A's rows run along k (and
// B's in g and u, by 128); tiles that would pass their offsets' range are left out, above 8.4 million columns.
inline cut choose_cut(int64_t M, int64_t N, int64_t K, int parts, int problems, int sums, bool near)
{
    const int64_t stages = std::max<int64_t>(1, (K + DEPTH - 1) / DEPTH * parts);
    cut best{256, 256, 2, 1, 1e30};
    for (const tile_kind &t : TILES) {
        if (near ? !rows_in_reach(t.tm, (K + 7) / 8 * 8) : t.tm == 192) continue;
        const int64_t tiles = (M + t.tm - 1) / t.tm * ((N + t.tn / sums - 1) / (t.tn / sums)) * problems;
        for (int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (splits > 1 && (sums == 2 || splits * 4 > stages || splits * tiles > 2 * t.slots)) break;
            const int64_t groups = tiles * splits, rounds = groups / t.slots, rest = groups % t.slots;
            const double each = (double)((stages + splits - 1) / splits);
            double us = rounds * (each * t.busy + t.ends);
            if (rest) us += each * (t.alone + (t.busy - t.alone) * rest / t.slots) + t.ends;
            if (splits > 1) us += JOIN_FIXED + 2.0 * 4.0 * splits * problems * (double)M * N / JOIN_BYTES;
            if (us < best.us) best = cut{t.tm, t.tn, t.bufs, splits, us};
        }
    }
    return best;
}

// How dx (in `splits`) and the weight gradients go in one launch of 128 x 128 tiles, and what it is expected to take.  Together they
// fill the chip where each alone does not, and a launch is saved: the backward from 8-bit checkpoints takes 14 us
// instead of 20 at 128 x 512 x 856, 36 instead of 43 at 512 x 1024 x 4096, 165 instead of 180 at 3000 x 1500 x 3000;
// at 2048 x 2048 x 2048 87 instead of 85.
struct pair_cut {
    int bufs, splits;
    double us;
};

inline pair_cut choose_pair(int64_t rows, int64_t d, int64_t f)
{
    const int64_t tiles_x = (rows + 127) / 128 * ((d + 127) / 128), tiles_w = 2 * ((f + 127) / 128) * ((d + 127) / 128);
    const int64_t stages_x = (f + DEPTH - 1) / DEPTH * 2, each_w = (rows + DEPTH - 1) / DEPTH;
    pair_cut best{2, 1, 1e30};
    for (const tile_kind &t : TILES) {
        if (t.tm != 128) continue;
        for (int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (splits > 1 && splits * 4 > stages_x) break;
            const int64_t each_x = (stages_x + splits - 1) / splits, groups = tiles_x * splits + tiles_w;
            const double longest = (double)std::max(each_x, each_w);
            double us;
            if (groups <= t.slots)
                us = longest * (t.alone + (t.busy - t.alone) * groups / t.slots) + t.ends;
            else
                us = ((double)(tiles_x * splits * each_x + tiles_w * each_w) * t.busy + groups * t.ends) / t.slots + 0.2 * longest * t.busy;
            if (splits > 1) us += JOIN_FIXED + 2.0 * 4.0 * splits * (double)rows * d / JOIN_BYTES;
            if (us < best.us) best = pair_cut{t.bufs, splits, us};
        }
    }
    return best;
}

constexpr int FEW_ROWS = 64;

// Whether the few-rows form is expected to beat tiles that take `tiles_us`.  Weights come at the rate of a large read, and
// with the rows that every workgroup reads again (from L2) at 7.3 TB/s in all, after 2.2 us of start and end.  At 1024 x 4096 one
// row takes 5.2 us and 64 take 9.1 (tiles: 9.4), at 4096 x 4096 14.5 and 26 (26), at 4096 x 11264 33 and 75 (30).  That rate
// needs N/16 workgroups that fill the chip and whole steps of 32 k: with 16 workgroups 4 x 4096 x 256 takes 11 us, and 33 at
// 4 x 4095 x 256, whose last step is loaded element by element (by tiles, 65 x 4096 x 256 takes 23).  What is kept has no
// say: h, and g and u made again, are the same bits in every form.
inline bool few_rows_win(int64_t M, int64_t N, int64_t K, double tiles_us)
{
    if (M > FEW_ROWS) return false;
    const double weights = 4.0 * N * K, again = (double)((N + 15) / 16) * M * K * 2.0;
    return 2.2 + std::max(weights / 5.5e6, (weights + again) / 7.3e6) < tiles_us;
}

// The three products of a gated block: g and u, dx, and dwg and dwu.
inline cut sums_cut(int64_t rows, int64_t d, int64_t f) { return choose_cut(rows, f, d, 1, 1, 2, true); }
inline cut dx_cut(int64_t rows, int64_t d, int64_t f) { return choose_cut(rows, d, f, 2, 1, 1, true); }
inline cut dw_cut(int64_t rows, int64_t d, int64_t f) { return choose_cut(f, d, rows, 1, 2, 1, false); }

// Up to so many elements of dg and du go into the products in two 16-bit parts each, so that only the results are rounded: a
// relative error of 1.7e-3 in bf16 instead of 2.4e-3, and 1.0 of a rounding's instead of up to 1.8 where a gradient is
// a single product.  That gain is the same at any size; the limit is one of cost, which is twice the products.  The backward of
// 1 x 64 x 64 takes 7.5 us so and 6.3 with one part, of 1 x 1024 x 4096 27 and 23, of 8 x 1024 x 4096 it would take 26
// instead of 20, and of 1024 x 1280 x 5120 133 instead of 75.
constexpr int64_t FINE_ELEMENTS = 4096;

// The backward's two products, one after the other or in one launch.
struct backward_cut {
    cut x, w;
    pair_cut both;
    bool together, fine;
    backward_cut(int64_t rows, int64_t d, int64_t f) : x(dx_cut(rows, d, f)), w(dw_cut(rows, d, f)), both(choose_pair(rows, d, f))
    {
        together = both.us < x.us + w.us + LAUNCH;
        fine = rows * f <= FINE_ELEMENTS;
    }
};

}  // namespace rkb
