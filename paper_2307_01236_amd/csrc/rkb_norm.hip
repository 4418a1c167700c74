// Layer norm, forward and backward (rk_block.h).
//
// Bound by memory: the forward reads x and writes y, the backward reads dy and x (or its 8-bit
// checkpoint) and writes dx.  A row stays in the registers of LANES lanes between the sums over it, so
// each matrix is read once; the mean is formed first and the variance from differences to
// it, which costs no second read and loses no digits where the mean is large.  At 16384 x 4096 (bf16) the
// forward takes 55 us (4.8 TB/s), the backward 78 (5.2 TB/s) and 5 for the columns; one row of 1024 takes 2.7 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "rkb_common.h"

namespace rkb {
namespace {

constexpr int NORM_BLOCK = 256;

// Sums over the lanes of one row, in every one of them.  Rows of more than a wave join their waves
// through LDS: successive calls use two places in turn, so that one barrier each is enough.
template <int LANES, int BLOCK, int COUNT>
struct row_sums {
    static constexpr int WAVES = LANES > WAVE ? LANES / WAVE : 1, ROWS = LANES > WAVE ? BLOCK / LANES : 1;
    using place = float[2][ROWS][COUNT][WAVES];
    place &part;
    int turn = 0;
    __device__ row_sums(place &p) : part(p) {}
    __device__ void operator()(float (&v)[COUNT])
    {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) v[c] = lane_sum<LANES < WAVE ? LANES : WAVE>(v[c]);
        if constexpr (LANES > WAVE) {
            const int row = threadIdx.x / LANES, wave = threadIdx.x % LANES / WAVE;
            if (threadIdx.x % WAVE == 0)
#pragma unroll
                for (int c = 0; c < COUNT; ++c) part[turn][row][c][wave] = v[c];
            __syncthreads();
#pragma unroll
            for (int c = 0; c < COUNT; ++c) {
                v[c] = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v[c] += part[turn][row][c][w];
            }
            turn ^= 1;
        }
    }
};

template <class T, class W>
__device__ inline void load_weight(const W *w, int64_t at, int64_t cols, float none, float (&v)[CHUNK<T>])
{
    constexpr int N = CHUNK<T>;
    if (!w) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = none;
    } else if constexpr (CHUNK<W> == N) {
        load_chunk<W>(w + at, cols - at, v);
    } else {  // 32-bit weights beside a 16-bit type: two chunks
        static_assert(2 * CHUNK<W> == N);
        float a[CHUNK<W>], b[CHUNK<W>];
        load_chunk<W>(w + at, cols - at, a);
        load_chunk<W>(w + at + CHUNK<W>, cols - at - CHUNK<W>, b);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            v[i] = a[i];
            v[N / 2 + i] = b[i];
        }
    }
}

// One row per LANES lanes, NV chunks of it in each.
template <class T, class W, int LANES, int NV, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_norm_fwd(int64_t rows, int cols, const T *__restrict__ x, int64_t xs,
                                                    const W *__restrict__ w, const W *__restrict__ b, float eps,
                                                    T *__restrict__ y, int64_t ys, float *__restrict__ mean,
                                                    float *__restrict__ rstd)
{
    constexpr int N = CHUNK<T>, ROWS = BLOCK / LANES;
    __shared__ typename row_sums<LANES, BLOCK, 1>::place part;
    row_sums<LANES, BLOCK, 1> sum(part);
    const int lane = threadIdx.x % LANES;
    const float n = (float)cols;  // divided by, so that a row of one value has exactly that mean
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES;
        const bool live = r < rows;  // the same in all lanes of a row; sums are taken by all
        float v[NV][N];
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
            load_chunk<T>(x + r * xs + at, live ? cols - at : 0, v[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) s[0] += v[k][i];
        }
        sum(s);
        const float m = s[0] / n;
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[k][i] -= m;
                s[0] += at + i < cols ? v[k][i] * v[k][i] : 0.0f;
            }
        }
        sum(s);
        const float inv = 1.0f / sqrtf(s[0] / n + eps);
        if (live) {
            if (lane == 0) {
                if (mean) mean[r] = m;
                if (rstd) rstd[r] = inv;
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int at = (k * LANES + lane) * N;
                if (at >= cols) continue;
                float ww[N], bb[N];
                load_weight<T>(w, at, cols, 1.0f, ww);
                load_weight<T>(b, at, cols, 0.0f, bb);
#pragma unroll
                for (int i = 0; i < N; ++i) v[k][i] = v[k][i] * inv * ww[i] + bb[i];
                store_chunk<T>(y + r * ys + at, cols - at, v[k]);
            }
        }
    }
}

// x of a backward pass: the matrix itself or its 8-bit checkpoint.
template <class T>
struct kept_matrix {
    const T *x;
    int64_t stride;
    const int8_t *codes;
    const uint8_t *exps;
};

// A chunk of it as it lies in memory.
template <class T, bool CKPT>
struct kept_chunk {
    static constexpr int N = CHUNK<T>;
    std::conditional_t<CKPT, vec<int8_t, N>, vec<T, N>> raw;
    uint8_t exp;
    __device__ void load(const kept_matrix<T> &x, int64_t r, int at, int cols, bool live)
    {
        if constexpr (!CKPT) {
            raw = load_raw<T>(x.x + r * x.stride + at, live ? cols - at : 0);
        } else {
            raw = {};
            exp = 0;
            if (live && at < cols) {  // a code row is whole groups: no partial chunk
                const int ld = (cols + GROUP - 1) / GROUP * GROUP;
                __builtin_memcpy(&raw, x.codes + r * ld + at, N);
                exp = x.exps[r * (ld / GROUP) + at / GROUP];
            }
        }
    }
    __device__ void values(float (&v)[N]) const
    {
        const float step = CKPT ? step_of(exp) : 1.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = CKPT ? (float)raw[i] * step : (float)raw[i];
    }
};

// dx of the rows that a block takes in turn, the next row's loads in flight while a row is summed; the columns' sums of
// dy xh and dy over those rows stay in registers and leave as one partial row [2, cols] per block (`sums`; no
// sums where it is NULL).
template <class T, class W, int LANES, int NV, int BLOCK, bool CKPT>
__global__ __launch_bounds__(BLOCK) void k_norm_bwd(int64_t rows, int cols, const T *__restrict__ dy, int64_t dys,
                                                    kept_matrix<T> x, const float *__restrict__ mean,
                                                    const float *__restrict__ rstd, const W *__restrict__ w,
                                                    T *__restrict__ dx, int64_t dxs, float *__restrict__ sums)
{
    constexpr int N = CHUNK<T>, ROWS = BLOCK / LANES;
    __shared__ typename row_sums<LANES, BLOCK, 2>::place part;
    constexpr int SLOTS = BLOCK / (LANES < WAVE ? WAVE : LANES);  // rows that are joined through LDS
    __shared__ __align__(16) float joined[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? LANES * NV * N : 4];
    row_sums<LANES, BLOCK, 2> sum(part);
    const int lane = threadIdx.x % LANES;
    const float n = (float)cols;
    float dw[NV][N] = {}, db[NV][N] = {}, ww[NV][N];
#pragma unroll
    for (int k = 0; k < NV; ++k) load_weight<T>(w, (k * LANES + lane) * N, cols, 1.0f, ww[k]);
    vec<T, N> next_dy[NV];
    kept_chunk<T, CKPT> next_x[NV];
    float next_m = 0.0f, next_inv = 0.0f;
    auto load = [&](int64_t r) {
        const bool live = r < rows;
        next_m = live ? mean[r] : 0.0f;
        next_inv = live ? rstd[r] : 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
            next_dy[k] = load_raw<T>(dy + r * dys + at, live ? cols - at : 0);
            next_x[k].load(x, r, at, cols, live);
        }
    };
    const int64_t step = (int64_t)gridDim.x * ROWS;
    load((int64_t)blockIdx.x * ROWS + threadIdx.x / LANES);
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < rows; r0 += step) {
        const int64_t r = r0 + threadIdx.x / LANES;
        const bool live = r < rows;
        const float m = next_m, inv = next_inv;
        float v[NV][N], xh[NV][N], s[2] = {};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[k][i] = (float)next_dy[k][i];
            next_x[k].values(xh[k]);
        }
        load(r + step);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // columns past the row's end take no part, whatever the row's statistics are
                xh[k][i] = live && at + i < cols ? (xh[k][i] - m) * inv : 0.0f;
                dw[k][i] += v[k][i] * xh[k][i];
                db[k][i] += v[k][i];
                v[k][i] *= ww[k][i];
                s[0] += v[k][i];
                s[1] += v[k][i] * xh[k][i];
            }
        }
        sum(s);
        const float s1 = s[0] / n, s2 = s[1] / n;
        if (live) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int at = (k * LANES + lane) * N;
                if (at >= cols) continue;
                float d[N];
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] = inv * (v[k][i] - s1 - xh[k][i] * s2);
                store_chunk<T>(dx + r * dxs + at, cols - at, d);
            }
        }
    }
    if (!sums) return;
    // join the rows of a wave, then the block's waves in their order, and write the block's partial sums
    if constexpr (LANES < WAVE) {
#pragma unroll
        for (int d = LANES; d < WAVE; d *= 2)
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dw[k][i] += __shfl_xor(dw[k][i], d);
                    db[k][i] += __shfl_xor(db[k][i], d);
                }
    }
    float *out = sums + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (SLOTS > 1) {
            if (which) __syncthreads();
            if (LANES >= WAVE || threadIdx.x % WAVE < LANES) {
                float *mine = joined[threadIdx.x / (BLOCK / SLOTS)];
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int i = 0; i < N; i += 4)
                        *(f32x4 *)&mine[(k * LANES + lane) * N + i] =
                            which ? f32x4{db[k][i], db[k][i + 1], db[k][i + 2], db[k][i + 3]}
                                  : f32x4{dw[k][i], dw[k][i + 1], dw[k][i + 2], dw[k][i + 3]};
            }
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += BLOCK) {
                float all = joined[0][c];
#pragma unroll
                for (int t = 1; t < SLOTS; ++t) all += joined[t][c];
                out[which * cols + c] = all;
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < N; i += 4) {
                    const int c = (k * LANES + lane) * N + i;
                    float four[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) four[e] = which ? db[k][i + e] : dw[k][i + e];
                    if (c < cols) store_chunk<float>(out + which * cols + c, cols - c, four);
                }
        }
    }
}

// Columns' sums from the blocks' partial rows: 16 shares of the rows, each in the blocks' order, for 64 columns of
// dw and db in a block.
template <class W>
__global__ __launch_bounds__(256) void k_norm_cols(int blocks, int cols, const float *__restrict__ sums,
                                                   W *__restrict__ dw, W *__restrict__ db)
{
    constexpr int SHARES = 16;
    __shared__ float share[SHARES][64];
    const int quad = threadIdx.x % 16, part = threadIdx.x / 16, c0 = blockIdx.x * 64 + quad * 4;
    W *out = blockIdx.y ? db : dw;
    if (!out) return;
    float s[4] = {};
    const float *from = sums + (int64_t)blockIdx.y * cols + c0;
#pragma unroll 8
    for (int b = part; b < blocks; b += SHARES) {
        float v[4];
        load_chunk<float>(from + (int64_t)b * 2 * cols, cols - c0, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] += v[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) share[part][quad * 4 + i] = s[i];
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= 64 || blockIdx.x * 64 + c >= cols) return;
    float all = 0.0f;
#pragma unroll
    for (int p = 0; p < SHARES; ++p) all += share[p][c];
    out[blockIdx.x * 64 + c] = (W)all;
}

// Blocks of a backward pass.  Each leaves a partial row of sums where columns' sums are wanted, so few are better: two of 256
// lanes or one of 1024 on every compute unit, and each should have several rows in turn: 1000 x 4096 (bf16)
// took 27 us with 500 blocks of one row at a time.  Not every layout's registers allow that.  64 lanes of 4 chunks in 16
// bits (1025 to 2048 columns) take 264 to 276, one block a compute unit, and half of the blocks wait: 8192 x 1280 (bf16) takes
// 37 us and 8192 x 2048 36, where 8192 x 1024 takes 18 and 8192 x 4096 43.  1024 lanes of 2 chunks in 16 bits and of 4 in 32
// (more than 8192 columns) do not fit 128: 28 to 60 and some 170 registers spill in the row loop, and 2048 x 16384 takes
// 86 us in bf16 (2.4 TB/s) and 173 in 32 bits.
int64_t bwd_blocks(int64_t rows, int rows_per_block, int block, bool want)
{
    const int64_t need = (rows + rows_per_block - 1) / rows_per_block, most = block == 256 ? 512 : 256;
    if (!want) return std::max<int64_t>(1, std::min<int64_t>(need, 4 * most));
    const int64_t in_turn = rows_per_block == 1 ? 6 : 2;
    return std::max<int64_t>(1, std::min(most, std::max(std::min<int64_t>(need, 128), need / in_turn)));
}

// The rows' layout: LANES lanes of a block of BLOCK, NV chunks each, as few lanes as keep a
// row in 4 chunks a lane.  N: elements of a chunk.  The backward pass (BWD) holds four values for each of the forward's one, and
// takes more lanes for the widest rows: 4096 x 8192 (bf16) goes in 49 us with 1024 lanes and in 75 with
// 256, its forward in 47 and 31.
template <bool BWD, int N, class F>
int with_layout(int64_t cols, F go)
{
    const int64_t chunks = (cols + N - 1) / N;
    using std::integral_constant;
#define RKB_LAYOUT(L, NV, B) return go(integral_constant<int, L>(), integral_constant<int, NV>(), integral_constant<int, B>())
    if (chunks <= 16) RKB_LAYOUT(16, 1, NORM_BLOCK);
    if (chunks <= 64) RKB_LAYOUT(64, 1, NORM_BLOCK);
    if (chunks <= 128) RKB_LAYOUT(64, 2, NORM_BLOCK);
    if (chunks <= 256) RKB_LAYOUT(64, 4, NORM_BLOCK);
    if (chunks <= 512) RKB_LAYOUT(256, 2, NORM_BLOCK);
    if (chunks <= 1024) {
        if constexpr (BWD)
            RKB_LAYOUT(1024, 1, 1024);
        else
            RKB_LAYOUT(256, 4, NORM_BLOCK);
    }
    if constexpr (N * 2048 < RKB_MAX_NORM_COLS)
        if (chunks > 2048) RKB_LAYOUT(1024, 4, 1024);
    RKB_LAYOUT(1024, 2, 1024);
#undef RKB_LAYOUT
}

template <class F>
int with_types(int dtype, int wdtype, F go)
{
    if (dtype == RKB_F32) return go((float *)nullptr, (float *)nullptr);
    if (dtype == RKB_F16) return wdtype == RKB_F32 ? go((f16 *)nullptr, (float *)nullptr) : go((f16 *)nullptr, (f16 *)nullptr);
    return wdtype == RKB_F32 ? go((bf16 *)nullptr, (float *)nullptr) : go((bf16 *)nullptr, (bf16 *)nullptr);
}

int64_t bwd_blocks_of(int dtype, int64_t rows, int64_t cols)
{
    auto blocks = [&](auto lanes, auto, auto block) { return (int)bwd_blocks(rows, block() / lanes(), block(), true); };
    return dtype == RKB_F32 ? with_layout<true, 4>(cols, blocks) : with_layout<true, 8>(cols, blocks);
}

bool good_norm(int dtype, int wdtype, int64_t rows, int64_t cols)
{
    return good_dtype(dtype) && (wdtype == dtype || wdtype == RKB_F32) && good_size(rows, cols) && cols <= RKB_MAX_NORM_COLS;
}

bool aligned_or_null(const void *p, int size) { return (uintptr_t)p % size == 0; }

}  // namespace
}  // namespace rkb

using namespace rkb;

extern "C" int rkb_layer_norm_fwd(int dtype, int wdtype, int64_t rows, int64_t cols, const void *x, int64_t x_stride,
                                  const void *w, const void *b, float eps, void *y, int64_t y_stride, float *mean,
                                  float *rstd, void *stream)
{
    if (!good_norm(dtype, wdtype, rows, cols) || !(eps >= 0.0f) || !(eps < INFINITY)) return RKB_E_INVAL;
    const int size = dtype_size(dtype), wsize = dtype_size(wdtype);
    if (!good_input(x, rows, x_stride, size) || !good_output(y, rows, cols, y_stride, size) ||
        !aligned_or_null(w, wsize) || !aligned_or_null(b, wsize) || !aligned_or_null(mean, 4) || !aligned_or_null(rstd, 4))
        return RKB_E_INVAL;
    if (rows == 0) return RKB_OK;
    return with_types(dtype, wdtype, [&](auto *t, auto *wt) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(wt)>;
        return with_layout<false, CHUNK<T>>(cols, [&](auto lanes, auto nv, auto block) {
            constexpr int ROWS = block() / lanes();
            // a launch's lanes are counted in 32 bits: more rows go in turn
            const int64_t blocks = std::min<int64_t>((rows + ROWS - 1) / ROWS, ((int64_t)1 << 30) / block());
            return launch(k_norm_fwd<T, W, lanes(), nv(), block()>, dim3((uint32_t)blocks), dim3(block()), (hipStream_t)stream, rows,
                          (int)cols, (const T *)x, x_stride, (const W *)w, (const W *)b, eps, (T *)y, y_stride, mean, rstd);
        });
    });
}

extern "C" int rkb_layer_norm_bwd_workspace(int dtype, int64_t rows, int64_t cols, size_t *bytes)
{
    if (!bytes || !good_norm(dtype, dtype, rows, cols)) return RKB_E_INVAL;
    *bytes = (size_t)bwd_blocks_of(dtype, rows, cols) * 2 * cols * sizeof(float);
    return RKB_OK;
}

extern "C" int rkb_layer_norm_bwd(int dtype, int wdtype, int64_t rows, int64_t cols, const void *dy, int64_t dy_stride,
                                  const void *x, int64_t x_stride, const int8_t *codes, const uint8_t *exps,
                                  const float *mean, const float *rstd, const void *w, void *dx, int64_t dx_stride,
                                  void *dw, void *db, void *workspace, size_t ws_bytes, void *stream)
{
    if (!good_norm(dtype, wdtype, rows, cols)) return RKB_E_INVAL;
    const int size = dtype_size(dtype), wsize = dtype_size(wdtype);
    const bool ckpt = codes != nullptr;
    if (!good_input(dy, rows, dy_stride, size) || !good_output(dx, rows, cols, dx_stride, size) ||
        !aligned_or_null(w, wsize) || !aligned_or_null(dw, wsize) || !aligned_or_null(db, wsize))
        return RKB_E_INVAL;
    if (rows > 0) {
        if (!mean || !rstd || !aligned_or_null(mean, 4) || !aligned_or_null(rstd, 4)) return RKB_E_INVAL;
        if (ckpt ? (x || !exps || (uintptr_t)codes % 16) : (exps || !good_input(x, rows, x_stride, size)))
            return RKB_E_INVAL;
    }
    const bool want = dw || db;
    if (want) {
        size_t need = 0;
        rkb_layer_norm_bwd_workspace(dtype, rows, cols, &need);
        if (!workspace || (uintptr_t)workspace % 256) return RKB_E_INVAL;
        if (ws_bytes < need) return RKB_E_NOMEM;
    } else if (rows == 0) {
        return RKB_OK;
    }
    float *sums = want ? (float *)workspace : nullptr;
    return with_types(dtype, wdtype, [&](auto *t, auto *wt) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(wt)>;
        const kept_matrix<T> kept{(const T *)x, x_stride, codes, exps};
        const hipStream_t st = (hipStream_t)stream;
        int64_t blocks = 0;
        int rc = with_layout<true, CHUNK<T>>(cols, [&](auto lanes, auto nv, auto block) {
            blocks = bwd_blocks(rows, block() / lanes(), block(), want);
            auto go = [&](auto kernel) {
                return launch(kernel, dim3((uint32_t)blocks), dim3(block()), st, rows, (int)cols, (const T *)dy, dy_stride, kept, mean,
                              rstd, (const W *)w, (T *)dx, dx_stride, sums);
            };
            return ckpt ? go(k_norm_bwd<T, W, lanes(), nv(), block(), true>) : go(k_norm_bwd<T, W, lanes(), nv(), block(), false>);
        });
        if (rc != RKB_OK || !want) return rc;
        return launch(k_norm_cols<W>, dim3((uint32_t)((cols + 63) / 64), 2), dim3(256), st, (int)blocks, (int)cols, sums, (W *)dw,
                      (W *)db);
    });
}
