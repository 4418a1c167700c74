// Layer norm, forward and backward (rk_block.h).
//
// Bound by memory: the forward reads x and writes y, the backward reads dy and x (or its 8-bit
// checkpoint) and writes dx.  A row stays in the registers of LANES lanes between the sums over it, so
// each matrix is read once; the mean is formed first and the variance from differences to
// it, which costs no second read and loses no digits where the mean is large.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "rkb_common.h"

namespace rkb {
namespace {

constexpr int NORM_BLOCK = 256;

// Sum over the lanes of one row, in every one of them.  Rows of more than a wave join their waves
// through LDS (`part`: one float per wave, and a barrier before each reuse).
template <int LANES>
__device__ inline float row_sum(float v, float *part)
{
    if constexpr (LANES <= WAVE) {
        return lane_sum<LANES>(v);
    } else {
        constexpr int WAVES = LANES / WAVE;
        v = lane_sum<WAVE>(v);
        __syncthreads();
        if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += part[w];
        return v;
    }
}

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
    __shared__ float part[LANES > WAVE ? LANES / WAVE : 1];
    const int lane = threadIdx.x % LANES;
    const float n = (float)cols;  // divided by, so that a row of one value has exactly that mean
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES;
        const bool live = r < rows;  // the same in all lanes of a row; sums are taken by all
        float v[NV][N];
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
            load_chunk<T>(x + r * xs + at, live ? cols - at : 0, v[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) s += v[k][i];
        }
        const float m = row_sum<LANES>(s, part) / n;
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[k][i] -= m;
                s += at + i < cols ? v[k][i] * v[k][i] : 0.0f;
            }
        }
        const float inv = 1.0f / sqrtf(row_sum<LANES>(s, part) / n + eps);
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

template <class T, bool CKPT>
__device__ inline void load_kept(const kept_matrix<T> &x, int64_t r, int at, int64_t cols, bool live,
                                 float (&v)[CHUNK<T>])
{
    constexpr int N = CHUNK<T>;
    if constexpr (!CKPT) {
        load_chunk<T>(x.x + r * x.stride + at, live ? cols - at : 0, v);
    } else if (live && at < cols) {  // a code row is whole groups: no partial chunk
        const int64_t ld = (cols + GROUP - 1) / GROUP * GROUP;
        vec<int8_t, N> q;
        __builtin_memcpy(&q, x.codes + r * ld + at, N);
        const float step = step_of(x.exps[r * (ld / GROUP) + at / GROUP]);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (float)q[i] * step;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.0f;
    }
}

// dx of the rows that a block takes in turn; the columns' sums of dy xh and dy over those rows stay in registers
// and leave as one partial row [2, cols] per block (`sums`; no sums where it is NULL).
template <class T, class W, int LANES, int NV, int BLOCK, bool CKPT>
__global__ __launch_bounds__(BLOCK) void k_norm_bwd(int64_t rows, int cols, const T *__restrict__ dy, int64_t dys,
                                                    kept_matrix<T> x, const float *__restrict__ mean,
                                                    const float *__restrict__ rstd, const W *__restrict__ w,
                                                    T *__restrict__ dx, int64_t dxs, float *__restrict__ sums)
{
    constexpr int N = CHUNK<T>, ROWS = BLOCK / LANES;
    __shared__ float part[LANES > WAVE ? LANES / WAVE : 1];
    __shared__ float joined[ROWS > 1 ? LANES * NV * N : 1];
    const int lane = threadIdx.x % LANES;
    const float n = (float)cols;
    float dw[NV][N] = {}, db[NV][N] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES;
        const bool live = r < rows;
        const float m = live ? mean[r] : 0.0f, inv = live ? rstd[r] : 0.0f;
        float v[NV][N], xh[NV][N];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
            load_chunk<T>(dy + r * dys + at, live ? cols - at : 0, v[k]);
            load_kept<T, CKPT>(x, r, at, cols, live, xh[k]);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * N;
            float ww[N];
            load_weight<T>(w, at, cols, 1.0f, ww);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // columns past the row's end take no part, whatever the row's statistics are
                xh[k][i] = at + i < cols ? (xh[k][i] - m) * inv : 0.0f;
                if (live) {
                    dw[k][i] += v[k][i] * xh[k][i];
                    db[k][i] += v[k][i];
                }
                v[k][i] *= ww[i];
                s1 += v[k][i];
                s2 += v[k][i] * xh[k][i];
            }
        }
        s1 = row_sum<LANES>(s1, part) / n;
        s2 = row_sum<LANES>(s2, part) / n;
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
    // join the block's rows, one after the other, and write the block's partial sums
    float *out = sums + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (ROWS > 1) {
            const int slot = threadIdx.x / LANES;
            for (int t = 0; t < ROWS; ++t) {
                __syncthreads();
                if (slot == t) {
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            float *j = &joined[(k * N + i) * LANES + lane];
                            const float mine = which ? db[k][i] : dw[k][i];
                            *j = t ? *j + mine : mine;
                        }
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += BLOCK) {
                const int k = c / (LANES * N), l = c / N % LANES, i = c % N;
                out[which * cols + c] = joined[(k * N + i) * LANES + l];
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int c = (k * LANES + lane) * N + i;
                    if (c < cols) out[which * cols + c] = which ? db[k][i] : dw[k][i];
                }
        }
    }
}

// Columns' sums from the blocks' partial rows, in the blocks' order within each of 8 shares.
template <class W>
__global__ __launch_bounds__(256) void k_norm_cols(int blocks, int cols, const float *__restrict__ sums,
                                                   W *__restrict__ dw, W *__restrict__ db)
{
    __shared__ float share[8][32];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32;
    W *out = blockIdx.y ? db : dw;
    float s = 0.0f;
    if (c < cols)
        for (int b = part; b < blocks; b += 8) s += sums[((int64_t)b * 2 + blockIdx.y) * cols + c];
    share[part][threadIdx.x % 32] = s;
    __syncthreads();
    if (part == 0 && c < cols && out) {
#pragma unroll
        for (int p = 1; p < 8; ++p) s += share[p][threadIdx.x];
        out[c] = (W)s;
    }
}

// Most blocks of a backward pass: each leaves a partial row of sums.
int64_t bwd_blocks(int64_t rows, int rows_per_block)
{
    const int64_t need = (rows + rows_per_block - 1) / rows_per_block;
    return need < 1 ? 1 : need < 512 ? need : 512;
}

// The rows' layout: LANES lanes of a block of BLOCK, NV chunks each, as few lanes as keep a
// row in 4 chunks a lane.  N: elements of a chunk.
template <int N, class F>
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
    if (chunks <= 1024) RKB_LAYOUT(256, 4, NORM_BLOCK);
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

int rows_per_block(int dtype, int64_t cols)
{
    auto rows = [](auto lanes, auto, auto block) { return block() / lanes(); };
    return dtype == RKB_F32 ? with_layout<4>(cols, rows) : with_layout<8>(cols, rows);
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
    if (!good_matrix(x, rows, cols, x_stride, size) || !good_matrix(y, rows, cols, y_stride, size) ||
        !aligned_or_null(w, wsize) || !aligned_or_null(b, wsize) || !aligned_or_null(mean, 4) || !aligned_or_null(rstd, 4))
        return RKB_E_INVAL;
    if (rows == 0) return RKB_OK;
    return with_types(dtype, wdtype, [&](auto *t, auto *wt) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(wt)>;
        return with_layout<CHUNK<T>>(cols, [&](auto lanes, auto nv, auto block) {
            constexpr int ROWS = block() / lanes();
            const int64_t blocks = std::min<int64_t>((rows + ROWS - 1) / ROWS, (int64_t)1 << 22);
            hipLaunchKernelGGL((k_norm_fwd<T, W, lanes(), nv(), block()>), dim3((uint32_t)blocks), dim3(block()), 0,
                               (hipStream_t)stream, rows, (int)cols, (const T *)x, x_stride, (const W *)w, (const W *)b,
                               eps, (T *)y, y_stride, mean, rstd);
            return launched();
        });
    });
}

extern "C" int rkb_layer_norm_bwd_workspace(int dtype, int64_t rows, int64_t cols, size_t *bytes)
{
    if (!bytes || !good_norm(dtype, dtype, rows, cols)) return RKB_E_INVAL;
    *bytes = (size_t)bwd_blocks(rows, rows_per_block(dtype, cols)) * 2 * cols * sizeof(float);
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
    if (!good_matrix(dy, rows, cols, dy_stride, size) || !good_matrix(dx, rows, cols, dx_stride, size) ||
        !aligned_or_null(w, wsize) || !aligned_or_null(dw, wsize) || !aligned_or_null(db, wsize))
        return RKB_E_INVAL;
    if (rows > 0) {
        if (!mean || !rstd || !aligned_or_null(mean, 4) || !aligned_or_null(rstd, 4)) return RKB_E_INVAL;
        if (ckpt ? (x || !exps || (uintptr_t)codes % 16) : (exps || !good_matrix(x, rows, cols, x_stride, size)))
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
        int rc = with_layout<CHUNK<T>>(cols, [&](auto lanes, auto nv, auto block) {
            blocks = bwd_blocks(rows, block() / lanes());
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(block()), 0, st, rows, (int)cols, (const T *)dy,
                                   dy_stride, kept, mean, rstd, (const W *)w, (T *)dx, dx_stride, sums);
            };
            if (ckpt)
                go(k_norm_bwd<T, W, lanes(), nv(), block(), true>);
            else
                go(k_norm_bwd<T, W, lanes(), nv(), block(), false>);
            return launched();
        });
        if (rc != RKB_OK || !want) return rc;
        hipLaunchKernelGGL((k_norm_cols<W>), dim3((uint32_t)((cols + 31) / 32), 2), dim3(256), 0, st, (int)blocks,
                           (int)cols, sums, (W *)dw, (W *)db);
        return launched();
    });
}
