// Checkpoints of activations in 8 bits: save and load (rk_block.h).
//
// Bound by memory: saving reads the matrix and writes its codes and exponents (17/32 of a
// 16-bit matrix), loading the reverse.  The step is a power of two taken from the maximum's bits,
// so neither way divides and both are exact but for the one rounding to a code.  Saving, a
// lane holds 16 columns: a group's maximum is one exchange between two lanes and codes leave 16
// bytes at a time.  Loading, it holds the 16 bytes of x that it stores, so that a wave's stores are
// contiguous.  At 16384 x 4096 (bf16) saving moves 6.0 TB/s (5.2 with 8 columns a lane) and loading
// 6.5; at 8192 x 4096 in 32 bits loading moves 6.4 (3.9 with 16 columns a lane).
#include <algorithm>

#include "rkb_common.h"

namespace rkb {
namespace {

constexpr int CKPT_BLOCK = 256, SAVE_SPAN = 16;

// Where a lane works: each block takes `rows_per_block` rows by up to 256 spans (a lane's columns).
struct span_map {
    int64_t rows, cols, ld;
    int spans, rows_per_block, magic;  // spans of a row; magic = ceil(65536 / min(spans, 256))
};

template <int SPAN>
__device__ inline void place(const span_map &m, int64_t row0, int64_t &row, int64_t &col, bool &live)
{
    const int t = threadIdx.x;
    // t / spans for t < 256 and spans <= 256: the product's error stays below one span's share
    const int r = m.spans < CKPT_BLOCK ? (t * m.magic) >> 16 : 0;
    const int s = m.spans < CKPT_BLOCK ? t - r * m.spans : (int)blockIdx.y * CKPT_BLOCK + t;
    row = row0 + r;
    col = (int64_t)s * SPAN;
    live = r < m.rows_per_block && row < m.rows && s < m.spans;
}

template <class T>
__global__ __launch_bounds__(CKPT_BLOCK) void k_ckpt_save(span_map m, const T *__restrict__ x, int64_t xs,
                                                          int8_t *__restrict__ codes, uint8_t *__restrict__ exps)
{
    constexpr int N = CHUNK<T>, SPAN = SAVE_SPAN, K = SPAN / N;
    for (int64_t row0 = (int64_t)blockIdx.x * m.rows_per_block; row0 < m.rows; row0 += (int64_t)gridDim.x * m.rows_per_block) {
        int64_t row, col;
        bool live;
        place<SPAN>(m, row0, row, col, live);
        float v[K][N];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            load_chunk<T>(x + row * xs + col + k * N, live ? m.cols - col - k * N : 0, v[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) top = max_bits(top, v[k][i]);
        }
        // spans come in pairs (a code row is whole groups), and a pair in neighbouring lanes
        top = max(top, dpp<DPP_XOR1>(top));
        if (!live) continue;
        const float most = __uint_as_float(top);
        const bool ok = finite(most);
        const int e = ok ? step_exp(most) : 0;
        float flat[SPAN];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) flat[k * N + i] = v[k][i];
        *(vec<uint32_t, SPAN / 4> *)(codes + row * m.ld + col) = codes_of<SPAN>(flat, ok ? two_to(-e) : 0.0f, e > CODE_TOP_EXP<T>);
        if (col % GROUP == 0) exps[row * (m.ld / GROUP) + col / GROUP] = ok ? (uint8_t)(e + 127) : (uint8_t)255;
    }
}

template <class T>
__global__ __launch_bounds__(CKPT_BLOCK) void k_ckpt_load(span_map m, const int8_t *__restrict__ codes,
                                                          const uint8_t *__restrict__ exps, T *__restrict__ x, int64_t xs)
{
    constexpr int N = CHUNK<T>;
    for (int64_t row0 = (int64_t)blockIdx.x * m.rows_per_block; row0 < m.rows; row0 += (int64_t)gridDim.x * m.rows_per_block) {
        int64_t row, col;
        bool live;
        place<N>(m, row0, row, col, live);
        if (!live) continue;
        const vec<int8_t, N> q = *(const vec<int8_t, N> *)(codes + row * m.ld + col);
        const float step = step_of(exps[row * (m.ld / GROUP) + col / GROUP]);
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (float)q[i] * step;
        store_chunk<T>(x + row * xs + col, m.cols - col, v);
    }
}

span_map make_map(int64_t rows, int64_t cols, int span)
{
    const int64_t ld = code_ld(cols);
    span_map m{rows, cols, ld, (int)(ld / span), 1, 0};
    if (m.spans < CKPT_BLOCK) {
        m.rows_per_block = CKPT_BLOCK / m.spans;
        m.magic = (65536 + m.spans - 1) / m.spans;
    }
    return m;
}

dim3 map_grid(const span_map &m)
{
    const int64_t blocks = (m.rows + m.rows_per_block - 1) / m.rows_per_block;
    return dim3((uint32_t)std::min<int64_t>(blocks, 1 << 20), (uint32_t)((m.spans + CKPT_BLOCK - 1) / CKPT_BLOCK));
}

}  // namespace
}  // namespace rkb

using namespace rkb;

extern "C" int rkb_ckpt8_save(int dtype, int64_t rows, int64_t cols, const void *x, int64_t x_stride, int8_t *codes,
                              uint8_t *exps, void *stream)
{
    if (!good_dtype(dtype) || !good_size(rows, cols) || !good_input(x, rows, x_stride, dtype_size(dtype)))
        return RKB_E_INVAL;
    if (rows == 0) return RKB_OK;
    if (!codes || !exps || (uintptr_t)codes % 16) return RKB_E_INVAL;
    const span_map m = make_map(rows, cols, SAVE_SPAN);
    auto go = [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return launch(k_ckpt_save<T>, map_grid(m), dim3(CKPT_BLOCK), (hipStream_t)stream, m, (const T *)x, x_stride, codes, exps);
    };
    return dtype == RKB_F32 ? go((float *)nullptr) : dtype == RKB_F16 ? go((f16 *)nullptr) : go((bf16 *)nullptr);
}

extern "C" int rkb_ckpt8_load(int dtype, int64_t rows, int64_t cols, const int8_t *codes, const uint8_t *exps, void *x,
                              int64_t x_stride, void *stream)
{
    if (!good_dtype(dtype) || !good_size(rows, cols) || !good_output(x, rows, cols, x_stride, dtype_size(dtype)))
        return RKB_E_INVAL;
    if (rows == 0) return RKB_OK;
    if (!codes || !exps || (uintptr_t)codes % 16) return RKB_E_INVAL;
    const span_map m = make_map(rows, cols, dtype == RKB_F32 ? CHUNK<float> : CHUNK<f16>);
    auto go = [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return launch(k_ckpt_load<T>, map_grid(m), dim3(CKPT_BLOCK), (hipStream_t)stream, m, codes, exps, (T *)x, x_stride);
    };
    return dtype == RKB_F32 ? go((float *)nullptr) : dtype == RKB_F16 ? go((f16 *)nullptr) : go((bf16 *)nullptr);
}
