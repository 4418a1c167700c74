// Products of the gated feed-forward block and of a linear layer's weight gradient
// (rk_block.h), on the matrix units.
#include <algorithm>
#include <type_traits>

#include "rkb_common.h"

namespace rkb {
namespace {

// ------------------------------------------------------------------ activations

// act(g) and act'(g).  1 / (1 + e^-g) is taken from e^-|g|, which cannot overflow.
template <int ACT>
__device__ inline void activate(float g, float &value, float &slope)
{
    if constexpr (ACT == RKB_SILU) {
        const float t = __expf(-fabsf(g)), s = (g >= 0.0f ? 1.0f : t) / (1.0f + t);
        value = g * s;
        slope = s * (1.0f + g * (1.0f - s));
    } else {
        const float below = 0.5f * erfcf(-0.70710678f * g);
        value = g * below;
        slope = below + 0.39894228f * g * __expf(-0.5f * g * g);
    }
}

// ------------------------------------------------------------------ matrix units

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

// ------------------------------------------------------------------ what becomes of a product
//
// A wave hands out its results in units of 16 rows by 32 columns: lane l has the 8 columns
// from 8 (l / 16) of row l % 16.  A unit's columns are one checkpoint group, held by 4 lanes.
// Units reach past the matrix's edge; `row` and `col` are compared with its size here.

template <class T>
struct out_matrix {
    T *p;
    int64_t stride, rows, cols;
    __device__ void put(int64_t row, int64_t col, const float (&v)[8]) const
    {
        if (p && row < rows && col < cols) store8<T>(p + row * stride + col, cols - col, v);
    }
};

// Codes of one unit's row (4 lanes of 8 columns each).
__device__ inline void put_codes(int64_t row, int64_t col, int64_t rows, int64_t cols, int8_t *codes, uint8_t *exps,
                                 const float (&v)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_bits(top, col + i < cols ? v[i] : 0.0f);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const int64_t ld = (cols + GROUP - 1) / GROUP * GROUP;
    if (row >= rows || col >= ld) return;
    const float most = __uint_as_float(top);
    const bool ok = finite(most);
    const int e = ok ? step_exp(most) : 0;
    const float inv = ok ? two_to(-e) : 0.0f, limit = e > CODE_TOP_EXP<float> ? 63.0f : 127.0f;
    vec<int8_t, 8> q;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = ok && col + i < cols ? (int8_t)code_of(v[i], inv, limit) : (int8_t)0;
    *(vec<int8_t, 8> *)(codes + row * ld + col) = q;
    if (col % GROUP == 0) exps[row * (ld / GROUP) + col / GROUP] = ok ? (uint8_t)(e + 127) : (uint8_t)255;
}

template <class T>
struct epi_store {
    static constexpr int SUMS = 1;
    out_matrix<T> c[2];  // of the first and the second problem of a launch
    __device__ void operator()(int which, int64_t row, int64_t col, const float (&v)[8]) const { c[which].put(row, col, v); }
};

// h = act(g) u, and g and u in the form that the backward pass will read.
template <class T, int ACT, int KEEP>
struct epi_gated_fwd {
    static constexpr int SUMS = 2;
    out_matrix<T> h;
    void *g, *u;
    uint8_t *ge, *ue;
    __device__ void operator()(int, int64_t row, int64_t col, const float (&gv)[8], const float (&uv)[8]) const
    {
        float out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float value, slope;
            activate<ACT>(gv[i], value, slope);
            out[i] = value * uv[i];
        }
        h.put(row, col, out);
        if constexpr (KEEP == RKB_KEEP_FULL || KEEP == RKB_KEEP_16BIT) {
            using K = std::conditional_t<KEEP == RKB_KEEP_FULL, float, T>;
            out_matrix<K>{(K *)g, h.cols, h.rows, h.cols}.put(row, col, gv);
            out_matrix<K>{(K *)u, h.cols, h.rows, h.cols}.put(row, col, uv);
        } else if constexpr (KEEP == RKB_KEEP_8BIT) {
            put_codes(row, col, h.rows, h.cols, (int8_t *)g, ge, gv);
            put_codes(row, col, h.rows, h.cols, (int8_t *)u, ue, uv);
        }
    }
};

// dg = dh u act'(g) and du = dh act(g), rounded to T: they are operands of the next products, whose
// matrix units take T; and h again where it is asked for.
template <class T, int ACT>
__device__ inline void gated_grads(const float (&g)[8], const float (&u)[8], const float (&d)[8], float (&dg)[8],
                                   float (&du)[8], float (&h)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float value, slope;
        activate<ACT>(g[i], value, slope);
        dg[i] = d[i] * u[i] * slope;
        du[i] = d[i] * value;
        h[i] = value * u[i];
    }
}

template <class T, int ACT>
struct epi_gated_bwd {
    static constexpr int SUMS = 2;
    const T *dh;
    int64_t dhs;
    out_matrix<T> dg, du, h;
    __device__ void operator()(int, int64_t row, int64_t col, const float (&gv)[8], const float (&uv)[8]) const
    {
        if (row >= dg.rows || col >= dg.cols) return;
        float d[8], a[8], b[8], c[8];
        load8<T>(dh + row * dhs + col, dg.cols - col, d);
        gated_grads<T, ACT>(gv, uv, d, a, b, c);
        dg.put(row, col, a);
        du.put(row, col, b);
        h.put(row, col, c);
    }
};

// ------------------------------------------------------------------ products

// Element (r, k) of an operand lies at p + r * row + k * red.
template <class T>
struct operand {
    const T *p;
    int64_t row, red;
};

// C[m, n] = sum over k < K of A(m, k) B(n, k).  SUMS of the epilogue = 1: the sum of `parts` products with operand
// pairs (a[i], b[i]); 2: the products a[0] b[0] and a[0] b[1] side by side.  gridDim.z = 2 runs two
// problems, the second with a[1] (and b[0]), where parts = 1.
template <class T>
struct problem {
    operand<T> a[2], b[2];
    int64_t M, N, K;
    int parts;
};

constexpr int ST = 64, SK = 32, SPAD = 8;  // tile side, depth, and LDS padding in elements

template <class T>
__device__ inline void stage(T (&to)[ST][SK + SPAD], const operand<T> &from, int64_t r0, int64_t rows, int64_t k0, int64_t K)
{
    const bool k_near = from.red == 1;  // neighbouring lanes read neighbouring addresses
#pragma unroll
    for (int i = 0; i < ST * SK / 256; ++i) {
        const int e = i * 256 + threadIdx.x;
        const int r = k_near ? e / SK : e % ST, k = k_near ? e % SK : e / ST;
        const bool in = r0 + r < rows && k0 + k < K;
        to[r][k] = in ? from.p[(r0 + r) * from.row + (k0 + k) * from.red] : (T)0.0f;
    }
}

template <class T, class EPI>
__global__ __launch_bounds__(256) void k_simple(problem<T> pr, EPI epi)
{
    constexpr int SUMS = EPI::SUMS;
    __shared__ T as[ST][SK + SPAD], bs[SUMS][ST][SK + SPAD];
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int64_t m0 = (int64_t)blockIdx.y * ST, n0 = (int64_t)blockIdx.x * ST;
    const int which = blockIdx.z;
    f32x4 acc[SUMS][4] = {};
    for (int part = 0; part < pr.parts; ++part) {
        for (int64_t k0 = 0; k0 < pr.K; k0 += SK) {
            __syncthreads();
            stage<T>(as, pr.a[part + which], m0, pr.M, k0, pr.K);
#pragma unroll
            for (int s = 0; s < SUMS; ++s) stage<T>(bs[s], pr.b[SUMS == 2 ? s : part], n0, pr.N, k0, pr.K);
            __syncthreads();
            const int r = lane % 16, k = lane / 16 * 8;
            const frag<T> fa = *(const frag<T> *)&as[wave * 16 + r][k];
#pragma unroll
            for (int s = 0; s < SUMS; ++s)
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    // fragment f of a unit holds its columns 8 q + 4 (f % 2) + i, q = 0..3, i = 0..3
                    const int n = f / 2 * 32 + r / 4 * 8 + f % 2 * 4 + r % 4;
                    acc[s][f] = mma(*(const frag<T> *)&bs[s][n][k], fa, acc[s][f]);
                }
        }
    }
#pragma unroll
    for (int unit = 0; unit < 2; ++unit) {
        const int64_t row = m0 + wave * 16 + lane % 16, col = n0 + unit * 32 + lane / 16 * 8;
        float v[SUMS][8];
#pragma unroll
        for (int s = 0; s < SUMS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[s][i] = acc[s][unit * 2 + i / 4][i % 4];
        if constexpr (SUMS == 1)
            epi(which, row, col, v[0]);
        else
            epi(which, row, col, v[0], v[1]);
    }
}

template <class T, class EPI>
int run_problem(const problem<T> &pr, int problems, const EPI &epi, hipStream_t st)
{
    const dim3 grid((uint32_t)((pr.N + ST - 1) / ST), (uint32_t)((pr.M + ST - 1) / ST), problems);
    hipLaunchKernelGGL((k_simple<T, EPI>), grid, dim3(256), 0, st, pr, epi);
    return launched();
}

// ------------------------------------------------------------------ the backward pass's elementwise step

// dg and du from what the forward kept; a lane has 8 columns of a row.
template <class T, int ACT, int KEEP>
__global__ __launch_bounds__(256) void k_gated_grads(const T *__restrict__ dh, int64_t dhs, const void *__restrict__ g,
                                                     const void *__restrict__ u, const uint8_t *__restrict__ ge,
                                                     const uint8_t *__restrict__ ue, out_matrix<T> dg, out_matrix<T> du,
                                                     out_matrix<T> h)
{
    const int64_t rows = dg.rows, cols = dg.cols, ld = (cols + GROUP - 1) / GROUP * GROUP;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= cols) return;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        float gv[8], uv[8], d[8], a[8], b[8], c[8];
        if constexpr (KEEP == RKB_KEEP_FULL || KEEP == RKB_KEEP_16BIT) {
            using K = std::conditional_t<KEEP == RKB_KEEP_FULL, float, T>;
            load8<K>((const K *)g + row * cols + col, cols - col, gv);
            load8<K>((const K *)u + row * cols + col, cols - col, uv);
        } else {
            const vec<int8_t, 8> gq = *(const vec<int8_t, 8> *)((const int8_t *)g + row * ld + col);
            const vec<int8_t, 8> uq = *(const vec<int8_t, 8> *)((const int8_t *)u + row * ld + col);
            const float gs = step_of(ge[row * (ld / GROUP) + col / GROUP]), us = step_of(ue[row * (ld / GROUP) + col / GROUP]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                gv[i] = (float)gq[i] * gs;
                uv[i] = (float)uq[i] * us;
            }
        }
        load8<T>(dh + row * dhs + col, cols - col, d);
        gated_grads<T, ACT>(gv, uv, d, a, b, c);
        dg.put(row, col, a);
        du.put(row, col, b);
        h.put(row, col, c);
    }
}

constexpr size_t WS_ALIGN = 256;
size_t padded_bytes(int64_t rows, int64_t cols) { return (size_t)round_up(rows * cols * 2, WS_ALIGN); }

bool good_workspace(const void *ws) { return ws && (uintptr_t)ws % WS_ALIGN == 0; }

template <class F>
int with_type16(int dtype, F go)
{
    return dtype == RKB_F16 ? go((f16 *)nullptr) : go((bf16 *)nullptr);
}

template <class F>
int with_act(int act, F go)
{
    return act == RKB_SILU ? go(std::integral_constant<int, RKB_SILU>()) : go(std::integral_constant<int, RKB_GELU>());
}

template <class F>
int with_kept(int keep, F go)
{
    if (keep == RKB_KEEP_FULL) return go(std::integral_constant<int, RKB_KEEP_FULL>());
    if (keep == RKB_KEEP_16BIT) return go(std::integral_constant<int, RKB_KEEP_16BIT>());
    return go(std::integral_constant<int, RKB_KEEP_8BIT>());
}

int load_ckpt(int dtype, int64_t rows, int64_t cols, const int8_t *codes, const uint8_t *exps, void *to, void *stream)
{
    return rkb_ckpt8_load(dtype, rows, cols, codes, exps, to, cols, stream);
}

}  // namespace
}  // namespace rkb

using namespace rkb;

extern "C" int rkb_weight_grad_workspace(int dtype, int64_t rows, int64_t n, int64_t k, int ckpt, size_t *bytes)
{
    if (!bytes || !good_dtype16(dtype) || !good_size(rows, n) || !good_size(rows, k)) return RKB_E_INVAL;
    *bytes = ckpt ? padded_bytes(rows, k) : 0;
    return RKB_OK;
}

extern "C" int rkb_weight_grad(int dtype, int64_t rows, int64_t n, int64_t k, const void *dy, int64_t dy_stride,
                               const void *x, int64_t x_stride, const int8_t *codes, const uint8_t *exps, void *dw,
                               int64_t dw_stride, void *workspace, size_t ws_bytes, void *stream)
{
    size_t need = 0;
    const bool ckpt = codes != nullptr;
    int rc = rkb_weight_grad_workspace(dtype, rows, n, k, ckpt, &need);
    if (rc != RKB_OK) return rc;
    if (!good_matrix(dy, rows, n, dy_stride, 2) || !good_matrix(dw, n, k, dw_stride, 2)) return RKB_E_INVAL;
    if (rows > 0 && (ckpt ? (x || !exps || (uintptr_t)codes % 16) : (exps || !good_matrix(x, rows, k, x_stride, 2))))
        return RKB_E_INVAL;
    if (need && !good_workspace(workspace)) return RKB_E_INVAL;
    if (ws_bytes < need) return RKB_E_NOMEM;
    if (ckpt && rows > 0) {
        rc = load_ckpt(dtype, rows, k, codes, exps, workspace, stream);
        if (rc != RKB_OK) return rc;
        x = workspace;
        x_stride = k;
    }
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        problem<T> pr{{{(const T *)dy, 1, dy_stride}}, {{(const T *)x, 1, x_stride}}, n, k, rows, 1};
        return run_problem<T>(pr, 1, epi_store<T>{{{(T *)dw, dw_stride, n, k}}}, (hipStream_t)stream);
    });
}

static bool good_gated(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f)
{
    return good_dtype16(dtype) && (act == RKB_SILU || act == RKB_GELU) && keep >= RKB_KEEP_NONE && keep <= RKB_KEEP_16BIT &&
           good_size(rows, d) && good_size(rows, f);
}

// What the forward kept of g and u, as the two directions are given it.
static bool good_kept(int keep, int64_t rows, const void *g, const void *u, const uint8_t *ge, const uint8_t *ue)
{
    if (keep == RKB_KEEP_NONE) return !g && !u && !ge && !ue;
    if (rows == 0) return true;
    if (!g || !u) return false;
    const int size = keep == RKB_KEEP_FULL ? 4 : 2;
    if (keep != RKB_KEEP_8BIT) return !ge && !ue && (uintptr_t)g % size == 0 && (uintptr_t)u % size == 0;
    return ge && ue && (uintptr_t)g % 16 == 0 && (uintptr_t)u % 16 == 0;
}

extern "C" int rkb_gated_fwd_workspace(int dtype, int64_t rows, int64_t d, int64_t f, size_t *bytes)
{
    if (!bytes || !good_gated(dtype, RKB_SILU, RKB_KEEP_NONE, rows, d, f)) return RKB_E_INVAL;
    *bytes = 0;
    return RKB_OK;
}

extern "C" int rkb_gated_fwd(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f, const void *x,
                             int64_t x_stride, const void *wg, int64_t wg_stride, const void *wu, int64_t wu_stride, void *h,
                             int64_t h_stride, void *g, void *u, uint8_t *ge, uint8_t *ue, void *workspace, size_t ws_bytes,
                             void *stream)
{
    if (!good_gated(dtype, act, keep, rows, d, f) || !good_matrix(x, rows, d, x_stride, 2) ||
        !good_matrix(wg, f, d, wg_stride, 2) || !good_matrix(wu, f, d, wu_stride, 2) || !good_matrix(h, rows, f, h_stride, 2) ||
        !good_kept(keep, rows, g, u, ge, ue))
        return RKB_E_INVAL;
    if (rows == 0) return RKB_OK;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const problem<T> pr{{{(const T *)x, x_stride, 1}}, {{(const T *)wg, wg_stride, 1}, {(const T *)wu, wu_stride, 1}}, rows, f, d, 1};
        return with_act(act, [&](auto a) {
            auto go = [&](auto kind) {
                epi_gated_fwd<T, a(), kind()> epi{{(T *)h, h_stride, rows, f}, g, u, ge, ue};
                return run_problem<T>(pr, 1, epi, (hipStream_t)stream);
            };
            if (keep == RKB_KEEP_NONE) return go(std::integral_constant<int, RKB_KEEP_NONE>());
            return with_kept(keep, go);
        });
    });
}

extern "C" int rkb_gated_bwd_workspace(int dtype, int keep, int64_t rows, int64_t d, int64_t f, size_t *bytes)
{
    if (!bytes || !good_gated(dtype, RKB_SILU, keep, rows, d, f)) return RKB_E_INVAL;
    *bytes = 2 * padded_bytes(rows, f);
    return RKB_OK;
}

extern "C" int rkb_gated_bwd(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f, const void *dh,
                             int64_t dh_stride, const void *x, int64_t x_stride, const void *wg, int64_t wg_stride,
                             const void *wu, int64_t wu_stride, const void *g, const void *u, const uint8_t *ge,
                             const uint8_t *ue, void *dx, int64_t dx_stride, void *dwg, void *dwu, int64_t dw_stride, void *h,
                             int64_t h_stride, void *workspace, size_t ws_bytes, void *stream)
{
    size_t need = 0;
    if (rkb_gated_bwd_workspace(dtype, keep, rows, d, f, &need) != RKB_OK || !good_gated(dtype, act, keep, rows, d, f))
        return RKB_E_INVAL;
    if (!good_matrix(dh, rows, f, dh_stride, 2) || !good_matrix(x, rows, d, x_stride, 2) ||
        !good_matrix(wg, f, d, wg_stride, 2) || !good_matrix(wu, f, d, wu_stride, 2) || !good_kept(keep, rows, g, u, ge, ue) ||
        (dx && !good_matrix(dx, rows, d, dx_stride, 2)) || (!dwg != !dwu) ||
        (dwg && (!good_matrix(dwg, f, d, dw_stride, 2) || !good_matrix(dwu, f, d, dw_stride, 2))) ||
        (h && !good_matrix(h, rows, f, h_stride, 2)))
        return RKB_E_INVAL;
    if (need && !good_workspace(workspace)) return RKB_E_INVAL;
    if (ws_bytes < need) return RKB_E_NOMEM;
    const hipStream_t st = (hipStream_t)stream;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        T *dg = (T *)workspace, *du = (T *)((char *)workspace + padded_bytes(rows, f));
        const out_matrix<T> og{dg, f, rows, f}, ou{du, f, rows, f}, oh{(T *)h, h_stride, rows, f};
        int rc = RKB_OK;
        if (rows > 0)
            rc = with_act(act, [&](auto a) {
                if (keep == RKB_KEEP_NONE) {
                    const problem<T> pr{{{(const T *)x, x_stride, 1}}, {{(const T *)wg, wg_stride, 1}, {(const T *)wu, wu_stride, 1}}, rows, f, d, 1};
                    return run_problem<T>(pr, 1, epi_gated_bwd<T, a()>{(const T *)dh, dh_stride, og, ou, oh}, st);
                }
                const dim3 grid((uint32_t)((f + 2047) / 2048), (uint32_t)std::min<int64_t>(rows, 32768));
                auto go = [&](auto kind) {
                    hipLaunchKernelGGL((k_gated_grads<T, a(), kind()>), grid, dim3(256), 0, st, (const T *)dh, dh_stride, g, u,
                                       ge, ue, og, ou, oh);
                    return launched();
                };
                return with_kept(keep, go);
            });
        if (rc == RKB_OK && dx && rows > 0) {
            const problem<T> pr{{{dg, f, 1}, {du, f, 1}}, {{(const T *)wg, 1, wg_stride}, {(const T *)wu, 1, wu_stride}}, rows, d, f, 2};
            rc = run_problem<T>(pr, 1, epi_store<T>{{{(T *)dx, dx_stride, rows, d}}}, st);
        }
        if (rc == RKB_OK && dwg) {
            const problem<T> pr{{{dg, 1, f}, {du, 1, f}}, {{(const T *)x, 1, x_stride}}, f, d, rows, 1};
            rc = run_problem<T>(pr, 2, epi_store<T>{{{(T *)dwg, dw_stride, f, d}, {(T *)dwu, dw_stride, f, d}}}, st);
        }
        return rc;
    });
}

extern "C" const char *rkb_strerror(int code)
{
    switch (code) {
    case RKB_OK: return "ok";
    case RKB_E_INVAL: return "invalid argument";
    case RKB_E_NOMEM: return "workspace too small";
    case RKB_E_DEVICE: return "HIP call failed";
    default: return "unknown error";
    }
}
