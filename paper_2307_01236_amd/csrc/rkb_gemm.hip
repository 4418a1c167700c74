// Products of the gated feed-forward block and of a linear layer's weight gradient
// (rk_block.h), on the matrix units.
#include <algorithm>
#include <type_traits>

#include "rkb_tile.h"

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

// ------------------------------------------------------------------ what becomes of a product
//
// A wave hands out its results in units of 16 rows by 32 columns: lane l has 8 neighbouring columns of
// row l % 16.  A unit's columns are one checkpoint group, held by the lanes l, l + 16, l + 32 and l + 48.
// Units reach past the matrix's edge; `row` and `col` are compared with its size here.

template <class T>
struct out_matrix {
    T *p;
    int64_t stride, rows, cols;
    // The same into rows whose columns go on to a multiple of 8: those past the end become 0.
    __device__ void put_padded(int64_t row, int64_t col, float (&v)[8]) const
    {
        if (row >= rows || col >= cols) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? v[i] : 0.0f;
        store8<T>(p + row * stride + col, 8, v);
    }
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
        dg.put_padded(row, col, a);
        du.put_padded(row, col, b);
        h.put(row, col, c);
    }
};

constexpr size_t WS_ALIGN = 256;

// ------------------------------------------------------------------ products

template <class T, class EPI, int TM, int TN, int WM, int WN, bool ANEAR, bool BNEAR>
int launch_product(product pr, const EPI &epi, hipStream_t st)
{
    pr.tiles_m = (int)((pr.M + TM - 1) / TM);
    pr.tiles_n = (int)((pr.N + TN / EPI::SUMS - 1) / (TN / EPI::SUMS));
    pr.splits = 1;
    pr.split_stages = (int)((pr.K + DEPTH - 1) / DEPTH) * pr.parts;
    const int64_t total = (int64_t)pr.tiles_m * pr.tiles_n * pr.problems * pr.splits;
    hipLaunchKernelGGL((k_product<T, EPI, TM, TN, WM, WN, ANEAR, BNEAR>), dim3((uint32_t)total), dim3(WM * WN * WAVE), 0, st,
                       pr, epi);
    return launched();
}

template <class T, bool ANEAR, bool BNEAR, class EPI>
int run_product(const product &pr, const EPI &epi, hipStream_t st)
{
    return launch_product<T, EPI, 128, 128, 2, 2, ANEAR, BNEAR>(pr, epi, st);
}

// ------------------------------------------------------------------ operands
//
// The products copy 16 bytes at a time from 16-byte aligned rows of a multiple of 8 columns.  A matrix that is laid
// out otherwise is copied into the workspace once, its rows ending in zeros: one more pass
// over that matrix, against the many that its product makes.

constexpr int64_t STRIDE_LIMIT = (int64_t)1 << 22;  // 256 rows' offsets stay in 32 bits

struct matrix {
    const void *p;
    int64_t stride, rows, cols;
    bool aligned() const
    {
        return cols % 8 == 0 && (uintptr_t)p % 16 == 0 && (rows <= 1 || (stride % 8 == 0 && stride <= STRIDE_LIMIT));
    }
};

size_t padded_bytes(int64_t rows, int64_t cols) { return (size_t)round_up(rows * round_up(cols, 8) * 2, WS_ALIGN); }

struct pad_job {
    const uint16_t *from;
    uint16_t *to;
    int64_t stride, rows;
    int cols, chunks;
};
struct pad_jobs {
    pad_job job[3];
};

__global__ __launch_bounds__(256) void k_pad(pad_jobs jobs)
{
    const pad_job j = jobs.job[blockIdx.y];
    const int64_t all = j.rows * j.chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / j.chunks;
        const int c = (int)(i - r * j.chunks) * 8, left = j.cols - c;
        const uint16_t *from = j.from + r * j.stride + c;
        vec<uint16_t, 8> v;
        if (left >= 8) {
            __builtin_memcpy(&v, from, 16);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < left ? from[e] : (uint16_t)0;
        }
        *(vec<uint16_t, 8> *)(j.to + i * 8) = v;
    }
}

// Takes scratch memory in order, and replaces matrices that are not aligned by copies in it.
struct workspace_taker {
    char *at, *end;
    pad_jobs jobs;
    int n_jobs = 0;

    workspace_taker(void *ws, size_t bytes) : at((char *)ws), end((char *)ws + bytes) {}
    void *take(size_t bytes)
    {
        char *p = at;
        at += bytes;
        return p;
    }
    bool fits() const { return at <= end; }
    void align(matrix &m, bool force = false)
    {
        if (m.rows <= 1) m.stride = round_up(m.cols, 8);
        if (m.rows == 0 || (m.aligned() && !force)) return;
        const int64_t ld = round_up(m.cols, 8);
        void *to = take(padded_bytes(m.rows, m.cols));
        jobs.job[n_jobs++] = pad_job{(const uint16_t *)m.p, (uint16_t *)to, m.stride, m.rows, (int)m.cols, (int)(ld / 8)};
        m.p = to;
        m.stride = ld;
    }
    int run(hipStream_t st)
    {
        if (!n_jobs) return RKB_OK;
        int64_t most = 0;
        for (int i = 0; i < n_jobs; ++i) most = std::max(most, jobs.job[i].rows * jobs.job[i].chunks);
        hipLaunchKernelGGL(k_pad, dim3((uint32_t)std::min<int64_t>((most + 255) / 256, 4096), n_jobs), dim3(256), 0, st, jobs);
        return launched();
    }
};

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
        dg.put_padded(row, col, a);
        du.put_padded(row, col, b);
        h.put(row, col, c);
    }
}

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

}  // namespace
}  // namespace rkb

using namespace rkb;

extern "C" int rkb_weight_grad_workspace(int dtype, int64_t rows, int64_t n, int64_t k, int ckpt, int aligned, size_t *bytes)
{
    if (!bytes || !good_dtype16(dtype) || !good_size(rows, n) || !good_size(rows, k)) return RKB_E_INVAL;
    *bytes = (ckpt || k % 8 || !aligned ? padded_bytes(rows, k) : 0) + (n % 8 || !aligned ? padded_bytes(rows, n) : 0);
    return RKB_OK;
}

extern "C" int rkb_weight_grad(int dtype, int64_t rows, int64_t n, int64_t k, const void *dy, int64_t dy_stride,
                               const void *x, int64_t x_stride, const int8_t *codes, const uint8_t *exps, void *dw,
                               int64_t dw_stride, void *workspace, size_t ws_bytes, void *stream)
{
    const bool ckpt = codes != nullptr;
    if (!good_dtype16(dtype) || !good_size(rows, n) || !good_size(rows, k) || !good_matrix(dy, rows, n, dy_stride, 2) ||
        !good_matrix(dw, n, k, dw_stride, 2))
        return RKB_E_INVAL;
    if (rows > 0 && (ckpt ? (x || !exps || (uintptr_t)codes % 16) : (exps || !good_matrix(x, rows, k, x_stride, 2))))
        return RKB_E_INVAL;
    const hipStream_t st = (hipStream_t)stream;
    workspace_taker ws(workspace, ws_bytes);
    matrix a{dy, dy_stride, rows, n}, b{x, x_stride, rows, k};
    if (ckpt && rows > 0) {
        b.p = ws.take(padded_bytes(rows, k));
        b.stride = round_up(k, 8);
    } else {
        ws.align(b);
    }
    ws.align(a);
    if (ws.at != workspace && !good_workspace(workspace)) return RKB_E_INVAL;
    if (!ws.fits()) return RKB_E_NOMEM;
    int rc = ws.run(st);
    if (rc == RKB_OK && ckpt && rows > 0) rc = rkb_ckpt8_load(dtype, rows, k, codes, exps, (void *)b.p, b.stride, stream);
    if (rc != RKB_OK) return rc;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const product pr{{(const char *)a.p, nullptr}, {(const char *)b.p, nullptr}, a.stride, b.stride, round_up(n, 8), round_up(k, 8), rows, 1, 1};
        return run_product<T, false, false>(pr, epi_store<T>{{{(T *)dw, dw_stride, n, k}}}, st);
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

extern "C" int rkb_gated_fwd_workspace(int dtype, int64_t rows, int64_t d, int64_t f, int aligned, size_t *bytes)
{
    if (!bytes || !good_gated(dtype, RKB_SILU, RKB_KEEP_NONE, rows, d, f)) return RKB_E_INVAL;
    *bytes = d % 8 || !aligned ? padded_bytes(rows, d) + 2 * padded_bytes(f, d) : 0;
    return RKB_OK;
}

// x, wg and wu as the products take them.
struct gated_operands {
    matrix x, wg, wu;
    void align(workspace_taker &ws)
    {
        ws.align(x);
        ws.align(wg);
        ws.align(wu);
        // a launch's pairs share their strides
        if (wg.stride != wu.stride) {
            if (wg.stride != round_up(wg.cols, 8)) ws.align(wg, true);
            if (wu.stride != round_up(wu.cols, 8)) ws.align(wu, true);
        }
    }
    product sums(int64_t rows, int64_t d, int64_t f) const  // g and u
    {
        return product{{(const char *)x.p, nullptr}, {(const char *)wg.p, (const char *)wu.p}, x.stride, wg.stride, rows, f, round_up(d, 8), 1, 1};
    }
};

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
    const hipStream_t st = (hipStream_t)stream;
    workspace_taker ws(workspace, ws_bytes);
    gated_operands in{{x, x_stride, rows, d}, {wg, wg_stride, f, d}, {wu, wu_stride, f, d}};
    in.align(ws);
    if (ws.at != workspace && !good_workspace(workspace)) return RKB_E_INVAL;
    if (!ws.fits()) return RKB_E_NOMEM;
    const int rc = ws.run(st);
    if (rc != RKB_OK) return rc;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return with_act(act, [&](auto a) {
            auto go = [&](auto kind) {
                const epi_gated_fwd<T, a(), kind()> epi{{(T *)h, h_stride, rows, f}, g, u, ge, ue};
                return run_product<T, true, true>(in.sums(rows, d, f), epi, st);
            };
            if (keep == RKB_KEEP_NONE) return go(std::integral_constant<int, RKB_KEEP_NONE>());
            return with_kept(keep, go);
        });
    });
}

extern "C" int rkb_gated_bwd_workspace(int dtype, int keep, int64_t rows, int64_t d, int64_t f, int aligned, size_t *bytes)
{
    if (!bytes || !good_gated(dtype, RKB_SILU, keep, rows, d, f)) return RKB_E_INVAL;
    *bytes = 2 * padded_bytes(rows, f) + (d % 8 || !aligned ? padded_bytes(rows, d) + 2 * padded_bytes(f, d) : 0);
    return RKB_OK;
}

extern "C" int rkb_gated_bwd(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f, const void *dh,
                             int64_t dh_stride, const void *x, int64_t x_stride, const void *wg, int64_t wg_stride,
                             const void *wu, int64_t wu_stride, const void *g, const void *u, const uint8_t *ge,
                             const uint8_t *ue, void *dx, int64_t dx_stride, void *dwg, void *dwu, int64_t dw_stride, void *h,
                             int64_t h_stride, void *workspace, size_t ws_bytes, void *stream)
{
    if (!good_gated(dtype, act, keep, rows, d, f) || !good_matrix(dh, rows, f, dh_stride, 2) ||
        !good_matrix(x, rows, d, x_stride, 2) || !good_matrix(wg, f, d, wg_stride, 2) || !good_matrix(wu, f, d, wu_stride, 2) ||
        !good_kept(keep, rows, g, u, ge, ue) || (dx && !good_matrix(dx, rows, d, dx_stride, 2)) || (!dwg != !dwu) ||
        (dwg && (!good_matrix(dwg, f, d, dw_stride, 2) || !good_matrix(dwu, f, d, dw_stride, 2))) ||
        (h && !good_matrix(h, rows, f, h_stride, 2)))
        return RKB_E_INVAL;
    const hipStream_t st = (hipStream_t)stream;
    workspace_taker ws(workspace, ws_bytes);
    const int64_t ld = round_up(f, 8);
    void *dg = ws.take(padded_bytes(rows, f)), *du = ws.take(padded_bytes(rows, f));
    gated_operands in{{x, x_stride, rows, d}, {wg, wg_stride, f, d}, {wu, wu_stride, f, d}};
    if (rows > 0) in.align(ws);
    if (ws.at != workspace && !good_workspace(workspace)) return RKB_E_INVAL;
    if (!ws.fits()) return RKB_E_NOMEM;
    int rc = ws.run(st);
    if (rc != RKB_OK) return rc;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const out_matrix<T> og{(T *)dg, ld, rows, f}, ou{(T *)du, ld, rows, f}, oh{(T *)h, h_stride, rows, f};
        if (rows > 0)
            rc = with_act(act, [&](auto a) {
                if (keep == RKB_KEEP_NONE)
                    return run_product<T, true, true>(in.sums(rows, d, f), epi_gated_bwd<T, a()>{(const T *)dh, dh_stride, og, ou, oh}, st);
                const dim3 grid((uint32_t)((f + 2047) / 2048), (uint32_t)std::min<int64_t>(rows, 32768));
                auto go = [&](auto kind) {
                    hipLaunchKernelGGL((k_gated_grads<T, a(), kind()>), grid, dim3(256), 0, st, (const T *)dh, dh_stride, g, u,
                                       ge, ue, og, ou, oh);
                    return launched();
                };
                return with_kept(keep, go);
            });
        if (rc == RKB_OK && dx && rows > 0) {
            const product pr{{(const char *)dg, (const char *)du}, {(const char *)in.wg.p, (const char *)in.wu.p}, ld, in.wg.stride, rows, round_up(d, 8), f, 2, 1};
            rc = run_product<T, true, false>(pr, epi_store<T>{{{(T *)dx, dx_stride, rows, d}}}, st);
        }
        if (rc == RKB_OK && dwg) {
            const product pr{{(const char *)dg, (const char *)du}, {(const char *)in.x.p, nullptr}, ld, in.x.stride, ld, round_up(d, 8), rows, 1, 2};
            rc = run_product<T, false, false>(pr, epi_store<T>{{{(T *)dwg, dw_stride, f, d}, {(T *)dwu, dw_stride, f, d}}}, st);
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
