// Products of the gated feed-forward block and of a linear layer's weight gradient
// (rk_block.h), on the matrix units.
#include <algorithm>
#include <type_traits>

#include "rkb_cut.h"
#include "rkb_tile.h"

namespace rkb {
namespace {

// ------------------------------------------------------------------ activations

// act(g) and act'(g).  1 / (1 + e^-g) is taken from e^-|g|, which cannot overflow.  Phi(-y) for y >= 0 is e^(-y^2/2)
// times a function that falls slowly from 1/2, here t P(t) with t = 1 / (1 + 0.3 y) and P of degree 7, fitted to the least largest
// relative error over 0 <= y <= 14 (1.5e-7, and 4.3e-7 as evaluated in 32 bits; the exponential's own grows with y^2 / 2, to
// 4e-6 of Phi at y = 13).  It shares its exponential with the slope;
// with the library's erfcf the forward of 5797 x 944 x 1040 took 41.8 us instead of 34.7.
template <int ACT>
__device__ inline void activate(float g, float &value, float &slope)
{
    if constexpr (ACT == RKB_SILU) {
        const float t = __expf(-fabsf(g)), s = (g >= 0.0f ? 1.0f : t) * __builtin_amdgcn_rcpf(1.0f + t);
        value = g * s;
        slope = s * (1.0f + g * (1.0f - s));
    } else {
        const float e = __expf(-0.5f * g * g), t = __builtin_amdgcn_rcpf(1.0f + 0.3f * fabsf(g));
        float p = 3.56748775e-02f;
        p = p * t + -1.57203496e-01f;
        p = p * t + 2.06354186e-01f;
        p = p * t + -5.36842421e-02f;
        p = p * t + 1.28561929e-01f;
        p = p * t + 9.99134108e-02f;
        p = p * t + 1.20753966e-01f;
        p = p * t + 1.19629301e-01f;
        p *= e * t;
        const float below = g < 0.0f ? p : 1.0f - p;
        value = g * below;
        slope = below + 0.39894228f * g * e;
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
    int64_t low = 0;  // distance to a second matrix that takes what rounding to T leaves over (0: none)
    // The same into rows whose columns go on to a multiple of 8: those past the end become 0.
    __device__ void put_padded(int64_t row, int64_t col, float (&v)[8]) const
    {
        if (row >= rows || col >= cols) return;
        const int left = (int)min(cols - col, (int64_t)8);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? v[i] : 0.0f;
        store8<T>(p + row * stride + col, 8, v);
        if (low) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float high = (float)(T)settled<T>(v[i]);
                v[i] = finite(fabsf(high)) ? v[i] - high : 0.0f;  // an infinity leaves nothing over (its difference would be NaN)
            }
            store8<T>(p + low + row * stride + col, 8, v);
        }
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
    const int left = (int)min(cols - col, (int64_t)8);
    float x[8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = i < left ? v[i] : 0.0f;
        top = max_bits(top, x[i]);
    }
    top = max_of_rows(top);
    const int64_t ld = (cols + GROUP - 1) / GROUP * GROUP;
    if (row >= rows || col >= ld) return;
    const float most = __uint_as_float(top);
    const bool ok = finite(most);
    const int e = ok ? step_exp(most) : 0;
    *(vec<uint32_t, 2> *)(codes + row * ld + col) = codes_of<8>(x, ok ? two_to(-e) : 0.0f, e > CODE_TOP_EXP<float>);
    if (col % GROUP == 0) exps[row * (ld / GROUP) + col / GROUP] = ok ? (uint8_t)(e + 127) : (uint8_t)255;
}

template <class T>
struct epi_store {
    static constexpr int SUMS = 1;
    out_matrix<T> c[2];  // of the first and the second problem of a launch
    __device__ void operator()(int which, int64_t row, int64_t col, const float (&v)[8]) const { c[which].put(row, col, v); }
};

// A split's partial sums, in 32 bits.
struct epi_part {
    static constexpr int SUMS = 1;
    float *p;
    int64_t rows, cols, ld;  // ld: cols rounded up to 8
    __device__ void operator()(int which, int64_t row, int64_t col, const float (&v)[8]) const
    {
        if (row < rows && col < cols) store8<float>(p + ((int64_t)which * rows + row) * ld + col, 8, v);
    }
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
// matrix units take T.  That adds an error like the results' own rounding (sqrt 2 of it in all), and in f16 values beyond 65504
// become infinite and below 6e-8 vanish.  Keeping what the rounding leaves over as a second operand doubles the products, so
// only few elements (FINE_ELEMENTS, where it is priced) have it.  And h again where it is asked for.
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

// Bytes of a cut's partial sums.
size_t split_bytes(const cut &c, int64_t M, int64_t N, int problems)
{
    return c.splits == 1 ? 0 : (size_t)round_up((int64_t)c.splits * problems * M * round_up(N, 8) * 4, WS_ALIGN);
}

template <class T, bool ANEAR, bool BNEAR, int PARTS, int TM, int TN, int WM, int WN, int BUFS, class EPI>
int launch_product(product pr, const cut &c, const EPI &epi, hipStream_t st)
{
    pr.tiles_m = (int)((pr.M + TM - 1) / TM);
    pr.tiles_n = (int)((pr.N + TN / EPI::SUMS - 1) / (TN / EPI::SUMS));
    const int stages = (int)((pr.K + DEPTH - 1) / DEPTH) * PARTS;
    pr.splits = c.splits;
    pr.split_stages = (stages + c.splits - 1) / c.splits;
    const int64_t total = (int64_t)pr.tiles_m * pr.tiles_n * pr.problems * pr.splits;
    if (total > MAX_TILES) return RKB_E_INVAL;
    return launch(k_product<T, EPI, TM, TN, WM, WN, BUFS, ANEAR, BNEAR, PARTS>, dim3((uint32_t)total), dim3(WM * WN * WAVE), st, pr, epi);
}

template <class T, bool ANEAR, bool BNEAR, int PARTS, class EPI>
int run_product(const product &pr, const cut &c, const EPI &epi, hipStream_t st)
{
    if (c.tm == 128)
        return c.bufs == 2 ? launch_product<T, ANEAR, BNEAR, PARTS, 128, 128, 4, 2, 2>(pr, c, epi, st)
                           : launch_product<T, ANEAR, BNEAR, PARTS, 128, 128, 4, 2, 4>(pr, c, epi, st);
    if constexpr (ANEAR)
        if (c.tm == 192) return launch_product<T, ANEAR, BNEAR, PARTS, 192, 256, 2, 4, 2>(pr, c, epi, st);
    return launch_product<T, ANEAR, BNEAR, PARTS, 256, 256, 2, 4, 2>(pr, c, epi, st);
}

// The two products of a backward pass in one launch: dx in the first `first` workgroups (they have the longer sums), the weights'
// gradients in the others.  FINE: dg and du come in two parts each.
template <class T, class EPI, int BUFS, bool FINE>
__global__ __launch_bounds__(512) void k_backward(product dx, EPI dx_epi, int first, product dw, epi_store<T> dw_epi)
{
    constexpr int X = STAGE_BYTES<T, 128, 128, 8, true, false, false>, W = STAGE_BYTES<T, 128, 128, 8, false, false, false>;
    constexpr int BYTES = X > W ? X : W;
    RKB_STAGE_BUFFERS(BYTES, BUFS);
    if ((int)blockIdx.x < first)
        product_tile<T, EPI, 128, 128, 4, 2, BUFS, true, false, FINE ? 4 : 2>(dx, dx_epi, blockIdx.x, lds);
    else
        product_tile<T, epi_store<T>, 128, 128, 4, 2, BUFS, false, false, FINE ? 2 : 1>(dw, dw_epi, blockIdx.x - first, lds);
}

// The splits' partial sums, in their order.
template <class T>
__global__ __launch_bounds__(256) void k_join(const float *__restrict__ parts, int splits, int64_t ld, epi_store<T> out)
{
    const out_matrix<T> c = out.c[blockIdx.y];
    const int64_t chunks = ld / 8, all = c.rows * chunks;
    parts += (int64_t)blockIdx.y * splits * c.rows * ld;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        float v[8] = {};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) {
            float w[8];
            load8<float>(parts + (int64_t)s * c.rows * ld + i * 8, 8, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += w[e];
        }
        const int64_t row = all >> 32 ? i / chunks : (uint32_t)i / (uint32_t)chunks;  // 64-bit division is slow
        c.put(row, (i - row * chunks) * 8, v);
    }
}

template <class T>
int join(const float *parts, int splits, int problems, const epi_store<T> &out, hipStream_t st)
{
    const int64_t ld = round_up(out.c[0].cols, 8), blocks = (out.c[0].rows * ld / 8 + 255) / 256;
    return launch(k_join<T>, dim3((uint32_t)std::min<int64_t>(blocks, 1 << 16), problems), dim3(256), st, parts, splits, ld, out);
}

// A product stored as it is; `scratch` has split_bytes.
template <class T, bool ANEAR, bool BNEAR, int PARTS>
int store_product(const product &pr, const cut &c, void *scratch, const epi_store<T> &out, hipStream_t st)
{
    if (c.splits == 1) return run_product<T, ANEAR, BNEAR, PARTS>(pr, c, out, st);
    const int64_t rows = out.c[0].rows, cols = out.c[0].cols, ld = round_up(cols, 8);
    const int rc = run_product<T, ANEAR, BNEAR, PARTS>(pr, c, epi_part{(float *)scratch, rows, cols, ld}, st);
    return rc != RKB_OK ? rc : join<T>((const float *)scratch, c.splits, pr.problems, out, st);
}

// Either product may be left out (no rows of output).
template <class T, bool FINE>
int run_pair(product dx, product dw, const pair_cut &c, void *scratch, const epi_store<T> &out_x, const epi_store<T> &out_w, hipStream_t st)
{
    auto tiles = [](product &pr, int splits, int stages) {
        pr.tiles_m = (int)((pr.M + 127) / 128);
        pr.tiles_n = (int)((pr.N + 127) / 128);
        pr.splits = splits;
        pr.split_stages = (stages + splits - 1) / splits;
        return (int64_t)pr.tiles_m * pr.tiles_n * pr.problems * splits;
    };
    const int64_t nx = tiles(dx, c.splits, (int)((dx.K + DEPTH - 1) / DEPTH) * (FINE ? 4 : 2)),
                  nw = tiles(dw, 1, (int)((dw.K + DEPTH - 1) / DEPTH) * (FINE ? 2 : 1));
    if (nx + nw > MAX_TILES) return RKB_E_INVAL;
    auto go = [&](auto epi) {
        using EPI = decltype(epi);
        auto by = [&](auto kernel) { return launch(kernel, dim3((uint32_t)(nx + nw)), dim3(512), st, dx, epi, (int)nx, dw, out_w); };
        if constexpr (!FINE)
            if (c.bufs == 4) return by(k_backward<T, EPI, 4, false>);
        return by(k_backward<T, EPI, 2, FINE>);
    };
    if (c.splits == 1 || nx == 0) return go(out_x);
    const int rc = go(epi_part{(float *)scratch, out_x.c[0].rows, out_x.c[0].cols, round_up(out_x.c[0].cols, 8)});
    return rc != RKB_OK ? rc : join<T>((const float *)scratch, c.splits, 1, out_x, st);
}

// ------------------------------------------------------------------ few rows
//
// g and u of at most 16 MT rows.  Bound by reading wg and wu once: each workgroup takes 16 NB columns of the
// hidden layer, its waves a share of d each, and a weight goes from memory to the matrix units' registers
// without a stop in LDS, whatever its alignment, the next steps' loads in flight while the present ones
// are multiplied.  The waves' sums are joined in LDS in their order.

constexpr int FEW_WAVES = 8, FEW_STEPS = 2;  // steps of 32 k that are loaded together

// 8 neighbouring k of a row, of which `left` exist (the others read as 0).
template <class T>
__device__ inline frag<T> load_frag(const T *p, int left)
{
    frag<T> v;
    if (left >= 8) {
        __builtin_memcpy(&v, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (T)0.0f;
    }
    return v;
}

template <class T, class EPI, int MT, int NB>
__global__ __launch_bounds__(FEW_WAVES *WAVE) void k_few(product pr, EPI epi)
{
    constexpr int F = 2 * NB;  // fragments of weights
    __shared__ f32x4 part[FEW_WAVES][MT][F][WAVE];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), r = lane % 16, q = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NB);
    const int K = (int)pr.K, steps = (K + 31) / 32, each = (steps + FEW_WAVES - 1) / FEW_WAVES;
    const int first = wave * each, last = min(steps, first + each);
    const T *x[MT], *w[F];
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = (const T *)pr.a[0] + min((int64_t)m * 16 + r, pr.M - 1) * pr.sa + q * 8;
#pragma unroll
    for (int f = 0; f < F; ++f)
        w[f] = (const T *)pr.b[f / NB] + min(n0 + f % NB * 16 + r, pr.N - 1) * (f < NB ? pr.sb : pr.sb2) + q * 8;
    f32x4 acc[MT][F] = {};
    frag<T> fw[2][FEW_STEPS][F], fx[2][FEW_STEPS][MT];
    auto load = [&](int at, int s) {  // steps from s on, past the share's end as zeros
#pragma unroll
        for (int i = 0; i < FEW_STEPS; ++i) {
            if (s + i >= last) {
#pragma unroll
                for (int f = 0; f < F; ++f) fw[at][i][f] = frag<T>{};
#pragma unroll
                for (int m = 0; m < MT; ++m) fx[at][i][m] = frag<T>{};
                continue;
            }
            const int k = (s + i) * 32, left = K - k - q * 8;
            if (K - k >= 32) {
#pragma unroll
                for (int f = 0; f < F; ++f) __builtin_memcpy(&fw[at][i][f], w[f] + k, 16);
#pragma unroll
                for (int m = 0; m < MT; ++m) __builtin_memcpy(&fx[at][i][m], x[m] + k, 16);
            } else {
#pragma unroll
                for (int f = 0; f < F; ++f) fw[at][i][f] = load_frag(w[f] + k, left);
#pragma unroll
                for (int m = 0; m < MT; ++m) fx[at][i][m] = load_frag(x[m] + k, left);
            }
        }
    };
    auto multiply = [&](int at) {
#pragma unroll
        for (int i = 0; i < FEW_STEPS; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int f = 0; f < F; ++f) acc[m][f] = mma(fw[at][i][f], fx[at][i][m], acc[m][f]);
    };
    load(0, first);
    for (int s = first; s < last; s += 2 * FEW_STEPS) {
        load(1, s + FEW_STEPS);
        multiply(0);
        load(0, s + 2 * FEW_STEPS);
        multiply(1);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int f = 0; f < F; ++f) part[wave][m][f][lane] = acc[m][f];
    __syncthreads();
    if (wave >= MT || q >= 2 * NB) return;
    // Column n of 16 of a fragment lies in lane n / 4 * 16 + row, element n % 4; this lane takes columns 8 q .. 8 q + 7.
    float v[2][8];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 sum = {};
#pragma unroll
            for (int from = 0; from < FEW_WAVES; ++from) sum += part[from][wave][which * NB + q / 2][(q % 2 * 2 + h) * 16 + r];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[which][h * 4 + e] = sum[e];
        }
    epi(0, wave * 16 + r, n0 + q * 8, v[0], v[1]);
}

template <class T, int NB, class EPI>
int launch_few(const product &pr, const EPI &epi, hipStream_t st)
{
    const dim3 grid((uint32_t)((pr.N + 16 * NB - 1) / (16 * NB))), block(FEW_WAVES * WAVE);
    if (pr.M <= 16) return launch(k_few<T, EPI, 1, NB>, grid, block, st, pr, epi);
    if (pr.M <= 32) return launch(k_few<T, EPI, 2, NB>, grid, block, st, pr, epi);
    return launch(k_few<T, EPI, 4, NB>, grid, block, st, pr, epi);
}

// g and u of a block, by tiles or by the few-rows form (which takes operands of any alignment).  WHOLE: the epilogue needs units
// of 32 columns (checkpoint groups).
template <class T, bool WHOLE, class EPI>
int run_sums(const product &pr, bool few, const cut &c, const EPI &epi, hipStream_t st)
{
    return few ? launch_few<T, WHOLE ? 2 : 1>(pr, epi, st) : run_product<T, true, true, 1>(pr, c, epi, st);
}

// ------------------------------------------------------------------ operands
//
// The products copy 16 bytes at a time from 16-byte aligned rows of a multiple of 8 columns.  A matrix that is laid
// out otherwise is copied into the workspace once, its rows ending in zeros: one more pass
// over that matrix (26803 x 1740: 31 us, 6 TB/s), against the many that its product makes.

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
        const int64_t r = all >> 32 ? i / j.chunks : (uint32_t)i / (uint32_t)j.chunks;  // 64-bit division is slow
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
        return launch(k_pad, dim3((uint32_t)std::min<int64_t>((most + 255) / 256, 4096), n_jobs), dim3(256), st, jobs);
    }
};

// ------------------------------------------------------------------ the backward pass's elementwise step

// dg and du from what the forward kept; a lane has 8 columns of a row.  Bound by memory: 8192 x 11264 takes 124 to 142 us
// from 8-bit checkpoints (5.2 TB/s), 172 from 16 bits and 241 from 32 (5.4 TB/s).
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
    *bytes = (ckpt || k % 8 || !aligned ? padded_bytes(rows, k) : 0) + (n % 8 || !aligned ? padded_bytes(rows, n) : 0) +
             split_bytes(choose_cut(n, k, rows, 1, 1, 1, false), n, k, 1);
    return RKB_OK;
}

extern "C" int rkb_weight_grad(int dtype, int64_t rows, int64_t n, int64_t k, const void *dy, int64_t dy_stride,
                               const void *x, int64_t x_stride, const int8_t *codes, const uint8_t *exps, void *dw,
                               int64_t dw_stride, void *workspace, size_t ws_bytes, void *stream)
{
    const bool ckpt = codes != nullptr;
    if (!good_dtype16(dtype) || !good_size(rows, n) || !good_size(rows, k) || !good_input(dy, rows, dy_stride, 2) ||
        !good_output(dw, n, k, dw_stride, 2))
        return RKB_E_INVAL;
    if (rows > 0 && (ckpt ? (x || !exps || (uintptr_t)codes % 16) : (exps || !good_input(x, rows, x_stride, 2))))
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
    const cut c = choose_cut(n, k, rows, 1, 1, 1, false);
    void *parts = ws.take(split_bytes(c, n, k, 1));
    if (ws.at != workspace && !good_workspace(workspace)) return RKB_E_INVAL;
    if (!ws.fits()) return RKB_E_NOMEM;
    int rc = ws.run(st);
    if (rc == RKB_OK && ckpt && rows > 0) rc = rkb_ckpt8_load(dtype, rows, k, codes, exps, (void *)b.p, b.stride, stream);
    if (rc != RKB_OK) return rc;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const product pr{{(const char *)a.p}, {(const char *)b.p, nullptr}, a.stride, b.stride, b.stride, round_up(n, 8), round_up(k, 8), rows, 1};
        return store_product<T, false, false, 1>(pr, c, parts, epi_store<T>{{{(T *)dw, dw_stride, n, k}}}, st);
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

// Of a backward pass, any way: a caller may want one of the two only.
static size_t backward_bytes(const backward_cut &c, int64_t rows, int64_t d, int64_t f)
{
    return std::max({split_bytes(c.x, rows, d, 1), split_bytes(c.w, f, d, 2), split_bytes(cut{128, 128, 2, c.both.splits, 0.0}, rows, d, 1)});
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
        return product{{(const char *)x.p}, {(const char *)wg.p, (const char *)wu.p}, x.stride, wg.stride, wu.stride, rows, f, d, 1};
    }
};

extern "C" int rkb_gated_fwd(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f, const void *x,
                             int64_t x_stride, const void *wg, int64_t wg_stride, const void *wu, int64_t wu_stride, void *h,
                             int64_t h_stride, void *g, void *u, uint8_t *ge, uint8_t *ue, void *workspace, size_t ws_bytes,
                             void *stream)
{
    if (!good_gated(dtype, act, keep, rows, d, f) || !good_input(x, rows, x_stride, 2) ||
        !good_input(wg, f, wg_stride, 2) || !good_input(wu, f, wu_stride, 2) || !good_output(h, rows, f, h_stride, 2) ||
        !good_kept(keep, rows, g, u, ge, ue))
        return RKB_E_INVAL;
    if (rows == 0) return RKB_OK;
    const hipStream_t st = (hipStream_t)stream;
    workspace_taker ws(workspace, ws_bytes);
    gated_operands in{{x, x_stride, rows, d}, {wg, wg_stride, f, d}, {wu, wu_stride, f, d}};
    const cut c = sums_cut(rows, d, f);
    const bool few = few_rows_win(rows, f, d, c.us);
    if (!few) in.align(ws);
    if (ws.at != workspace && !good_workspace(workspace)) return RKB_E_INVAL;
    if (!ws.fits()) return RKB_E_NOMEM;
    const int rc = ws.run(st);
    if (rc != RKB_OK) return rc;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return with_act(act, [&](auto a) {
            auto go = [&](auto kind) {
                const epi_gated_fwd<T, a(), kind()> epi{{(T *)h, h_stride, rows, f}, g, u, ge, ue};
                return run_sums<T, kind() == RKB_KEEP_8BIT>(in.sums(rows, d, f), few, c, epi, st);
            };
            if (keep == RKB_KEEP_NONE) return go(std::integral_constant<int, RKB_KEEP_NONE>());
            return with_kept(keep, go);
        });
    });
}

extern "C" int rkb_gated_bwd_workspace(int dtype, int keep, int64_t rows, int64_t d, int64_t f, int aligned, size_t *bytes)
{
    if (!bytes || !good_gated(dtype, RKB_SILU, keep, rows, d, f)) return RKB_E_INVAL;
    *bytes = (rows * f <= FINE_ELEMENTS ? 4 : 2) * padded_bytes(rows, f) + (d % 8 || !aligned ? padded_bytes(rows, d) + 2 * padded_bytes(f, d) : 0) +
             backward_bytes(backward_cut(rows, d, f), rows, d, f);
    return RKB_OK;
}

extern "C" int rkb_gated_bwd(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f, const void *dh,
                             int64_t dh_stride, const void *x, int64_t x_stride, const void *wg, int64_t wg_stride,
                             const void *wu, int64_t wu_stride, const void *g, const void *u, const uint8_t *ge,
                             const uint8_t *ue, void *dx, int64_t dx_stride, void *dwg, void *dwu, int64_t dw_stride, void *h,
                             int64_t h_stride, void *workspace, size_t ws_bytes, void *stream)
{
    if (!good_gated(dtype, act, keep, rows, d, f) || !good_input(dh, rows, dh_stride, 2) ||
        !good_input(x, rows, x_stride, 2) || !good_input(wg, f, wg_stride, 2) || !good_input(wu, f, wu_stride, 2) ||
        !good_kept(keep, rows, g, u, ge, ue) || (dx && !good_output(dx, rows, d, dx_stride, 2)) || (!dwg != !dwu) ||
        (dwg && (!good_output(dwg, f, d, dw_stride, 2) || !good_output(dwu, f, d, dw_stride, 2))) ||
        (h && !good_output(h, rows, f, h_stride, 2)))
        return RKB_E_INVAL;
    const hipStream_t st = (hipStream_t)stream;
    workspace_taker ws(workspace, ws_bytes);
    const int64_t ld = round_up(f, 8);
    const backward_cut cuts(rows, d, f);
    const size_t part = padded_bytes(rows, f);
    char *dg = (char *)ws.take(part), *du = (char *)ws.take(part);  // and what their rounding left over, at the same distance
    if (cuts.fine) ws.take(2 * part);
    gated_operands in{{x, x_stride, rows, d}, {wg, wg_stride, f, d}, {wu, wu_stride, f, d}};
    if (rows > 0) in.align(ws);
    void *parts = ws.take(backward_bytes(cuts, rows, d, f));
    if (ws.at != workspace && !good_workspace(workspace)) return RKB_E_INVAL;
    if (!ws.fits()) return RKB_E_NOMEM;
    int rc = ws.run(st);
    if (rc != RKB_OK) return rc;
    return with_type16(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const int64_t low = cuts.fine ? (int64_t)part : 0;  // 2 matrices of `part` bytes on, in elements of 2
        const out_matrix<T> og{(T *)dg, ld, rows, f, low}, ou{(T *)du, ld, rows, f, low}, oh{(T *)h, h_stride, rows, f};
        if (rows > 0)
            rc = with_act(act, [&](auto a) {
                if (keep == RKB_KEEP_NONE) {
                    const epi_gated_bwd<T, a()> epi{(const T *)dh, dh_stride, og, ou, oh};
                    const cut c = sums_cut(rows, d, f);
                    return run_sums<T, false>(in.sums(rows, d, f), few_rows_win(rows, f, d, c.us), c, epi, st);
                }
                const dim3 grid((uint32_t)((f + 2047) / 2048), (uint32_t)std::min<int64_t>(rows, 32768));
                auto go = [&](auto kind) {
                    return launch(k_gated_grads<T, a(), kind()>, grid, dim3(256), st, (const T *)dh, dh_stride, g, u, ge, ue, og, ou, oh);
                };
                return with_kept(keep, go);
            });
        if (rc != RKB_OK) return rc;
        const bool want_x = dx && rows > 0;
        const char *gl = dg + 2 * part, *ul = du + 2 * part;
        product px{{dg, du, gl, ul}, {(const char *)in.wg.p, (const char *)in.wu.p}, ld, in.wg.stride, in.wg.stride, rows, round_up(d, 8), f, 1};
        product pw{{dg, du}, {(const char *)in.x.p, nullptr}, ld, in.x.stride, in.x.stride, ld, round_up(d, 8), rows, 2};
        const epi_store<T> ox{{{(T *)dx, dx_stride, rows, d}}}, ow{{{(T *)dwg, dw_stride, f, d}, {(T *)dwu, dw_stride, f, d}}};
        if (cuts.fine) {
            if (!want_x) px.M = 0;
            if (!dwg) pw.M = 0;
            pw.a[0] = dg, pw.a[1] = gl, pw.a[2] = du, pw.a[3] = ul;
            return px.M || pw.M ? run_pair<T, true>(px, pw, cuts.both, parts, ox, ow, st) : RKB_OK;
        }
        if (want_x && dwg && cuts.together) return run_pair<T, false>(px, pw, cuts.both, parts, ox, ow, st);
        if (want_x) rc = store_product<T, true, false, 2>(px, cuts.x, parts, ox, st);
        if (rc == RKB_OK && dwg) rc = store_product<T, false, false, 1>(pw, cuts.w, parts, ow, st);
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
