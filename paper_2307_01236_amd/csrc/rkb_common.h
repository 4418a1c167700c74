// Shared by the kernels of librkblock (rk_block.h): types, 16-byte row chunks, sums over
// lanes, and the arithmetic of the 8-bit checkpoints.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <tuple>
#include <type_traits>

#include "rk_block.h"

namespace rkb {

using bf16 = __bf16;
using f16 = _Float16;
template <class T, int N>
using vec = T __attribute__((ext_vector_type(N)));
using f32x4 = vec<float, 4>;
using f32x8 = vec<float, 8>;
using u32x4 = vec<uint32_t, 4>;

constexpr int WAVE = 64;
constexpr int GROUP = RKB_GROUP;

template <class T>
constexpr int CHUNK = 16 / sizeof(T);  // elements of a 16-byte chunk

// Largest power of two 2^e at which a group's codes may pass 63 (see rk_block.h): above it
// 64 * 2^e is no finite value of T.
template <class T>
inline constexpr int CODE_TOP_EXP = 121;  // bf16 and f32: 64 * 2^122 = 2^128
template <>
inline constexpr int CODE_TOP_EXP<f16> = 9;  // 64 * 2^10 = 65536

// Chunk of a row, `left` of whose elements exist (any number; the others read as 0).  The
// pointer has the alignment of T only: global loads take any address on gfx950.
template <class T>
__device__ inline vec<T, CHUNK<T>> load_raw(const T *p, int64_t left)
{
    constexpr int N = CHUNK<T>;
    vec<T, N> t;
    if (left >= N) {
        __builtin_memcpy(&t, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = i < left ? p[i] : (T)0.0f;
    }
    return t;
}

template <class T>
__device__ inline void load_chunk(const T *p, int64_t left, float (&v)[CHUNK<T>])
{
    const auto t = load_raw<T>(p, left);
#pragma unroll
    for (int i = 0; i < CHUNK<T>; ++i) v[i] = (float)t[i];
}

// A 32-bit result before it is rounded to T.  The compiler may fold a product into its rounding to
// f16 in one place and not in another (one rounding or two); here it is two everywhere, so that what
// is made again is bit for bit what it was.
template <class T>
__device__ inline float settled(float v)
{
    if constexpr (std::is_same_v<T, f16>) asm("" : "+v"(v));
    return v;
}

template <class T>
__device__ inline void store_chunk(T *p, int64_t left, const float (&v)[CHUNK<T>])
{
    constexpr int N = CHUNK<T>;
    if (left >= N) {
        vec<T, N> t;
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = (T)settled<T>(v[i]);
        __builtin_memcpy(p, &t, 16);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = (T)settled<T>(v[i]);
    }
}

// Eight columns: one chunk of a 16-bit type, two of a 32-bit one.
template <class T>
__device__ inline void load8(const T *p, int64_t left, float (&v)[8])
{
    constexpr int N = CHUNK<T>;
#pragma unroll
    for (int k = 0; k < 8; k += N) {
        float c[N];
        load_chunk<T>(p + k, left - k, c);
#pragma unroll
        for (int i = 0; i < N; ++i) v[k + i] = c[i];
    }
}

template <class T>
__device__ inline void store8(T *p, int64_t left, const float (&v)[8])
{
    constexpr int N = CHUNK<T>;
#pragma unroll
    for (int k = 0; k < 8; k += N) {
        float c[N];
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = v[k + i];
        store_chunk<T>(p + k, left - k, c);
    }
}

__device__ inline float two_to(int e)  // 2^e for -126 <= e <= 127
{
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Exponent of a group's step from max|x|: the least e >= -126 with top <= 127 * 2^e.  With
// top = m * 2^k, 1 <= m < 2, that is k - 6 for m <= 127/64 (its fraction bits 0x7e0000), else k - 5.
__device__ inline int step_exp(float top)
{
    const uint32_t b = __float_as_uint(top);
    const int e = (int)(b >> 23) - 127 - ((b & 0x7fffffu) <= 0x7e0000u ? 6 : 5);
    return max(e, -126);
}

__device__ inline bool finite(float top)  // top >= 0 or NaN
{
    return __float_as_uint(top) < 0x7f800000u;
}

// max(a, |b|) that keeps NaN: bit patterns of non-negative floats are ordered as the
// floats, infinity and then NaN above them.
__device__ inline uint32_t max_bits(uint32_t a, float b)
{
    return max(a, __float_as_uint(b) & 0x7fffffffu);
}

// Codes of N values of one group: round-half-even(x * 2^-e).  Scaling by a power of two is exact, and adding 1.5 * 2^23
// rounds to a whole number whose low byte is the code, so one instruction does both.  A value is at most 127 steps by
// the choice of e; only where the type's range ends (`top`: 64 steps would pass it) is it limited to 63.
template <int N>
__device__ inline vec<uint32_t, N / 4> codes_of(const float (&x)[N], float inv_step, bool top)
{
    vec<uint32_t, N / 4> q;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v = x[i + j];
            if (top) v = fminf(fmaxf(v, -63.0f / inv_step), 63.0f / inv_step);
            b[j] = __float_as_uint(__builtin_fmaf(v, inv_step, 12582912.0f));
        }
        const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400), hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400);
        q[i / 4] = __builtin_amdgcn_perm(hi, lo, 0x05040100);
    }
    return q;
}

// The value that stands for a group's stored exponent byte: its step, or NaN.
__device__ inline float step_of(uint8_t exp_byte)
{
    return exp_byte == 255 ? __uint_as_float(0x7fc00000u) : two_to((int)exp_byte - 127);
}

// Exchanges between lanes in vector instructions (an exchange through LDS takes some hundred cycles).  Each leaves both partners
// with the same pair.
template <int CTRL>
__device__ inline uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e;      // quad permutations
constexpr int DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;  // of 8 and of 16 lanes

// Sum over groups of LANES (16 or 64) neighbouring lanes, in every lane and the same bits in each.
template <int LANES>
__device__ inline float lane_sum(float v)
{
    static_assert(LANES == 16 || LANES == 64);
    auto f = [](uint32_t u) { return __uint_as_float(u); };
    v += f(dpp<DPP_XOR1>(__float_as_uint(v)));
    v += f(dpp<DPP_XOR2>(__float_as_uint(v)));
    v += f(dpp<DPP_HALF_MIRROR>(__float_as_uint(v)));
    v += f(dpp<DPP_MIRROR>(__float_as_uint(v)));
    if constexpr (LANES == 64) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(a[0]) + f(a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(b[0]) + f(b[1]);
    }
    return v;
}

// Maximum over the lanes l, l + 16, l + 32 and l + 48, in each.
__device__ inline uint32_t max_of_rows(uint32_t v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

inline bool good_dtype(int dtype) { return dtype == RKB_F32 || dtype == RKB_F16 || dtype == RKB_BF16; }
inline bool good_dtype16(int dtype) { return dtype == RKB_F16 || dtype == RKB_BF16; }
inline int dtype_size(int dtype) { return dtype == RKB_F32 ? 4 : 2; }

inline bool good_size(int64_t rows, int64_t cols)
{
    return rows >= 0 && rows <= RKB_MAX_ROWS && cols >= 1 && cols <= RKB_MAX_COLS;
}

// A matrix argument: present, aligned to its type, and for an output with rows that do not overlap (a stride is not read for
// one row).
inline bool good_input(const void *p, int64_t rows, int64_t stride, int size)
{
    return rows == 0 || (p && (uintptr_t)p % size == 0 && (rows == 1 || (stride >= 0 && stride <= ((int64_t)1 << 40))));
}
inline bool good_output(const void *p, int64_t rows, int64_t cols, int64_t stride, int size)
{
    return good_input(p, rows, stride, size) && (rows <= 1 || stride >= cols);
}

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
inline int64_t code_ld(int64_t cols) { return round_up(cols, GROUP); }

// Queues a kernel.  The launch's own result is looked at, not the thread's last error, which an earlier call of someone
// else's may have left: that is neither reported here nor taken from whoever asks for it.
template <class... P, class... A>
int launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t st, const A &...a)
{
    static_assert(sizeof...(P) == sizeof...(A));
    std::tuple<P...> values(a...);
    const hipError_t e = std::apply(
        [&](auto &...v) {
            void *at[] = {(void *)&v...};
            return hipLaunchKernel((const void *)kernel, grid, block, at, 0, st);
        },
        values);
    if (e == hipSuccess) return RKB_OK;
    (void)hipGetLastError();
    return RKB_E_DEVICE;
}

}  // namespace rkb
