/*
 * rk_block.h -- C ABI of librkblock, the steps that a re-materialization schedule runs, on
 * AMD Instinct MI355X (gfx950).
 *
 * rk.h plans which intermediates each block of a chain keeps from its forward F^o to its
 * backward B^o.  This library holds operators that such blocks are made of, in the forms
 * that the plan chooses between:
 *   - layer norm, forward and backward;
 *   - checkpoints of activations in 8 bits (a saving option with half the memory of a
 *     16-bit activation), and backward steps that read them;
 *   - the gated feed-forward block h = act(x Wg^T) * (x Wu^T), whose backward reads
 *     g = x Wg^T and u = x Wu^T as they were, from 8-bit checkpoints, or makes them again;
 *   - the weight gradient of a linear layer whose input was kept in 8 bits.
 *
 * Matrices are row-major with neighbouring columns adjacent; `..._stride` is the distance
 * between rows in elements (not read for matrices of at most one row): at least the number of columns
 * for an output, any number from 0 (one row for all) to 2^40 for an input.  All pointers but *bytes are device memory of the device that is current.
 * Outputs must not overlap inputs, other outputs or the workspace.  Sums, statistics and
 * products accumulate in 32 bits whatever the type; outputs are rounded once, to nearest even.
 *
 * Every call checks its arguments, queues kernels on `stream` (a hipStream_t; NULL is the
 * device's default stream) and returns without waiting.  Nothing is allocated, copied from
 * the host or kept between calls, and no call records anything but kernels, so all may be
 * captured into a HIP graph.  Calls that need scratch memory take a caller's workspace, 256-byte
 * aligned, of at least the bytes that the matching ..._workspace call reports; its contents
 * matter only while the call's kernels run.  Products read their operands (x, dy, wg, wu) in 16-byte
 * chunks; `aligned` of a ..._workspace call says that each of them starts at a multiple of 16 bytes and
 * has a row stride that is a multiple of 8 elements and at most 2^22 (wg and wu the same stride), and 0 asks for
 * room for copies that are.  Results do not depend on what ran before or
 * beside: every sum has a fixed order.  Calls are thread-safe.  Nothing is thrown across the
 * ABI.
 */
#ifndef RK_BLOCK_H
#define RK_BLOCK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    RKB_OK = 0,
    RKB_E_INVAL = -1,   /* bad argument (NULL, negative, out of range, misaligned), or a
                           product of more than 2^22 tiles (128 x 128 at least)         */
    RKB_E_NOMEM = -3,   /* workspace too small                                          */
    RKB_E_DEVICE = -4   /* a HIP call failed (no device, launch error, ...)             */
};

enum { RKB_F32 = 0, RKB_F16 = 1, RKB_BF16 = 2 };       /* types                          */
enum { RKB_SILU = 0, RKB_GELU = 1 };                   /* g/(1+e^-g); g Phi(g), Phi the
                                                          normal distribution            */
enum { RKB_KEEP_NONE = 0, RKB_KEEP_FULL = 1, RKB_KEEP_8BIT = 2, RKB_KEEP_16BIT = 3 };

#define RKB_MAX_NORM_COLS 16384                        /* widest row of a layer norm     */
#define RKB_MAX_ROWS ((int64_t)1 << 30)                /* most rows and ...              */
#define RKB_MAX_COLS ((int64_t)1 << 24)                /* ... columns of any matrix      */
#define RKB_GROUP 32                                   /* columns that share a scale     */

/*
 * Layer norm of each row: y = (x - mean) rstd w + b with mean and (biased) variance of the
 * row and rstd = 1 / sqrt(variance + eps).  w, b: [cols] of type wdtype (dtype or RKB_F32), or
 * NULL for ones and zeros.  mean, rstd: [rows] 32-bit, either may be NULL.  The variance is the mean of
 * squared differences from the mean.  1 <= cols <= RKB_MAX_NORM_COLS; eps >= 0.
 */
int rkb_layer_norm_fwd(int dtype, int wdtype, int64_t rows, int64_t cols, const void *x, int64_t x_stride,
                       const void *w, const void *b, float eps, void *y, int64_t y_stride, float *mean,
                       float *rstd, void *stream);

/*
 * Its backward: with xh = (x - mean) rstd and v = dy w,
 *   dx = rstd (v - rowmean(v) - xh rowmean(v xh)),  dw = sum over rows of dy xh,  db = of dy.
 * x is given as it was (x, x_stride; codes and exps NULL) or as its 8-bit checkpoint (codes, exps; x
 * NULL); mean and rstd are the forward's.  dw, db: [cols] of type wdtype, either may be NULL.  The workspace holds
 * partial sums of dw and db (none is needed without them).
 */
int rkb_layer_norm_bwd_workspace(int dtype, int64_t rows, int64_t cols, size_t *bytes);
int rkb_layer_norm_bwd(int dtype, int wdtype, int64_t rows, int64_t cols, const void *dy, int64_t dy_stride,
                       const void *x, int64_t x_stride, const int8_t *codes, const uint8_t *exps,
                       const float *mean, const float *rstd, const void *w, void *dx, int64_t dx_stride,
                       void *dw, void *db, void *workspace, size_t ws_bytes, void *stream);

/*
 * Checkpoints in 8 bits.  Each RKB_GROUP neighbouring columns of a row share 2^e, the least
 * power of two with max|x| <= 127 * 2^e (e >= -126); a value is kept as the whole number
 * q = round-half-even(x 2^-e), |q| <= 127 (63 where 64 * 2^e would pass dtype's largest
 * finite value), and stands for q * 2^e, which every dtype holds exactly where x's type held x.
 * So |x - q 2^e| <= 2^(e-1) < max|x| / 127 for e > -126 (below 2^e where 63 limits).  A group with an infinity or NaN stands for NaN as a whole, whatever
 * its codes, so that such a value still reaches the gradients.
 *   codes [rows, ld] with ld = cols rounded up to RKB_GROUP (the rest zero), 16-byte aligned
 *   exps  [rows, ld / RKB_GROUP]: e + 127, or 255 for NaN
 */
int rkb_ckpt8_save(int dtype, int64_t rows, int64_t cols, const void *x, int64_t x_stride, int8_t *codes,
                   uint8_t *exps, void *stream);
int rkb_ckpt8_load(int dtype, int64_t rows, int64_t cols, const int8_t *codes, const uint8_t *exps, void *x,
                   int64_t x_stride, void *stream);

/*
 * Weight gradient of y = x W^T: dw [n, k] = dy^T x, summed over rows; dy [rows, n], x [rows, k], given as it
 * was or as its checkpoint, as above.  A checkpoint is loaded whole into the workspace first, as the 16-bit matrix that it
 * stands for.  dtype: RKB_F16 or RKB_BF16.  rows == 0 gives zeros.
 * ckpt of the workspace call: whether x is given as its checkpoint.
 */
int rkb_weight_grad_workspace(int dtype, int64_t rows, int64_t n, int64_t k, int ckpt, int aligned, size_t *bytes);
int rkb_weight_grad(int dtype, int64_t rows, int64_t n, int64_t k, const void *dy, int64_t dy_stride,
                    const void *x, int64_t x_stride, const int8_t *codes, const uint8_t *exps, void *dw,
                    int64_t dw_stride, void *workspace, size_t ws_bytes, void *stream);

/*
 * Gated feed-forward: g = x wg^T, u = x wu^T, h = act(g) u; x [rows, d], wg and wu [f, d],
 * h [rows, f].  dtype: RKB_F16 or RKB_BF16.  keep:
 *   RKB_KEEP_NONE  g, u, ge, ue are NULL
 *   RKB_KEEP_FULL  g, u [rows, f] (contiguous) receive g and u in 32 bits, as they were
 *                  summed, so that the backward pass loses nothing; ge, ue NULL
 *   RKB_KEEP_16BIT the same, rounded to dtype
 *   RKB_KEEP_8BIT  g, u receive the codes and ge, ue the exps of the checkpoints of g and u, taken
 *                  from the 32-bit sums (as of type RKB_F32)
 */
int rkb_gated_fwd_workspace(int dtype, int64_t rows, int64_t d, int64_t f, int aligned, size_t *bytes);
int rkb_gated_fwd(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f, const void *x,
                  int64_t x_stride, const void *wg, int64_t wg_stride, const void *wu, int64_t wu_stride, void *h,
                  int64_t h_stride, void *g, void *u, uint8_t *ge, uint8_t *ue, void *workspace,
                  size_t ws_bytes, void *stream);

/*
 * Its backward, from dh [rows, f] and what the forward kept (RKB_KEEP_NONE makes g and u again from x, wg
 * and wu): with dg = dh u act'(g) and du = dh act(g),
 *   dx = dg wg + du wu,  dwg = dg^T x,  dwu = du^T x.
 * dg and du enter the products rounded to dtype.  That adds as much error to the gradients as their own rounding, and a dg or
 * du beyond dtype's largest value (65504 in f16) is an infinity, one below its smallest 0.  Where there are at most 4096
 * of them (rows * f), what the rounding leaves over enters as well, which saves the error but not the range.  dx [rows, d],
 * dwg and dwu [f, d] of dtype, dx or both of dwg and dwu may be NULL.  h: NULL, or [rows, f] of dtype, receives
 * act(g) u of the same g and u, for the weight gradient of the layer that follows.  rows == 0 gives zero weight gradients.
 */
int rkb_gated_bwd_workspace(int dtype, int keep, int64_t rows, int64_t d, int64_t f, int aligned, size_t *bytes);
int rkb_gated_bwd(int dtype, int act, int keep, int64_t rows, int64_t d, int64_t f, const void *dh,
                  int64_t dh_stride, const void *x, int64_t x_stride, const void *wg, int64_t wg_stride,
                  const void *wu, int64_t wu_stride, const void *g, const void *u, const uint8_t *ge,
                  const uint8_t *ue, void *dx, int64_t dx_stride, void *dwg, void *dwu, int64_t dw_stride, void *h,
                  int64_t h_stride, void *workspace, size_t ws_bytes, void *stream);

/* Short English description of an RKB_* code. */
const char *rkb_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* RK_BLOCK_H */
