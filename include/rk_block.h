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
 *   - the weight gradient of a linear layer whose input was kept in 8 bits;
 *   - attention to keys and values of another length, forward and backward, with a learned bias by
 *     relative position, and from a cache of keys and values in 8 bits.
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
#define RKB_MAX_DIM 256                                /* widest head of an attention    */
#define RKB_MAX_TOKENS ((int64_t)1 << 28)              /* most queries or keys of a sequence */
#define RKB_MAX_BUCKETS 128                            /* most buckets of a bias and ... */
#define RKB_MAX_DISTANCE 1024                          /* ... its largest max_distance   */

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

/*
 * Attention.  A rkb_heads is a [batch, rows, heads, dim] tensor whose neighbouring columns are adjacent, with its strides in
 * elements (those of a size of one are not read): 0 to 2^40 for an input; an output's elements must not overlap.
 */
typedef struct rkb_heads {
    void *p;
    int64_t batch, row, head;
} rkb_heads;

/*
 * What a call attends to what.  For each sequence b and head h, whose keys and values are those of head h / (heads / kv_heads):
 *   s_ij = scale q_i . k_j + table[bucket(j - pos_i), h]   for each key j that lives for query i,
 *   lse_i = ln sum_j e^s_ij,  p_ij = e^(s_ij - lse_i),  o_i = sum_j p_ij v_j.
 * pos_i = first + firsts[b] + i is where query i stands among the keys (within 2^30; beyond, as if there).
 * Key j lives if j < lens[b] (taken to lie in 0 .. k_rows), mask[b * mask_stride + j] is not 0 and, where `causal`, j <= pos_i.
 * lens, firsts and mask are device memory, or NULL: all keys, 0, all keys.  A query without live keys has o_i = 0 and lse_i = -inf.
 * What lies at a key that lives for no query (a length or the mask says so) is not looked at, whatever it is; one that
 * only `causal` hides from a query counts 0 times its value there, which is NaN for an infinity or NaN.
 *
 * table: [buckets, heads] of type table_dtype (dtype or RKB_F32), or NULL for none.  Of the relative position n = j - pos_i, a two-sided
 * bias has half of its buckets for n <= 0 and the other half for n > 0, by distance |n|; a one-sided one has all
 * for the distance max(-n, 0).  Of nb buckets of a side the first e = nb / 2 (rounded down) are one distance each; from e on,
 * the bucket is e + floor((nb - e) ln(d / e) / ln(max_distance / e)), at most nb - 1, as exact arithmetic has it.
 * nb is 2 .. RKB_MAX_BUCKETS (and so is twice nb, where two-sided), e < max_distance <= RKB_MAX_DISTANCE.  An entry of -1e30 or less, -inf
 * among them, hides its keys as a mask does, and its gradient is 0; one of 2^127 or more may count as an infinity, whose rows are NaN.
 *
 * dtype: RKB_F16 or RKB_BF16; 1 <= dim <= RKB_MAX_DIM; heads a multiple of kv_heads; 0 < scale, and scale / ln 2 finite in 32 bits; batch * heads times
 * q_rows (rounded up to 128) at most 2^28, and for the backward pass batch * kv_heads times k_rows likewise.
 */
typedef struct rkb_attn {
    int dtype, causal;
    int64_t batch, q_rows, k_rows, heads, kv_heads, dim;
    float scale;
    int64_t first;
    const int32_t *firsts, *lens;
    const uint8_t *mask;
    int64_t mask_stride;
    const void *table;
    int table_dtype, buckets, max_distance, two_sided;
} rkb_attn;

/*
 * A cache of keys and values in 8 bits.  For each sequence and head, RKB_GROUP neighbouring tokens (a block) share 2^e, the least power of
 * two with max|x| <= 127 * 2^e (e >= -126), over all their columns; values are kept as in the 8-bit checkpoints above:
 * round-half-even(x 2^-e), at most 63 where 64 * 2^e would pass dtype's largest finite value, and exactly what they stand for in dtype.
 *   codes [2, batch, kv_heads, room, ld]: keys, then values; room = tokens rounded up to RKB_GROUP, ld = dim rounded up to 16,
 *         16-byte aligned; columns past dim are 0
 *   exps  [2, batch, kv_heads, room / RKB_GROUP]: e + 127; 255 for a block that stands for NaN as a whole, because it took an infinity
 *         or NaN; 0 for a block that stands for zeros, as memory cleared beforehand does
 */
typedef struct rkb_kv8 {
    int8_t *codes;
    uint8_t *exps;
    int64_t tokens;  /* most of a sequence */
} rkb_kv8;

/*
 * Writes k and v [batch, rows, kv_heads, dim] into a cache: row i of sequence b becomes its token first + firsts[b] + i, if i < counts[b]
 * (NULL: all rows).  Rows that would lie before token 0 or behind the last are not written.  A block that holds
 * tokens before the first one written keeps them: where the new ones need a larger step, 2^e', their codes become
 * round-half-even(code 2^(e - e')).  What a block held from the first token written on is dropped: the places behind the
 * last one written are zeros.  Other blocks stay as they were.
 * At most 2^22 blocks of all sequences and heads may be touched by a call: batch * kv_heads times the lesser of
 * (rows + 62) / 32, rounded down (what rows tokens touch wherever they begin, and whatever counts says), and a head's blocks.
 */
int rkb_kv8_write(int dtype, int64_t batch, int64_t rows, int64_t kv_heads, int64_t dim, const rkb_heads *k, const rkb_heads *v,
                  int64_t first, const int32_t *firsts, const int32_t *counts, const rkb_kv8 *cache, void *stream);

/* The values that a cache stands for: k and v [batch, tokens, kv_heads, dim], either may have p NULL. */
int rkb_kv8_load(int dtype, int64_t batch, int64_t kv_heads, int64_t dim, const rkb_kv8 *cache, const rkb_heads *k,
                 const rkb_heads *v, void *stream);

/*
 * Attention forward.  q and o [batch, q_rows, heads, dim]; k and v [batch, k_rows, kv_heads, dim], or both NULL and `cache` given, with
 * k_rows <= cache->tokens (codes of tokens from k_rows on are not read).  o32: NULL, or [batch, q_rows, heads, dim] (contiguous, 16-byte
 * aligned) receives o in 32 bits, as it was summed; lse: NULL, or [batch, heads, q_rows].  Probabilities are rounded to dtype on their way into the
 * second product, relative to the row's largest (within 2^8), so that what is lost of one is at most as much as its
 * rounding; sums are not.
 * `aligned` of the workspace call: q, k and v start at multiples of 16 bytes, dim and all their strides are multiples of 8 and
 * row strides at most 2^22; 0 asks for room for copies that are.
 */
int rkb_attn_fwd_workspace(const rkb_attn *a, int cache, int aligned, size_t *bytes);
int rkb_attn_fwd(const rkb_attn *a, const rkb_heads *q, const rkb_heads *k, const rkb_heads *v, const rkb_kv8 *cache,
                 const rkb_heads *o, float *o32, float *lse, void *workspace, size_t ws_bytes, void *stream);

/*
 * Its backward, from do [batch, q_rows, heads, dim] and what the forward kept: lse, and o as it was returned (o) or in 32 bits
 * (o32); with neither (o, o32 and lse NULL) they are made again.  With dp_ij = do_i . v_j and ds_ij = p_ij (dp_ij - do_i . o_i),
 *   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i,
 *   dtable[c, h] = sum of ds_ij over the i, j of bucket c and all sequences,
 * dk and dv summed over the heads that share them too.  p and ds enter the products rounded to dtype; in f16, scaled
 * so that neither overflows nor loses bits that its size would not lose in any type.  do_i . o_i would take over the error of o (its rounding, where o is
 * not given in 32 bits, and that of the probabilities it was summed from); what a row's ds add up to, 0 otherwise, tells that error, which
 * is taken out of all of them.
 * dq, dk, dv of dtype, each may have p NULL (dk and dv both); dtable of table_dtype, NULL for none.  What q and do hold at
 * a query without live keys is not looked at, whatever it is; its dq is 0.
 * aligned: as above, of do too.
 */
int rkb_attn_bwd_workspace(const rkb_attn *a, int again, int aligned, size_t *bytes);
int rkb_attn_bwd(const rkb_attn *a, const rkb_heads *d_o, const rkb_heads *q, const rkb_heads *k, const rkb_heads *v,
                 const rkb_heads *o, const float *o32, const float *lse, const rkb_heads *dq, const rkb_heads *dk,
                 const rkb_heads *dv, void *dtable, void *workspace, size_t ws_bytes, void *stream);

/* Short English description of an RKB_* code. */
const char *rkb_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* RK_BLOCK_H */
