/*
 * libmpic -- what goes along with a linked context: fresh rows on their way into it
 * (norms of the query and key heads, rotation to their positions), the context held in
 * 4 bits, and attention over it.  Same conventions as mpic.h: plain C ABI, every call
 * returns an mpic_status, arguments are checked on the host before anything is
 * enqueued, calls are stream-ordered and can be captured into a graph (the context must
 * then be bound to the GPU already, which any earlier GPU call of it does).
 *
 * A context linked by mpic_assemble_kv is read once by the prefill and then by every
 * decode step.  In 4 bits such a step reads 144 bytes per token and kv head instead of 512
 * (bf16, head_dim 128) and a GPU holds 3.5 times as many contexts.  The rows of a
 * context can be written as they are produced, a prefill's all at once and then the new
 * token of every step.  None of these calls uses a plan: lengths, pages and slots are
 * device arrays, so one captured graph serves a whole generation.
 */
#ifndef MPIC_Q4_H
#define MPIC_Q4_H

#include "mpic.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Position fresh rows: every head of q and k is normed (if eps >= 0) and rotated to the
 * position of its row, in one pass.
 *   y = x * rsqrt(mean(x^2) + eps) * weight          (eps >= 0; a NULL weight is all ones)
 *   pair i of y is turned by pos[axis(i)][row] * rope_theta^(-2i/D)
 * in fp32, with one rounding at the end.  rope_theta, the pairing (rope_interleaved), D, the
 * head counts and the type are those of the context.  Angles are reduced to a turn in
 * 64-bit integers, so that positions of any size lose nothing.
 * The result is what contexts without fresh_pre_rope take as fresh rows.
 *
 * With several axes (rows of images and videos: time, height, width) each pair follows one
 * of them.  A stored chunk whose rows were positioned this way, counted from its own
 * origin, is moved by the same distance on every axis, and the distance that
 * mpic_assemble_kv moves it by is the token index of its first token in the request.  So
 * a chunk of several axes may be linked only where its origin lies at that index on all
 * axes, and the fresh rows around it have to be positioned by the same count.  Models
 * whose positions go on by less than a chunk's tokens behind it (by 24 behind an image of
 * 24 x 24) do not link so, and nothing in the rows tells: no plan gives another distance.
 * Their stored keys are turned by the difference first, on every axis: this call without
 * norms, positions = wanted origin - token index, negative or not, and one rounding more.
 *
 *   q [n_rows][Hq][D], k [n_rows][Hkv][D]  device, rows q_stride / k_stride elements apart
 *                     (so both may be parts of the rows of one projection): multiples of 16
 *                     bytes, at least Hq * D and Hkv * D
 *   pos               device [n_axes][n_rows], any int32 values
 *   n_axes            1 .. 4
 *   pair_axis         host [D/2], the axis of each pair, 0 .. n_axes - 1; NULL = all of axis 0
 *   q_weight, k_weight  device [D] in the context's type; may be NULL; must be NULL for eps < 0
 *   eps               finite; negative: rows are rotated without norms
 *   q_out, k_out      device, like q and k.  May be q and k themselves with the same strides;
 *                     must not overlap them otherwise
 * A row of zeros stays zeros for eps > 0; with eps = 0 it becomes NaN, as the formula says.
 * Squares are fp32: a head whose sum of squares passes 2^128 becomes zeros, and squares below
 * 2^-149 are zero.
 * Errors: MPIC_ERR_INVALID, MPIC_ERR_UNSUPPORTED (launch beyond the grid's limits), MPIC_ERR_HIP.
 */
int mpic_position_rows(mpic_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                       int64_t n_rows, const int32_t* pos, int32_t n_axes, const int32_t* pair_axis,
                       const void* q_weight, const void* k_weight, double eps, void* q_out,
                       int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream);

/*
 * A cache in 4 bits holds n_slots rows of K and V in one device buffer of mpic_q4_bytes
 * bytes (rounded up to 16 slots; the layout is the library's own).  Every 64 neighbouring
 * values of a head share a scale and a minimum, both of the context's type:
 *   low   = least of the 64 values
 *   scale = (greatest - low) / 15: difference and quotient in fp32, then rounded to the type;
 *           a scale below 2^-100 is taken as zero
 *   code  = the whole number nearest to (x - low) / scale (the difference rounded to fp32, the
 *           quotient exact, halves upwards), at most 15; 0 if the scale is zero
 *   value = low + code * scale, in fp32, rounded to the type where it is read back
 * So the least value of a group is held exactly and no value is off by more than half a
 * scale and the rounding of the scale (times the code).  A group with a value that is not
 * finite, or whose range overflows fp32, stands for 64 NaN.
 * Errors: MPIC_ERR_INVALID, MPIC_ERR_UNSUPPORTED (more bytes than 64 bits hold).
 */
int mpic_q4_bytes(const mpic_ctx* ctx, int64_t n_slots, int64_t* bytes);

/*
 * Write rows into the cache: row r of k and v goes to slot slots[r] (slots == NULL: to slot r).
 *   k, v [n_rows][Hkv][D]  device, rows k_stride / v_stride elements apart (multiples of 16
 *                     bytes, at least Hkv * D)
 *   slots             device [n_rows] or NULL.  A row whose slot is not in 0 .. n_slots - 1 is
 *                     left out (padding).  A slot must not be named twice in a call: its content
 *                     is then undefined (part of one row, part of another)
 *   cache             device, 16-byte aligned; other slots keep what they hold
 *   cache_bytes       size of the buffer, at least mpic_q4_bytes for n_slots
 * Errors: MPIC_ERR_INVALID, MPIC_ERR_UNSUPPORTED (launch beyond the grid's limits), MPIC_ERR_HIP.
 */
int mpic_q4_write(mpic_ctx* ctx, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  int64_t n_rows, const int32_t* slots, void* cache, int64_t cache_bytes, int64_t n_slots,
                  void* stream);

/*
 * Read rows back: k and v row r = the values that slot slots[r] holds.  Same arguments; a row
 * whose slot is not in 0 .. n_slots - 1 is left as it was; a slot may be read into several rows.
 */
int mpic_q4_read(mpic_ctx* ctx, const void* cache, int64_t cache_bytes, int64_t n_slots,
                 const int32_t* slots, int64_t n_rows, void* k, int64_t k_stride, void* v,
                 int64_t v_stride, void* stream);

/*
 * Attention over contexts held in 4 bits.  Request b has lens[b] tokens, token j of them in slot
 *   page_table[b][j / page_size] * page_size + j % page_size
 * of the cache, and n_b new queries, which belong to its last n_b tokens (their rows have been
 * written to the cache already): query i sits at position p = lens[b] - n_b + i and sees the
 * positions 0 .. p.  For every query and query head h (kv head h / (Hq/Hkv)):
 *   s_j = softmax_scale * <q, K_j>,  out = sum_j softmax(s)_j V_j,  lse = log sum_j exp(s_j)
 * over the values that the codes stand for.  A query that sees nothing (p < 0, or an empty
 * request) gets zeros and lse = -infinity.
 * BF16: products on the matrix cores with fp32 accumulation over the codes themselves, which are
 * exact; the weights (times the scale of V) are rounded to bf16 before the second product, those
 * that meet V's minima are held in 16 bits or more; one final rounding of out.  F32: factors split
 * into three bf16 parts (24 bits), fp32 otherwise.
 *
 *   q                 device [n_rows][Hq][D], rows q_stride elements apart (as above)
 *   q_off             device [n_requests + 1], queries of request b are rows q_off[b] ..
 *                     q_off[b + 1] - 1 (never decreasing); NULL: one query per request, n_rows =
 *                     n_requests.  Rows of no request are left as they were
 *   max_q             most queries of a request, >= 1 (shapes the launch; queries beyond it are
 *                     not computed)
 *   page_table        device [n_requests][table_width]; entries behind a request's last page may
 *                     hold anything.  Tokens whose block of 16 slots is not inside the cache are
 *                     not seen
 *   page_size         a positive multiple of 16.  Contiguous caches are those with one page per
 *                     request
 *   lens              device [n_requests]; negative = 0, more than max_len = max_len
 *   max_len           bound on lens, 0 .. table_width * page_size (shapes the launch: a bound near
 *                     the lengths makes it faster)
 *   softmax_scale     2^-126 .. 2^123
 *   out               device [n_rows][Hq][D]
 *   lse               device float [n_rows][Hq]; may be NULL
 *   workspace         device, 16-byte aligned, at least mpic_q4_attn_workspace bytes for the same
 *                     counts and bounds (smaller bounds may need more; may be NULL for 0 bytes), any
 *                     content.  It is the caller's so that graphs and streams
 *                     that may run beside each other can have one each; calls that may overlap
 *                     must not share one
 * Scores and sums are fp32: |V| up to 2^80 cannot overflow them.
 * Values that are not finite reach the queries that see them and no others, those of V only the 64
 * neighbouring columns that share their group.
 * Errors: MPIC_ERR_INVALID, MPIC_ERR_UNSUPPORTED (launch beyond the grid's limits), MPIC_ERR_HIP.
 */
int mpic_q4_attn_workspace(const mpic_ctx* ctx, int32_t n_requests, int64_t n_rows, int32_t max_q,
                           int64_t max_len, int64_t* bytes);
int mpic_q4_attn(mpic_ctx* ctx, const void* q, int64_t q_stride, int64_t n_rows, const int32_t* q_off,
                 int32_t max_q, const void* cache, int64_t cache_bytes, int64_t n_slots,
                 const int32_t* page_table, int64_t table_width, int32_t page_size, const int32_t* lens, int32_t n_requests,
                 int64_t max_len, double softmax_scale, void* out, float* lse, void* workspace,
                 int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
