/*
 * radar_cache.h -- C ABI of the cache operators beside the decode path of
 * radar.h: rotary positions for the rows on their way into the cache, exact
 * attention of a batch over a prefix that its sequences share, exact
 * attention that accumulates the weight of every cache row, and eviction of
 * the rows with the least of it.
 *
 * Conventions are those of radar.h: device pointers owned by the caller and
 * aligned to 16 bytes, dense row-major layouts unless strides are given, no
 * allocation, no synchronisation, launches on `stream` only, every argument
 * checked before anything is launched, no C++ exception across the boundary.
 * K and V may lie in pinned host memory mapped for the device. Of the
 * radar_config these calls read batch, n_q_heads, n_kv_heads, head_dim,
 * capacity, kv_dtype and n_sink, with radar.h's limits; the fields of the
 * index and the selection are not read. Workspaces: contents on entry do not
 * matter, and one workspace must not be used by two calls at the same time
 * (two graphs that hold the same one must not be replayed concurrently).
 *
 * The measurement hook of radar.h books their kernels under the kinds that it
 * has: rotations and the eviction's move as RADAR_K_APPEND, the attention's
 * blocks as _ATTEND, what follows them (merge and masses) as _COMBINE, the
 * eviction's choice of rows as _TOPK.
 */
#ifndef RADAR_CACHE_H
#define RADAR_CACHE_H

#include "radar.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions ----------------------------------------------------
 * Pair i < rot_dim / 2 of a head's dims, (i, i + rot_dim / 2) or, interleaved,
 * (2 i, 2 i + 1), is turned by the angle p * inv_freq[i] at position p:
 *   a' = mscale (a cos - b sin),   b' = mscale (b cos + a sin);
 * dims from rot_dim on are copied. The angle is reduced in 64 bits and the
 * sine, cosine and products are taken in 32, with one rounding to the output
 * type. The transposed map (the gradient) has -sin. */
typedef struct {
  int32_t rot_dim;         /* even, 2 .. head_dim                            */
  int32_t interleaved;     /* 0: pairs (i, i + rot_dim / 2); 1: (2 i, 2 i + 1) */
  float mscale;            /* factor on the rotated dims                     */
  const double* inv_freq;  /* device [rot_dim / 2], radians per position     */
} radar_rope;

/* Rows [batch][tokens][heads][head_dim] with the strides of the first three
 * axes in elements (multiples of 16 bytes; the last axis is dense). */
typedef struct {
  void* data;
  int64_t seq, token, head;
} radar_rows;

/* Rotates q (n_q_heads heads) into q_out and k (n_k_heads) into k_out in one
 * launch; with n_k_heads = 0 only q (k and k_out may be NULL). An output may
 * be its own input (the same address and strides); no other overlap. Token
 * (b, t) stands at position pos0 + t, with pos (nullable, device int64) at
 * pos[b] + t, with pos_per_token too at pos[b * tokens + t]. lens (nullable,
 * device int64 [batch]): only tokens t < lens[b] are read and written.
 * inverse: the transposed map. head_dim: a multiple of 16, at most 256;
 * batch * tokens < 2^31. tokens = 0 launches nothing. */
radar_status radar_rotary(const radar_rope* rope, int32_t batch, int64_t tokens,
                          int32_t head_dim, radar_dtype dtype,
                          int32_t n_q_heads, const radar_rows* q,
                          const radar_rows* q_out, int32_t n_k_heads,
                          const radar_rows* k, const radar_rows* k_out,
                          int64_t pos0, const int64_t* pos,
                          int32_t pos_per_token, const int64_t* lens,
                          int32_t inverse, hipStream_t stream);

/* A chunk of tokens on its way into the cache, in one launch: token (b, t)'s
 * rotated k and its v go to row row0 + t (with rows, nullable device int64
 * [batch], rows[b] + t) of K and V, and with q (nullable) its rotated q to
 * q_out. Positions and lens as for radar_rotary; rows outside [0, capacity)
 * are skipped, as are tokens from lens[b] on, and no other row is touched.
 * The summaries are not: radar_build_index follows. k and v hold n_kv_heads
 * heads, q and q_out n_q_heads. Requires 0 <= row0 and row0 + tokens <=
 * capacity where rows is NULL. */
radar_status radar_rotary_fill(const radar_config* cfg, const radar_rope* rope,
                               int64_t tokens, const radar_rows* q,
                               const radar_rows* q_out, const radar_rows* k,
                               const radar_rows* v, void* K, void* V,
                               int64_t row0, const int64_t* rows, int64_t pos0,
                               const int64_t* pos, int32_t pos_per_token,
                               const int64_t* lens, hipStream_t stream);

/* ---- attention over a shared prefix --------------------------------------
 * One query per (b, q head) attends the prefix_len rows of the prefix
 * Kp, Vp [n_kv_heads][prefix_capacity][head_dim], which all sequences share,
 * and rows [0, t) (with lens, nullable device int64 [batch], [0, lens[b]),
 * t their bound) of the sequence's own K and V: exact softmax attention with
 * the scale 1/sqrt(head_dim). Of the batch * n_q_heads / n_kv_heads query rows
 * of a kv head up to 128 share one read of a prefix row (fp32: 16, 64 or 128);
 * more read it again. 0 <= prefix_len <= prefix_capacity < 2^31, 0 <= t <=
 * capacity; Kp and Vp may be NULL with prefix_len = 0, K and V with t = 0. A
 * query that attends no row gets a zero output; lens[b] outside [0, t] makes
 * that sequence's outputs NaN. With a bf16 cache the weights enter the product
 * with V in 16 bits where at most 16 query rows share a read, and rounded to
 * bf16 where more do (the output's error is then up to 1.4 times that of its own
 * rounding); everything else is fp32. */
radar_status radar_attend_prefix(const radar_config* cfg, const void* q,
                                 const void* Kp, const void* Vp,
                                 int64_t prefix_len, int64_t prefix_capacity,
                                 const void* K, const void* V, int64_t t,
                                 const int64_t* lens, void* out,
                                 void* workspace, size_t workspace_bytes,
                                 hipStream_t stream);

/* Scratch bytes for every call with this config, at most this prefix_len and
 * at most this t (0 if the arguments are invalid). */
size_t radar_attend_prefix_workspace_bytes(const radar_config* cfg,
                                           int64_t prefix_len, int64_t t);

/* ---- attention that accumulates the rows' weights -------------------------
 * One query per (b, q head) attends rows [0, t) (lens: [0, lens[b])) of K and
 * V exactly, as above; and the softmax weight that row i gets from the query
 * heads of kv head h, summed over them, is added to mass[b][h][i] (fp32,
 * [batch][n_kv_heads][capacity]; entries from the length on are not touched).
 * 1 <= t <= capacity; lens[b] outside [1, t] makes that sequence's outputs NaN
 * and leaves its masses alone. The order of the additions is fixed: the same
 * inputs give the same bits. */
radar_status radar_attend_accumulate(const radar_config* cfg, const void* q,
                                     const void* K, const void* V, float* mass,
                                     int64_t t, const int64_t* lens, void* out,
                                     void* workspace, size_t workspace_bytes,
                                     hipStream_t stream);

/* Scratch bytes for every call with this config and at most this t. */
size_t radar_attend_accumulate_workspace_bytes(const radar_config* cfg, int64_t t);

/* ---- eviction --------------------------------------------------------------
 * Cuts a cache of t rows (lens: lens[b], t their bound) to n = n_sink + heavy
 * + recent: of every (b, kv head) the first n_sink rows stay, the last
 * `recent`, and of the rows between them the `heavy` with the largest mass
 * (ties: the lower row; a NaN counts as larger than every number). The kept
 * rows of K, V and mass move to rows 0 .. n - 1 in their order, the masses of
 * rows n .. len - 1 become 0, and the rows of K and V from n on are left as
 * they were. A sequence of at most n rows is not changed, nor is one with
 * lens[b] outside [0, t]. new_lens (nullable, device int64 [batch]) receives
 * min(lens[b], n) (an invalid lens[b] as it is; it may be lens itself); kept
 * (nullable, device int32 [batch][n_kv_heads][min(n, t)]) the rows that were
 * kept, ascending, -1 behind them. 0 <= t <= capacity, t below 2^31 - 2^14;
 * heavy, recent >= 0; n below 2^31; a head's kept rows of K at most 2^39 - 2^17
 * bytes. The summaries of the index are not touched: they hold for the old
 * rows, and radar_build_index follows. */
radar_status radar_evict(const radar_config* cfg, void* K, void* V, float* mass,
                         int64_t t, const int64_t* lens, int64_t heavy,
                         int64_t recent, int64_t* new_lens, int32_t* kept,
                         void* workspace, size_t workspace_bytes,
                         hipStream_t stream);

/* Scratch bytes for every call with this config, at most this t and this many
 * kept rows or fewer. */
size_t radar_evict_workspace_bytes(const radar_config* cfg, int64_t t,
                                   int64_t heavy, int64_t recent);

#ifdef __cplusplus
}
#endif

#endif /* RADAR_CACHE_H */
