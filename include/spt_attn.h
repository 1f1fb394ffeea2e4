/*
 * C ABI of full attention over packed sequences, of a paged cache of keys and values, and of the
 * attention of one new token over that cache: what a decoder needs around the routed FFN of spt.h
 * to be trained with all keys and to be served (the sparse attention of spt_mha.h sees no mask, one
 * length for all sequences, and no cache).  Part of libspt.so.
 *
 * Conventions are those of spt.h: device pointers unless they say "host"; every call validates on
 * the host, enqueues on `stream` (a hipStream_t), never synchronises, never allocates; outputs are
 * overwritten; same calls give bit-identical outputs (no floating-point atomics; the order of sums, and so a sequence's last
 * bits, may change with the sizes of the call that it is in).  Return codes are
 * those of spt.h (SPT_OK, SPT_ERR_ARG, SPT_ERR_UNSUPPORTED, SPT_ERR_WORKSPACE, SPT_ERR_HIP).
 * Calls on several streams may overlap as long as they share no output and no workspace.  Outputs and workspaces share no
 * memory with one another or with inputs.  What is not finite among the keys and values that a query sees makes what depends on
 * it not finite; what it does not see does not matter.
 *
 * Heads: H query heads, Hk key heads, H % Hk == 0; query head h reads key head h / (H / Hk).
 * Head dimension dh: 64 or 128.
 */
#ifndef SPT_ATTN_H
#define SPT_ATTN_H
#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Attention over packed sequences ------------------------------------------------------
 * Sequence b owns rows cu_q[b] .. cu_q[b+1]-1 of Q (nq of them) and rows cu_k[b] .. cu_k[b+1]-1
 * of K and V (nk).  Query i of a sequence sees its keys j < nk, with `causal` only those with
 * j <= i + nk - nq: the last query sees all keys, so that nq < nk is a part of a prompt behind keys
 * that are there already, and with nq > nk the first nq - nk queries see nothing. */
typedef struct {
  int32_t B;      /* sequences, 1 .. 4096; any of them may be empty */
  int32_t Tq, Tk; /* rows of Q, of K and V: at least one; cu_q[B] <= Tq, cu_k[B] <= Tk */
  int32_t H, Hk;  /* query heads, at most 65535, and key heads; Tq H / 128 + B H and (Tk / 128 + B) Hk at most 2^23 - 16 */
  int32_t dh;     /* 64 or 128 */
  int32_t causal; /* 0 or 1 */
  float scale;    /* logits are scale * q.k; positive, at most 2e38 */
} spt_attn_shape_t;

/* y_i = sum_j p_ij v_j, p_ij = exp(s_ij - lse_i), s_ij = scale q_i.k_j, lse_i = log sum_j exp(s_ij),
 * over the keys that query i sees.  A query that sees none (or none with a score above -inf) gets
 * y = 0 and lse = -inf.  Keys that a query does not see do not touch its row, whatever they hold
 * (infinities and NaN included); rows of Y and lse behind cu_q[B] are left as they were.  q.k and the scores may have any size that
 * fp32 holds (scores: times log2 e); rows of a workgroup that meets one above 2^27 are taken one by one.
 *   Q, Y    bf16 [Tq][H][dh]     K, V  bf16 [Tk][Hk][dh]     (16-byte aligned)
 *   strides host, or NULL for dense tensors: elements from a row to the next and from a head to the
 *           next, of Q, K, V, Y: 8 numbers.  Multiples of 8, not negative, below 2^23; dh is
 *           always dense; rows and heads of outputs must not overlap.
 *   cu_q, cu_k  int32 [B+1], ascending from 0 (values outside 0 .. Tq, Tk are taken to the nearest of the two)
 *   lse     out fp32 [H][Tq], or NULL when no backward follows
 * P is rounded to bf16 (nearest even) in front of the second product; sums and statistics are fp32. */
int spt_attn_prompt_fwd(const spt_attn_shape_t* shape, const void* Q, const void* K, const void* V,
                        const int64_t* strides, const int32_t* cu_q, const int32_t* cu_k, void* Y, float* lse,
                        void* stream);

/* Backward: dQ, dK, dV (bf16) from dY, the forward's Y and lse.
 *   D_i = dy_i.y_i;  dS_ij = p_ij (dy_i.v_j - D_i);  dv_j = sum p_ij dy_i;
 *   dq_i = scale sum_j dS_ij k_j;  dk_j = scale sum dS_ij q_i   (sums of dk, dv over the queries of all heads of the group)
 * A query that sees no key has dq = 0, a key that no query sees dk = dv = 0; rows behind cu_q[B], cu_k[B] are left as they were.
 *   strides  host, or NULL: of Q, K, V, Y, dY, dQ, dK, dV: 16 numbers
 *   ws       spt_attn_prompt_workspace_bytes(shape) bytes, 256-byte aligned
 * In front of their products P is rounded to bf16, dS to bf16 or, where there are few rows (Tq H <= 128 B Hk or
 * (Tq / 32) H <= 256, by the sizes of the call: a sequence alone may have the one, in a large batch the other), to the sum of two.  What the
 * rounding of Y leaves in the sum of a row's dS, which is 0, is taken off D.  P comes from scores and an lse of 32 bits: it is off by up to
 * |lse| 2^-22 of itself, bf16's rounding at 2^14; from 2^29 on gradients may not be finite. */
int spt_attn_prompt_bwd(const spt_attn_shape_t* shape, const void* Q, const void* K, const void* V,
                        const void* Y, const void* dY, const float* lse, const int64_t* strides,
                        const int32_t* cu_q, const int32_t* cu_k, void* dQ, void* dK, void* dV, void* ws,
                        size_t ws_bytes, void* stream);

/* Bytes of workspace spt_attn_prompt_bwd needs (0 for an invalid shape). */
size_t spt_attn_prompt_workspace_bytes(const spt_attn_shape_t* shape);

/* ---- Paged cache of keys and values --------------------------------------------------------
 * A pool of pages of `page` tokens: Kc, Vc [pages][Hk][page][dh].  Token t of sequence b lies in
 * page table[b][t / page], at t % page.
 *   SPT_CACHE_BF16  values as bf16; ks, vs NULL
 *   SPT_CACHE_E4M3  values as 8-bit codes (e4m3: 4 exponent bits, 3 fraction bits, no infinities), and a byte for
 *                   every row of dh values in ks, vs [pages][Hk][page]: value = code * 2^(byte - 127).  The
 *                   exponent is the least from -127 on with which the row's largest finite magnitude is at most 448,
 *                   rounding is to nearest even (not up to 2^128: at most 240 2^120), values that are not finite become
 *                   the NaN code.  Every value so held is exact in bf16. */
typedef struct {
  int32_t pages;     /* pages of the pool */
  int32_t page;      /* tokens of a page: 16, 32, 64, 128 or 256 */
  int32_t Hk, dh;    /* Hk at most 65535 */
  int32_t format;    /* SPT_CACHE_BF16 or SPT_CACHE_E4M3 */
  int32_t B;         /* sequences, 1 .. 65535 */
  int32_t max_pages; /* row length of table: a sequence has at most max_pages * page tokens (below 2^31) */
} spt_cache_shape_t;

#define SPT_CACHE_BF16 0
#define SPT_CACHE_E4M3 1

/* Rows of K, V [T][Hk][dh] bf16 into the pages of their sequences: sequence b owns rows cu[b] .. cu[b+1]-1,
 * and they become its tokens start[b], start[b] + 1, ...  A token whose number lies outside 0 .. max_pages * page - 1, or whose
 * entry of table outside 0 .. pages - 1, is not written; nothing else in the pool is touched.  Sequences that
 * share a page must not write the same token of it in one call.
 *   strides  host, or NULL for dense: elements per row and head of K, V: 4 numbers, as above
 *   table int32 [B][max_pages];  start int32 [B];  cu int32 [B+1] as above, cu[B] <= T;  T: 1 .. 2^26 - 1 */
int spt_cache_write(const spt_cache_shape_t* shape, int32_t T, const void* K, const void* V, const int64_t* strides,
                    const int32_t* table, const int32_t* start, const int32_t* cu, void* Kc, void* Vc,
                    uint8_t* ks, uint8_t* vs, void* stream);

/* The reverse: rows cu[b] .. cu[b+1]-1 of K, V become what the cache holds for tokens start[b], start[b] + 1, ... of
 * sequence b (zeros for a token that spt_cache_write would not write); rows behind cu[B] are left as they were. */
int spt_cache_read(const spt_cache_shape_t* shape, int32_t T, void* K, void* V, const int64_t* strides,
                   const int32_t* table, const int32_t* start, const int32_t* cu, const void* Kc,
                   const void* Vc, const uint8_t* ks, const uint8_t* vs, void* stream);

/* Attention of one query for each sequence over the first lens[b] tokens of its pages (its own among them, once
 * spt_cache_write has put it there):  Y[b][h] = softmax_j(scale Q[b][h].K[j]) V.  A length of zero or below, or no key with
 * a score above -inf, gives zeros; lengths above max_pages * page count as that; tokens whose entry of table lies outside
 * 0 .. pages - 1 are left out.  What lies in a page behind the last token does not matter.
 *   Q, Y bf16 [B][H][dh];  strides host, or NULL for dense: of Q, Y: 4 numbers, as above
 *   lens int32 [B];  scale positive, at most 2e38
 *   ws: spt_attn_decode_workspace_bytes(shape, H) bytes, 256-byte aligned
 * H is at most 65535, B * Hk * ceil(max_pages * page / 32) * ceil(H / Hk / 16) below 2^31, B * H at most 2^23 - 16.
 * Sixteen query heads of a key head are taken at a time: where more share one, its part of the cache is read again for every sixteen.
 * In tables of many tokens the lengths are gone through for every sequence and head: 4096 sequences of 64 tokens, 8 heads on 2,
 * take 2.7 times as long as in a table of 64 tokens, 16384 take 8 times as long.  Of values below 2^-117 that are held in 8 bits
 * the products with their weights lose bits. */
int spt_attn_decode(const spt_cache_shape_t* shape, int32_t H, float scale, const void* Q, const int64_t* strides,
                    const void* Kc, const void* Vc, const uint8_t* ks, const uint8_t* vs, const int32_t* table,
                    const int32_t* lens, void* Y, void* ws, size_t ws_bytes, void* stream);

/* Bytes of workspace spt_attn_decode needs (0 for an invalid shape). */
size_t spt_attn_decode_workspace_bytes(const spt_cache_shape_t* shape, int32_t H);

#ifdef __cplusplus
}
#endif
#endif /* SPT_ATTN_H */
