/*
 * libtva -- the new tokens' way through a layer: rotary positions of their q and k heads (with the heads' norms, where the
 * model has them), their K/V to the end of each sequence's cache, and their attention over that cache: a chunk of a prompt
 * of any length or a draft tree, over everything or over a sliding window and the first few tokens.
 * Same conventions as tva.h: device pointers owned by the caller, work queued on `stream` (hipStream_t as void*), nothing
 * allocated, no host synchronisation, negative tva_status on rejected arguments (then nothing is queued).
 */
#ifndef TVA_LAYER_H
#define TVA_LAYER_H

#include <stddef.h>
#include <stdint.h>

#include "tva_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * How fast each pair of elements turns, in radians per position: freq[j] = base^(-2j/dims), j < dims/2, and its forms for
 * contexts longer than the model was trained for, by `factor` (>= 1):
 *   PLAIN       as above (factor, original, low, high are ignored)
 *   LINEAR      freq / factor (positions interpolated)
 *   BASE        base is raised to base * factor^(dims / (dims-2)): the fastest pair stays, the slowest is divided by factor
 *   WAVELENGTH  by the turns a pair makes over `original` positions, n_j = original * freq[j] / 2 pi: those of `high` and more
 *               stay, those of `low` and less are divided by factor, between them the two are mixed linearly in n_j
 *   RAMP        the same choice, mixed linearly in j between the pairs that make `high` and `low` turns (the first rounded
 *               down, the second up, both kept within 0 .. dims-1); *magnitude = 0.1 ln(factor) + 1
 * HOST function on HOST memory; freq has dims/2 entries.  *magnitude (may be NULL) is what the rotated elements are multiplied
 * by, 1 but for RAMP.  dims even and >= 4, base > 1; WAVELENGTH and RAMP: original > 0, 0 < low < high.
 */
typedef enum { TVA_ROTARY_PLAIN = 0, TVA_ROTARY_LINEAR = 1, TVA_ROTARY_BASE = 2, TVA_ROTARY_WAVELENGTH = 3, TVA_ROTARY_RAMP = 4 } tva_rotary_scaling;
int tva_rotary_frequencies(int32_t scaling, int32_t dims, double base, double factor, double original, double low, double high,
                           double *freq, double *magnitude);

/*
 * The heads of q and k of new tokens, each normed (where a norm is given) and turned by its token's position.
 * Row r = cu_T[b] + i is token i of sequence b; its position P is pos[r], or without pos L[b] + i, or with anc_mask (without
 * pos) L[b] + d, d = the number of bits set in the row less one: a draft tree's node at depth d.
 *   norm     x'[e] = w[e] * x[e] / sqrt(mean over e of x[e]^2 + eps), over all D elements of a head
 *   turn     pair j < dims/2 is elements (j, j + dims/2), or with `interleaved` (2j, 2j+1) of the first `dims` ones:
 *            u' = magnitude * (u cos a - v sin a), v' = magnitude * (v cos a + u sin a), a = P * freq[j]; elements from
 *            dims on stay
 * Angles are reduced in 64 bits (any int32 position), sums and products are fp32, the result is rounded to bf16 once.  (A
 * norm's sum of squares is an fp32 number: from 2^128 on it is infinite, and the head becomes 0, but for elements that are infinite
 * themselves; with eps 0 a head whose squares all vanish in it has no finite norm.)
 * Rows before cu_T[0] and from cu_T[B] on are left as they are.  q_out may be q with the same stride, k_out k (in place); other
 * overlaps are not allowed.  q or k may be NULL (then so is its output).
 */
typedef struct tva_rotate_args {
  int32_t B, Hq, Hkv, D;        /* D: 64 or 128 */
  int32_t sum_T;                /* rows of q and k; at least cu_T[B] (rows behind it are not looked at) */
  int32_t dims;                 /* 0 (nothing is turned) .. D, a multiple of 16 */
  int32_t interleaved;
  int32_t mask_words;           /* 64-bit words per anc_mask row, 1 or 2 */
  float magnitude;              /* 0 is read as 1 */
  float eps;                    /* >= 0 */
  const int32_t *cu_T, *L;      /* device [B+1], [B]; with pos both may be NULL: all sum_T rows are taken */
  const int32_t *pos;           /* device [sum_T] or NULL */
  const uint64_t *anc_mask;     /* device [sum_T, mask_words] (tva_build_ancestor_mask) or NULL */
  const double *freq;           /* device [dims/2] */
  const void *q, *k;            /* device bf16: head h of row r at r * stride + h * D */
  const void *q_norm, *k_norm;  /* device bf16 [D] or NULL: w */
  void *q_out, *k_out;          /* device bf16 */
  int64_t q_stride, k_stride;   /* elements between rows, multiples of 8, at least the heads' own; 0 = packed */
  int64_t q_out_stride, k_out_stride;
} tva_rotate_args;

int tva_rotate(const tva_rotate_args *a, void *stream);
size_t tva_sizeof_rotate_args(void);

/*
 * The same, and K and V of the new tokens go to the cache: token i of sequence b takes position L[b] + i (whatever position
 * it was turned by).  What is stored is the bf16 row that tva_rotate gives (V: as it is), in the cache's kind:
 *   BF16  as it is;  E4M3  the nearest code to the fp32 quotient by k_scale / v_scale (ties to even), magnitudes above 448
 *   become 448, infinities among them, NaN becomes 0;  E2M1  as tva_cache_store rounds it.
 * r.k is required, r.k_out may be NULL or get the turned keys besides; r.q may be NULL.  r.cu_T and r.L are required.
 * A position outside the sequence's room, or whose entry in the page table is below 0, is left out and, if err_flag is given (zero on
 * entry), stores 1 + b there.  Pages (rows) that are reached belong to one sequence.  L_out[b] = L[b] + T_b if given (not L itself).
 */
typedef struct tva_append_args {
  tva_rotate_args r;
  const void *v;    /* device bf16: head h of row r at r * v_stride + h * D */
  int64_t v_stride;
  tva_cache cache;  /* any kind */
  int32_t *L_out;   /* device [B] or NULL */
  int32_t *err_flag; /* device int32[1] or NULL */
} tva_append_args;

int tva_cache_append(const tva_append_args *a, void *stream);
size_t tva_sizeof_append_args(void);

/*
 * Attention of new tokens whose K/V the cache holds already (token i of sequence b at position L[b] + i: tva_cache_append),
 * T_b = cu_T[b+1]-cu_T[b] of them, any number; L[b] >= 0 cached tokens before them.
 *   without anc_mask  a chunk: token i has position P = L[b] + i and sees the new tokens j <= i
 *   with anc_mask     a draft tree: node i has position P = L[b] + (bits set in its row) - 1 and sees the nodes j whose bit is
 *                     set (T_b <= TVA_MAX_TREE, bits from T_b on are 0)
 * and of the cached tokens all.  With window > 0 a token at position P sees, of those, only keys whose own position is above
 * P - window, or below n_first (window 1: itself and the first ones).  Query head h reads KV head h / (Hq/Hkv).
 *     lse = log sum exp(scale * <q, K>),  out = sum exp(scale * <q, K> - lse) V     over the keys that are seen
 * out is bf16, rounded once from fp32; lse fp32, natural logarithm, may be NULL.  Sums and softmax weights are fp32; as a factor of V
 * a weight is rounded to bf16 (half a step, 2^-8 of it at most), with plan_rows 32 to 16 bits.  Where the library chooses the rows
 * (plan_rows 0), which of the two a row gets therefore goes by the shapes of the call; batches of single tokens with up to 32 query
 * heads to a KV head get 32 rows, and plan_rows 32 gives them to any call.
 * A row that sees nothing gets out = 0, lse = -inf.  A key or value that is not finite reaches the rows that see it, and no others.
 * Rows before cu_T[0] and from cu_T[B] on are left as they are.  Positions outside the sequence's room are not read; a page none of
 * whose positions any token sees may have an entry below 0 in the page table (given back: page 0 is read in its place, to no effect),
 * others below L[b] + T_b are pages.  E2M1 caches are read by tva_tree_verify_attn_4bit: TVA_UNSUPPORTED here.
 * max_T and max_L size the launch: rows i >= max_T are not computed; max_L only shapes the plan.
 * The workspace holds partial results where keys are split (0 bytes when nothing is); what it holds before does not matter, and
 * calls that overlap need one each.  There are 65535 row blocks at most, sum_T * Hq / Hkv / (rows per workgroup) + B (TVA_UNSUPPORTED).
 */
typedef struct tva_chunk_args {
  int32_t B, Hq, Hkv, D;        /* D: 64 or 128 */
  int32_t sum_T, max_T, max_L;  /* host-side: rows of q (at least cu_T[B]), bounds of T_b and L[b] */
  int32_t mask_words;           /* words per anc_mask row, >= ceil(max_T/64), <= 2 */
  int32_t window, n_first;      /* 0 = no window (n_first is then ignored) */
  float scale;                  /* > 0 */
  int32_t num_splits;           /* the most parts a row block's keys are split into; 0 = the library chooses */
  int32_t plan_rows;            /* query rows (tokens x heads of a KV head) per workgroup: 32, 128 or 256; 0 = the library
                                   chooses.  A tuning and testing aid: every value computes the same, to the roundings above */
  int32_t reserved;
  const int32_t *cu_T, *L;      /* device [B+1], [B] */
  const void *q;                /* device bf16, head h of row r at r * q_stride + h * D */
  int64_t q_stride;             /* elements, multiple of 8; 0 = packed */
  const uint64_t *anc_mask;     /* device [sum_T, mask_words] or NULL */
  tva_cache cache;              /* kind BF16 or E4M3; stride_tok below 2^25 */
  void *out;                    /* device bf16 [sum_T, Hq, D] */
  float *lse;                   /* device fp32 [sum_T, Hq] or NULL */
  void *workspace;              /* device, 16-byte aligned */
  size_t workspace_bytes;       /* >= tva_chunk_workspace_bytes(a) */
} tva_chunk_args;

int tva_chunk_attn(const tva_chunk_args *a, void *stream);
size_t tva_chunk_workspace_bytes(const tva_chunk_args *a); /* reads shapes only; (size_t)-1 on invalid ones */
int32_t tva_chunk_plan_rows(const tva_chunk_args *a);      /* query rows per workgroup; -1 on invalid shapes */
int32_t tva_chunk_plan_splits(const tva_chunk_args *a);    /* the most parts of a row block's keys; -1 on invalid shapes */
size_t tva_sizeof_chunk_args(void);

#ifdef __cplusplus
}
#endif
#endif /* TVA_LAYER_H */
