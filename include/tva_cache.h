/*
 * libtva -- long caches: K/V rows held in 4 bits (store, read back, the verification attention over them), and
 * eviction (how much attention each cached key has received, which keys stay, the move that closes the gaps).
 * Same conventions as tva.h: device pointers owned by the caller, work queued on `stream` (hipStream_t as void*),
 * nothing allocated, no host synchronisation, negative tva_status on rejected arguments (then nothing is queued).
 *
 * The 4-bit row (TVA_ROWS_E2M1).  An element is a code of the OCP 4-bit floating point format E2M1 (1 sign, 2 exponent,
 * 1 mantissa bit): the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6.  A row of D elements (one token, one KV head) is D/2 bytes,
 * element 2i in the low four bits of byte i.
 *   K: value = code * 2^(x - 127), one byte x for every 32 consecutive elements (D/32 bytes per row).
 *   V: value = code * s, one s per row, a bf16 number with at most 4 significant bits.
 * (K's scales are powers of two because the matrix cores multiply such blocks as they are; V's scale is per row
 * because it is taken into the softmax weight of the key.)  All values are exact in bf16.
 */
#ifndef TVA_CACHE_H
#define TVA_CACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TVA_ROWS_BF16 = 0, /* 2 bytes per element */
  TVA_ROWS_E4M3 = 1, /* 1 byte per element (tva_args.kv_fp8), K = k_scale * value, V = v_scale * value */
  TVA_ROWS_E2M1 = 2  /* 4 bits per element and the scales above */
} tva_row_kind;

/*
 * A K/V cache, dense or paged as in tva_args (exactly one of cu_L, page_table):
 *   dense : position t of sequence b is row cu_L[b] + t; sequence b has the room cu_L[b+1] - cu_L[b]
 *   paged : position t is slot t % page_size of page page_table[b*max_pages + t/page_size]; the room is max_pages pages
 * The first element of KV head g of a position is element page*stride_page + slot*stride_tok + g*stride_head, strides
 * counted in ELEMENTS whatever the kind (page = 0, slot = row in the dense form).  0 = the packed default, [.., Hkv, D]
 * token-major.  BF16: multiples of 8, E4M3: of 16, E2M1: of D (a row's scales are found by element / D).
 * Positions are below 2^30; E2M1 row numbers (element / D) below 2^32, and stride_tok below 2^25 (2^24 bytes).
 * Head-major ([.., Hkv, page_size, D]: stride_tok = D, stride_head = page_size*D) keeps a head's keys together.
 * tva_cache_store and tva_evict_move write in place: a page (or row) that they reach belongs to one sequence.  Sequences that
 * share a prefix's pages are given pages of their own before either is called for those positions; the other calls only read.
 */
typedef struct tva_cache {
  int32_t kind; /* a tva_row_kind */
  int32_t page_size, max_pages;
  float k_scale, v_scale;           /* E4M3 only: one scale per tensor, 0 is read as 1 */
  int32_t reserved;
  void *k, *v;                      /* device, 16-byte aligned */
  void *k_row_scale, *v_row_scale;  /* E2M1 only, device: uint8 [rows, D/32] and bf16 [rows], row = element / D */
  const int32_t *cu_L;              /* device [B+1] or NULL */
  const int32_t *page_table;        /* device [B, max_pages] or NULL */
  int64_t stride_page, stride_tok, stride_head;
} tva_cache;

/*
 * tva_cache_store: rows in bf16 are rounded to the cache's 4-bit rows (kind E2M1; others: TVA_UNSUPPORTED).
 * tva_cache_load: the inverse, the values of 4-bit rows written to bf16 rows (exact).
 *
 * Sequence b has n_b rows: path_len[b] of them, row j being row cu_T[b] + path[b*max_rows + j] of k_rows / v_rows (an
 * accepted path, tva_accept_greedy's outputs), or without path all rows cu_T[b] .. cu_T[b+1]-1 in order (a prompt).
 * Row j is position L[b] + j of the cache.  At most max_rows rows of a sequence are taken.
 *
 * Rounding of a K group of 32 and of a V row, a the largest finite magnitude in it:
 *   K: the smallest power of two s with a <= 6 s, kept within 2^-96 .. 2^124;
 *   V: the smallest s with 4 significant bits and a <= 6 s, kept within the same range.
 * An element becomes the code nearest to element / s, of two equally near the one with an even code; magnitudes above
 * 6 s become 6 s, infinities among them; NaN becomes 0.  A row without a magnitude has s = 2^-96.
 *
 * A position outside the sequence's room, or a path entry that is not one of the sequence's rows, is left out and, if
 * err_flag is given (zero on entry), stores 1 + b there.  L_out[b] = L[b] + min(n_b, max_rows) if given (not L itself;
 * store only).  Path entries of a load are distinct.  n_layers > 1: layer l's cache starts layer_stride_cache elements (a multiple of D) behind layer l-1's,
 * its rows layer_stride_rows elements behind.  D is 64 or 128; the K/V head count is free.
 */
typedef struct tva_rows_args {
  int32_t B, Hkv, D;
  int32_t max_rows;               /* host-side bound of n_b, row length of path */
  const int32_t *cu_T;            /* device [B+1] */
  const int32_t *L;               /* device [B], the first position */
  const int32_t *path, *path_len; /* device [B, max_rows], [B]; or both NULL */
  void *k_rows, *v_rows;          /* device bf16 [cu_T[B], Hkv, D]: read by store, written by load */
  tva_cache cache;
  int32_t *L_out;    /* device [B] or NULL */
  int32_t *err_flag; /* device int32[1] or NULL */
  int32_t n_layers;  /* 0 or 1: one layer */
  int64_t layer_stride_cache, layer_stride_rows;
} tva_rows_args;

int tva_cache_store(const tva_rows_args *a, void *stream);
int tva_cache_load(const tva_rows_args *a, void *stream);
size_t tva_sizeof_rows_args(void);

/*
 * tva_tree_verify_attn (tva.h) over a cache of 4-bit rows: sequence b's T_b = cu_T[b+1]-cu_T[b] tree tokens (one: plain
 * decoding) against its L[b] cached tokens and, in bf16, the tree's own K/V under the ancestor sets.  Same shapes,
 * same definition with K and V the values of the rows; out is bf16, rounded once from the fp32 result (the next product
 * takes bf16), lse may be NULL.  Sums and softmax weights are fp32; as a factor of V a weight has 16 bits, that of a cached key
 * with no more than an eighth of its row possibly 8 (half a step, 2^-8 of that weight, as in tva_tree_verify_attn).
 * A row that attends to nothing gets out = 0, lse = -inf; a tree token's K or V that is not finite reaches the rows that see
 * it, and no others.  num_splits: into how many parts the keys of each sequence are split, 0 = the library chooses, and may
 * deal several sequences' keys out together.  The workspace holds partial results (0 bytes when nothing is split); what it
 * holds before does not matter, and calls that overlap need one each.
 */
typedef struct tva_attn4_args {
  int32_t B, Hq, Hkv, D;
  int32_t sum_T, max_T;   /* cu_T[B], host-side bound of T_b (<= TVA_MAX_TREE) */
  int32_t mask_words;     /* 64-bit words per ancestor-mask row, >= ceil(max_T/64), <= 2; ignored with parent */
  int32_t max_L;          /* host-side bound of L[b] (a value below some L[b] truncates that sequence's context) */
  float scale;
  int32_t num_splits;
  int32_t plan_rows;           /* query rows (nodes x heads of a KV head) per workgroup: 32, 64 or 128; 0 = the library chooses.  A
                                  tuning and testing aid: every value computes the same for every input, to the roundings above */
  int32_t reserved;
  const int32_t *cu_T, *L;     /* device [B+1], [B] */
  const void *q;               /* device bf16 [sum_T, Hq, D] */
  const void *k_tree, *v_tree; /* device bf16 [sum_T, Hkv, D] */
  const uint64_t *anc_mask;    /* device [sum_T, mask_words], or NULL and parent is given */
  const int32_t *parent;       /* device [sum_T] (parent[i] < i, -1 = root), read when anc_mask is NULL */
  tva_cache cache;             /* kind E2M1 */
  void *out;                   /* device bf16 [sum_T, Hq, D] */
  float *lse;                  /* device fp32 [sum_T, Hq] or NULL */
  void *workspace;             /* device, 16-byte aligned */
  size_t workspace_bytes;      /* >= tva_attn4_workspace_bytes(a) */
} tva_attn4_args;

int tva_tree_verify_attn_4bit(const tva_attn4_args *a, void *stream);
size_t tva_attn4_workspace_bytes(const tva_attn4_args *a); /* reads shapes only; (size_t)-1 on invalid ones */
int32_t tva_attn4_plan_splits(const tva_attn4_args *a);    /* parts per sequence, or per 64 sequences dealt out together; -1 on invalid shapes */
size_t tva_sizeof_attn4_args(void);

/*
 * The attention that cached keys receive, added up: what eviction goes by.  Called after the attention and the commit
 * of a step.  Sequence b's n_b newest tokens (rows as in tva_rows_args: an accepted path, or all of cu_T; max_rows at most,
 * as many as tva_cache_store took) sit at positions L[b]-n_b .. L[b]-1 of its cache, and row i of them saw the positions
 * t <= L[b]-n_b+i.  With q and lse of those rows (the attention's input and output), for every KV head g and position t
 *     weight[b,g,t] = (t < L[b]-n_b ? weight[b,g,t] : 0) + sum over rows i that saw t, query heads h of g,
 *                                                          exp(scale * <q[i,h,:], K[t,g,:]> - lse[i,h])
 * so what the new tokens' entries held before does not matter.  A row whose lse is -inf adds nothing, and neither does a path
 * entry that is not one of the sequence's rows.  Entries from L[b] on are left as they are.  pos, if given, gets
 * first_pos[b] + i at the new tokens' entries: the age that eviction can protect.  Sums are fp32, in an order that does not
 * change from call to call.
 * Each head of each sequence has ld entries (>= every L[b]) in weight and pos.  max_L truncates as in tva_args.
 */
typedef struct tva_key_weight_args {
  int32_t B, Hq, Hkv, D;
  int32_t max_rows, max_L;
  float scale;
  int32_t reserved;
  const int32_t *cu_T;            /* device [B+1] */
  const int32_t *path, *path_len; /* device [B, max_rows], [B]; or both NULL */
  const int32_t *L;               /* device [B]: the lengths with the new tokens */
  const void *q;                  /* device bf16 [cu_T[B], Hq, D] */
  const float *lse;               /* device fp32 [cu_T[B], Hq] */
  tva_cache cache;                /* any kind; only its K is read */
  float *weight;                  /* device fp32 [B, Hkv, ld] */
  int32_t *pos;                   /* device int32 [B, Hkv, ld] or NULL */
  const int32_t *first_pos;       /* device int32 [B], with pos */
  int64_t ld;
} tva_key_weight_args;

int tva_key_weights(const tva_key_weight_args *a, void *stream);
size_t tva_sizeof_key_weight_args(void);

#define TVA_EVICT_MAX_SLOTS 262144 /* max_L of tva_evict_select */

/*
 * Which slots stay.  Each of the H weight rows of a sequence (one per KV head; or H = 1 for a choice that all heads share)
 * keeps n = min(keep[b], L[b]) of its first L[b] slots: first the protected ones, then by weight, largest first; among
 * equal ones the lower slot.  Protected: slots below n_first, and those whose age counts as new: pos[slot] >= newest[b]
 * (without pos: slot >= newest[b]; without newest: none).  Protected slots are equals: if there are more of them than n, the
 * lower ones stay, whatever their age, so keep is no less than n_first and the new ones together where these are meant to
 * stay.  A NaN weight is below all others; -0 equals 0.
 *
 * Softmax does not depend on the order of the keys, so nothing is shifted: kept slots below n stay where they are, and
 * the m-th gap below n (in ascending order) is given the m-th kept slot from n on.  src[.., j] for j < n is the slot whose
 * row lies in slot j afterwards; entries from n on are not written.  L_out[b] = n.
 * n_layers > 1: weight, pos and src are [n_layers, B, H, ld / ld_src], lengths and bounds are the same for every layer.
 */
typedef struct tva_evict_select_args {
  int32_t n_layers, B, H, max_L; /* max_L: host-side bound of L[b] (longer sequences are taken to end there) */
  int32_t n_first, reserved;
  const int32_t *L, *keep;       /* device [B] */
  const int32_t *newest;         /* device [B] or NULL */
  const float *weight;           /* device fp32 [n_layers, B, H, ld] */
  const int32_t *pos;            /* device int32, like weight, or NULL */
  int64_t ld;                    /* >= max_L */
  int32_t *src;                  /* device int32 [n_layers, B, H, ld_src] */
  int64_t ld_src;                /* >= the largest n (a row keeps no more than it) */
  int32_t *L_out;                /* device [B] or NULL; not L or keep */
} tva_evict_select_args;

int tva_evict_select(const tva_evict_select_args *a, void *stream);
size_t tva_sizeof_evict_select_args(void);

/*
 * The move that follows: slot j < n[b] of every head takes the rows (K, V, their scales, and the entries of weight and
 * pos where given) of slot src[.., j] where that is not j itself.  Sources lie at n[b] or behind (tva_evict_select's
 * do), so nothing that is read is written.  An entry below n[b] other than j, outside the sequence's room, or with weight or pos outside ld, is left
 * out and, if err_flag is given (zero on entry), stores 1 + b there; so does a slot j outside the room.
 * H: weight rows per sequence, Hkv or 1 (then src is shared by the heads, and weight and pos have one row).
 * At most max_keep slots of a sequence are looked at.  D: 64 or 128.
 */
typedef struct tva_evict_move_args {
  int32_t n_layers, B, H, Hkv, D;
  int32_t max_keep;    /* host-side bound of n[b] */
  const int32_t *n;    /* device [B]: tva_evict_select's L_out */
  const int32_t *src;  /* device int32 [n_layers, B, H, ld_src] */
  int64_t ld_src;
  tva_cache cache;     /* any kind */
  int64_t layer_stride_cache; /* elements */
  float *weight;       /* device fp32 [n_layers, B, H, ld] or NULL */
  int32_t *pos;        /* device int32, like weight, or NULL */
  int64_t ld;
  int32_t *err_flag;   /* device int32[1] or NULL */
} tva_evict_move_args;

int tva_evict_move(const tva_evict_move_args *a, void *stream);
size_t tva_sizeof_evict_move_args(void);

#ifdef __cplusplus
}
#endif
#endif /* TVA_CACHE_H */
