/*
 * caote_paged.h — attention over packed prompts and over a K/V cache in pages, and eviction from such a cache by accumulated
 * attention weight. Part of libcaote.so; conventions (streams, errors, ownership, workspaces, alignment) are those of caote.h.
 *
 * How they go together: a prompt is attended whole (caote_prompt_attend), its K and V rows and the weight each of its tokens
 * received go into pages (caote_paged_append), and the lightest tokens beyond the budget are evicted (caote_paged_evict).
 * From then on every call brings new tokens of some sequences, one or a block of each: caote_paged_append,
 * caote_paged_attend, caote_paged_evict.
 *
 * Layout. Innermost dimension last; T = total_new rows of all sequences' new tokens, one sequence behind another:
 *   cu           [B + 1]            int32; the new tokens of sequence b are rows cu[b] .. cu[b + 1] - 1 (none is allowed)
 *   q            [T, Hq,  d]        I/O dtype; rows of q_stride elements from one token to the next
 *   k, v (new)   [T, Hkv, d]        I/O dtype; rows of kv_stride elements from one token to the next
 *   o            [T, Hq,  d]        I/O dtype: the fp32 sums are rounded once
 *   lse          [T, Hq]            fp32: log of the row's sum of exponentials
 *   K, V         [n_pages, Hkv, page_size, d]  I/O dtype
 *   mass         [n_pages, Hkv, page_size]     fp32: the attention weight that the token has received, summed over the G
 *                                              query heads of its KV head; of prompts [T, Hkv]
 *   pos          [n_pages, Hkv, page_size]     int32: the token's original position
 *   page_table   [B, max_pages]     int32: slot j of sequence b lies in page page_table[b, j / page_size]. Entries behind a
 *                                   sequence's length are not read.
 *   len, n_seen, budget, n_evict [B] int32: tokens in the cache, tokens ever appended, tokens to keep, tokens evicted
 * Values: weighted values are summed in fp32, with weights of up to 2^20 in bf16 (2^0 in fp32) before they are divided by their sum, so
 * |v| n has to stay below 2^107 (2^127). A row that sees a NaN or a logit of +inf is NaN in o and lse, and so are the weights that it
 * gives; a row all of whose logits are -inf is NaN in o. A NaN or infinity in v may also reach the rows of the tokens before it.
 * Outputs must not overlap inputs. Strides in elements, 0 = dense; q, k and v may be slices of one buffer. q, k, v, K, V, o must be
 * 16-byte aligned, and so must their strides in bytes; the other arrays 4-byte aligned.
 *
 * Calls that write pages (append, evict, attend with mass) need pages that belong to one sequence each. Calls that only read
 * them do not: sequences may share pages.
 *
 * What only the device can see goes to the workspace's status word (caote_read_status): CAOTE_ERR_BAD_LENGTH (cu outside
 * [0, T], more than max_new new tokens, len outside [new tokens, max_pages * page_size]: the sequence is skipped; cu not ascending:
 * append moves no length on, the other calls' outputs mean nothing), CAOTE_ERR_BAD_PAGE (a page index outside [0, n_pages); nothing is
 * read or written out of bounds, nor in other sequences' pages; attend: the outputs of that sequence and what its own tokens' weights
 * grow by mean nothing, append: the sequence keeps its length, evict: it is skipped), CAOTE_ERR_OVERFLOW as in caote.h.
 */
#ifndef CAOTE_PAGED_H_
#define CAOTE_PAGED_H_

#include "caote.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t batch;      /* B >= 1                                                                    */
  int32_t n_q_heads;  /* Hq, a multiple of n_kv_heads; G = Hq / Hkv <= 16                          */
  int32_t n_kv_heads; /* Hkv >= 1                                                                  */
  int32_t head_dim;   /* d in {64, 128}                                                            */
  int32_t page_size;  /* tokens per page: 16, 32, 64, 128 or 256. Prompts alone: 0                 */
  int32_t n_pages;    /* pages in the pool; n_pages * Hkv * page_size < 2^31. Prompts alone: 0     */
  int32_t max_pages;  /* columns of the page table, max_pages * page_size <= 2^31 - 2^16; prompts: 0 */
  int32_t total_new;  /* T >= 1, T * G < 2^28                                                      */
  int32_t max_new;    /* most new tokens of one sequence in this call, 1 .. T                      */
  int32_t dtype;      /* caote_dtype_t of q, k, v, K, V, o                                         */
  float scale;        /* logits are scale * <q, k>                                                 */
  int32_t flags;      /* reserved, must be 0                                                       */
} caote_paged_params_t;

/* Bytes of scratch for all calls below with these parameters; 0 if they are invalid. A workspace made for larger total_new
 * and max_new (everything else equal) serves smaller ones. Its first 256 bytes are as in caote_workspace_bytes. With bf16 pages it holds
 * the logits of up to 16 rows for every slot of the page table, batch * Hkv * max_pages * page_size * 32 (rows <= 8) or 64 bytes, so
 * max_pages is best no larger than the longest cache needs. */
CAOTE_API size_t caote_paged_workspace_bytes(const caote_paged_params_t* params);

/* Causal attention inside every packed prompt (Sec. 2, prompt prefill): for token i of a prompt
 *   o_i = sum_{j <= i} softmax_j(scale * <q_i, k_j>) v_j,   lse_i = log sum_{j <= i} exp(scale * <q_i, k_j>),
 *   mass[j, h] = sum over the G heads and the tokens i >= j of the weight of j  (f_score of H2O, Sec. 2).
 * lse, mass nullable. Page fields of params are not looked at. */
CAOTE_API int caote_prompt_attend(const caote_paged_params_t* params, const void* q, int64_t q_stride, const void* k,
                                  const void* v, int64_t kv_stride, const int32_t* cu, void* o, float* lse, float* mass,
                                  void* workspace, size_t workspace_bytes, caote_stream_t stream);

/* New rows into the pages: for token i of sequence b, slot len[b] + i gets its K and V row, pos = n_seen[b] + i and
 * mass = mass_new[cu[b] + i, h] (0 where mass_new is NULL); then len[b] and n_seen[b] grow by the number of new tokens.
 * mass, pos, n_seen, mass_new nullable (pos without n_seen: the slot). */
CAOTE_API int caote_paged_append(const caote_paged_params_t* params, void* K, void* V, float* mass, int32_t* pos,
                                 const int32_t* page_table, int32_t* len, int32_t* n_seen, const void* k_new,
                                 const void* v_new, int64_t kv_stride, const float* mass_new, const int32_t* cu,
                                 void* workspace, size_t workspace_bytes, caote_stream_t stream);

/* Attention of every sequence's new tokens, which are the last ones of its cache (append first): with n = len[b] and m new
 * tokens, token i attends to slots j <= n - m + i (Sec. 2, block-wise prefill and generation). o, lse as above;
 * mass, nullable: += the weight that every slot received, summed over the G heads and the m tokens. lse nullable. */
CAOTE_API int caote_paged_attend(const caote_paged_params_t* params, const void* q, int64_t q_stride, const void* K,
                                 const void* V, float* mass, const int32_t* page_table, const int32_t* len,
                                 const int32_t* cu, void* o, float* lse, void* workspace, size_t workspace_bytes,
                                 caote_stream_t stream);

/* Eviction by accumulated attention weight: k = max(0, len[b] - budget[b]) (a budget below 1 counts as 1) tokens of every KV
 * head of sequence b go, the first in the order (sheltered, bits of mass, pos); sheltered are tokens with pos < sinks or
 * pos >= n_seen[b] - recent, which go last, the oldest first. mass >= +0 (other bits sort as unsigned numbers). Then the
 * survivors of the last k slots fill the holes, len[b] -= k: pages behind the new length are free.
 *   evict_idx [B, Hkv, max_evict] out: the slots that went, ascending;  n_evict [B] out: k. */
CAOTE_API int caote_paged_evict(const caote_paged_params_t* params, void* K, void* V, float* mass, int32_t* pos,
                                const int32_t* page_table, int32_t* len, const int32_t* n_seen, const int32_t* budget,
                                int32_t sinks, int32_t recent, int32_t* evict_idx, int32_t max_evict, int32_t* n_evict,
                                void* workspace, size_t workspace_bytes, caote_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* CAOTE_PAGED_H_ */
