/*
 * ssv_round.h -- C ABI of the operators around a verification round (same library as ssv_nsa.h, whose conventions,
 * error codes and element types hold here: device pointers owned by the caller, host parameters, nothing allocated,
 * everything enqueued on `stream` without synchronising, nothing launched when an error code is returned).
 *
 * One round of speculative verification: the verifier's attention over committed and draft tokens (ssv_nsa_verify, or
 * ssv_prefix_verify where a batch shares a long prefix and the layer is dense), the verifier's logits turned into one
 * token per draft node (ssv_sample), the drafts that these tokens accept (ssv_accept), the accepted rows of every layer's
 * cache moved behind the committed ones (ssv_commit), and the compressed cache extended (ssv_nsa_compress from
 * seq_lens to committed).
 *
 * Draft nodes as in ssv_nsa.h: node i of sequence b occupies slot seq_lens[b] + i; tree_parents[b*T+i] is -1 (child of the
 * last committed token) or the index (< i) of its parent (other values count as -1); NULL: a chain.  n_query[b] (NULL: T)
 * nodes of sequence b exist.  Lengths read from device memory are clamped to the host-side bounds of the parameters.
 * The threads of a launch are counted in 32 bits: problems that need more are SSV_EUNSUPPORTED.
 */
#ifndef SSV_ROUND_H
#define SSV_ROUND_H

#include "ssv_nsa.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ssv_prefix_params {
    int32_t B, T;             /* sequences; draft nodes per sequence (row capacity), 1..SSV_MAX_T */
    int32_t H, H_kv;          /* query heads, KV heads; H / H_kv in {1,2,4,8,16} */
    int32_t d_k, d_v;         /* head dims; supported (dtype, d_k, d_v): those of ssv_nsa_supported */
    int32_t n_prefix;         /* prefixes; B % n_prefix == 0: sequence b reads prefix b / (B / n_prefix) */
    int32_t dtype;            /* SSV_F32 or SSV_BF16: type of q, all K and V, out */
    float   scale;            /* softmax scale, 2^-100 to 2^100; 0 => 1/sqrt(d_k) */
    int32_t max_prefix_len;   /* host-side bound on prefix_lens[g]: rows of k_prefix / v_prefix per (prefix, KV head); 0: no prefix */
    int32_t max_seq_len;      /* host-side bound on seq_lens[b]; k and v hold at least max_seq_len + T rows per (sequence, KV head) */
    int64_t kp_stride[3], vp_stride[3];   /* elements: prefix, KV head, row */
    int64_t k_stride[3], v_stride[3];     /* elements: sequence, KV head, row */
    int64_t q_stride[3], out_stride[3];   /* elements: sequence, node, head; all zero = contiguous [B,T,H,d]; rows of out do not overlap */
} ssv_prefix_params;

/*
 * Dense verification attention for a batch that shares prefixes: every draft node attends to the prefix_lens[g] rows of its
 * sequence's prefix, to the seq_lens[b] committed rows of its own sequence behind it, to itself and to its ancestors;
 * softmax over all of them together.  The rows of a prefix are read for all its sequences at once.  Decoding without drafts is
 * T = 1, a batch without a common prefix max_prefix_len = 0 (k_prefix, v_prefix, prefix_lens may then be NULL).
 *   q [B,T,H,d_k]; k_prefix, v_prefix [n_prefix,H_kv,rows,d]; k, v [B,H_kv,rows,d]; out [B,T,H,d_v]; strides above, the feature
 *   dimension is contiguous; K and V bases and strides are multiples of 16 bytes.
 *   prefix_lens [n_prefix], seq_lens [B], n_query [B] or NULL, tree_parents [B,T] or NULL: device int32.
 *   Rows of out of nodes i >= n_query[b] are 0.  Rows beyond the lengths may hold anything; a row that some node of the
 *   sequence attends to must hold finite values.
 *   Up to 2^19 sequences (and prefixes) times KV heads times groups of rows, a group being 16 of a sequence's T H / H_kv rows (or of those
 *   of a prefix's sequences), of more than 16 rows 256 (bf16) or 32 (fp32); else SSV_EUNSUPPORTED, as are rows 32 MiB apart and more.
 *   workspace: >= ssv_prefix_workspace_bytes(p) bytes, 256-byte aligned; contents need not be preserved or initialised;
 *   calls sharing a workspace must not overlap in time.
 * Scores, softmax statistics and sums are fp32; with bf16 inputs the probabilities are rounded to bf16 for the matrix
 * instructions, the result is rounded once to the type of out.  Scores times the scale stay within +-2^27: a reference maximum
 * is subtracted in fp32, and its rounding is a factor of all weights of a row, which has to stay in range.
 */
int ssv_prefix_verify(const void* q, const void* k_prefix, const void* v_prefix, const void* k, const void* v,
                      const int32_t* prefix_lens, const int32_t* seq_lens, const int32_t* n_query, const int32_t* tree_parents,
                      const ssv_prefix_params* p, void* out, void* workspace, size_t workspace_bytes, void* stream);

/* Scratch bytes ssv_prefix_verify needs for p; 0 if p is invalid. */
size_t ssv_prefix_workspace_bytes(const ssv_prefix_params* p);

typedef struct ssv_sample_params {
    int32_t B, T;             /* sequences; nodes per sequence */
    int32_t V;                /* vocabulary size, 1..SSV_SAMPLE_MAX_V */
    int32_t dtype;            /* SSV_F32 or SSV_BF16: type of logits */
    int64_t logits_stride[2]; /* elements: sequence, node; all zero = contiguous [B,T,V]; the vocabulary is contiguous */
} ssv_sample_params;

#define SSV_SAMPLE_MAX_V (1 << 20)

/*
 * One token per node from the verifier's logits and a given random number each.  With x the node's logits (NaN counts
 * as -inf), M = max x and w_j = exp((x_j - M) / temperature): order the vocabulary by descending x, ties by ascending index, and
 * keep its first n = min(n_k, n_p, n_m) entries, n_k = top_k, n_p = the fewest entries that hold at least top_p of the sum of w
 * over the first n_k, n_m = the entries with w >= min_p.  The token is the lowest index j with
 *   (sum of w over the kept indices <= j)  >  u * (sum of w over all kept indices),
 * its probability w_j / (sum over the kept).  The same u in [0, 1) gives the same token, run after run.
 *   temperature, top_k, top_p, min_p [B] (device; one value per sequence; each may be NULL = 1, all, 1, 0).
 *   temperature <= 0 or NaN: the lowest index with x = M, probability 1.  top_k <= 0 or >= V: all.  top_p >= 1 or NaN: all, <= 0: the
 *   first entry alone.  min_p <= 0 or NaN: all; >= 1 counts as 1.  M = +inf: the entries at +inf have weight 1, the others 0.
 *   u [B,T] (device float32; NaN and values below 0 count as 0, values of 1 and more give the last kept index of positive weight).
 *   n_query [B] or NULL: logits of nodes i >= n_query[b] are not read.
 *   tokens [B,T] int32, probs [B,T] float32 or NULL (device, written): -1 and 0 for nodes i >= n_query[b] and for nodes
 *   without a logit above -inf.
 *   workspace: >= ssv_sample_workspace_bytes(p) bytes, 256-byte aligned, as in ssv_prefix_verify.
 * Weights and their sums are computed in 64 bits: a token of a large vocabulary has a weight far below the rounding of a 32-bit
 * sum, and a rounding of the running sum moves every border behind it.  The sums that top_p is compared with are 64-bit integers,
 * off by V 2^-63 of the whole sum at most, with top_k by 2^-40 of the sum over the first top_k at most.
 */
int ssv_sample(const void* logits, const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
               const float* u, const int32_t* n_query, const ssv_sample_params* p, int32_t* tokens, float* probs,
               void* workspace, size_t workspace_bytes, void* stream);

/* Scratch bytes ssv_sample needs for p; 0 if p is invalid. */
size_t ssv_sample_workspace_bytes(const ssv_sample_params* p);

/*
 * Drafts accepted by the verifier's tokens.  Starting at the last committed token, whose next token is root_tokens[b], the
 * walk goes to the child whose draft token equals the token that the verifier put behind its parent (the lowest index among equal
 * siblings) and ends where there is none.  Whatever the drafts are, the accepted tokens and the one that follows them are
 * distributed as the verifier's own samples.
 *   draft_tokens [B,T]: token of every draft node; sampled [B,T]: the verifier's token behind every node (ssv_sample;
 *   negative: matches nothing); root_tokens [B]: its token behind the last committed one.
 *   path [B,T] (written): accepted nodes in order, padded with -1; n_accepted [B]; next_tokens [B]: the verifier's token
 *   behind the last accepted node (root_tokens of the next round); committed [B] = seq_lens + n_accepted.  next_tokens may be the
 *   buffer of root_tokens and committed that of seq_lens.
 * All pointers are device int32; 1 <= T <= SSV_MAX_T.
 */
int ssv_accept(const int32_t* draft_tokens, const int32_t* root_tokens, const int32_t* sampled, const int32_t* seq_lens,
               const int32_t* n_query, const int32_t* tree_parents, int32_t B, int32_t T, int32_t* path, int32_t* n_accepted,
               int32_t* next_tokens, int32_t* committed, void* stream);

typedef struct ssv_commit_params {
    int32_t layers;           /* caches addressed by the first stride; 1: one layer */
    int32_t B, T, H_kv;
    int32_t d_k, d_v;         /* row lengths; times the element size multiples of 16 bytes */
    int32_t dtype;            /* SSV_F32 or SSV_BF16 */
    int32_t kv_capacity;      /* rows of k / v per (layer, sequence, KV head) */
    int64_t k_stride[4], v_stride[4];   /* elements: layer, sequence, KV head, row; multiples of 16 bytes; caches do not overlap */
} ssv_commit_params;

/*
 * Moves the accepted draft rows to the front of the draft slots, in place: row seq_lens[b] + path[b][j] of K and V becomes row
 * seq_lens[b] + j, j < n_accepted[b], in every layer and KV head.  seq_lens are the lengths before the round (those of
 * ssv_accept's input).  Paths ascend, as ssv_accept's do: a sequence's rows from the first entry on that is negative, not
 * above the one before it, T or more, or beyond kv_capacity are left as they are.  No other row changes.
 */
int ssv_commit(void* k, void* v, const int32_t* path, const int32_t* n_accepted, const int32_t* seq_lens,
               const ssv_commit_params* p, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SSV_ROUND_H */
