/*
 * nacl.h -- C ABI of the MI355X (gfx950) implementation of NaCl's one-shot
 * encoding-phase KV-cache eviction.
 *
 * Paper: Chen et al., "NaCl: A General and Effective KV Cache Eviction
 * Framework for LLMs at Inference Time", arXiv 2408.03675.
 *
 * For every layer l, batch row b and head h (heads are independent; head-wise
 * eviction, Section 6.3):
 *   score   F[j] = sum over proxy tokens p_i of softmax_j(s * <Q[p_i], K[j]>),
 *           keys j <= p_i only (causal)            -- Section 5.1, F_score
 *   select  S = Pi  u  top-Cp of F over R  u  Cr tokens sampled without
 *           replacement from Softmax(F) over the rest, |S| = C
 *                                                  -- Section 5.1 argmax,
 *                                                     Section 5.2, Algorithm 1
 *   compact K' = K[S], V' = V[S]                   -- Section 3, encoding phase
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Device pointers are HIP device memory of the current device.  Host
 *   pointers are marked HOST.  The library allocates nothing, keeps no state
 *   between calls (apart from the thread-local error text), never
 *   synchronises, and enqueues all work on `stream` (a hipStream_t; NULL is
 *   the default stream).  Outputs are complete once the stream reaches them.
 * - Every function returns a nacl_status.  Arguments are validated on the
 *   host before anything is enqueued; on any error nothing is enqueued and
 *   outputs are untouched.  nacl_last_error_detail() explains the failure.
 * - Q, K, V are [B, H, L, D] tensors addressed by element strides for
 *   (b, h, l); d is contiguous.  Base pointers and every row start must be
 *   16-byte aligned.
 * - Scores are fp32 [B, H, L] contiguous; keep_idx is int32 [B, H, C]
 *   contiguous, strictly ascending per head; k_out / v_out are [B, H, C, D]
 *   contiguous in the input dtype and overlap no input, or are K and V
 *   themselves (in-place compaction, see nacl_compact).
 * - Overlapping calls that share a workspace race; give concurrent calls
 *   their own workspaces.
 */
#ifndef NACL_H
#define NACL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NACL_VERSION 2
#define NACL_MAX_P 4096          /* proxy tokens per head */
#define NACL_MAX_L (1 << 19)     /* prompt length */

typedef enum {
  NACL_OK = 0,
  NACL_ERR_INVALID_ARG = 1,  /* an argument is out of range or inconsistent */
  NACL_ERR_UNSUPPORTED = 2,  /* valid in principle, not supported by the library */
  NACL_ERR_WORKSPACE = 3,    /* workspace missing, misaligned or too small */
  NACL_ERR_HIP = 4           /* a HIP runtime call or kernel launch failed */
} nacl_status;

typedef enum { NACL_F32 = 0, NACL_BF16 = 1 } nacl_dtype;

/* Distribution of the random eviction (Section 5.2).  SOFTMAX is the paper's
 * Softmax(F) (weights exp(F[j])); PROPORTIONAL uses weights F[j]; UNIFORM
 * uses equal weights (the ablation's uniform sampling). */
typedef enum {
  NACL_SAMPLE_SOFTMAX = 0,
  NACL_SAMPLE_PROPORTIONAL = 1,
  NACL_SAMPLE_UNIFORM = 2
} nacl_sampling;

/* The eviction problem of one layer (Section 3, encoding-phase eviction). */
typedef struct nacl_problem {
  int32_t B, H, L, D;        /* batch, heads, prompt length, head dim (64 or 128) */
  int32_t dtype;             /* nacl_dtype of Q, K, V (and of k_out, v_out) */
  int32_t P;                 /* number of proxy tokens, 1 <= P <= min(L, NACL_MAX_P) */
  int32_t n_protect;         /* the last n_protect proxies are always kept (0..P);
                                the paper keeps all proxies: n_protect = P */
  float sm_scale;            /* logit scale s > 0, normally 1/sqrt(D) */
  int64_t q_stride[3];       /* element strides of Q for b, h, l */
  int64_t k_stride[3];       /* element strides of K for b, h, l */
  int64_t v_stride[3];       /* element strides of V for b, h, l */
  const int32_t* proxy_pos;  /* HOST, P positions, strictly increasing, in [0, L);
                                shared by every b and h (Section 5.1) */
  const int32_t* proxy_pos_dev; /* optional DEVICE copy of proxy_pos (same values);
                                NULL: the library stages proxy_pos through the
                                workspace with a stream-ordered copy */
  int32_t q_group;           /* query heads per K/V head (grouped-query attention;
                                0 or 1: multi-head, 1..64).  H counts K/V heads:
                                K, V, scores, keep_idx and the outputs have H
                                heads, Q has H * q_group heads (q_stride[1] steps
                                one query head), and K/V head h is scored by the
                                proxy rows of query heads h*q_group ..
                                h*q_group + q_group - 1, so its score mass is
                                P * q_group.  lse (nacl_score) is then
                                [B, H * q_group, P]. */
} nacl_problem;

/* Workspace bytes the score, select and evict calls need for problem *p
 * (0 on invalid input).  The workspace is device memory, 256-byte aligned,
 * owned by the caller; its contents need no initialisation. */
size_t nacl_workspace_bytes(const nacl_problem* p);

/* Proxy-token scores F (Section 5.1, F_score; Appendix A.7 for the blockwise
 * recomputation).  q, k: device [B,H,L,D].  lse: optional device fp32
 * [B,H,P], the natural log-sum-exp of each proxy row's scaled causal logits
 * as a FlashAttention-2 forward returns it (Appendix A.7, Algorithm 2); with
 * it only the column reduction runs.  NULL: the library computes it (two
 * passes over K).  scores: device fp32 [B,H,L], fully overwritten; keys after
 * the last proxy get 0.
 * Health words (score and evict calls): uint32 word 1 of the workspace
 * (byte offset 4) is this call's, cleared by the call itself; word 2 (byte
 * offset 8) is sticky: every call ORs its bits into it and no call clears it,
 * so it covers every call since the caller last zeroed it (zero it when the
 * workspace is allocated; the Python binding does).  Bit 0: a wave gave up
 * waiting for a head's log-sum-exp after its bounded spin.  Bit 2 (evict
 * only): the compaction met a keep index outside [0, L).  Bit 3 (evict only,
 * heads of more than 32768 tokens): a work-group of the selection gave up
 * waiting for the other slices of its head, or its search for a threshold
 * ran out of rounds.  Never expected; whenever a call's word is non-zero once
 * the stream has completed it, that call's scores, keep_idx, k_out and v_out
 * are not valid. */
int nacl_score(const nacl_problem* p, const void* q, const void* k, const float* lse,
               float* scores, void* ws, size_t ws_bytes, void* stream);

/* Keep set S per head (Section 5.1 argmax, Section 5.2, Algorithm 1).
 * scores: device fp32 [B,H,L] (finite, >= 0).  C: total budget, with
 * n_protect + Cr <= C <= L; Cr: tokens drawn by the random eviction;
 * Cp = C - n_protect - Cr come from the top-Cp scores over the unprotected
 * tokens.  Ties go to the lower token index.  The random draw uses
 * Philox4x32-10 with key = seed and counter (j/4, h, b, layer), token j
 * taking word j mod 4, u = (word + 1/2) / 2^32, Gumbel g = -ln(-ln u) in
 * binary64, key = binary32(log-weight + g); the Cr largest keys among the
 * remaining tokens are kept (Gumbel-top-k).  keep_idx: device int32 [B,H,C],
 * ascending. */
int nacl_select(const nacl_problem* p, const float* scores, int32_t C, int32_t Cr,
                int32_t sampling, uint64_t seed, uint32_t layer, int32_t* keep_idx,
                void* ws, size_t ws_bytes, void* stream);

/* Cache update K0, V0 <- K_S, V_S (Section 3).  k, v: device [B,H,L,D] with
 * the problem's strides; keep_idx: device int32 [B,H,C], strictly ascending
 * per head (as nacl_select writes it); an entry outside [0, L) gives a row
 * of zeros (no memory outside the head is read).  Two output forms:
 *  - k_out, v_out: device [B,H,C,D] contiguous, overlapping no input;
 *  - in place (k_out == k and v_out == v, K and V disjoint): row c of each
 *    head takes row keep_idx[c] of the same head, in the input's own layout,
 *    for c < C; rows C..L-1 keep their old contents.  This is the cache
 *    update of the generation phase (Section 3, "Generation Phase Eviction"),
 *    where the cache is a fixed buffer of L rows per head.
 * Bit-exact row copies. */
int nacl_compact(const nacl_problem* p, const void* k, const void* v,
                 const int32_t* keep_idx, int32_t C, void* k_out, void* v_out,
                 void* stream);

/* Slot form of the in-place cache update, for a generation-phase cache whose
 * rows need not stay in token order (Section 3, "Generation Phase Eviction":
 * the paper fixes which entries stay, not where they sit).  keep_idx: device
 * int32 [B,H,C], the ascending keep set as nacl_select writes it (read only).
 * In each head of k, v (device [B,H,L,D] with the problem's strides, K and V
 * disjoint) the kept rows below C stay where they are and the kept rows at or
 * past C move, in ascending order, into the slots below C whose rows were
 * not kept (taken in ascending order); nothing else is written, so only the
 * kept rows past C are copied.  slot_idx: device int32 [B,H,C] (overlapping
 * nothing above) receives, for each slot c < C, the old row it holds
 * afterwards.  A keep list that is not an ascending set of rows in [0, L)
 * gives zero rows in the slots whose mover lies outside [C, L).  Bit copies. */
int nacl_compact_slots(const nacl_problem* p, void* k, void* v, const int32_t* keep_idx, int32_t C,
                       int32_t* slot_idx, void* stream);

/* Append of decode steps to the cache (Algorithm 1, generation phase: the
 * new token's key and value join the cache): rows [row0, row0 + m) of every
 * head of k, v (device [B,H,L,D] with the problem's k/v strides) take the m
 * rows of k_new, v_new (device [B,H,m,D] contiguous, overlapping neither
 * cache; K and V caches disjoint).  0 <= row0, row0 + m <= L.  Bit copies. */
int nacl_append(const nacl_problem* p, void* k, void* v, int32_t row0,
                const void* k_new, const void* v_new, int32_t m, void* stream);

/* The whole step for one layer: score, select, compact on one stream
 * (Algorithm 1, encoding phase).  Arguments as above; k_out, v_out may be
 * k, v themselves (in-place compaction).  The health words of nacl_score
 * apply: keep_idx, k_out and v_out are not valid when the call's word is
 * non-zero.
 * Generation-phase eviction (Section 3, "Generation Phase Eviction"; the
 * Generation function of Algorithm 1) is the same call at decode shapes:
 * the cache is a [B,H,L,D] buffer with L = C + m rows per head; after the
 * m decoding steps appended their rows (nacl_append at row0 = C + t), call
 * with the current token as the only proxy (proxy_pos = {L - 1},
 * n_protect = 1), its query as a [B,H,1,D] tensor with q_stride[2] = 0, and
 * k_out = k, v_out = v: the C kept entries move to rows 0..C-1 and the next
 * m steps append after them.  Use a different seed per eviction round so
 * the random draws differ between rounds. */
int nacl_evict(const nacl_problem* p, const void* q, const void* k, const void* v,
               int32_t C, int32_t Cr, int32_t sampling, uint64_t seed, uint32_t layer,
               float* scores, int32_t* keep_idx, void* k_out, void* v_out,
               void* ws, size_t ws_bytes, void* stream);

/* Generation-phase eviction with the slot form of the cache update
 * (Section 3, "Generation Phase Eviction"; the Generation function of
 * Algorithm 1): nacl_score, nacl_select and nacl_compact_slots on one stream,
 * in place in k, v.  Arguments as nacl_evict; keep_idx receives the
 * ascending keep set and slot_idx (device int32 [B,H,C]) the old row each
 * slot below C holds afterwards.  At decode shapes (L = C + m, the current
 * token as the only, protected, proxy) only the kept rows among the m newest
 * move, instead of nearly every kept row as in nacl_evict's in-place form.
 * The health words of nacl_score apply. */
int nacl_evict_slots(const nacl_problem* p, const void* q, void* k, void* v, int32_t C, int32_t Cr,
                     int32_t sampling, uint64_t seed, uint32_t layer, float* scores, int32_t* keep_idx,
                     int32_t* slot_idx, void* ws, size_t ws_bytes, void* stream);

/* The whole step without a caller workspace, for callers that cannot
 * allocate device memory (code under HIP graph capture, serving loops,
 * harnesses that forbid hipMalloc).  Arguments and results as nacl_evict,
 * which it runs; p->proxy_pos_dev is required (no host-to-device copy).  The
 * workspace is a built-in device array of NACL_NOALLOC_WORKSPACE_MAX bytes,
 * one per GPU, held until the process ends; problems needing more
 * (nacl_workspace_bytes) return NACL_ERR_UNSUPPORTED.  Nothing is allocated:
 * no hipMalloc, hipFree or allocating library routine.  Every call on a GPU
 * shares that GPU's array, so calls on one GPU that overlap in time (other
 * streams, other threads) race and must be serialised by the caller.
 * health: optional device uint32[2] that receives the call's health words
 * (this call's, then the sticky one accumulated over every such call on the
 * GPU; see nacl_score), copied on the stream after the eviction. */
#define NACL_NOALLOC_WORKSPACE_MAX (64u << 20)
int nacl_evict_noalloc(const nacl_problem* p, const void* q, const void* k, const void* v,
                       int32_t C, int32_t Cr, int32_t sampling, uint64_t seed, uint32_t layer,
                       float* scores, int32_t* keep_idx, void* k_out, void* v_out,
                       uint32_t* health, void* stream);

/* Causal attention of the prefill with the log-sum-exp of every query row:
 * the FlashAttention-2 forward pass whose log-sum-exp Appendix A.7 reuses,
 * so that the score of a layer runs as the single column reduction of
 * Algorithm 2 (nacl_score with lse = lse_proxy reads K once).  bf16 only
 * (NACL_ERR_UNSUPPORTED otherwise); D = 64 or 128; grouped query heads as in
 * the problem struct: query head hq reads K/V head hq / q_group.
 * q: device [B, H*q_group, L, D] with q_stride; k, v: device [B,H,L,D] with
 * k_stride, v_stride; every row stride at least D.
 * out: device bf16 [B, H*q_group, L, D] contiguous, row i of a query head =
 * sum over j <= i of softmax_j(sm_scale <q_i, k_j>) v_j (fp32 accumulation,
 * the probabilities rounded to bf16 for the value product, the row rounded
 * to bf16 once).
 * lse: device fp32 [B, H*q_group, L], the natural log of
 * sum over j <= i of exp(sm_scale <q_i, k_j>).
 * lse_proxy: optional device fp32 [B, H*q_group, P] receiving lse at the
 * proxy rows, the layout of nacl_score's lse argument; it needs
 * p->proxy_pos_dev.  out, lse and lse_proxy overlap nothing else.  The
 * problem is validated as for every call (its proxy fields included), but
 * the proxies change nothing except which rows lse_proxy receives. */
int nacl_attention(const nacl_problem* p, const void* q, const void* k, const void* v, void* out,
                   float* lse, float* lse_proxy, void* stream);

/* ------------------------------------------------------------------------
 * The decoding step between two evictions (Algorithm 1, generation phase):
 * the new tokens' queries and keys are normalised and rotated and join the
 * cache (nacl_rotate_append), attend to it and to a prefix that a group of
 * sequences shares (nacl_prefix_attention), and the next token is drawn from
 * the model's logits (nacl_sample).  The problem describes the cache, as for
 * nacl_append: B, H, L rows per head, D, dtype, q_group, sm_scale, k_stride
 * and v_stride; its proxies and q_stride are validated and not used.
 * ------------------------------------------------------------------------ */

/* The new tokens of one step: T per sequence, a prompt's or a decoding
 * step's.  Token t of sequence b belongs in row row0 + lens[b] + t of each of
 * the sequence's heads. */
typedef struct nacl_step {
  int32_t T;               /* 1..NACL_MAX_L */
  int32_t row0;            /* >= 0; added to every length */
  const int32_t* lens;     /* optional DEVICE [B]: rows each sequence holds before the step (NULL: 0) */
  const int32_t* n_new;    /* optional DEVICE [B]: of sequence b's T tokens the first n_new[b] are
                              real, the others padding (NULL: all real) */
  int64_t q_stride[3];     /* element strides of the new tokens' Q for b, query head, t */
  int64_t k_stride[3];     /* and of their K and V for b, h, t (nacl_rotate_append) */
  int64_t v_stride[3];
  int64_t q_out_stride[3]; /* of nacl_rotate_append's rotated Q */
} nacl_step;

/* Norm and rotation of nacl_rotate_append. */
typedef struct nacl_rotation {
  int32_t rot;             /* the leading entries of a head that are rotated: a multiple of 16, 0..D */
  int32_t interleaved;     /* 0: entry i pairs with i + rot/2; 1: entry 2i with 2i + 1 */
  float eps;               /* >= 0, added to the mean square */
  const void* q_weight;    /* optional DEVICE [D] of the problem's dtype: the norm's weights (NULL: no norm) */
  const void* k_weight;
  const float* inv_freq;   /* DEVICE [rot/2]: radians per position of each pair (unused if rot is 0) */
  int64_t pos_stride;      /* elements between two sequences' positions (0: shared by the batch) */
} nacl_rotation;

/* The step's queries and keys, each head normalised by its root mean square
 * and the weights (where given), then rotated by the token's position, and the
 * keys and values written into the cache:
 *   y = x / sqrt(mean(x^2) + eps) * weight           (y = x without weights)
 *   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin),
 *   angle = positions[b, t] * inv_freq[pair]
 *   q_out = Q',  cache K row row0 + lens[b] + t = K',  cache V row = V (bit copy)
 * in fp32 (the angle in fp64, so far positions keep their accuracy), rounded
 * once to the dtype.  An evicted cache holds fewer rows than the sequence has
 * tokens, so positions are given apart from the rows.
 * q_new: device [B, H*q_group, T, D], k_new, v_new: device [B,H,T,D], with the
 * step's strides (one projection's [B, T, (H*q_group + 2 H) D] output, say).
 * positions: device int32, T consecutive entries per sequence (NULL only if
 * rot is 0).  q_out: device, [B, H*q_group, T, D] with q_out_stride; it may be
 * q_new with the same strides (in place), and overlaps nothing else.  k, v: the
 * cache, [B,H,L,D] with the problem's strides, K and V disjoint and apart from
 * the new tokens, no two rows of them at one place (strides of at least D).
 * Padding tokens (t >= n_new[b]) are not
 * read, and q_out and the cache keep what they hold in their places.  A
 * token whose row lies outside [0, L) joins no cache (its q_out is written).
 * Sequences may not share cache rows.  Base pointers 16-byte aligned, strides
 * multiples of 16 bytes, B * T below 2^28. */
int nacl_rotate_append(const nacl_problem* p, const nacl_step* s, const nacl_rotation* r, const int32_t* positions,
                       const void* q_new, const void* k_new, const void* v_new, void* q_out, void* k, void* v,
                       void* stream);

/* A prefix that groups of sequences share: B / G consecutive sequences read
 * the same rows, sequence b those of group b / (B / G). */
typedef struct nacl_prefix {
  int32_t G;               /* groups, a divisor of B */
  int32_t L;               /* rows per head of the prefix buffers, 1..NACL_MAX_L */
  int64_t k_stride[3];     /* element strides for group, h, row; row strides of at least D */
  int64_t v_stride[3];
  const void* k;           /* DEVICE [G,H,L,D], of the problem's dtype */
  const void* v;
  const int32_t* lens;     /* optional DEVICE [G]: rows in use (NULL: L); clamped to [0, L] */
} nacl_prefix;

/* Workspace bytes of nacl_prefix_attention (0 on invalid input).  Device
 * memory, 256-byte aligned; its contents need no initialisation. */
size_t nacl_prefix_workspace_bytes(const nacl_problem* p, const nacl_step* s, const nacl_prefix* x);

/* Attention of the step's queries to the cache and the shared prefix: query
 * row (b, hq, t) sees the rows in use of its group's prefix (none if x is
 * NULL) and its sequence's cache rows j < row0 + lens[b] + t + 1 (at most L),
 * so the step's own tokens causally.  B * H * q_group * T below 2^26.
 * The prefix's K and V are read once for all the group's rows.
 * q: device [B, H*q_group, T, D] with the step's q_stride (16-byte aligned
 * base, strides multiples of 16 bytes); k, v: the cache, row strides at least
 * D; query head hq reads K/V head hq / q_group.
 * out: device [B, H*q_group, T, D] contiguous, of the problem's dtype: the
 * softmax of sm_scale <q, k_j> over the visible rows times their values (fp32
 * accumulation; for bf16 the row is rounded once, and where more than 32 rows
 * read the same keys the probabilities are too, for the value product).  lse: optional device fp32
 * [B, H*q_group, T], the natural log-sum-exp of the row's scaled logits; for
 * T = 1 it is the lse argument of nacl_score with the current token as the
 * proxy.  A row that sees nothing (padding among them, which sees nothing) and
 * a row whose logits are all -infinity get zeros and lse -infinity.  Rows of
 * the cache or prefix that a query does not see do not touch its result,
 * whatever they hold.  out, lse and ws overlap nothing else. */
int nacl_prefix_attention(const nacl_problem* p, const nacl_step* s, const nacl_prefix* x, const void* q,
                          const void* k, const void* v, void* out, float* lse, void* ws, size_t ws_bytes,
                          void* stream);

/* Settings of nacl_sample; each array is optional DEVICE [N]. */
typedef struct nacl_draw {
  int32_t N, V;            /* rows, 1..65535, and tokens of the vocabulary, 1..NACL_MAX_V */
  int32_t dtype;           /* nacl_dtype of the logits */
  int64_t stride;          /* elements between rows, at least V */
  const float* temperature; /* <= 0 or NaN: greedy, the first largest logit (NULL: 1) */
  const int32_t* top_k;    /* <= 0: no limit (NULL: none) */
  const float* top_p;      /* >= 1 or NaN: no limit (NULL: none); <= 0: the first largest */
  const float* min_p;      /* <= 0 or NaN: no limit (NULL: none); > 1 counts as 1 */
} nacl_draw;
#define NACL_MAX_V (1 << 20)

/* Workspace bytes of nacl_sample (0 on invalid input), the same for both
 * dtypes.  Device memory, 256-byte aligned; its contents need no
 * initialisation. */
size_t nacl_sample_workspace_bytes(const nacl_draw* d);

/* The next token of every row of logits [N, V] (row stride d->stride, element
 * alignment) from given uniform numbers u [N] in [0, 1):
 *   w_i = exp((x_i - max x) / temperature); tokens in order of falling logit,
 *   equal logits by index; kept are the first top_k, of these the fewest
 *   leading ones whose weights reach top_p of the weights' sum (at least one),
 *   and of these those with w_i >= min_p;
 *   tokens[n] = the first kept i, in order of index, at which the kept weights
 *   up to and with i exceed u times their sum.
 * logprobs (optional): ln of the probability it was drawn with, w_i over the
 * kept weights' sum.  A NaN logit counts as -infinity; infinite logits share a row
 * evenly; a row without a logit above -infinity gives token -1 and logprob -infinity.
 * (Hide tokens by -infinity: logits near the type's lowest value, or by a large finite
 * amount below the others, give the same tokens by a path several times slower.)
 * Weights are fp32 exponentials; their sums are 64-bit integers or fp64 in an order
 * that V fixes, so a row's result depends on the row and its settings alone.
 * (Of the top k <= 1024, a token below 2^-32 of the largest counts as nothing.)
 * tokens: device int32 [N]; logprobs: device fp32 [N]. */
int nacl_sample(const nacl_draw* d, const void* logits, const float* u, int32_t* tokens, float* logprobs, void* ws,
                size_t ws_bytes, void* stream);

/* Static text for a status code. */
const char* nacl_status_string(int status);

/* Thread-local text describing the last failed call on this thread ("" if
 * none).  Valid until the next call on the same thread. */
const char* nacl_last_error_detail(void);

/* NACL_VERSION of the built library. */
int nacl_version(void);

#ifdef __cplusplus
}
#endif

#endif /* NACL_H */
