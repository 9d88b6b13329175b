/*
 * adsa.h -- C ABI of the MI355X (gfx950) ADSA decode library.
 *
 * One call processes ONE transformer layer for a batch of independent
 * sequences: the per-step decode attention of Adaptive Dynamic Sparse Attention
 * (paper Section 4.1) restricted to prefix + local window + globally ranked
 * tokens, and the dynamic KV-cache update that evicts and compacts
 * (Section 4.2).  Every entry point only ENQUEUES work on the caller's HIP
 * stream: no host synchronisation, no allocation, no global state (the
 * optional timing hook at the end of this file aside).  The library never
 * touches host memory behind the pointers it is given except `adsa_params`
 * (a host struct, read during the call).
 *
 * Pointers are DEVICE pointers owned by the caller unless marked [host].
 * Return value: ADSA_OK or a negative adsa_status; argument errors are found
 * on the host before anything is launched.  Conditions only the device can see
 * (a full cache, a malformed state) set `adsa_seq.status` of that sequence,
 * which the caller reads when it next synchronises; such a sequence is
 * skipped by every call until the caller clears the status, and its output
 * row is zero-filled.
 *
 * Cache layout.  Element (slot, head, d) of a sequence's K (same for V) lives
 * at  k + slot*kv_slot_stride + head*kv_head_stride + d  (strides in
 * elements).  [head][slot][D] (slot stride = head_dim, head stride >= cap*head_dim):
 * a head's rows are contiguous, one workgroup streams one head -- the fast
 * path; [slot][head][D] (slot stride = n_heads*head_dim, head stride =
 * head_dim) is supported too.  Base pointers must be 16-byte aligned and both
 * strides multiples of 16 bytes.
 *
 * Decode-step convention.  `step` = s = number of image tokens in the context
 * INCLUDING the query token; the query token is image token s-1, at grid cell
 * (row, col) = ((s-1) / grid_w, (s-1) % grid_w) and absolute position
 * grid_origin + s - 1.  s = 0 means the query is the last prefix token
 * (nothing is appended).  0 <= s <= grid_h*grid_w.  A sequence with step < 0
 * is inactive and skipped.
 */
#ifndef ADSA_H
#define ADSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ADSA_VERSION 1
#define ADSA_MAX_CAP 8192      /* largest `cap` (slots per sequence) the select/compact kernels accept */
#define ADSA_STATIC_SCRATCH_BYTES (4u << 20)   /* built-in scratch of adsa_step_static, per GPU */
#define ADSA_MIN_PAGE 16       /* smallest `page_size` of a paged cache */
#define ADSA_MAX_VOCAB (1 << 18)               /* most logits of a row of adsa_sample */

typedef enum {
  ADSA_OK = 0,
  ADSA_ERR_NULL = -1,          /* a required pointer is NULL */
  ADSA_ERR_SHAPE = -2,         /* a size or window parameter is out of range */
  ADSA_ERR_DTYPE = -3,         /* unknown dtype / score mode */
  ADSA_ERR_ALIGN = -4,         /* pointer or stride not 16-byte aligned */
  ADSA_ERR_CAPACITY = -5,      /* cap or sel_cap too small / above ADSA_MAX_CAP */
  ADSA_ERR_WORKSPACE = -6,     /* workspace missing or smaller than adsa_workspace_bytes() */
  ADSA_ERR_LAUNCH = -7,        /* the HIP runtime refused a launch */
  ADSA_ERR_UNSUPPORTED = -8,   /* valid request this build does not implement */
  ADSA_ERR_STATIC_SCRATCH = -9 /* adsa_step_static: these parameters need more than ADSA_STATIC_SCRATCH_BYTES */
} adsa_status;

typedef enum { ADSA_F32 = 0, ADSA_BF16 = 1 } adsa_dtype;

/* How the "previous" tokens are ranked for Eq. 4 (which K of them are kept). */
typedef enum {
  ADSA_SCORE_ATTN_MASS = 0,    /* accumulated softmax probability received so far; keep LARGEST */
  ADSA_SCORE_VCOS = 1,         /* mean pairwise cosine of V (Eq. 2-3) over the candidates; keep SMALLEST */
  ADSA_SCORE_EXT_LARGEST = 2,  /* caller-maintained score[]; keep largest */
  ADSA_SCORE_EXT_SMALLEST = 3, /* caller-maintained score[]; keep smallest */
  ADSA_SCORE_VCOS_FUSED = 4    /* the same Eq. 2-3 ranking as ADSA_SCORE_VCOS for ADSA_EVICT_REUSE_SLOT, without
                                  separate passes over V: the attention launch, which streams every resident
                                  V row anyway, also takes each row's squared norm and its dot product with
                                  the running sum u of the candidates' normalised V vectors (adsa_seq.vcos_u,
                                  kept up to date by adsa_compact: minus the evicted row, plus the row that
                                  leaves the local window next).  The next eviction ranks from those numbers.
                                  Needs [head][slot][D] caches, q_per_kv <= 1, win_recent_m >= 2 and
                                  16*n_heads*head_dim + cap (rounded up to 16) <= 65536 (else ADSA_ERR_UNSUPPORTED).  Whenever the running state
                                  does not belong to the step at hand (first use, a cache edited by the
                                  caller) the call falls back to the two-pass computation, so results never
                                  depend on it being warm */
} adsa_score_mode;

/* When the dynamic cache evicts (Section 4.2). */
typedef enum {
  ADSA_EVICT_ROW_END = 0,      /* once per completed grid row: keep prefix + last R rows + top-B of the rest */
  ADSA_EVICT_WHEN_FULL = 1,    /* the paper's own rule: when n_res == cap and a token is about to be inserted,
                                  evict the ONE last-ranked candidate (most redundant) before the insertion;
                                  needs win_recent_m > 0 (a token that left a 1-D window is never local again).
                                  Attention then covers everything resident (Tables 1-2: context == KV cache):
                                  the budget fields are ignored.  The hole is closed: slots stay in position
                                  order, at the price of moving every row behind the hole */
  ADSA_EVICT_REUSE_SLOT = 2    /* the same rule and the same evicted token (among equal scores the newest
                                  position goes), but nothing moves: the evicted slot is recorded in
                                  adsa_seq.hole and the incoming token takes it.  From the first eviction on,
                                  slot order is no longer position order (pos[] says who lives where) */
} adsa_evict_policy;

/* Device-side per-sequence status bits (adsa_seq.status). */
#define ADSA_SEQ_OK            0
#define ADSA_SEQ_CACHE_FULL    1   /* append would exceed cap */
#define ADSA_SEQ_BAD_STATE     2   /* n_res/step out of range, or an entry newer than the query */
#define ADSA_SEQ_SEL_OVERFLOW  4   /* attended set larger than sel_cap */

/* Flags of adsa_select / adsa_attend / adsa_compact / adsa_step and of the prompt side. */
#define ADSA_FLAG_NO_COMPACT    1u  /* caller guarantees no sequence closes a grid row in this step */
#define ADSA_FLAG_NO_ACCUMULATE 2u  /* adsa_attend: do not add attention mass to score[] */
#define ADSA_FLAG_PLAN_APPEND   4u  /* adsa_select: reserve slot n_res for the query token (pos, zero score,
                                       n_res += 1, pending_slot) and rank with it in place (it is always
                                       local); its K/V rows arrive with adsa_attend(ADSA_FLAG_APPEND).
                                       Once per decode step */
#define ADSA_FLAG_APPEND        8u  /* adsa_attend: write (k_new, v_new) into pending_slot while attending */
#define ADSA_FLAG_NEW_F32      32u  /* adsa_attend / adsa_step with a bf16 cache: k_new and v_new are fp32
                                       [n_seq][n_heads][head_dim]; each value is rounded to the nearest bf16
                                       (ties to even) once, as it enters the cache, and the launch attends the
                                       rounded row.  No effect with an fp32 cache */
#define ADSA_FLAG_ADVANCE      16u  /* adsa_attend / adsa_compact: step += 1 for every active sequence when
                                       the call is done; give it to the LAST call of a decode step only
                                       (adsa_compact tests the row end on the step before the increment) */

#define ADSA_FLAG_SPLIT_P      64u  /* adsa_prefill and adsa_prefill_paged with a bf16 cache: probabilities meet V with 16 bits in calls of any size, as
                                       those of the other calls do, for half as many products again.  Without it
                                       they may be rounded to bf16, by 2^-8 of themselves at most (calls of more
                                       than 32 rows a cache head).  No effect with an fp32 cache */

/* [host] Launch-wide parameters (Section 4.1's n, m, K and the problem shape). */
typedef struct adsa_params {
  int32_t n_seq;               /* sequences in this launch (>= 1) */
  int32_t n_heads;             /* key/value (cache) heads; the query has n_heads * max(q_per_kv, 1) heads */
  int32_t head_dim;            /* 64 or 128 */
  int32_t grid_h, grid_w;      /* image-token grid H x W, raster order */
  int32_t win_rows_back;       /* R: rows above the query's row that belong to the local window */
  int32_t win_col_radius;      /* w: column radius in those rows; w >= grid_w-1 gives the paper's
                                  1-D "most recent m tokens" window */
  int32_t sel_groups;          /* 1: one attended set per sequence shared by all heads.
                                  n_heads: one set, and one eviction history, PER (cache) HEAD (Eq. 4 does not say
                                  which).  Every (sequence, head) then is a sequence of one head: `seqs` holds
                                  n_seq * n_heads records, record b * n_heads + h describing head h of sequence b
                                  (k / v point at that head's first row, rows kv_slot_stride apart -- either cache
                                  nesting works, kv_head_stride is not used --, its own pos, score, n_res, step...);
                                  sel_idx, sel_cnt and keep_map carry one row per record ([n_seq][n_heads][...]);
                                  q, k_new, v_new, out, lse keep their layouts.  n_seq * n_heads <= 65535.
                                  Any other value: ADSA_ERR_UNSUPPORTED */
  int32_t dtype;               /* adsa_dtype of q, K, V, out */
  int32_t score_mode;          /* adsa_score_mode */
  int32_t cap;                 /* slots allocated per sequence (<= ADSA_MAX_CAP) */
  int32_t sel_cap;             /* entries per row of sel_idx: the longest list.  Attention launches are planned for lists
                                  of this length (the counts are on the device), so a tight bound is the fast one */
  int64_t kv_slot_stride;      /* elements */
  int64_t kv_head_stride;      /* elements */
  float   softmax_scale;       /* 0 => 1/sqrt(head_dim).  With bf16 caches it is applied to the fp32 sum q.k, which has
                                  to be finite without it */
  int32_t win_recent_m;        /* > 0: the paper's own 1-D local region (Section 4.1), the m most recent image
                                  tokens incl. the query token, instead of the 2-D window (R, w ignored) */
  int32_t evict_policy;        /* adsa_evict_policy */
  int32_t q_per_kv;            /* G: query heads per cache head.  0 or 1: multi-head attention.  2..16:
                                  grouped-query attention, query head j reads cache head floor(j/G); bf16 only,
                                  one head's rows must span less than 4 GiB
                                  (cap * kv_slot_stride * 2 bytes: the kernel addresses them with 32-bit
                                  offsets), else ADSA_ERR_UNSUPPORTED */
} adsa_params;

/* Device array of n_seq entries (96 bytes each): the ragged per-sequence state.  The kernels read AND update
   n_res, step, status, compacted, so one launch serves sequences at different positions. */
typedef struct adsa_seq {
  void*    k;                  /* this sequence's K cache (dtype elements) */
  void*    v;                  /* this sequence's V cache */
  int32_t* pos;                /* [cap] absolute position of each resident slot, strictly ascending (under
                                  ADSA_EVICT_REUSE_SLOT only until the first eviction; always distinct) */
  float*   score;              /* [score_rows][cap] ranking score of each resident slot: the rank of slot i
                                  is the sum over rows (ascending, fp32) of score[row][i].
                                  ADSA_SCORE_ATTN_MASS: score_rows = n_heads, one accumulator per head
                                  (each head's workgroup updates only its own row).
                                  ADSA_SCORE_VCOS_FUSED: score_rows = 2*n_heads, rows 2h and 2h+1 hold head h's
                                  share of |v|^2 and of v.u per slot (written by the attention launch; not a
                                  rank by themselves).  Else score_rows = 1 */
  int32_t  n_res;              /* resident slots */
  int32_t  step;               /* s (see the decode-step convention above); < 0: inactive */
  int32_t  grid_origin;        /* P: absolute position of image token 0 (= prefix length) */
  int32_t  n_keep_prefix;      /* positions below this are pinned (never ranked, never evicted) */
  int32_t  budget;             /* B: global tokens kept, when budget_den == 0 */
  int32_t  budget_num;         /* else B = floor((P + s) * budget_num / budget_den) */
  int32_t  budget_den;
  int32_t  status;             /* ADSA_SEQ_* bits, set by the device, cleared by the caller */
  int32_t  compacted;          /* 1 if the last adsa_step/adsa_compact evicted+compacted this sequence */
  int32_t  pending_slot;       /* slot adsa_select(PLAN_APPEND) reserved for the query token, whose K/V rows
                                  the next adsa_attend(APPEND) fills; -1 if none.  Written by adsa_select */
  int32_t  hole;               /* ADSA_EVICT_REUSE_SLOT: 1 + the slot the last eviction freed, 0 if none (start
                                  with 0).  A freed slot still counts in n_res but is in no list; the next
                                  adsa_select(PLAN_APPEND) gives it to the query token and clears hole */
  int32_t  reserved;
  float*   vcos_u;             /* ADSA_SCORE_VCOS_FUSED: [n_heads*head_dim + 4] floats owned by the caller and
                                  maintained by the library: the running sum u, then two step tags (as floats)
                                  that say which step u and the score rows belong to.  Zero it when the cache
                                  or `step` is changed by hand.  NULL otherwise */
  int64_t  reserved2;
} adsa_seq;

/* Bytes of device scratch the entry points need for these parameters (0 if they are invalid). */
size_t adsa_workspace_bytes(const adsa_params* p);

/*
 * Prepare a workspace (256-byte aligned, >= adsa_workspace_bytes(p)) for use with parameters p:
 * checks the arguments and zeroes the words at its head with a small fill kernel on `stream`.  No result depends on
 * those words or on any other content of the memory (every call writes what its kernels read), so the call may be
 * left out.  A workspace may be shared by calls that are ordered on one stream, not by concurrent ones.
 */
int adsa_workspace_init(const adsa_params* p, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Eq. 1 + Eq. 4: partition every sequence's resident slots into prefix / local / candidate for
 * the query of its current `step`, rank the candidates, and write the attended set
 *   PREFIX u LOCAL u top-min(B, |candidates|)
 * as an ascending slot list.  Ties go to the lower slot; -0 == +0; NaN scores are a
 * precondition violation.  Reads seqs[].pos/score/n_res/step, writes pending_slot (and, with
 * ADSA_FLAG_PLAN_APPEND, pos / score / n_res of the reserved slot); VCOS mode first writes Eq. 3's
 * S_i into score[] at the candidate slots (reads V, needs the workspace; other modes accept a
 * NULL workspace).  The ranking does not depend on the query token's q/k/v, so one call may
 * cover the sequences of every layer of a model (n_seq = layers x batch) before the layers run.
 * flags: ADSA_FLAG_PLAN_APPEND.
 *   sel_idx  int32 [n_seq][sel_cap]   out
 *   sel_cnt  int32 [n_seq]            out
 */
int adsa_select(const adsa_params* p, adsa_seq* seqs, int32_t* sel_idx, int32_t* sel_cnt,
                uint32_t flags, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Eq. 5 + attention: per sequence and query head, softmax(q.K_sel^T * scale) V_sel over the slots
 * listed in sel_idx (gathered in place, never materialised), fp32 accumulation.  With
 * hq = n_heads * max(q_per_kv, 1) query heads:
 *   q    dtype [n_seq][hq][head_dim]
 *   out  dtype [n_seq][hq][head_dim]
 *   lse  float [n_seq][hq]   natural-log sum-exp of the scaled logits
 *   k_new, v_new  dtype [n_seq][n_heads][head_dim], only read with ADSA_FLAG_APPEND (else may be NULL)
 * For ADSA_SCORE_ATTN_MASS and unless ADSA_FLAG_NO_ACCUMULATE is set, score[slot] of every
 * attended slot gains, in row h of score[], the probability the query head(s) of cache head h gave it
 * (grouped queries: their sum in ascending head order).
 * ADSA_FLAG_APPEND (Section 4.2, new tokens go to the end of the cache): the row (k_new, v_new)
 * is written to the slot adsa_select(ADSA_FLAG_PLAN_APPEND) reserved (pending_slot >= 0), and that
 * slot is attended from k_new / v_new directly.
 * flags: ADSA_FLAG_NO_ACCUMULATE, ADSA_FLAG_APPEND, ADSA_FLAG_NEW_F32, ADSA_FLAG_ADVANCE.
 */
int adsa_attend(const adsa_params* p, adsa_seq* seqs, const void* q, const void* k_new,
                const void* v_new, const int32_t* sel_idx, const int32_t* sel_cnt, void* out,
                float* lse, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Section 4.2 in per-row form.  For every sequence whose query token closes a grid row
 * ((s-1) % grid_w == grid_w-1, s >= 1): keep the pinned prefix, the last R completed rows and
 * the top min(B, |rest|) of the rest by the same ranking as adsa_select; write
 *   keep_map int32 [n_seq][cap]: new slot of old slot i, or -1 (entries >= old n_res untouched)
 * move K, V, pos and every score row to the front in place, order preserved, and set n_res, compacted.
 * Other sequences are untouched (compacted = 0, keep_map row untouched).  Like adsa_select it
 * may cover every layer's sequences in one call.  flags: ADSA_FLAG_ADVANCE.
 * With ADSA_EVICT_WHEN_FULL / ADSA_EVICT_REUSE_SLOT the call acts instead on the sequences whose cache is full
 * (n_res == cap, step >= 1), BEFORE the step's adsa_select: it removes the one candidate ranked
 * last for the incoming query's partition (ties: the highest slot goes) and closes the hole.
 */
int adsa_compact(const adsa_params* p, adsa_seq* seqs, int32_t* keep_map, uint32_t flags,
                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * One whole decode step of one layer, in one call: adsa_select(PLAN_APPEND), adsa_attend(APPEND)
 * and, unless ADSA_FLAG_NO_COMPACT, adsa_compact in stream order, the last of them advancing: the query
 * token is appended at slot n_res (skipped when s == 0), the attended set is chosen and attended,
 * attention mass is accumulated (ATTN_MASS), sequences that closed a row are evicted+compacted,
 * and step += 1.  keep_map may be NULL only with ADSA_FLAG_NO_COMPACT.
 * With ADSA_EVICT_WHEN_FULL / ADSA_EVICT_REUSE_SLOT the order is the paper's: evict one if full, then
 * append/select/attend.
 */
int adsa_step(const adsa_params* p, adsa_seq* seqs, const void* q, const void* k_new,
              const void* v_new, void* out, float* lse, int32_t* sel_idx, int32_t* sel_cnt,
              int32_t* keep_map, uint32_t flags, void* workspace, size_t workspace_bytes,
              void* stream);

/*
 * adsa_step for callers that cannot allocate device memory or carry a workspace around: code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation.  Same arguments, same kernels and
 * same results as adsa_step, but the scratch memory is a built-in array of ADSA_STATIC_SCRATCH_BYTES that
 * every GPU the library runs on holds until the process ends; the call allocates nothing (its address is
 * looked up once per device, at the first call there).  Parameters whose adsa_workspace_bytes() exceeds
 * ADSA_STATIC_SCRATCH_BYTES are rejected with ADSA_ERR_STATIC_SCRATCH before anything is launched.
 * All calls on one GPU share the one array: calls ordered on one stream are fine, calls that may
 * overlap on the same GPU (different streams or host threads) race.
 */
int adsa_step_static(const adsa_params* p, adsa_seq* seqs, const void* q, const void* k_new,
                     const void* v_new, void* out, float* lse, int32_t* sel_idx, int32_t* sel_cnt,
                     int32_t* keep_map, uint32_t flags, void* stream);

/* ---------------------------------------------------------------------------------------------------------------------------------
 * Prompts: rotary positions, tokens that enter the caches many at a time, their attention, and decode attention for sequences that
 * share a prompt.  The entry points below take the same parameters and records as those above, one layer per call; sel_groups != 1
 * is ADSA_ERR_UNSUPPORTED in all of them.  A workspace of adsa_prefill or adsa_attend_shared holds partial results between the launches of
 * one call: calls that may run at the same time (on streams without an order between them, or replays of graphs) need one each.
 */
#define ADSA_MAX_AXES 3

typedef enum { ADSA_PAIR_HALVES = 0,       /* pair i of a row: elements i and i + head_dim/2 */
               ADSA_PAIR_NEIGHBOURS = 1    /* elements 2i and 2i + 1 */
} adsa_pairing;

/* [host] Rotary positions with up to three axes (row and column; time, height and width; a plain line).  A token with the
   coordinates c has pair i of its q and k rows turned by the angle  sum over a of c[a] * freq[a][i]  radians:
   (x, y) -> (x cos - y sin, y cos + x sin).  A pair that an axis does not turn has frequency 0 there.  Angles are formed and reduced
   in 64 bits, so far positions lose nothing.  A token at absolute position t has, where none are given, the coordinates
     t < grid_origin (P):                      c[a] = text[a] * t
     image token at (row r, column c) else:    c[a] = origin[a] * P + row[a] * r + col[a] * c */
typedef struct adsa_rope {
  const double* freq;          /* device [n_axes][head_dim/2]; 16-byte aligned */
  int32_t n_axes;              /* 1..ADSA_MAX_AXES */
  int32_t pairing;             /* adsa_pairing */
  int32_t text[ADSA_MAX_AXES], origin[ADSA_MAX_AXES], row[ADSA_MAX_AXES], col[ADSA_MAX_AXES];
} adsa_rope;

/* [host] New tokens of a batch, packed one sequence behind the other.  Token begin[b] + j of sequence b belongs in slot slot0[b] + j.
   The slots of a sequence have to be in position order (under ADSA_EVICT_REUSE_SLOT: before its first eviction). */
typedef struct adsa_tokens {
  int32_t n_tokens;            /* T >= 1: tokens of all sequences */
  int32_t max_len;             /* no sequence has more new tokens than this; 1..cap */
  const int32_t* begin;        /* device [n_seq + 1], ascending from 0 to n_tokens */
  const int32_t* slot0;        /* device [n_seq] */
  const int32_t* pos0;         /* device [n_seq] absolute position of each sequence's first new token, or NULL: one behind that of slot
                                  slot0 - 1, 0 in an empty cache.  (Members of a shared prompt have caches that begin behind it) */
  const int32_t* coords;       /* device [T][n_axes] coordinates instead of those that follow from positions, or NULL */
  int64_t q_stride, k_stride, v_stride;   /* elements from one token's row to the next in q, k, v of adsa_append (rows of a packed
                                             projection); 0: no gap.  Multiples of 16 bytes */
} adsa_tokens;

typedef enum { ADSA_MASK_CAUSAL = 0,       /* a token sees itself and the slots before its own */
               ADSA_MASK_PREFIX = 1        /* besides, tokens among the first n_keep_prefix slots see each other both ways */
} adsa_mask;

/* [host] What is done to scaled scores z = q.k * softmax_scale before the softmax; NULL: nothing, causal. */
typedef struct adsa_mods {
  float softcap;               /* > 0: z <- softcap * tanh(z / softcap); 0: not.  softmax_scale / softcap and 1.45 softcap have to be normal fp32 numbers */
  int32_t mask;                /* adsa_mask (adsa_prefill) */
  const float* slopes;         /* device, one per query head: z <- z - slopes[head] * |difference of absolute positions|, after the cap; or NULL */
  const int32_t* doc;          /* device [n_seq][doc_stride]: document of every slot; a token sees only its own document's slots, and a
                                  negative number marks a slot that neither sees nor is seen; or NULL (adsa_prefill only) */
  int64_t doc_stride;          /* >= cap */
} adsa_mods;

/* [host] Prompts that sequences of a launch share: group g's prompt is the resident slots of a record of its own (filled by adsa_append
   like any other, with strides and a capacity of its own, same head count, head_dim and dtype), and its members are the sequences
   members[g] .. members[g+1] - 1.  Members' own caches hold only what comes behind the prompt. */
typedef struct adsa_shared {
  int32_t n_groups;            /* 1..n_seq */
  int32_t max_prompt;          /* capacity of the prompts' records: none has more slots (<= ADSA_MAX_CAP) */
  int32_t max_members;         /* no group has more members; 1..n_seq */
  int32_t reserved;
  const adsa_seq* prompts;     /* device [n_groups]; k, v, pos, n_res and status are read */
  const int32_t* members;      /* device [n_groups + 1], ascending from 0 to n_seq */
  int64_t kv_slot_stride, kv_head_stride;    /* of the prompts' caches, elements */
} adsa_shared;

/*
 * Rotate the query token's q and k of every sequence, at the position its record's step says (grid_origin + step - 1), or at
 * coords [n_seq][n_axes]:
 *   q, k      [n_seq] rows of n_heads * max(q_per_kv, 1) and of n_heads heads, q_stride and k_stride elements apart (0: no gap);
 *             dtype, or fp32 with ADSA_FLAG_NEW_F32 and a bf16 cache
 *   q_out, k_out  dtype [n_seq][heads][head_dim]; may be q and k themselves where those are dtype without gaps
 * Rotated in fp32, rounded once.  Inactive sequences (step < 0 or a status) get zeros.  flags: ADSA_FLAG_NEW_F32.
 */
int adsa_rotate(const adsa_params* p, const adsa_rope* rope, const adsa_seq* seqs, const int32_t* coords, const void* q,
                const void* k, int64_t q_stride, int64_t k_stride, void* q_out, void* k_out, uint32_t flags, void* stream);

/*
 * New tokens enter the caches: k rows rotated, v rows as they are, q rows rotated to q_out (dtype [T][heads][head_dim]; q and q_out may
 * both be NULL).  rope NULL: nothing is turned.  q, k, v are dtype, or fp32 with ADSA_FLAG_NEW_F32 and a bf16 cache (rounded once).
 * Per sequence with new tokens (whatever its step): slot0 <= n_res is required, slots from slot0 on are overwritten, and n_res becomes
 * slot0 + its number of tokens; the same call may be made again, and a smaller slot0 takes tokens back.  pos and zero scores
 * are written, pending_slot,
 * compacted and the running V-cosine state are reset, and step becomes the number of image tokens resident, as if the last
 * token were the query token; ADSA_FLAG_ADVANCE adds 1 to it.  Sequences without new tokens are left alone.
 * A record that does not fit (n_res, slot0 or a count out of range, a hole, positions beyond the grid: ADSA_SEQ_BAD_STATE;
 * more tokens than slots: ADSA_SEQ_CACHE_FULL) gets its status set, nothing else, and zeros in q_out.
 * flags: ADSA_FLAG_NEW_F32, ADSA_FLAG_ADVANCE.
 */
int adsa_append(const adsa_params* p, const adsa_tokens* tokens, const adsa_rope* rope, adsa_seq* seqs, const void* q,
                const void* k, const void* v, void* q_out, uint32_t flags, void* stream);

/*
 * Attention of those tokens over slots 0 .. slot0 + tokens - 1 of their sequences (already resident), masked and with scores changed
 * as mods say, any number of tokens from one on:
 *   q    dtype [T][heads][head_dim] (rotated)        out  dtype [T][heads][head_dim]        lse  float [T][heads]
 * A row that sees nothing gives zeros and lse = -INFINITY; what masked slots hold, infinities and NaN included, changes nothing.
 * For ADSA_SCORE_ATTN_MASS and unless ADSA_FLAG_NO_ACCUMULATE is set, score[h][slot] gains the probability that the tokens' query
 * heads of cache head h gave the slot.  Sums are taken in the same order whatever the launch does: results repeat bit by bit.
 * A sequence with a status or without those slots (ADSA_SEQ_BAD_STATE) gets zeros; one without new tokens is left alone.
 * flags: ADSA_FLAG_NO_ACCUMULATE, ADSA_FLAG_SPLIT_P, ADSA_FLAG_ADVANCE (step += 1 for every sequence with new tokens, where adsa_append did not).
 */
int adsa_prefill(const adsa_params* p, const adsa_tokens* tokens, const adsa_mods* mods, adsa_seq* seqs, const void* q,
                 void* out, float* lse, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream);
size_t adsa_prefill_workspace_bytes(const adsa_params* p, const adsa_tokens* tokens);   /* 0 if the parameters are invalid */

/*
 * adsa_attend for sequences that share prompts, with scores changed as mods say (mask and doc: NULL or not read): softmax over the group's prompt and
 * the sequence's own list (sel_idx, sel_cnt, as adsa_select leaves them), one pass over a prompt for all its members.  Arguments as in
 * adsa_attend, whose scores, append and advance happen alike; own lists may be empty (only the prompt is attended), a sequence with
 * nothing at all gives zeros and lse = -INFINITY; one that is inactive, has a status, or whose prompt's record has one or more slots
 * than max_prompt, zeros.  ADSA_SCORE_VCOS_FUSED: ADSA_ERR_UNSUPPORTED.
 * flags: ADSA_FLAG_NO_ACCUMULATE, ADSA_FLAG_APPEND, ADSA_FLAG_NEW_F32, ADSA_FLAG_ADVANCE.
 */
int adsa_attend_shared(const adsa_params* p, const adsa_shared* shared, const adsa_mods* mods, adsa_seq* seqs, const void* q,
                       const void* k_new, const void* v_new, const int32_t* sel_idx, const int32_t* sel_cnt, void* out,
                       float* lse, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream);
size_t adsa_shared_workspace_bytes(const adsa_params* p, const adsa_shared* shared);    /* 0 if the parameters are invalid */

/* ---------------------------------------------------------------------------------------------------------------------------------
 * Caches in pages: the K and V rows of all sequences of a launch lie in two pools of equal pages, and a table says which page holds which
 * slots.  pos, score and the counters of a sequence stay in its record, so adsa_select, which reads no cache row, works as it is; a
 * record's k and v are not used and may be NULL, nor are kv_slot_stride and kv_head_stride of the parameters (they have to be valid).
 * ADSA_SCORE_VCOS and ADSA_SCORE_VCOS_FUSED, which rank by V, and sel_groups != 1 are ADSA_ERR_UNSUPPORTED in the calls below.
 * Table entries of slots a sequence does not have are not read as pages; a sequence with resident slots on an entry that is no page of
 * the pool gets ADSA_SEQ_BAD_STATE and zeros (adsa_append_paged: ADSA_SEQ_CACHE_FULL where it is the new tokens' slots), and its pages stay
 * as they are.  A page may be in several sequences' tables as long as no call writes to it: pinned prefixes do not move.  A step whose new token's slot,
 * which adsa_select has reserved, has no page is such a case: ADSA_SEQ_BAD_STATE, and n_res counts the slot already.
 */
typedef struct adsa_pages {    /* [host] */
  void* k;                     /* device: page 0 of the pool of K (dtype elements); 16-byte aligned, as is v */
  void* v;                     /* ... of V; may be the same memory as k, with strides that keep them apart */
  const int32_t* table;        /* device [n_seq][table_stride]: entry i of a row is the page of slots i * page_size .. + page_size - 1 */
  int64_t page_stride;         /* elements from a page to the next, from a slot's row to the next slot's in a page, and from a head's row to the next head's; */
  int64_t slot_stride;         /* multiples of 16 bytes, nested [page][head][slot][D] or [page][slot][head][D]; a page's below 4 GiB and a slot's below */
  int64_t head_stride;         /* 16 MiB, else ADSA_ERR_UNSUPPORTED */
  int32_t page_size;           /* slots of a page: a power of two from ADSA_MIN_PAGE to ADSA_MAX_CAP */
  int32_t n_pages;             /* pages of a pool; n_pages * page_stride, in units of the largest power of two (16 bytes at least) that divides the
                                  three strides, below 2^31 (rows of 128 bytes, one behind the other: 256 GiB), else ADSA_ERR_UNSUPPORTED */
  int32_t table_stride;        /* entries of a row: at least cap / page_size, rounded up; at most 65535 */
  int32_t reserved;
} adsa_pages;

/* adsa_append, adsa_prefill, adsa_attend and adsa_compact over pages: what those say holds, but for where rows lie. */
int adsa_append_paged(const adsa_params* p, const adsa_pages* pages, const adsa_tokens* tokens, const adsa_rope* rope, adsa_seq* seqs, const void* q,
                      const void* k, const void* v, void* q_out, uint32_t flags, void* stream);
int adsa_prefill_paged(const adsa_params* p, const adsa_pages* pages, const adsa_tokens* tokens, const adsa_mods* mods, adsa_seq* seqs, const void* q,
                       void* out, float* lse, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream);
size_t adsa_prefill_paged_workspace_bytes(const adsa_params* p, const adsa_pages* pages, const adsa_tokens* tokens);   /* 0 if something is invalid */
/* Listed slots have to be resident.  A sequence with a status is skipped and gets zeros, whatever its list.
   flags: ADSA_FLAG_NO_ACCUMULATE, ADSA_FLAG_APPEND, ADSA_FLAG_NEW_F32, ADSA_FLAG_ADVANCE. */
int adsa_attend_paged(const adsa_params* p, const adsa_pages* pages, adsa_seq* seqs, const void* q, const void* k_new, const void* v_new,
                      const int32_t* sel_idx, const int32_t* sel_cnt, void* out, float* lse, uint32_t flags, void* workspace, size_t workspace_bytes,
                      void* stream);
/* The table is not changed: pages behind the new n_res are the caller's to give to others. */
int adsa_compact_paged(const adsa_params* p, const adsa_pages* pages, adsa_seq* seqs, int32_t* keep_map, uint32_t flags, void* workspace,
                       size_t workspace_bytes, void* stream);
size_t adsa_paged_workspace_bytes(const adsa_params* p);       /* of adsa_attend_paged and adsa_compact_paged; 0 if the parameters are invalid */

/* ---------------------------------------------------------------------------------------------------------------------------------
 * The next token of every row of logits, from random numbers that the caller brings.
 *   z[i]   the logit; guided: fp32(u + guidance * (c - u)), formed in 64 bits, of the conditional row's c and its partner's u; -infinity where c or u is
 *          (a token that either row masks is masked); with guidance 1 it is c, whatever u is
 *   w[i]   exp((z[i] - max z) / temperature)
 * In descending order of z (equal ones: the lower index first) the candidates are the first top_k, of these as few as have together top_p of
 * their sum of w, and of these those with w >= min_p (relative to the largest, whose w is 1).  The token is the first candidate in ascending
 * order of index at which the running sum of the candidates' w exceeds uniform times their whole sum; logprob the natural logarithm of its share.
 * Temperature 0: the largest (the first of several), logprob 0.  A NaN counts as -infinity; where +infinities are, only these are
 * candidates; a row without a logit above -infinity gets token -1 and logprob -infinity.  Weights are summed as whole numbers of 2^-44, whatever
 * the order, so results repeat bit by bit; what is less than half of that, 31.19 temperatures below the largest, is 0.  A temperature between 0 and
 * 2^-100 counts as 2^-100.
 */
typedef struct adsa_sampling { /* [host] */
  int32_t n_rows;              /* tokens to draw: 1..2^20 */
  int32_t vocab;               /* logits of a row: 1..ADSA_MAX_VOCAB */
  int32_t dtype;               /* adsa_dtype of the logits */
  int32_t guided;              /* 0: n_rows rows of logits.  1: 2 * n_rows, row n_rows + r being the unconditional partner of row r */
  int64_t row_stride;          /* elements from a row of logits to the next; 0: vocab.  Any alignment of elements */
  float   guidance;            /* finite; 1: the conditional row alone */
  float   temperature;         /* >= 0, finite */
  int32_t top_k;               /* <= 0, or vocab and more: not limited */
  float   top_p;               /* 1 and more: not limited; 0 and less: the largest alone */
  float   min_p;               /* 0 and less: not limited; more than 1 counts as 1 */
  int32_t reserved;
  const float* temperatures;   /* device [n_rows], or NULL: the number above for every row (negative or NaN counts as 0; +infinity: all that is above -infinity weighs alike) */
  const int32_t* top_ks;       /* the same for the others (a NaN: not limited) */
  const float* top_ps;
  const float* min_ps;
} adsa_sampling;

/*
 *   logits   dtype rows, aligned to their elements, as all arrays are (else ADSA_ERR_ALIGN)      uniform  float [n_rows] in [0, 1) (outside: the nearest that is)
 *   token    int32 [n_rows], guided [2 * n_rows]: the partner gets the same token      logprob  float [n_rows], or NULL
 *   seqs     NULL, or as many records as token has numbers: a row whose record is inactive (step < 0 or a status) gets token -1 and logprob 0;
 *            a pair goes by the record of its conditional row
 */
int adsa_sample(const adsa_sampling* s, const adsa_seq* seqs, const void* logits, const float* uniform, int32_t* token, float* logprob, void* stream);

/* Timing hook for benchmarks: when enabled, adsa_attend/adsa_step attach a start and a stop HIP
   event to every attention-kernel dispatch on the caller's stream (in adsa_step, where that kernel ranks for itself or plans
   evictions, those are part of it; kernels that merge split lists are not).  adsa_profile_read
   synchronises those events and returns, through its arguments, the number of timed launches and
   their summed duration in milliseconds since the last adsa_profile_enable(1); [host] pointers.
   adsa_profile_enable(0) switches the hook off and destroys its events.  Process-wide state, not thread-safe. */
int adsa_profile_enable(int on);
int adsa_profile_read(int64_t* n_launches, double* total_ms);

const char* adsa_strerror(int code);
int adsa_version(void);

#ifdef __cplusplus
}
#endif
#endif
