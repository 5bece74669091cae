/*
 * tfe.h -- C ABI of the B200 Engram lookup-and-inject library (libtfe.so).
 *
 * The library implements the per-token side pathway of an Engram-style memory
 * as TF-Engram uses it at inference time: from the token ids ending at each
 * position form the trailing n-gram phrase keys, look each key up in an
 * exact-match (non-colliding) phrase index, decide which matched phrase is
 * retained, see in which storage tier its memory vector lives, fetch the
 * vectors that are in the GPU tier and add them to the hidden state through a
 * gate; phrases whose vectors are not in the GPU tier are reported so the host
 * DRAM / SSD tier and the prefetcher can stage them, and staged vectors are
 * written into the GPU tier by a separate call.
 *
 * Everything below is plain C: opaque context, PODs, raw pointers.  Each
 * pointer is marked HOST or DEVICE.  "stream" is a cudaStream_t passed as
 * void* (NULL = the legacy default stream).  All device work of one context
 * must be issued in stream order (one stream, or streams the caller orders);
 * two calls on the same context that overlap on the GPU race.  A context (and
 * a head) is also not safe for concurrent calls from several host threads:
 * each entry point updates host-side state of its object without locking.
 * Different contexts are independent.
 *
 * No entry point throws, aborts or traps.  Argument errors are found on the
 * host before anything is launched and leave the context unchanged.
 */
#ifndef TFE_H
#define TFE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tfe_ctx tfe_ctx;

typedef enum {
    TFE_OK = 0,
    TFE_ERR_INVALID_ARG = 1,
    TFE_ERR_DUPLICATE_PHRASE = 2,   /* two phrases with the same token tuple                    */
    TFE_ERR_KEY_COLLISION = 3,      /* two different tuples of a hashed order share a 64-bit key */
    TFE_ERR_CAPACITY = 4,           /* more phrases than load_factor * index slots, or > 2^32-2 */
    TFE_ERR_SLOT_RANGE = 5,         /* GPU-tier slot outside [0, gpu_slots) or used twice       */
    TFE_ERR_UNKNOWN_PHRASE = 6,
    TFE_ERR_ALREADY_RESIDENT = 7,
    TFE_ERR_MISS_OVERFLOW = 8,      /* caller's miss buffers are smaller than the miss count    */
    TFE_ERR_PROBE_LIMIT = 9,        /* index build could not place a key within max_kicks moves   */
    TFE_ERR_CUDA = 10,              /* a CUDA runtime call failed; see tfe_last_cuda_error()    */
    TFE_ERR_INTERNAL = 11           /* the device reported an inconsistent state or a bounded wait ran out */
} tfe_status;

/* Table geometry, fixed at build time. */
typedef struct {
    int32_t d;                  /* row width in elements; multiple of 8, >= 8                         */
    int32_t vocab;              /* token ids are valid in [0, vocab); anything else is padding        */
    int32_t n_orders;           /* 1..4                                                               */
    int32_t orders[4];          /* n-gram orders, strictly ascending, each in [1,4]                   */
    int64_t n_phrases;          /* N                                                                  */
    int64_t gpu_slots;          /* C, rows of the GPU tier                                            */
    float   load_factor;        /* index slots = ceil(N / load_factor), rounded up to 4-slot buckets  */
    int32_t hidden_dtype;       /* 0 = bf16 hidden states, 1 = fp32 hidden states (rows always bf16)  */
    int32_t max_kicks;          /* cuckoo moves allowed per insertion at build, 0 = default (2000)    */
} tfe_config;

enum { TFE_POLICY_LONGEST = 0, TFE_POLICY_ALL = 1 };
enum { TFE_GATE_CONST = 0, TFE_GATE_COSINE = 1 };
enum { TFE_FLAG_ABSENT = 0, TFE_FLAG_GPU_HIT = 1, TFE_FLAG_HOST_MISS = 2, TFE_FLAG_SSD_MISS = 3 };
#define TFE_NO_PHRASE 0xFFFFFFFFu

/* Per-call injection rule. */
typedef struct {
    int32_t policy;   /* LONGEST: keep the matched phrase of greatest order.  ALL: keep every match
                         and aggregate m = sum_i alpha_i e_i, alpha_i = n_i / sum of matched orders  */
    int32_t gate;     /* CONST: g = lambda.  COSINE: g = lambda * sigmoid(cos(h, m))                 */
    float   lambda;   /* the memory injection scale                                                  */
} tfe_inject_params;

/*
 * tfe_index_build -- build the exact-match phrase index and the per-phrase
 * metadata (paper Sec. 4.2: an index in two levels, from token prefixes to phrase ids and from
 * phrase ids to memory addresses; per phrase its length, the address of its vector, its tier).
 *
 *   cfg            HOST.
 *   phrase_tokens  HOST int32 [N][4]; phrase i is the first phrase_len[i] entries, the rest -1.
 *   phrase_len     HOST uint8 [N]; must be one of cfg->orders.
 *   init_slot      HOST int32 [N]; >= 0: GPU-tier slot holding the vector; -1: host DRAM; -2: SSD.
 *   gpu_rows       DEVICE bf16 [C][d] row-major, 16-byte aligned, CALLER-OWNED, already holding
 *                  the vectors of the resident phrases.  The library keeps the pointer and writes
 *                  to it only in tfe_cache_install.
 *   stream         work is issued here; the call synchronises it before returning.
 *   out            receives the context (phrase id = index into the arrays above).
 *
 * Errors (nothing is kept): INVALID_ARG (geometry, length not an order, token outside [0,vocab)),
 * DUPLICATE_PHRASE, KEY_COLLISION, CAPACITY, SLOT_RANGE, PROBE_LIMIT, CUDA.
 */
tfe_status tfe_index_build(const tfe_config *cfg, const int32_t *phrase_tokens,
                           const uint8_t *phrase_len, const int32_t *init_slot, void *gpu_rows,
                           void *stream, tfe_ctx **out);

/*
 * tfe_index_build_device -- the same construction with the phrase table already on the DEVICE
 * (phrase_tokens int32 [N][4] 16-byte aligned, phrase_len uint8 [N], init_slot int32 [N]) and
 * every step on the GPU: key formation and input checks, two-choice cuckoo placement with
 * 128-bit compare-and-swap / exchange on whole index slots, and a final pass in which every
 * phrase looks itself up (which is also how equal tuples and colliding hashes are found).  The
 * paper's index construction is its dominant offline cost (Sec. 5.3); this is that step for
 * tables that are produced or kept on the GPU.  Results of later calls do not depend on which
 * of the two builds made the context (only the mapping is defined, not the slot a key sits in).
 * Two kernel launches, one synchronisation of `stream`; the host-side copy of the residency
 * state that tfe_cache_install checks its arguments against is fetched on its first call.
 * Errors as tfe_index_build; when several problems are present
 * the one reported may differ.
 */
tfe_status tfe_index_build_device(const tfe_config *cfg, const int32_t *phrase_tokens,
                                  const uint8_t *phrase_len, const int32_t *init_slot,
                                  void *gpu_rows, void *stream, tfe_ctx **out);

/*
 * tfe_cache_install -- write n fetched vectors into GPU-tier slots and make
 * their phrases GPU-resident (paper Sec. 4.3: an entry read from DRAM / SSD is
 * inserted into a faster tier when it arrives; Sec. 4.4: prefetched entries
 * are moved into the GPU cache before they are needed).
 *
 *   phrase_ids  HOST uint32 [n]; valid, pairwise distinct, currently NOT GPU-resident.
 *   src_rows    bf16 [n][d]; HOST (pinned memory makes the copy asynchronous; it must stay valid
 *               until the stream has passed this call) or DEVICE.
 *   dst_slots   HOST int32 [n]; pairwise distinct, in [0, C).  A slot that holds another phrase
 *               is overwritten and that phrase falls back to the host-DRAM tier.
 *   Asynchronous on `stream`; a lookup issued later on the same stream sees the new state.
 *   phrase_ids / dst_slots may be reused as soon as the call returns.
 *
 * Errors (state unchanged): INVALID_ARG, UNKNOWN_PHRASE, ALREADY_RESIDENT, SLOT_RANGE, CUDA.
 */
tfe_status tfe_cache_install(tfe_ctx *ctx, int32_t n, const uint32_t *phrase_ids,
                             const void *src_rows, const int32_t *dst_slots, void *stream);

/*
 * tfe_cache_install_device -- the same insertion with the whole batch on the DEVICE and no check
 * by the host: what a prefetch loop that stays on the GPU produces (candidate phrases from
 * tfe_prefetch_candidates, destination slots from tfe_cache_select_victims_device, rows staged in
 * device memory).  Entries that cannot be applied are skipped instead of refusing the batch.
 * Judged against the state before the call, entry k is a candidate if phrase_ids[k] is a phrase,
 * that phrase is not GPU-resident, dst_slots[k] is a slot and no earlier entry names the same
 * phrase; it is applied if in addition no earlier candidate names the same slot.  Applied
 * entries take effect as in tfe_cache_install.
 *
 *   n              0..4096
 *   phrase_ids     DEVICE uint32 [n];  src_rows DEVICE [n][d] bf16, 16-byte aligned;
 *   dst_slots      DEVICE int32 [n]
 *   applied        DEVICE uint8 [n], receives 1 / 0 per entry, or NULL
 *   applied_count  DEVICE uint32, receives the number applied, or NULL
 * Asynchronous on `stream`, two kernel launches, never synchronises.  The first call on a context
 * allocates 4 bytes per phrase and per slot (with a device synchronisation: make it outside a stream
 * capture); every later call keeps no state on the host and may be captured into a CUDA graph and
 * replayed with new contents in the same buffers.  Once this function has been used, the host-side
 * residency copy that tfe_cache_install checks against is re-read from the device (one
 * synchronisation) on every call of that function.
 * Errors: INVALID_ARG, CUDA.
 */
tfe_status tfe_cache_install_device(tfe_ctx *ctx, int32_t n, const uint32_t *phrase_ids,
                                    const void *src_rows, const int32_t *dst_slots, uint8_t *applied,
                                    uint32_t *applied_count, void *stream);

/*
 * tfe_lookup_inject -- the hot path, one kernel launch (paper Sec. 2.2: key
 * from token n-grams, lookup m_t = M(q_t), aggregation m_t = sum alpha_i v_i,
 * injection h'_t = h_t + g_t * m_t; Sec. 4.2: longest-match selection;
 * Sec. 4.3: tier walk).
 *
 *   tokens      DEVICE int32 [B][T] row-major.
 *   q_start     queries are the positions t in [q_start, T) of every sequence,
 *               numbered q = b*(T-q_start) + (t-q_start); Q = B*(T-q_start).  An n-gram ends at
 *               its query position and never reaches before t = 0 of its sequence.
 *   h           DEVICE [Q][d] hidden states (bf16 or fp32 per cfg.hidden_dtype), 16-byte aligned.
 *   out         DEVICE [Q][d], same dtype; may be the same pointer as h (then only injected
 *               positions are touched); must not partially overlap h.
 *   params      HOST.
 *   sel_phrase  DEVICE uint32 [Q] (LONGEST) or [Q][n_orders] (ALL, column = index into orders);
 *   sel_slot    DEVICE int32, same shape: slot (hit), -1 host, -2 SSD, -3 absent;
 *   flags       DEVICE uint8, same shape: TFE_FLAG_*.   Any of the three may be NULL.
 *
 * Positions whose retained phrase is GPU-resident get out = round(h + g*m) (fp32 arithmetic,
 * round-to-nearest-even into the hidden dtype); every other position gets out = h bit for bit.
 * A retained phrase that is not GPU-resident is NOT replaced by a shorter resident one; it goes to
 * the miss list.  Asynchronous; launches exactly one kernel and never synchronises.
 * Errors: INVALID_ARG, CUDA (a first call with a larger Q than any before grows context buffers).
 */
tfe_status tfe_lookup_inject(tfe_ctx *ctx, const int32_t *tokens, int32_t B, int32_t T,
                             int32_t q_start, const void *h, void *out,
                             const tfe_inject_params *params, uint32_t *sel_phrase,
                             int32_t *sel_slot, uint8_t *flags, void *stream);

/*
 * tfe_lookup_inject_host -- the same call for HOST buffers (tokens, h, out and the optional
 * result arrays all in host memory; pinned memory lets the copies run asynchronously and
 * overlap): copies the inputs to context-owned device buffers, runs the kernel, copies the
 * results back, without synchronising the host.  Everything is ordered after the work already
 * queued on `stream`, and `stream` continues only when the last result byte is in host memory,
 * so the caller sees the call as one operation on `stream`.  The buffers must stay valid until
 * the stream has passed the call.
 *
 * LONGEST / CONST calls with at least 16 MiB of hidden state are issued in pieces (query ranges;
 * up to 32, small at both ends, up to 8 MiB in the middle) through two context-owned copy
 * streams, so that one piece's kernel runs while the next piece comes in and the previous one
 * goes back; the last piece's launch builds the miss list of the whole call.  Results are the
 * same as for the single launch.  Other variants copy, launch once and copy back on `stream`.
 * The first piecewise call on a context creates the two streams and their events.
 */
tfe_status tfe_lookup_inject_host(tfe_ctx *ctx, const int32_t *tokens, int32_t B, int32_t T,
                                  int32_t q_start, const void *h, void *out,
                                  const tfe_inject_params *params, uint32_t *sel_phrase,
                                  int32_t *sel_slot, uint8_t *flags, void *stream);

/*
 * tfe_miss_list -- the compacted, order-stable list of retained phrases that were not
 * GPU-resident in the most recent lookup of this context (paper Sec. 4.3: such entries are staged
 * from DRAM or read asynchronously from SSD; Sec. 4.4: the prefetcher consumes the same records).
 * Entries are in ascending (q, order); duplicates are kept; tier is TFE_FLAG_HOST_MISS / SSD_MISS.
 *
 *   q_idx, phrase_id, tier   HOST buffers of `cap` entries (may be NULL if cap == 0).
 *   count                    HOST, always receives the full miss count.
 *   Synchronises `stream`.  Errors: MISS_OVERFLOW (count > cap; the first cap entries are
 *   returned), INTERNAL, CUDA.
 */
tfe_status tfe_miss_list(tfe_ctx *ctx, uint32_t *q_idx, uint32_t *phrase_id, uint8_t *tier,
                         int64_t cap, int64_t *count, void *stream);

/*
 * tfe_lookup_inject_noalloc -- tfe_lookup_inject for callers that must not allocate.  (The paper
 * has no counterpart for this entry point; it exists for the sake of the embedding runtime.)
 *
 * tfe_lookup_inject lets the context cudaMalloc its per-call scratch on first use and again when
 * a larger call arrives.  A runtime that has given all free device memory to its own pool, or a
 * latency-critical loop that cannot tolerate the device-wide synchronisation an allocation or a
 * free brings, calls this instead: it allocates and frees nothing, on the host or on the device.
 * Its scratch is a fixed area inside the loaded library image (2 MiB: one 8-byte result record per
 * entry; present on every GPU that loads the library until the process ends), which bounds the call:
 *
 *     Q * (policy == ALL ? n_orders : 1)  <=  262,144      otherwise TFE_ERR_CAPACITY.
 *
 *   tokens ... flags   as for tfe_lookup_inject (DEVICE; sel_phrase / sel_slot / flags may be NULL).
 *   miss_q, miss_phrase, miss_tier
 *                      DEVICE, CALLER-OWNED, each with room for Q * (ALL ? n_orders : 1) entries;
 *                      receive the ordered miss list (the context's own list and tfe_miss_list are
 *                      not involved).  Required.
 *   miss_count         DEVICE uint32, receives the number of entries written.  Required.
 *
 * The context's device must be the current device.  The first call on a device looks up the
 * address of the scratch area (cudaGetSymbolAddress); make that first call outside any stream
 * capture.  All calls on one device share the area, whatever their context, and it keeps what the
 * last call left: a call puts the launch state back to zero on its stream (a call refused for its
 * arguments touches nothing), and records carry the number of the call that wrote them, so a record
 * left by an earlier call is never taken for one of this call.  Two calls that overlap on the GPU
 * (different streams, no dependency) race.  Results are those of tfe_lookup_inject.
 * Errors: INVALID_ARG, CAPACITY, CUDA.
 */
tfe_status tfe_lookup_inject_noalloc(tfe_ctx *ctx, const int32_t *tokens, int32_t B, int32_t T,
                                     int32_t q_start, const void *h, void *out,
                                     const tfe_inject_params *params, uint32_t *sel_phrase,
                                     int32_t *sel_slot, uint8_t *flags, uint32_t *miss_q,
                                     uint32_t *miss_phrase, uint8_t *miss_tier, uint32_t *miss_count,
                                     void *stream);

/* The same list as DEVICE pointers owned by the context, valid until the next lookup; no sync. */
tfe_status tfe_miss_list_device(tfe_ctx *ctx, const uint32_t **q_idx, const uint32_t **phrase_id,
                                const uint8_t **tier, const uint32_t **count);

/*
 * GPU-tier retention ranking (paper Sec. 4.3 names the signals an implementation may rank entries by --
 * access frequency and recency among them -- and gives no formula; the ranking below is this
 * library's reading).
 *
 * tfe_cache_policy_enable -- starts the bookkeeping: from now on every lookup of this context
 * (tfe_lookup_inject, tfe_lookup_inject_host; not tfe_lookup_inject_noalloc) adds 1 to `freq` and
 * stores the call's epoch in `last` for every GPU-tier slot it injects from, and every
 * tfe_cache_install sets {freq, last} = {1, epoch} for the slots it fills.  The epoch is a device
 * counter of completed lookups (a replayed launch advances it like a fresh one).  Calling it
 * again clears the counters and the epoch.  Allocates 8 bytes per GPU-tier slot and 8.2 MiB of work
 * space for the selection on the first call; waits for the device then.  Launches recorded earlier (a captured CUDA graph) keep the arguments they were
 * recorded with and do no bookkeeping; record them again after enabling.
 * Errors: INVALID_ARG, CUDA.
 */
tfe_status tfe_cache_policy_enable(tfe_ctx *ctx, void *stream);

/*
 * tfe_cache_select_victims -- the n slots least worth keeping at the current epoch `now`:
 *     age     = now - last                                  (unsigned 32-bit)
 *     decayed = freq >> min(31, age / half_life)            (half_life <= 0: no decay)
 *     key     = min(decayed, 65535) << 16 | (65535 - min(age, 65535));  key = 0 for a free slot
 * in ascending (key, slot): free slots first, then by decayed frequency, ties by least recent
 * use, then by slot.  half_life -> large gives least-frequently-used order, equal frequencies
 * give least-recently-used order.
 *
 *   n        0..4096;  half_life at most 2^26 - 1;  slots HOST int32 [n], or NULL;  keys HOST uint32 [n] or NULL;
 *   count    HOST: entries written = min(n, gpu_slots).
 * One cooperative kernel launch on `stream` (one block per SM; its blocks wait for one another at
 * two or more step boundaries, every wait bounded).  The
 * per-slot bookkeeping is read once; a threshold taken from a sample of the slots keeps the work
 * after that pass to a candidate list, and the result does not depend on the sample: a threshold
 * that turns out too low or too high only makes the call walk the table again.  With host `slots`
 * the results are copied there and the stream is synchronised (they feed tfe_cache_install, which
 * takes host arrays); with slots = NULL nothing is copied and nothing synchronises.
 * tfe_cache_select_victims_device returns the DEVICE copies of the most recent selection (owned
 * by the context, valid until the next one; they feed tfe_cache_install_device).
 * One selection at a time per context (the work space is the context's).
 * Errors: INVALID_ARG (also: policy not enabled, half_life too large), CUDA, INTERNAL (a wait inside the
 * kernel ran out or its counts contradicted one another; the outputs are not valid.  Reported by the
 * form with host `slots`, which also clears the condition; until then later selections do nothing).
 */
tfe_status tfe_cache_select_victims(tfe_ctx *ctx, int32_t n, int32_t half_life, int32_t *slots,
                                    uint32_t *keys, int32_t *count, void *stream);
tfe_status tfe_cache_select_victims_device(tfe_ctx *ctx, const int32_t **slots, const uint32_t **keys);

/*
 * tfe_cache_select_tuning -- sizes of the selection's internal steps, for tests and tuning; the
 * result of tfe_cache_select_victims does not depend on them.  list_cap: entries of the candidate
 * list (1..1048576), final_cap: numbers the last step ranks (..8192; at least n + 1 is used; a table
 * with more slots than either is sampled for a threshold), n_samples: slots sampled
 * (..2048).  0 or less: the default.  Takes effect with the next selection.
 * Errors: INVALID_ARG.
 */
tfe_status tfe_cache_select_tuning(tfe_ctx *ctx, int32_t list_cap, int32_t final_cap, int32_t n_samples);

/*
 * tfe_cache_stats -- copies the bookkeeping to the host: freq_last HOST uint32 [gpu_slots][2]
 * ({freq, last} per slot) and/or the epoch (either may be NULL).  Synchronises `stream`.
 */
tfe_status tfe_cache_stats(tfe_ctx *ctx, uint32_t *freq_last, uint32_t *epoch, void *stream);

/* Scoring of prefetch candidates. */
typedef struct {
    float   benefit_host;   /* c_i of an entry that sits in host DRAM (>= 0)                           */
    float   benefit_ssd;    /* c_i of an entry that sits only on SSD (>= 0); GPU-resident entries: 0   */
    int32_t budget;         /* at most this many candidates are returned, 0..4096                      */
} tfe_prefetch_params;

/*
 * tfe_prefetch_candidates -- candidate phrase expansion and priority for early-exit guided
 * prefetching (paper Sec. 4.4: each predicted token is put behind the sequence's recent history, the
 * n-grams that result are looked up in the token-to-phrase index and give the candidate set Q_t;
 * a candidate's priority is s_i = p_i * r_i * c_i, and the budget goes to the highest priorities,
 * the rest is dropped).  The top-K tokens and their probabilities are inputs: they come from the
 * early-exit head, tfe_head_topk below, or from anywhere else.
 *
 *   history      DEVICE int32 [B][H]: the last H tokens of every sequence (H >= n_max - 1 to let
 *                every order contribute; an order n with n - 1 > H contributes nothing).
 *   cand_tokens  DEVICE int32 [B][K]: predicted next tokens;  cand_prob DEVICE float [B][K]: p.
 *   usefulness   DEVICE float [N]: r of every phrase, or NULL for r = 1.
 *   params       HOST.
 * For every sequence b, token k and configured order n the n-gram (history[b][H-n+1..H-1],
 * cand_tokens[b][k]) is looked up; a phrase found outside the GPU tier is a candidate with
 * s = (p * r) * c in fp32, dropped if s <= 0.  Outputs (DEVICE, `budget` entries each): phrase id,
 * tier (TFE_FLAG_HOST_MISS / TFE_FLAG_SSD_MISS), s, and source b*K + k of the `budget` best, in
 * descending s, equal s in ascending (b, k, order); duplicates of one phrase are kept.
 * out_count DEVICE uint32 [2]: entries written, candidates found before the cut.  The phrase ids
 * beyond the entries written are set to TFE_NO_PHRASE (the other arrays are left as they were), so
 * the whole array can be handed to tfe_cache_install_device, which skips ids that are no phrase.
 * Asynchronous on `stream`, two kernel launches; a first call with more entries than any before
 * grows context buffers.  Errors: INVALID_ARG, CUDA.
 */
tfe_status tfe_prefetch_candidates(tfe_ctx *ctx, const int32_t *history, int32_t B, int32_t H,
                                   const int32_t *cand_tokens, const float *cand_prob, int32_t K,
                                   const float *usefulness, const tfe_prefetch_params *params,
                                   uint32_t *out_phrase, uint8_t *out_tier, float *out_score,
                                   uint32_t *out_src, uint32_t *out_count, void *stream);

/* Frees everything the context owns (not gpu_rows).  NULL is allowed. */
void tfe_destroy(tfe_ctx *ctx);

const char *tfe_status_string(tfe_status s);

/* Text of the last CUDA error seen by this thread's calls ("" if none). */
const char *tfe_last_cuda_error(void);

/*
 * Introspection used by tests and the benchmark (HOST only, no device work).
 *   tfe_index_geometry  buckets (of 4 slots of 16 bytes), bytes of the device index, bytes of per-phrase metadata.
 *   tfe_phrase_key64    the 64-bit index key of a token tuple (0 if n or a token is invalid) and
 *                       whether that order is packed injectively (exact) or hashed + verified.
 *   tfe_home_bucket     the first bucket probed for a key.
 *   tfe_launch_geometry grid size, block size and queries per warp round of the last lookup.
 */
tfe_status tfe_index_geometry(const tfe_ctx *ctx, int64_t *n_buckets, int64_t *index_bytes,
                              int64_t *metadata_bytes);
uint64_t tfe_phrase_key64(int32_t vocab, const int32_t *tokens, int32_t n, int32_t *is_exact);
uint64_t tfe_home_bucket(uint64_t key, uint64_t n_buckets);
tfe_status tfe_launch_geometry(const tfe_ctx *ctx, int32_t *grid, int32_t *block, int32_t *batch_queries);

/*
 * Tuning knob (HOST only; results never depend on it).  A lookup warp takes batches of 1..8
 * consecutive queries: it probes the whole batch at once (one lane per query and order), then
 * streams the batch's rows.  0 = the library picks per call (small calls 1, the lowest latency;
 * large calls 4).
 */
tfe_status tfe_set_tuning(tfe_ctx *ctx, int32_t batch_queries);

/*
 * Early-exit prefetch head (paper Sec. 4.4): p_early(x_{t+1} | x_<=t) = softmax(W_pref h_t^{L-r})
 * and T_early = TopK(p_early) -- the K most likely next tokens of every sequence with their
 * probabilities, which are the inputs of tfe_prefetch_candidates.  The only dense contraction of
 * the method; it runs on the tensor cores.  A head is independent of any phrase index.
 *
 * tfe_head_create -- w_pref DEVICE bf16 [V][d] row-major, 16-byte aligned, CALLER-OWNED; it is
 * copied into the head in the order the GEMM reads it (pieces of 128 rows x 64 columns, 16
 * contiguous KB each) and may be released when the call returns (the call waits for the device);
 * d a multiple of 64; max_batch 1..256.  Allocates that copy (V * d * 2 bytes, rounded up to
 * whole 128-row tiles per CTA: 349 MB for V = 151,936, d = 1,024), the logits buffer
 * (max_batch * V * 4 bytes) and small work areas on the current device.
 * Errors: INVALID_ARG, CUDA.
 */
typedef struct tfe_head tfe_head;
tfe_status tfe_head_create(const void *w_pref, int32_t V, int32_t d, int32_t max_batch, tfe_head **out);
void       tfe_head_destroy(tfe_head *head);

/*
 * tfe_head_topk -- hidden DEVICE bf16 [B][d] (16-byte aligned), 0 <= B <= max_batch, 1 <= K <= 128,
 * K <= V.  Outputs DEVICE: cand_tokens int32 [B][K], cand_prob float [B][K], per sequence in
 * descending probability, equal logits in ascending token id.  Logits are bf16 products
 * accumulated in fp32 (tensor cores); selection and softmax in fp32.  Asynchronous on `stream`,
 * two kernel launches, never synchronises.  Errors: INVALID_ARG, CUDA, INTERNAL.
 */
tfe_status tfe_head_topk(tfe_head *head, const void *hidden, int32_t B, int32_t K, int32_t *cand_tokens,
                         float *cand_prob, void *stream);

/* DEVICE views of the most recent call: logits fp32 [B][ld] and log-sum-exp fp32 [B]; owned by the head. */
tfe_status tfe_head_buffers(tfe_head *head, const float **logits, int64_t *ld, const float **lse);

/*
 * tfe_head_status -- synchronises `stream` and reads the device status word: 0, or a bit set by a
 * wait inside the kernel that ran out (1 loader, 2 MMA issuer, 4 epilogue); then INTERNAL.
 */
tfe_status tfe_head_status(tfe_head *head, uint32_t *device_flags, void *stream);

/* Launch geometry: CTAs, vocabulary rows per CTA, rows of each CTA's short last tile. */
tfe_status tfe_head_geometry(const tfe_head *head, int32_t *grid, int32_t *rows_per_cta, int32_t *tail_rows);

/*
 * N-gram extraction with a frequency threshold (paper Sec. 4.2, construction pipeline: candidate
 * phrases such as bigrams and trigrams are selected by a frequency threshold; Sec. 5.3: this
 * tokenizer-level n-gram extraction dominates the offline cost of building a table).  Independent of
 * any context; its output is the phrase table that tfe_index_build_device takes.
 *
 *   tokens         DEVICE int32 [L], the tokenised corpus; an id outside [0, vocab) separates documents:
 *                  no window contains one.  0 <= L <= TFE_MINE_MAX_TOKENS.
 *   orders         HOST int32 [n_orders], strictly ascending, each in 1..4.
 *   window         for an order n and an end position t >= n - 1 whose n ids x_{t-n+1} .. x_t are all
 *                  valid, that tuple occurs once at t.  count(tuple) = number of occurrences,
 *                  first(tuple) = its smallest end position.
 *   result         the tuples with count >= min_count (0 means 1) in ascending (first, n) order:
 *                  phrase_tokens DEVICE int32 [cap][4] (16-byte aligned; unused trailing ids -1),
 *                  phrase_len DEVICE uint8 [cap], phrase_count DEVICE uint32 [cap]; may be NULL if cap = 0.
 *   n_found        HOST: how many tuples qualify; min(n_found, cap) entries were written (the first ones
 *                  in that order) -- n_found > cap is not an error, the caller raises min_count or cap.
 *   distinct       HOST int64 [n_orders] or NULL: different tuples per order.
 *   hist           HOST int64 [TFE_MINE_HIST_BINS] or NULL: hist[c] = different tuples, all orders together,
 *                  that occur exactly c times; the last bin collects every c >= TFE_MINE_HIST_BINS - 1.
 *                  sum_{c >= m} hist[c] is n_found for min_count = m, so one call tells which threshold
 *                  yields a table of a wanted size.
 *
 *   workspace      DEVICE scratch of workspace_bytes >= tfe_mine_workspace_bytes(L, n_orders) (about 24..48
 *                  bytes per token for the counting table plus 4 bytes per token and order (+ 1); smaller:
 *                  TFE_ERR_CAPACITY), contents undefined before and after; or NULL with workspace_bytes = 0:
 *                  the call allocates and frees it (several milliseconds per call at 10^8 tokens).
 *
 * Launches on `stream` and synchronises it.  Exact for every vocabulary: orders whose ids do not fit one
 * 64-bit key side by side are keyed through the exact names of their halves.  Errors:
 * TFE_ERR_INVALID_ARG, TFE_ERR_CAPACITY, TFE_ERR_CUDA (the workspace could not be allocated),
 * TFE_ERR_INTERNAL (a bounded probe ran out).
 */
#define TFE_MINE_HIST_BINS 1024
#define TFE_MINE_MAX_TOKENS (1ll << 30)
tfe_status tfe_mine_ngrams(const int32_t *tokens, int64_t L, int32_t vocab, int32_t n_orders, const int32_t *orders,
                           uint32_t min_count, int64_t cap, int32_t *phrase_tokens, uint8_t *phrase_len,
                           uint32_t *phrase_count, int64_t *n_found, int64_t *distinct, int64_t *hist,
                           void *workspace, int64_t workspace_bytes, void *stream);
int64_t tfe_mine_workspace_bytes(int64_t L, int32_t n_orders);   /* -1 for invalid arguments */

/*
 * Initial residency from corpus counts (paper Sec. 4.3: the GPU tier is reserved for the most frequently
 * accessed entries, DRAM holds warm entries, SSD absorbs the long tail).  Turns the counts that
 * tfe_mine_ngrams returns into the init_slot array that tfe_index_build_device takes.
 *
 *   count           DEVICE uint32 [N];  init_slot DEVICE int32 [N] (output);  0 <= N, gpu_slots < 2^31
 *   rule            the G = min(gpu_slots, N) phrases of largest count start in the GPU tier, among equal
 *                   counts the smaller id first; GPU-tier slots are handed out in id order (the chosen
 *                   phrase with the k-th smallest id gets slot k).  Of the others, count >= host_min_count
 *                   means host DRAM (-1), a smaller count SSD (-2).
 *   tiers           HOST int64 [3] or NULL: phrases per tier (GPU, host, SSD).
 *
 * Allocates a few bytes per 1,024 phrases, launches on `stream`, synchronises it.
 * Errors: TFE_ERR_INVALID_ARG, TFE_ERR_CUDA, TFE_ERR_INTERNAL (the selection's totals do not add up).
 */
tfe_status tfe_assign_residency(const uint32_t *count, int64_t N, int64_t gpu_slots, uint32_t host_min_count,
                                int32_t *init_slot, int64_t *tiers, void *stream);

/*
 * Rows of logits.  The calls below work on DEVICE matrices of vocabulary logits, one row per position,
 * row r starting `ld` elements after row r - 1 (ld >= V, at most 2^34; rows need no alignment beyond the
 * element's own), as fp32 or bf16.  They come from a head (tfe_head_buffers, tfe_matmul_fp8) or from the model
 * itself.  A logit at or below -1e30 is a masked one: -inf, or the lowest value of either type.
 * These calls keep no state (but tfe_matmul_fp8's status word and switch), allocate nothing, never synchronise (but
 * tfe_matmul_fp8_status) and may be captured into a CUDA graph; they
 * work on the current device, which has to be the one that holds the buffers.  Calls on different streams are
 * independent.  Argument errors are found on the host before anything is launched.  Results must not touch
 * operands unless a call says that they may.
 */
enum { TFE_DTYPE_BF16 = 0, TFE_DTYPE_F32 = 1 };
#define TFE_ROWS_MAX (1 << 27)

/*
 * The vocabulary product in 8 bits: the head's contraction (paper Sec. 4.4) with one byte per weight.  Both operands
 * are e4m3 with an fp32 scale for each block of 128 columns: per row for activations, per 128 rows for weights.
 *
 * tfe_quantize_fp8 -- x DEVICE [R][ld], dtype TFE_DTYPE_*, to q DEVICE e4m3 [R][C] (rows side by side) and
 * scale DEVICE float [ceil(R / block_rows)][ceil(C / 128)];  block_rows 1 (activations) or 128 (weights);
 * 1 <= C <= TFE_FP8_MAX_COLS, fewer than 2^31 blocks.  scale = max(largest |x| of the block / 448, 2^-126) and
 * q = x / scale, the quotients correctly rounded to fp32 and then to the nearest e4m3 (ties to even).  A
 * block that holds an infinity or NaN has it as its scale and reads back as NaN.  One launch.
 *
 * tfe_quantize_fp8_ld -- the same with q's rows `ldq` bytes apart (C <= ldq <= 2^34; the bytes between them stay as they
 * were): the operands of tfe_matmul_fp8 have rows a multiple of 16 bytes apart.
 *
 * tfe_matmul_fp8 --
 *     out[m][n] = sum_b a_scale[m][b] * w_scale[n / 128][b] * (sum of a[m][k] * w[n][k] over block b's 128 k)
 *   a DEVICE e4m3 [M][lda], a_scale DEVICE float [M][kb];  w DEVICE e4m3 [N][ldw], w_scale DEVICE float
 *   [ceil(N / 128)][kb], kb = ceil(K / 128);  out DEVICE [M][ldo], fp32 or bf16.  0 <= M, 1 <= N <= TFE_ROWS_MAX,
 *   1 <= K <= TFE_FP8_MAX_COLS; a and w 16-byte aligned, lda and ldw multiples of 16.  A block's products are
 *   summed by the tensor cores, blocks in fp32, and the result is rounded once.  The product of a block's two scales is
 *   formed in fp32 first: below 2^-126 it loses bits, from 2^128 on the results are infinite or NaN.  Elements of out beyond N stay as
 *   they were.  One launch.
 *
 *   Every wait inside the kernel is bounded.  Should one run out, the results that the call has not stored by then are NaN,
 *   from which tfe_sample_tokens draws -1.
 *
 * tfe_matmul_fp8_status -- synchronises `stream`, reads the library's status word on the current device and clears what
 * it read: 0, or bits set by waits inside the kernel that ran out (1 loader, 2 MMA issuer, 4 scales, 8 epilogue); then
 * INTERNAL.  The word is one for all calls on the device, whatever their stream: it says that some product since the
 * last report failed, and the NaN in its results which.
 *
 * tfe_matmul_fp8_give_up, for tests of how a caller takes a failure -- 0: as usual; 2: in the products that follow, of the whole process, the
 * MMA issuers' waits count as run out after their first tile, with copies and MMAs under way; another number: all waits do from the start.
 * Errors of all five: INVALID_ARG, CUDA.
 */
#define TFE_FP8_MAX_COLS (1 << 16)
tfe_status tfe_quantize_fp8(const void *x, int32_t dtype, int32_t R, int32_t C, int64_t ld, int32_t block_rows,
                            void *q, float *scale, void *stream);
tfe_status tfe_quantize_fp8_ld(const void *x, int32_t dtype, int32_t R, int32_t C, int64_t ld, int32_t block_rows,
                               void *q, int64_t ldq, float *scale, void *stream);
tfe_status tfe_matmul_fp8(const void *a, int64_t lda, const float *a_scale, int32_t M, const void *w, int64_t ldw,
                          const float *w_scale, int32_t N, int32_t K, void *out, int32_t out_dtype, int64_t ldo,
                          void *stream);
tfe_status tfe_matmul_fp8_status(uint32_t *device_flags, void *stream);
tfe_status tfe_matmul_fp8_give_up(int32_t how);

/*
 * tfe_sample_tokens -- the next token of every sequence from its logits and one given random number per sequence
 * (the lookups are keyed by the token ids that decoding produces; the paper names no sampling rule).  Per row, in
 * the order of descending logits, equal logits by ascending id, with w_i = exp((z_i - z_max) / temperature):
 *     min-p   entries with w_i >= min_p                               (min_p <= 0: all of them)
 *     top-k   the first top_k of those                                (top_k <= 0: all)
 *     top-p   the shortest prefix of those whose sum of w reaches top_p of theirs; at least one entry (top_p >= 1: all)
 *     token   the first entry of those whose running sum exceeds u of theirs;  prob = its w over their sum.
 * A temperature that is not greater than 0 takes the first entry (prob 1).  Masked (-inf) and NaN logits are never
 * drawn; a row without any other gives token -1 and prob 0.  Logits of +inf, if any, share the draw.  (The lowest value of
 * a type needs no rule here: its weight is 0 next to any other logit.)
 *
 *   logits        DEVICE [B][ld], dtype TFE_DTYPE_*;  0 <= B <= TFE_ROWS_MAX, 1 <= V <= TFE_SAMPLE_MAX_VOCAB.
 *   params        HOST; four DEVICE arrays of B values, or NULL for: temperature 1, no restriction.  Values
 *                 outside a parameter's range act as its nearest end; NaN as "no restriction" (temperature: greedy).
 *   u             DEVICE float [B], in [0, 1): values outside are brought to the nearest end, NaN to 0.
 *   tokens, prob  DEVICE int32 [B], DEVICE float [B] (prob may be NULL).
 * Weights are evaluated in fp64 and summed as whole numbers of a unit, 2^-45 of the greatest weight (beyond 2^17
 * entries coarser by as many bits), so a row's result does not depend on the rest of the batch, on its place in it, or on
 * the order of any addition; an entry that weighs less than half a unit adds nothing and is not drawn.  Every entry is
 * rounded for itself: an end may lie off by half a unit for each entry before it.  One launch.
 * Errors: INVALID_ARG, CUDA.
 */
#define TFE_SAMPLE_MAX_VOCAB (1 << 24)
typedef struct {
    const float   *temperature;
    const int32_t *top_k;
    const float   *top_p;
    const float   *min_p;
} tfe_sample_params;
tfe_status tfe_sample_tokens(const void *logits, int32_t dtype, int32_t B, int32_t V, int64_t ld,
                             const tfe_sample_params *params, const float *u, int32_t *tokens, float *prob,
                             void *stream);

/*
 * Distillation of a teacher's top logits (paper Sec. 4.4: the early-exit projection predicts the full model's
 * next tokens; the paper gives no training rule, this is the library's: the divergence from the teacher's
 * distribution over its K best tokens to the predictor's over the whole vocabulary).  Per row, with q the
 * softmax of teacher_logits / tau over the row's valid entries and lse = ln sum_v exp(z_v / tau):
 *     loss = tau^2 * sum_k q_k (ln q_k - z[id_k] / tau + lse)
 *     grad_v = grad_loss * tau * (exp(z_v / tau - lse) - sum of q_k with id_k = v)
 *
 *   logits           DEVICE [N][ld], dtype TFE_DTYPE_*;  0 <= N <= TFE_ROWS_MAX.
 *   teacher_ids      DEVICE int32 [N][K];  an id outside [0, V) is no entry.  Equal ids in a row are terms of their own in
 *                    the loss and add up in the gradient.
 *   teacher_logits   DEVICE float [N][K];  logits or log-probabilities (q does not change by a constant), such as the
 *                    logarithm of tfe_head_topk's probabilities; -inf is a weight of zero.
 *   K, tau           1 <= K <= TFE_DISTILL_MAX_TOP;  1e-6 <= tau <= 1e6.
 *   loss, lse        DEVICE float [N].  Sums run in fp32 and are joined in fp64; each result is rounded once.
 *   grad_loss        DEVICE float [N]: the gradient that arrives at each row's loss.
 *   grad_logits      DEVICE [N][ld_grad] of the logits' type, rounded once; may be the logits themselves (same
 *                    pointer and ld_grad = ld), and must not touch them otherwise, nor any other operand (refused).
 *                    Elements beyond V stay as they were.
 * A row without a teacher weight, or without an unmasked logit, has loss 0 and gradient 0 (lse = -inf for the
 * latter), and so has a row whose grad_loss is 0.  A masked logit has probability 0; a teacher weight on it makes the
 * loss +inf and its gradient -grad_loss * tau * q.  NaN propagates, and a logit of +inf makes its row's results NaN.  The loss
 * keeps its precision for logits of any size; the gradient's probabilities are relative to lse as it is given, which
 * as an fp32 number is off by up to |lse| 2^-24.  One launch each.  Errors: INVALID_ARG, CUDA.
 */
#define TFE_DISTILL_MAX_TOP 1024
tfe_status tfe_distill_forward(const void *logits, int32_t dtype, int32_t N, int32_t V, int64_t ld,
                               const int32_t *teacher_ids, const float *teacher_logits, int32_t K, float tau,
                               float *loss, float *lse, void *stream);
tfe_status tfe_distill_backward(const void *logits, int32_t dtype, int32_t N, int32_t V, int64_t ld,
                                const int32_t *teacher_ids, const float *teacher_logits, int32_t K, float tau,
                                const float *lse, const float *grad_loss, void *grad_logits, int64_t ld_grad,
                                void *stream);

/*
 * Softmax cross entropy from hidden states and the vocabulary projection, without keeping the logits (paper Sec. 4.4: the
 * early-exit projection predicts the next token; the paper gives no training rule, this is the library's).  Per row, with
 * z_v = weight[v] . hidden[n], t the target and lse = ln sum_v exp(z_v):
 *     loss = lse - z_t
 *     grad_hidden[n] = sum_v G[n][v] weight[v],  grad_weight[v] = sum_n G[n][v] hidden[n],  G[n][v] = grad_loss[n] (exp(z_v - lse) - [v = t])
 *
 *   hidden, weight   DEVICE bf16 [N][ld_hidden], [V][ld_weight]: rows of d elements, 16-byte aligned, distances multiples of 8;
 *                    0 <= N, 1 <= V <= TFE_XENT_MAX_ROWS, d a multiple of 8 up to TFE_XENT_MAX_COLS.
 *   target           DEVICE int32 [N]; a row whose target is outside [0, V) has loss, lse and gradient 0 and takes part in no sum,
 *                    whatever its hidden state holds; so does, for the gradients, a row whose grad_loss is 0.
 *   loss, lse        DEVICE float [N].  Products are summed by the tensor cores in fp32, exponentials in fp32, and joined in fp64.
 *   grad_loss        DEVICE float [N]: the gradient that arrives at each row's loss.  lse: as tfe_xent_forward left it.
 *   grad_hidden, grad_weight   DEVICE bf16, rows as above, every row written; one of them may be NULL.  They must touch no operand
 *                    and not each other.  G is rounded to bf16 for the two products with it (the tensor cores take both operands in one
 *                    type; a G of its own error 2^-9 on average adds as much to a gradient as the gradient's own rounding), but for its
 *                    entries at the targets, whose rounding is made up for in fp32 and which are minus the sum of the row's others: a row
 *                    that is sure of its target has gradients as exact as any other.  Sums are fp32 and rounded once.
 *   workspace        DEVICE scratch, 256-byte aligned, of at least tfe_xent_*_workspace_bytes(N, V, d) bytes (smaller: TFE_ERR_CAPACITY);
 *                    contents undefined before and after.  It bounds what exists of the logits at a time.  With N rounded up to a multiple of
 *                    256, forward takes up to 64 MiB + 16 N bytes of partial results and, where N > 256, the hidden states once more (2 N d)
 *                    and 12 N; backward a piece of G of up to 256 MiB (of 4,096 columns where N > 32,768) and a 64th of that, the hidden states
 *                    (2 N d), sums for grad_hidden of up to 256 MiB (or 4 N d, d rounded up to 256, up to 128 where it is less than 256), the rows of
 *                    grad_weight that targets have (4 min(N, V) d), and 32 N + 5 V bytes.
 * NaN propagates, and a logit of +inf makes its row's results NaN; a target whose logit is -inf has a loss of +inf.  The order of every sum
 * is fixed by the sizes and the targets.
 * Forward two or three launches; backward two for each piece of the vocabulary and
 * three more.
 *
 * Every wait inside the kernels is bounded.  Should one run out, the loss and lse of the rows concerned, or all gradients, are NaN.
 * tfe_xent_status synchronises `stream`, reads the status word of the current device and clears what it read: 0, or bits set by
 * waits that ran out (1 loader, 2 MMA issuer, 4 epilogue); then INTERNAL.  tfe_xent_give_up, for tests of how a caller takes a failure --
 * 0: as usual; 2: in the calls that follow, of the whole process, the MMA issuers' waits count as run out after their first sum, with copies and
 * MMAs under way; another number: all waits do from the start.
 * Errors: INVALID_ARG, CAPACITY, CUDA.
 */
#define TFE_XENT_MAX_ROWS (1 << 24)
#define TFE_XENT_MAX_COLS (1 << 16)
int64_t tfe_xent_forward_workspace_bytes(int32_t N, int32_t V, int32_t d);     /* -1 for invalid arguments */
int64_t tfe_xent_backward_workspace_bytes(int32_t N, int32_t V, int32_t d);
tfe_status tfe_xent_forward(const void *hidden, int64_t ld_hidden, int32_t N, const void *weight, int64_t ld_weight, int32_t V,
                            int32_t d, const int32_t *target, float *loss, float *lse, void *workspace,
                            int64_t workspace_bytes, void *stream);
tfe_status tfe_xent_backward(const void *hidden, int64_t ld_hidden, int32_t N, const void *weight, int64_t ld_weight, int32_t V,
                             int32_t d, const int32_t *target, const float *lse, const float *grad_loss, void *grad_hidden,
                             int64_t ld_grad_hidden, void *grad_weight, int64_t ld_grad_weight, void *workspace,
                             int64_t workspace_bytes, void *stream);
tfe_status tfe_xent_status(uint32_t *device_flags, void *stream);
tfe_status tfe_xent_give_up(int32_t how);

/*
 * Injection between two norms (paper Sec. 2.2: h' = h + g m with a gate that is a "scalar, vector, or learned function"; the norms are
 * this library's): a norm on the memory vector, a learned gate, the residual scale lam, and the norm that the next block starts
 * with, in one pass, and its gradients in another.  Per row, with rms(x) = sqrt(mean(x^2) + eps) and s = gate, or 1 / (1 + exp(-gate))
 * with `sigmoid`, or 1 without a gate:
 *     out = h + lam s (post_weight m / rms(m)),      normed = next_weight out / rms(out)
 *
 *   h, m             DEVICE [Q][ld], rows of d elements of type dtype (TFE_DTYPE_*); 0 <= Q <= TFE_ROWS_MAX,
 *                    1 <= d <= TFE_INJECT_NORM_MAX_COLS, ld >= d; rows need no alignment beyond the element's own (16-byte rows
 *                    of a multiple of 8 elements are faster).
 *   gate             TFE_GATE_SCALAR: DEVICE float [Q];  TFE_GATE_VECTOR: DEVICE [Q][ld_gate] of type dtype;  TFE_GATE_NONE: not read.
 *   weights          DEVICE [d] each, of type weight_dtype.
 *   lam, eps         lam finite, 0 <= eps <= 1.
 *   out, normed      DEVICE [Q][ld] of type dtype, rounded once each (normed comes from out before its rounding).  out may be h itself
 *                    (same pointer and distance); they must not touch an operand or each other otherwise.
 *   grads            gradients that arrive (grad_out, grad_normed; NULL: zero, one at least is given) and those to make, of the
 *                    operands' types and shapes (grad_gate float [Q] for a scalar gate), NULL where not wanted; none may touch
 *                    anything else.  Sums run in fp32 in an order that the sizes fix; each result is rounded once.
 *   workspace        for grad_post and grad_next: DEVICE scratch, 16-byte aligned, of tfe_inject_norm_workspace_bytes(Q, d) bytes
 *                    (smaller: TFE_ERR_CAPACITY), contents undefined before and after.
 * A row of zeros has a norm of sqrt(eps) (with eps = 0 it gives NaN); mean squares must lie within fp32's range.  NaN stays in its row
 * and in the weights' gradients.  One launch forward, one or two backward.  Errors: INVALID_ARG, CAPACITY, CUDA.
 */
#define TFE_INJECT_NORM_MAX_COLS 8192
enum { TFE_GATE_NONE = 0, TFE_GATE_SCALAR = 1, TFE_GATE_VECTOR = 2 };
typedef struct {
    int32_t     dtype, Q, d;
    int32_t     gate_kind, sigmoid, weight_dtype;
    const void *h, *m, *gate;
    int64_t     ld_h, ld_m, ld_gate;
    const void *post_weight, *next_weight;
    float       lam, eps;
} tfe_inject_norm_params;
typedef struct {
    const void *grad_out, *grad_normed;
    int64_t     ld_grad_out, ld_grad_normed;
    void       *grad_h, *grad_m, *grad_gate;
    int64_t     ld_grad_h, ld_grad_m, ld_grad_gate;
    void       *grad_post, *grad_next;
} tfe_inject_norm_grads;
tfe_status tfe_inject_norm_forward(const tfe_inject_norm_params *params, void *out, int64_t ld_out, void *normed, int64_t ld_normed,
                                   void *stream);
int64_t tfe_inject_norm_workspace_bytes(int32_t Q, int32_t d);      /* -1 for invalid arguments */
tfe_status tfe_inject_norm_backward(const tfe_inject_norm_params *params, const tfe_inject_norm_grads *grads, void *workspace,
                                    int64_t workspace_bytes, void *stream);

/*
 * The norm of many gradients taken together, and clipping by it (no counterpart in the paper: the end of a training step).
 *     norm = sqrt(sum of x^2 over all elements of all tensors),   results = x min(1, max_norm / norm)
 *   tensors          HOST array of n DEVICE addresses; numel HOST int64 [n] (0 is a tensor without elements; at most 2^40 each, fewer
 *                    than 2^45 together); dtype HOST int32 [n], TFE_DTYPE_*.  0 <= n <= TFE_CLIP_MAX_TENSORS.  Elements lie side by side.
 *   results          HOST array of n DEVICE addresses of the same sizes and types, or NULL: in place.  A result may be its own tensor;
 *                    otherwise nothing that is written may touch anything else.  In place, nothing is written where norm <= max_norm.
 *   max_norm         >= 0 (+inf: clips nothing).
 *   norm             DEVICE float: the norm before clipping.  Squares are summed in fp32 by fours or eights, those sums in fp64, and
 *                    squares beyond fp32's range are formed in fp64.  Where it is not finite (an element was not, or it is beyond
 *                    fp32) the elements stay as they are.
 *   workspace        DEVICE scratch, 8-byte aligned, of tfe_clip_workspace_bytes(n) bytes (smaller: TFE_ERR_CAPACITY), contents
 *                    undefined before and after.
 * Each result is rounded once; the order of the sums depends on the sizes alone.  The lists are read before the calls return.  Two
 * launches for each 900 tensors.  tfe_grad_norm gives the norm alone.  Errors: INVALID_ARG, CAPACITY, CUDA, INTERNAL (no host memory).
 */
#define TFE_CLIP_MAX_TENSORS (1 << 20)
int64_t tfe_clip_workspace_bytes(int32_t n);                        /* -1 for invalid arguments */
tfe_status tfe_grad_norm(const uint64_t *tensors, const int64_t *numel, const int32_t *dtype, int32_t n, float *norm, void *workspace,
                         int64_t workspace_bytes, void *stream);
tfe_status tfe_clip_grad_norm(const uint64_t *tensors, const uint64_t *results, const int64_t *numel, const int32_t *dtype, int32_t n,
                              float max_norm, float *norm, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * tfe_describe_tensors -- the lists of the two calls above from n tensors that a Python program holds, HOST only: asking for each
 * property of each tensor from Python takes longer than clipping 400 of them.
 *   objects, item    a list object, and the function that gives its i-th element as a borrowed reference (PyList_GetItem)
 *   describe         dltensor_from_py_object_no_sync of the DLPack exchange interface (DLPack 1.3) that the tensors' class offers;
 *                    every element must be of that class.  The caller holds the interpreter's lock.
 *   outputs          HOST [n] each; device: the CUDA device of all.  reason: HOST, 0 or why a tensor is refused: 1 not on a CUDA
 *                    device, or on another than the first, 2 neither bf16 nor fp32, 3 its elements do not lie side by side in order,
 *                    4 describe failed and has set the interpreter's error.
 * Errors: INVALID_ARG.
 */
tfe_status tfe_describe_tensors(void *objects, void *(*item)(void *, int64_t), int (*describe)(void *, void *), int32_t n, uint64_t *tensors,
                                int64_t *numel, int32_t *dtype, int32_t *device, int32_t *reason);

/*
 * Streaming copy (the paper has no counterpart: a yardstick for the measurements, not a step of the method).
 * Copies `bytes` bytes from `src` to `dst` (DEVICE, 16-byte aligned, bytes a multiple of 16, ranges must not
 * overlap) with the load / store instructions the lookup kernels stream hidden states with, one asynchronous
 * launch on `stream`, graph-capturable.  The benchmark times it on a transfer of the lookup call's own footprint:
 * what a plain copy of that many bytes reaches on the device is the ceiling the lookup's rate is read against.
 * Errors: TFE_ERR_INVALID_ARG, TFE_ERR_CUDA.
 */
tfe_status tfe_stream_copy(void *dst, const void *src, int64_t bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TFE_H */
