/*
 * stmoe.h — C ABI of the B200 (sm_100a) decode-time MoE layer step with the
 * spatio-temporal expert predictor of ST-MoE.
 *
 * One layer step = gating network (RMSNorm, router GEMV, softmax, top-K;
 * Section 2) -> verification + table update (Algorithm 3) and prediction of
 * the next layer's experts (Algorithm 2, Eq. 1) -> miss loading and prefetch
 * of predicted experts from a pinned host store into fixed HBM slots
 * (Sections 4.1, 4.3.4) -> routed SwiGLU expert FFNs, probability-weighted
 * sum (Section 2) and the residual update of the stack harness.
 *
 * Conventions
 *   - Every function returns STMOE_OK (0) or a negative STMOE_ERR_* code; no
 *     exception, abort or output crosses this boundary.
 *   - Pointers are aligned to their element type; the MX4 and balance entry points refuse others.
 *   - "device" pointers are CUDA global memory of the device that was current
 *     in stmoe_create; "host" pointers are ordinary or pinned host memory.
 *   - load_* calls copy what they are given; the caller keeps its buffers.
 *     The library owns its weight storage, pinned host store, slot cache,
 *     copy stream, events and scratch.
 *   - cuda_stream arguments are cudaStream_t handles passed as void*.
 *   - There is no CPU fallback: without a CUDA device every call fails.
 */
#ifndef STMOE_H
#define STMOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define STMOE_OK 0
#define STMOE_ERR_BAD_ARG (-1)
#define STMOE_ERR_OOM (-2)
#define STMOE_ERR_CUDA (-3)
#define STMOE_ERR_TIMEOUT (-4)
#define STMOE_ERR_STATE (-5)
#define STMOE_ERR_UNIMPLEMENTED (-6)
#define STMOE_ERR_TOO_LARGE (-7)

/* weight_dtype */
#define STMOE_F32 0
#define STMOE_BF16 1
#define STMOE_FP8_E4M3 2 /* e4m3 codes + one bf16 scale per output channel */
#define STMOE_MX4 3      /* e2m1 codes + one e8m0 scale per 32 elements of a row (see stmoe_mx4_quantize) */
#define STMOE_F16 4      /* element type of the MX4 and balance operators only */

/* predictor_mode: which sources feed Algorithm 2 (tables evolve identically) */
#define STMOE_PRED_OFF 0
#define STMOE_PRED_TEMPORAL 1 /* history table only            */
#define STMOE_PRED_SPATIAL 2  /* cross-layer table only        */
#define STMOE_PRED_ST 3       /* both, combined as in Eq. 1    */

/* flags */
#define STMOE_FLAG_RENORM_TOPK 1 /* divide the K gate weights by their sum (off: Section 2 uses
                                    the plain softmax probabilities) */

#define STMOE_FLAG_NO_PERSISTENT 2 /* resident stacks: decode steps as per-layer kernels (replayed as a
                                      CUDA graph) instead of the single persistent kernel */

#define STMOE_FLAG_NO_DENSE 4 /* never use the tensor-core FFN kernels: by default resident bf16 and fp8
                                stacks run decode steps of at least stmoe_set_dense_min_batch() sequences
                                (default 2) with one work-list entry per expert on tcgen05 tiles,
                                rounding the hidden state and the gated activations to bf16 (bf16
                                stacks) or to the sum of three e5m2 values (fp8 stacks, whose e4m3
                                weights are multiplied as stored): relative 2^-9 either way */

#define STMOE_FLAG_NO_FUSED 8 /* resident stacks, one sequence: by default stmoe_decode_token runs a kernel
                                that streams each expert's gate, up and (from a transposed copy made at
                                load time: one third more weight memory) down rows together, one
                                streaming phase and two grid barriers per layer; its sums are exact in
                                fixed point, so results are reproducible but differ in the last bits
                                from the three-phase kernels.  This flag keeps the three-phase kernel. */

/* per-sequence result flags of a layer step */
#define STMOE_TOKEN_NEAR_TIE 1u /* K-th and (K+1)-th router logit closer than 1e-4 */

typedef struct stmoe stmoe_t;

typedef struct {
    int32_t n_layers;
    int32_t n_experts;      /* routed experts per layer, <= 256 (8-bit ids in the CCT) */
    int32_t top_k;          /* K of the gating network = candidates per CCT row, <= 32 */
    int32_t n_shared;       /* always-on experts per layer (weight 1, not predicted)   */
    int32_t hidden;         /* H, multiple of 16 (STMOE_MX4: of 32)                     */
    int32_t inter;          /* I, multiple of 16 (STMOE_MX4: of 32)                     */
    int32_t max_batch;      /* sequences decoded together, <= 64                       */
    int32_t weight_dtype;   /* expert weights; the router is fp32 for STMOE_F32, else bf16 */
    int64_t cache_slots;    /* 0: all experts resident in HBM; else number of HBM expert
                               slots (>= max_batch*top_k), experts live in pinned host memory */
    int32_t profile_tokens; /* P of Algorithm 1: decode steps spent counting co-activations */
    int32_t predictor_mode;
    int32_t flags;
    int32_t prefetch_limit; /* max prefetch copies issued per layer step, 0 = no limit */
    float rms_eps;
    float residual_scale;   /* r in h' = h + r * MoE(RMSNorm(h))                       */
} stmoe_config_t;

typedef struct {
    int64_t decode_steps;     /* completed decode steps (one per pass over all layers)   */
    int64_t runtime_steps;    /* (layer, sequence) steps after profiling                  */
    int64_t routed;           /* experts routed in those steps                            */
    int64_t predicted;        /* experts predicted for those steps                        */
    int64_t hits;             /* routed experts that were in the predicted set            */
    int64_t near_ties;        /* sequences flagged STMOE_TOKEN_NEAR_TIE (all steps)       */
    int64_t cache_hits;       /* routed experts found in an HBM slot                      */
    int64_t cache_misses;     /* routed experts demand-loaded from the host store         */
    int64_t prefetch_issued;
    int64_t prefetch_useful;  /* prefetched experts used before eviction                  */
    int64_t prefetch_wasted;  /* prefetched experts evicted unused                        */
    int64_t prefetch_dropped; /* predictions not prefetched (no slot / over the limit)    */
    int64_t prefetch_resident;/* predictions already in a slot                            */
    int64_t h2d_bytes_demand;
    int64_t h2d_bytes_prefetch;
    double transfer_ms;       /* device time of all host->HBM expert copies               */
    double exposed_ms;        /* time the compute stream waited for such copies           */
    int64_t kernel_launches;  /* kernels launched by layer steps since creation           */
    int64_t timed_ffn_launches; /* layer steps whose FFN kernels were timed (see below)   */
    double gate_up_ms;        /* summed device time of the timed gate/up kernels          */
    double down_ms;           /* summed device time of the timed down kernels             */
    double router_ms;         /* summed device time of the timed router kernels           */
    int64_t recovered_faults; /* slot-table inconsistencies found at verification and repaired by a demand load */
} stmoe_stats_t;

/* Create a stack for the current CUDA device.  Allocates weight storage (HBM
 * for resident stacks, pinned host memory plus cache_slots HBM slots
 * otherwise), predictor tables (Co, CCT per adjacent layer pair, HT per layer
 * and sequence) and scratch.  *out is NULL on failure. */
int stmoe_create(const stmoe_config_t *cfg, stmoe_t **out);
int stmoe_destroy(stmoe_t *s);
const char *stmoe_strerror(int code);

/* Router matrix of one layer, [E][H] row-major (w_j of Section 2 in row j), fp32 for
 * STMOE_F32 stacks and bf16 otherwise.  w: host or device.  Synchronous. */
int stmoe_load_router(stmoe_t *s, int layer, const void *w);

/* Weights of experts first_expert .. first_expert+count-1 of one layer (is_shared: the
 * always-on experts).  gate, up: [count][I][H]; down: [count][H][I]; row-major in
 * weight_dtype.  scales (fp8 only, else NULL): [count][2I+H] bf16 = gate rows, up rows,
 * down rows.  STMOE_MX4: gate, up [count][I][H/2] and down [count][H][I/2] bytes of codes, scales
 * [count][3*H*I/32] bytes = the scale bytes of gate, of up, of down.  Pointers may be host or device.  Synchronous: the sources are read during the call
 * (a device source must be complete: synchronise the stream that produced it first). */
int stmoe_load_experts(stmoe_t *s, int layer, int first_expert, int count, const void *gate,
                       const void *up, const void *down, const void *scales, int is_shared);

/* One layer step for `batch` sequences.  Layers must be called in order 0..L-1 for each
 * decode step (else STMOE_ERR_STATE).
 *   h_in, h_out    device fp32 [batch][H]; may alias
 *   routed_ids     device int32 [batch][K], ascending ids            (NULL: not returned)
 *   routed_w       device fp32  [batch][K], gate weights              (NULL: not returned)
 *   predicted_ids  device int32 [batch][max_pred], ascending ids of the prefetch set for
 *                  layer+1 (after the last layer: layer 0 of the next decode step), padded
 *                  with -1; max_pred = stmoe_max_predicted()          (NULL: not returned)
 *   n_predicted    device int32 [batch]                              (NULL: not returned)
 *   flags          device uint32 [batch], STMOE_TOKEN_*               (NULL: not returned)
 * Resident stacks: the call only enqueues work on cuda_stream.  Stacks with cache_slots > 0:
 * the call waits on the host (bounded, STMOE_ERR_TIMEOUT) for this layer's routing, issues
 * demand and prefetch copies on the library's copy stream and fences them with events.
 * Prediction never changes routing or output (Section 4.3.4).
 * A step that returns an error other than STMOE_ERR_BAD_ARG / STMOE_ERR_STATE may already have
 * applied Algorithm 3 and the history overwrite for this layer; the stack is then marked failed
 * and every further step returns STMOE_ERR_STATE until stmoe_import_state restores a consistent
 * image (retrying the layer would apply the update twice). */
int stmoe_decode_step(stmoe_t *s, int layer, int batch, const float *h_in, float *h_out,
                      int32_t *routed_ids, float *routed_w, int32_t *predicted_ids,
                      int32_t *n_predicted, uint32_t *flags, void *cuda_stream);

/* All layers of one decode step: h_out = stack(h_in).  The per-layer outputs are as in
 * stmoe_decode_step with a leading [n_layers] dimension; any of them may be NULL.  Resident
 * stacks run the whole step as one persistent cooperative kernel (one CTA per SM, bounded grid
 * barriers between the phases of a layer; a barrier that times out makes stmoe_stats return
 * STMOE_ERR_TIMEOUT). */
int stmoe_decode_token(stmoe_t *s, int batch, const float *h_in, float *h_out,
                       int32_t *routed_ids, float *routed_w, int32_t *predicted_ids,
                       int32_t *n_predicted, uint32_t *flags, void *cuda_stream);

/* stmoe_decode_token for callers whose buffers are in HOST memory (pinned for the copies to run
 * at link speed; pageable works): copies h_in_host [batch][H] to the device, runs the decode step,
 * copies h_out_host [batch][H] and, if not NULL, routed_ids_host [n_layers][batch][K] back, and
 * waits for cuda_stream.  The device staging buffers belong to the stack (allocated at the first
 * call).  Errors as stmoe_decode_token; a failed copy or wait returns STMOE_ERR_CUDA. */
int stmoe_decode_token_host(stmoe_t *s, int batch, const float *h_in_host, float *h_out_host,
                            int32_t *routed_ids_host, void *cuda_stream);

int stmoe_max_predicted(const stmoe_t *s); /* min(E, K*K+K) */

/* on != 0: bracket the expert-FFN kernels of every following layer step with CUDA events
 * on the caller's stream (the router kernel too); their summed durations appear in stmoe_stats.
 * Off by default. */
int stmoe_set_kernel_timing(stmoe_t *s, int on);

/* Offloaded stacks: prefetch only queue entries whose score (Eq. 1, summed over the batch's
 * sequences) is at least min_score; entries below it are ignored as if they had not been
 * predicted (they are neither copied nor protected from eviction).  0 (default) prefetches the
 * whole predicted set, the paper's policy; higher values trade recall for fewer wasted copies.
 * Between decode steps; routing, outputs and predictor tables are unaffected. */
int stmoe_set_prefetch_min_score(stmoe_t *s, int min_score);

/* Set threshold of Algorithm 2: an expert is predicted when its score (sum of the confidences of
 * its stored candidates in the routed experts' rows, plus binary 10 if it is in the history table,
 * Eq. 1) reaches `threshold`.  Section 4.2 fixes it at binary 10 = 2 (default); 1 predicts every
 * stored candidate of non-zero confidence, larger values trade recall for precision (threshold
 * sweep of the ablation).  Tables evolve identically for every value.  Between decode steps. */
int stmoe_set_predict_threshold(stmoe_t *s, int threshold);

/* Replacement rule of Algorithm 3.  When a stored candidate misses at confidence 0 the listing
 * replaces it by a routed expert the row does not hold and leaves open which.  live_counts = 0 (default): the
 * lowest such id; the co-activation counts stay as profiling (Algorithm 1) left them.
 * live_counts = 1: counting goes on at run time (for every sequence, in index order, the K x K
 * pairs of (previous layer's routing, this layer's routing) are counted right before that
 * sequence's table update) and the new candidate is the routed expert with the largest count in
 * the row, equal counts -> the lower id.  The exported state then carries the live counts.
 * Between decode steps. */
int stmoe_set_replacement_rule(stmoe_t *s, int live_counts);

/* Replacement policy of the HBM slot cache (the paper stages predicted experts and fetches
 * misses at once, Section 4.3.4, and names no replacement policy).  Victims are taken in this
 * order among the slots not needed by the step in progress: empty slots; the expert with the
 * fewest uses in its history window (history_window bits per expert: routed at its layer's turn i
 * decode steps ago; 0: not counted); with by_turn, the expert whose layer's next turn in the
 * cyclic layer walk is furthest away; the least recently used; the lowest slot.  0, 0 is plain
 * LRU.  prefetch_floor >= 0: a prefetch only takes a slot whose expert has at most that many uses
 * in its window (0: only slots without recent use), otherwise the prediction is dropped; -1: no
 * such test (every predicted expert is prefetched, the paper's behaviour).  A floor needs a
 * history window (history_window > 0), else STMOE_ERR_BAD_ARG.
 * Default: LRU when a decode step cannot touch more experts than there are slots
 * (n_layers * min(n_experts, max_batch * top_k) <= cache_slots), else a 16-step window with
 * by_turn (LRU has hit rate zero on a cyclic walk that is larger than the cache); floor -1.
 * Only before the first decode step of an offloaded stack. */
int stmoe_set_cache_policy(stmoe_t *s, int history_window, int by_turn, int prefetch_floor);

/* Bandwidth sensitivity (the paper's off-chip bandwidth axis): expert copies host -> HBM are issued
 * in chunks of chunk_bytes with gap_us of idle time on the copy stream after each, which lowers
 * the effective link speed to chunk_bytes / (chunk_bytes / link + gap_us).  0, 0: whole images at
 * full speed (default).  Offloaded stacks, between decode steps. */
int stmoe_set_copy_throttle(stmoe_t *s, int64_t chunk_bytes, int gap_us);

/* Host-side fault injection for tests (nothing here faults or hangs the GPU).  Offloaded stacks,
 * between decode steps:
 *   DROP_PREFETCH n   the next n prefetch requests are lost (counted as dropped); the experts
 *                     are demand-loaded if routed
 *   FAIL_COPY n       the n-th next expert copy reports failure: the layer step returns
 *                     STMOE_ERR_CUDA and the stack is failed until stmoe_import_state
 *   DELAY_COPY_US us  the next expert copy is preceded by us microseconds (<= 10000) of idle
 *                     time on the copy stream; the consuming kernels wait on the slot's event
 *   CORRUPT_TAG slot  the slot's tag is overwritten: verification finds the mismatch, reloads
 *                     the expert and counts it in recovered_faults
 *   HOST_WAIT_MS ms   limit of the host's wait for a layer's routing (default 20000); when it
 *                     runs out the step returns STMOE_ERR_TIMEOUT
 * Any stack: POLL_LIMIT n = polls after which a grid-barrier wait of the single-sequence
 * persistent kernel gives up (default 2^22).
 * No stack (s NULL): MX4_POLL_LIMIT n = polls, of about 4 us each, after which a wait inside the MX4
 * product and FFN kernels and the adapters' tile kernels gives up, in every launch of the process from then on (default and most 2^22;
 * 0: at once; a captured graph keeps the limit it was captured with). */
#define STMOE_HOOK_DROP_PREFETCH 1
#define STMOE_HOOK_FAIL_COPY 2
#define STMOE_HOOK_DELAY_COPY_US 3
#define STMOE_HOOK_CORRUPT_TAG 4
#define STMOE_HOOK_HOST_WAIT_MS 5
#define STMOE_HOOK_POLL_LIMIT 6
#define STMOE_HOOK_MX4_POLL_LIMIT 7
int stmoe_test_hook(stmoe_t *s, int what, int64_t value);

/* Runs the bounded waits of the persistent kernels on barriers that nobody completes, with a poll
 * limit of a few thousand: which = 0 the grid barrier of the three-phase kernel, 1 the grid barrier
 * of the single-sequence kernel, 2 an mbarrier wait of the tensor-core kernels, 3 the mbarrier wait
 * of the single-sequence kernel's copy ring, 4 the wait of the tensor-core kernel's down-projection
 * loads for an entry's gate/up tiles.  Each wait gives up, the stack's error word is set
 * and stmoe_stats returns STMOE_ERR_TIMEOUT from then on (destroy the stack afterwards); the
 * kernel itself ends normally.  Asynchronous on cuda_stream. */
int stmoe_selftest_bounded_wait(stmoe_t *s, int which, int poll_limit, void *cuda_stream);

/* On-chip staging in the single-sequence persistent decode step of resident stacks: the paper's
 * idea of fetching experts before they are needed (Sections 4.1, 4.3.4), one memory level down.
 * Weight rows are hinted into L2 while HBM would otherwise idle at a grid barrier; results never
 * depend on it (bit-identical on or off).
 *   known_bytes      weights whose addresses are already known: the down projection of the routed
 *                    experts (known since the top-K) ahead of the barrier in front of it, at most
 *                    known_bytes per expert and SM, and the next layer's shared experts ahead of
 *                    its router.  0 = off (default: measured neutral to slower, the phases
 *                    it overlaps with are not idle enough).
 *   predicted_bytes  per layer, summed over the GPU: leading gate/up rows of the experts in
 *                    Algorithm 2's prefetch set for the next layer, hinted ahead of that layer's
 *                    router and top-K.  0 = off (default).
 * Between decode steps. */
int stmoe_set_onchip_staging(stmoe_t *s, int64_t known_bytes, int64_t predicted_bytes);

/* Smallest batch that takes the tensor-core FFN path (see STMOE_FLAG_NO_DENSE); between decode
 * steps.  min_batch < 2 or a stack without that path: STMOE_ERR_BAD_ARG. */
int stmoe_set_dense_min_batch(stmoe_t *s, int min_batch);

/* Counters and timings; synchronises the device. */
int stmoe_stats(stmoe_t *s, stmoe_stats_t *out);

/* Predictor tables as a canonical image: 8 int32 {magic 0x53544D50, version 1, L, E, K, B, P,
 * built}, int64 decode steps, Co u32 [L-1][E][E], CCT ids u8 [L-1][E][K], CCT confidences u8
 * [L-1][E][K], HT i16 [B][L][K] (-1 = empty).  buf == NULL: only *bytes is set.  Host buffer.
 * Synchronises the device.  import restores such an image between decode steps. */
int stmoe_export_state(stmoe_t *s, void *buf, size_t *bytes);
int stmoe_import_state(stmoe_t *s, const void *buf, size_t bytes);

/* tags[slot] = layer*E+expert held by each HBM slot, -1 if empty (host int32 [cache_slots]). */
int stmoe_export_cache_tags(stmoe_t *s, int32_t *tags, int64_t n);

/* ---- single kernels behind the step, exposed for testing and reuse -------------------- */

/* Gating network of Section 2 for `batch` tokens: x = RMSNorm(h), z = W_r x, s = softmax(z),
 * top-K by logit (ties: lower id), ids ascending, w = s[ids].  All pointers device.
 * wr_dtype: STMOE_F32 or STMOE_BF16.  logits: fp32 [batch*E + batch]; receives the logits
 * [batch][E] followed by the per-sequence factors 1/sqrt(mean(h^2)+eps). */
int stmoe_router_topk(const float *h, const void *w_router, int wr_dtype, int batch, int n_experts,
                      int hidden, int top_k, float rms_eps, int renorm, float *logits,
                      int32_t *ids, float *w, uint32_t *flags, void *cuda_stream);

/* Predictor only (Algorithms 1-3 on the stack's tables) driven by given routing:
 * routed_ids device int32 [batch][K] ascending.  Same ordering rules and outputs as
 * stmoe_decode_step; used to replay routing traces. */
int stmoe_predictor_step(stmoe_t *s, int layer, int batch, const int32_t *routed_ids,
                         int32_t *predicted_ids, int32_t *n_predicted, void *cuda_stream);

/* Routed SwiGLU expert FFN, weighted sum and residual for given routing:
 *   h_out[b] = h[b] + r * sum_k w[b][k] * W_d^e ( silu(W_g^e x_b) * (W_u^e x_b) ),
 *   x_b = h[b] * inv_rms[b],  e = ids[b][k].
 * experts: device array of n_experts expert images, each `stmoe_expert_image_bytes` long:
 * gate [I][H], up [I][H], down [H][I], then (fp8) bf16 scales [2I+H].
 * scratch: device, stmoe_moe_ffn_scratch_bytes(batch, top_k, hidden, inter) bytes,
 * 256-byte aligned; contents need not be initialised.
 *
 * STMOE_MX4: an image is the codes of gate [I][H/2], up [I][H/2], down [H][I/2] bytes, then the scale
 * bytes of gate, up, down; hidden and inter multiples of 32, experts 16-byte aligned, scratch
 * stmoe_mx4_ffn_scratch_bytes(batch, top_k, hidden, inter) bytes, which also serve every smaller batch
 * and top_k (a call of exactly that size may take less).  The weights go to the tensor cores
 * as stored; an activation is held as a sum of eight 4-bit values that leaves less than 2^-22 of the
 * largest magnitude among its 32 neighbours (or 2^-128, where that is more: 4-bit scales end at 2^-127), and sums are fp32, so results have the precision of fp32
 * activations.  A non-finite activation makes the 32 neighbours, and what depends on them, NaN; pairs
 * whose id is outside [0, n_experts) add nothing.  Should a bounded wait inside a kernel run out, the
 * outputs that depend on it are NaN. */
size_t stmoe_expert_image_bytes(int hidden, int inter, int weight_dtype);
size_t stmoe_moe_ffn_scratch_bytes(int batch, int top_k, int hidden, int inter);
size_t stmoe_mx4_ffn_scratch_bytes(int batch, int top_k, int hidden, int inter);
int stmoe_moe_ffn(const float *h, const float *inv_rms, const int32_t *ids, const float *w,
                  const void *experts, int weight_dtype, int batch, int n_experts, int top_k,
                  int hidden, int inter, float residual_scale, float *h_out, void *scratch,
                  size_t scratch_bytes, void *cuda_stream);

/* stmoe_moe_ffn without a scratch argument and without any allocation (the paper has no
 * counterpart; this serves hosts, not the method).  For callers that must not allocate device
 * memory once they are running: serving loops where cudaMalloc could stall the device or fail
 * because a framework already owns all of HBM, and plug-in hosts that forbid allocator calls.
 * The work list, activations and partial sums live in an 8 MiB area built into the library
 * image; each GPU that loads the library holds those 8 MiB until the process exits.
 *   - Same arguments, layout and results as stmoe_moe_ffn; inputs and outputs stay with the
 *     caller.  Calls no cudaMalloc/cudaFree or other allocating routine.
 *   - Returns STMOE_ERR_TOO_LARGE when stmoe_moe_ffn_scratch_bytes(batch, top_k, hidden, inter)
 *     (STMOE_MX4: what a call of exactly that size takes) exceeds 8 MiB (for example batch 64, top_k 8, hidden 4096, inter 14336).
 *   - The first call on each device looks up the area's device address (with that device
 *     current); make that first call before starting any stream capture, and from one host
 *     thread (later calls may come from any thread).
 *   - Arguments out of range are STMOE_ERR_BAD_ARG, as in stmoe_moe_ffn; only a well-formed
 *     problem that does not fit is STMOE_ERR_TOO_LARGE.
 *   - All calls on a device share the one area, which keeps whatever the last call left; the
 *     call clears the counters that must start at zero itself.  Two calls whose kernels can
 *     overlap on the GPU (different streams, no ordering between them) race on it: order
 *     them, or use stmoe_moe_ffn with separate scratch buffers. */
int stmoe_moe_ffn_static(const float *h, const float *inv_rms, const int32_t *ids, const float *w,
                         const void *experts, int weight_dtype, int batch, int n_experts, int top_k,
                         int hidden, int inter, float residual_scale, float *h_out, void *cuda_stream);

/* One expert's SwiGLU FFN (Section 2: the expert network of a routed token) for m tokens that
 * share the expert, as bf16 tensor-core GEMMs (tcgen05.mma, accumulators in tensor memory):
 *   y[t] = W_d ( bf16( silu(W_g x_t) * (W_u x_t) ) ),  x_t = bf16( h[t] * inv_rms[t] ),
 * products exact, sums in fp32.  This is the regime where the per-expert token count makes the
 * FFN a real dense contraction; the decode step itself streams weights through the CUDA cores.
 *   h        device fp32 [m][hidden]; inv_rms device fp32 [m] or NULL (= 1).
 *   image    device, one STMOE_BF16 expert image (gate [I][H], up [I][H], down [H][I]).
 *   y        device fp32 [m][hidden], overwritten.
 *   flags    device uint32, caller-zeroed; set to 1 when a bounded wait inside a kernel ran out
 *            (y is then undefined).
 *   scratch  device, stmoe_expert_ffn_dense_scratch_bytes(m, hidden, inter) bytes, 256-byte
 *            aligned, contents need not be initialised.
 * m in 1..64; hidden and inter multiples of 64; else STMOE_ERR_BAD_ARG.  Asynchronous on
 * cuda_stream. */
size_t stmoe_expert_ffn_dense_scratch_bytes(int m, int hidden, int inter);
int stmoe_expert_ffn_dense(const float *h, const float *inv_rms, const void *image, int m, int hidden,
                           int inter, float *y, uint32_t *flags, void *scratch, size_t scratch_bytes,
                           void *cuda_stream);

/* ---- microscaled 4-bit floating point (MX4) ------------------------------------------------
 *
 * A row of `cols` elements is cut into blocks of 32 (nb = ceil(cols / 32), the last one filled up
 * with zeros).  A block is 16 bytes of e2m1 codes, two to a byte, the even element in the low
 * half (values 0, .5, 1, 1.5, 2, 3, 4, 6; bit 3 of a code is the sign), and one e8m0 scale byte
 * worth 2^(byte-127); byte 255 means that the block is NaN.  Codes are [rows][nb*16] bytes,
 * scales [rows][nb] bytes; row strides are free. */

/* x [rows][cols] -> codes, scales.  byte = clamp(floor(log2 amax) - 2 + 127, 0, 254), amax the block's
 * largest magnitude (0 for a block of zeros, 255 for a block that holds a NaN or an infinity);
 * code = x / 2^(byte-127) to the nearest value, ties to the even code, magnitudes above 6 to 6.
 *   dtype: STMOE_F32, STMOE_BF16 or STMOE_F16.  x_stride in elements, >= cols; code_stride (a
 *   multiple of 4, codes 4-byte aligned) and scale_stride in bytes.  rows may be 0.  All pointers
 *   device; asynchronous on cuda_stream.  16-byte aligned rows of x are read 16 bytes at a time,
 *   others element by element. */
int stmoe_mx4_quantize(const void *x, int dtype, int64_t rows, int64_t cols, int64_t x_stride, uint8_t *codes,
                       int64_t code_stride, uint8_t *scales, int64_t scale_stride, void *cuda_stream);
/* The reverse: x [rows][cols] = value(code) * 2^(byte-127), rounded once to dtype (exact for fp32 and
 * bf16 unless it overflows).  Elements of x behind column `cols` stay as they were. */
int stmoe_mx4_dequantize(const uint8_t *codes, int64_t code_stride, const uint8_t *scales, int64_t scale_stride, int64_t rows,
                         int64_t cols, void *x, int dtype, int64_t x_stride, void *cuda_stream);

/* out[t][i] = sum_k a[t][k] * b_g(t)[i][k], both operands MX4, on the tensor cores' block-scaled
 * 4-bit form: products exact, sums fp32, one rounding to out_dtype.
 *   a        [m] rows (tokens), sorted by group; k_blocks scale blocks each
 *   b        [n_groups][n] rows of k_blocks blocks (the experts' matrices, one after the other)
 *   counts   device int32 [n_groups]: rows of a that belong to each group, in order (the counts of
 *            stmoe_router_balance); rows of a behind their sum have no group, and their rows of out stay
 *            as they were.  Counts below 0 read as 0, and counts that lead past m are cut.
 *            NULL: one group (n_groups = 1) with all m rows.
 *   out      [m][n] in out_dtype (STMOE_F32, STMOE_BF16, STMOE_F16), out_stride in elements
 *   flags    device uint32, caller-zeroed, or NULL; set to 1 when a bounded wait inside the kernel ran
 *            out (the affected outputs are then NaN)
 * Codes 16-byte aligned with strides that are multiples of 16; scale strides are free (rows on
 * 8-byte boundaries are read fastest).  The part of a row's last block behind its end has to hold
 * zero codes, as stmoe_mx4_quantize writes them.  A block with scale 255 makes every sum it enters
 * NaN.  n <= 2^24, n_groups <= 256, n_groups * n < 2^31; m may be 0.  The same call gives the same
 * bits every time.  No workspace; asynchronous on cuda_stream. */
int stmoe_mx4_matmul(const uint8_t *a_codes, int64_t a_code_stride, const uint8_t *a_scales, int64_t a_scale_stride, int64_t m,
                     const uint8_t *b_codes, int64_t b_code_stride, const uint8_t *b_scales, int64_t b_scale_stride,
                     int n_groups, int n, int k_blocks, const int32_t *counts, void *out, int out_dtype,
                     int64_t out_stride, uint32_t *flags, void *cuda_stream);

/* ---- router statistics over many tokens ----------------------------------------------------- */

/* Balance loss, z loss and per-expert counts of a router (the gating network of Section 2):
 *   p_t = softmax(logits_t), lse_t = log sum exp logits_t, over the n rows that count;
 *   counts[e] = how often e stands in ids of those rows;  f_e = counts[e] / (n top_k);
 *   loss[0] = n_experts * sum_e f_e * (1/n) sum_t p_te;   loss[1] = (1/n) sum_t lse_t^2.
 * A row does not count where its mask byte is 0 (it may then hold anything, NaN included) or where
 * all its logits are -infinity; a row filled with any finite value counts, with uniform p.  A NaN or
 * +infinity in a row that counts makes both losses and the row's gradient NaN.  With n = 0 everything is 0.
 *   logits   [tokens][n_experts] in dtype (STMOE_F32, STMOE_BF16, STMOE_F16), stride in elements
 *   ids      int32 [tokens][top_k]; entries outside [0, n_experts) (-1 for a dropped choice) are not
 *            counted, an expert that stands twice in a row counts twice
 *   mask     uint8 [tokens] or NULL
 *   loss     fp32 [2], counts int32 [n_experts], rows int32 [1] (= n): written
 *   scratch  stmoe_router_balance_scratch_bytes(tokens, n_experts) bytes (0 for short batches: NULL is
 *            fine), 4-byte aligned, contents free; calls that can overlap need scratch of their own
 * All pointers device.  n_experts <= 256, top_k <= n_experts, tokens * top_k < 2^31; tokens may be 0.  The same call
 * gives the same bits every time.  Asynchronous on cuda_stream. */
size_t stmoe_router_balance_scratch_bytes(int64_t tokens, int n_experts);
int stmoe_router_balance(const void *logits, int dtype, int64_t stride, const int32_t *ids, const uint8_t *mask, int64_t tokens,
                         int n_experts, int top_k, float *loss, int32_t *counts, int32_t *rows, void *scratch,
                         size_t scratch_bytes, void *cuda_stream);
/* Gradient of grad_loss[0] * loss[0] + grad_loss[1] * loss[1] with respect to the logits (counts held
 * constant), from the forward call's counts and rows:
 *   grad_logits[t][e] = g0 E/n p_te (f_e - sum_j f_j p_tj) + g1 2/n lse_t p_te,
 * 0 in rows that do not count.  grad_loss: device fp32 [2].  grad_logits: dtype as the logits,
 * [tokens][n_experts], every element written; the two may not overlap. */
int stmoe_router_balance_backward(const void *logits, int dtype, int64_t stride, const uint8_t *mask, int64_t tokens,
                                  int n_experts, int top_k, const int32_t *counts, const int32_t *rows, const float *grad_loss,
                                  void *grad_logits, int64_t grad_stride, void *cuda_stream);

/* ---- choice of experts for many tokens ---------------------------------------------------------- */

#define STMOE_SELECT_SIGMOID 1 /* scores are sigmoids of the logits (off: their softmax)    */
#define STMOE_SELECT_RENORM 2  /* weights are divided by the sum of the chosen scores       */

/* The gating network's choice from given logits z [tokens][n_experts] (stmoe_router_topk makes them for a decode
 * step), for routers beyond the plain softmax of Section 2:
 *   s = softmax(z) or sigmoid(z);  v = s + bias;  groups of n_experts / n_groups neighbouring experts are ranked
 *   by the sum of their group_best (1 or 2) largest v and the best top_groups stay;  ids = the top_k largest v in
 *   them, ascending;  w = scale * s[ids], divided by the sum of s[ids] with STMOE_SELECT_RENORM.
 * Equal values: the lower index, of groups too; values are compared as the formula's in 64 bits, so the choice
 * does not depend on their rounding to 32.  Where the order of the scores is that of the logits (bias NULL, and groups, if any have to go,
 * ranked by their best one) the logits are compared, which differ also where scores are equal in 64 bits: sigmoids of 40 and 50, a softmax's
 * values 800 below its largest.  With a bias, be it zeros, such scores are equal and the lower index is chosen.
 * A logit or bias of -infinity, or a NaN, is never chosen and counts as -infinity in its group's sum; a row with fewer than top_k left has id -1 and weight 0 behind the last.  So has a row whose mask byte is 0, which may hold
 * anything.  A NaN in a row that counts (softmax: +infinity too) makes its weights NaN.
 *   logits  STMOE_F32, STMOE_BF16 or STMOE_F16, stride in elements;  bias fp32 [n_experts] or NULL;  mask uint8 [tokens] or NULL
 *   ids     int32 [tokens][top_k], w fp32 [tokens][top_k]: written
 * n_experts <= 256 and a multiple of n_groups <= 32, top_k <= 32, tokens * top_k < 2^31; tokens may be 0.  Asynchronous on cuda_stream. */
int stmoe_router_select(const void *logits, int dtype, int64_t stride, const float *bias, const uint8_t *mask, int64_t tokens, int n_experts,
                        int top_k, int n_groups, int top_groups, int group_best, int flags, float scale, int32_t *ids, float *w, void *cuda_stream);
/* Gradient of sum grad_w . w with respect to the logits (the choice held constant), from the forward call's ids and w, flags and
 * scale: 0 for experts that were not chosen, except under a softmax without STMOE_SELECT_RENORM.  Rows without a choice have zero
 * gradient, rows with NaN weights NaN.  grad_w: fp32 [tokens][top_k], not read where the id is -1.  grad_logits: dtype as the logits,
 * every element written; the two may not overlap. */
int stmoe_router_select_backward(const void *logits, int dtype, int64_t stride, int64_t tokens, int n_experts, int top_k, int flags, float scale,
                                 const int32_t *ids, const float *w, const float *grad_w, void *grad_logits, int64_t grad_stride, void *cuda_stream);

/* ---- rows grouped by expert, there and back --------------------------------------------------- */

/* Grouping of the pairs (t, k) of ids [rows][top_k] by id, in 0 .. n_groups - 1 (others have no group):
 *   counts [n_groups], starts [n_groups + 1]   pairs of each group, and where it begins (last: pairs in groups)
 *   order  [rows * top_k]   the pair t * top_k + k at each slot: groups one after the other, pairs of a group in their order,
 *                           pairs without a group behind the last
 *   slots  [rows][top_k]    slot of each pair, -1 without a group
 * All int32, device.  The counts are what stmoe_mx4_matmul takes, the grouping of rows by adapter (top_k 1) what stmoe_lora takes.
 *   scratch  stmoe_group_rows_scratch_bytes(rows, top_k, n_groups) bytes (0 for few pairs: NULL is fine), 4-byte
 *            aligned, contents free; calls that can overlap need scratch of their own
 * n_groups <= 1024, rows * top_k <= 2^30; rows may be 0.  Asynchronous on cuda_stream. */
size_t stmoe_group_rows_scratch_bytes(int64_t rows, int top_k, int n_groups);
int stmoe_group_rows(const int32_t *ids, int64_t rows, int top_k, int n_groups, int32_t *counts, int32_t *starts, int32_t *order,
                     int32_t *slots, void *scratch, size_t scratch_bytes, void *cuda_stream);

/* out[slots[t][k]] = x[t], rows of row_bytes bytes (of any type; strides in bytes).  Slots outside [0, out_rows) are left out.
 *   n_rows  int32 [1]: rows of out from there to rows * top_k become 0 (starts[n_groups] of the grouping); NULL: they stay as they were
 * x and out may not overlap.  Asynchronous on cuda_stream. */
int stmoe_dispatch_rows(const void *x, int64_t row_bytes, int64_t x_stride, int64_t rows, int top_k, const int32_t *slots, const int32_t *n_rows,
                        void *out, int64_t out_rows, int64_t out_stride, void *cuda_stream);

/* out[t] = residual[t] + scale * sum_k w[t][k] y[slots[t][k]], summed in fp32 in the order of k and rounded once.
 *   y        [y_rows][cols] in y_dtype (STMOE_F32, STMOE_BF16, STMOE_F16); slots outside [0, y_rows) add nothing, whatever their weight
 *   w        fp32 [tokens][top_k], or NULL: 1
 *   residual, out  [tokens][cols] in out_dtype (y's or STMOE_F32); residual may be NULL (0) or out itself; nothing else may overlap
 * Strides in elements.  With w NULL and scale 1 it is the gradient of stmoe_dispatch_rows.  Asynchronous on cuda_stream. */
int stmoe_combine_rows(const void *y, int y_dtype, int64_t y_stride, int64_t y_rows, const int32_t *slots, const float *w, const void *residual,
                       int64_t residual_stride, float scale, int64_t tokens, int top_k, int64_t cols, void *out, int out_dtype,
                       int64_t out_stride, void *cuda_stream);
/* Its gradients: grad_y[slots[t][k]] = scale * w[t][k] * grad[t] and grad_w[t][k] = scale * <grad[t], y[slots[t][k]]> (0 without a slot;
 * grad_w NULL: not wanted); the residual's gradient is grad itself.  grad [tokens][cols] in grad_dtype (y's or STMOE_F32), grad_y in y's type.
 *   n_rows  as in stmoe_dispatch_rows, for the rows of grad_y.  grad_y may overlap neither y nor grad. */
int stmoe_combine_rows_backward(const void *grad, int grad_dtype, int64_t grad_stride, const void *y, int y_dtype, int64_t y_stride, int64_t y_rows,
                                const int32_t *slots, const float *w, float scale, int64_t tokens, int top_k, int64_t cols, const int32_t *n_rows,
                                void *grad_y, int64_t grad_y_stride, float *grad_w, void *cuda_stream);

/* ---- low-rank adapters of many requests beside a shared projection ----------------------------- */

/* out[t] = base[t] + alpha * scale[g] * (x[t] A_g^T) B_g^T, g = ids[t]; rows whose id is outside [0, n_adapters): out = base.
 *   x      [tokens][inner] in dtype (STMOE_BF16 or STMOE_F16); A [n_adapters][rank][inner], B [n_adapters][outer][rank] in the same type
 *   ids    int32 [tokens];  order, counts, starts: what stmoe_group_rows makes of them (top_k 1, n_adapters groups)
 *   scale  fp32 [n_adapters], or NULL: 1
 *   base, out  [tokens][outer] in out_dtype (dtype or STMOE_F32); base may be NULL (0) or out itself; nothing else may overlap
 *   hidden fp32 [tokens][rank], or NULL: receives x A^T (0 for rows without an adapter), which the gradient of B needs
 *   scratch  stmoe_lora_scratch_bytes(...) bytes (which serve fewer tokens too), 16-byte aligned, contents free; calls that can overlap need scratch of their own
 * Strides in elements; a_group, b_group: from one adapter to the next.  Sums in fp32, one rounding of out; x A^T is kept to 2^-17 (out fp32:
 * 2^-24) of itself or, fp16, to 2^-38 of the largest of its row, whichever is more.  n_adapters <= 1024, rank <= 256, inner and outer <= 2^22; tokens may be 0 (or 1: a decode step).  The same call gives the same bits every
 * time.  16-byte aligned rows (rank a multiple of 8 for B) are read 16 bytes at a time, others element by element.  Should a bounded wait inside a kernel run out, the outputs that depend on it are NaN.  Asynchronous on cuda_stream. */
size_t stmoe_lora_scratch_bytes(int64_t tokens, int n_adapters, int rank, int inner, int outer);
int stmoe_lora(const void *x, int dtype, int64_t x_stride, int64_t tokens, const void *a, int64_t a_group, int64_t a_row, const void *b, int64_t b_group,
               int64_t b_row, int n_adapters, int rank, int inner, int outer, const int32_t *ids, const int32_t *order,
               const int32_t *counts, const int32_t *starts, const float *scale, float alpha, const void *base, int64_t base_stride, void *out, int out_dtype, int64_t out_stride, float *hidden, void *scratch,
               size_t scratch_bytes, void *cuda_stream);
/* Gradients for grad [tokens][outer] in dtype: grad_x [tokens][inner] = c u A with u = grad B (0 for rows without an adapter; the base's gradient
 * is grad itself), grad_a [n][rank][inner] = c sum_t u^T x, grad_b [n][outer][rank] = c sum_t grad^T hidden, c = alpha * scale[g]; contiguous, in dtype,
 * each rounded once, 0 for adapters without rows; grad_a and grad_b may be NULL.  u and hidden are kept to 2^-17 of themselves or, fp16, to 2^-38 of
 * the largest of their row (of all rows of their adapter for grad_a and grad_b), whichever is more.  tokens may be 0: grad_a and grad_b are cleared.
 * scale is held constant.  scratch: stmoe_lora_backward_scratch_bytes(...) bytes, 256-byte aligned.  grad_x may overlap neither grad nor x. */
size_t stmoe_lora_backward_scratch_bytes(int64_t tokens, int n_adapters, int rank, int inner, int outer);
int stmoe_lora_backward(const void *grad, int dtype, int64_t grad_stride, const void *x, int64_t x_stride, int64_t tokens, const void *a, int64_t a_group,
                        int64_t a_row, const void *b, int64_t b_group, int64_t b_row, int n_adapters, int rank, int inner, int outer,
                        const int32_t *ids, const int32_t *order, const int32_t *counts, const int32_t *starts, const float *scale, float alpha,
                        const float *hidden, void *grad_x, int64_t grad_x_stride, void *grad_a, void *grad_b, void *scratch, size_t scratch_bytes,
                        void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* STMOE_H */
