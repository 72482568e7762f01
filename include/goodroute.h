/*
 * libgoodroute: the batched routing math of GoodServe's predict-and-rectify
 * request router, for one AMD MI355X (gfx950).
 *
 * The three calls follow the paper's statement of the routing problem:
 *
 *   gr_build_status  the per-instance status that Eq. 2 (Sec. 3.1) needs (queuing
 *                    delay q_g, decode speed d_g) and the expected end-to-end
 *                    finish time of every request an instance already holds;
 *   gr_score_route   Alg. 1 ("Backend Selection Algorithm", Appendix) for a
 *                    batch of incoming requests: T(r,g) of Eq. 2 for every
 *                    (request, instance) pair, feasibility T <= D_r, the
 *                    just-enough choice of Sec. 3.4, the least-violation
 *                    fallback;
 *   gr_risk_scan     the periodic SLO-violation re-check of Sec. 3.4 over all
 *                    active requests, with a just-enough migration target for
 *                    every request found at risk.
 *
 * Time model.  Sec. 3.3 estimates q_g, p_g, d_g black-box; this library takes
 * them from an explicit model of a continuously batching instance of GPU
 * class c:  prefill costs delta_c seconds per prompt token, and one decode
 * step of a batch of B requests whose context lengths sum to C costs
 * alpha_c + beta_c*B + gamma_c*C seconds.  Queued requests are prefilled back
 * to back before decoding resumes; every step emits one token per batch
 * member.  "Now" is time 0 of every call.
 *
 * Conventions.  Every function returns GR_OK (0) or a negative GR_ERR_* code;
 * nothing throws or aborts.  Pointers marked DEVICE are device memory owned by
 * the caller (readable/writable by kernels on the current device); pointers
 * marked HOST are ordinary host memory read during the call.  Work is queued
 * on the given HIP stream (a hipStream_t passed as void*, NULL = default
 * stream) and the calls do not wait for it; outputs are valid once the stream
 * has been synchronised.  The handle owns its tables and workspace, sized at
 * gr_create; no call after gr_create allocates.  Calls on one handle must not
 * overlap.  Token counts are int32; times are seconds.
 *
 * The calls that take a stream only launch kernels on it (no copy, no memset,
 * no synchronisation), so a sequence of them can be recorded into a HIP graph
 * and replayed on the same buffers.  What the host decides at call time is
 * recorded with it: sizes, the blend weight and caps in force, and how a
 * batch is scored (gr_set_small_batch_pairs).  Direct calls on the same handle
 * before, between and after replays work on the tables as the last call or
 * replay on the device left them.  gr_create, gr_destroy, the
 * gr_set_* calls, gr_profile_* and gr_device_status copy or synchronise and
 * are not for use inside a capture.
 *
 * Input contract for device data (not validated on the host): remaining and
 * predicted lengths in [1, max_len]; prompt >= 1; generated >= 0; entries per
 * instance <= max_entries_per_inst; CSR offsets non-decreasing, starting at 0.
 * Kernels stay in bounds when the contract is broken (lengths are clamped,
 * surplus entries dropped) and raise a sticky bit readable with
 * gr_device_status.  gr_risk_scan writes no finish time and no flag for running
 * entries that it drops or that no instance's offsets cover; a target is looked
 * for wherever out_flag then reads nonzero.
 */
#ifndef GOODROUTE_H
#define GOODROUTE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gr_fleet gr_fleet;

enum {
    GR_OK = 0,
    GR_ERR_INVALID_ARG = -1, /* NULL where a pointer is required, negative size, bad class id */
    GR_ERR_TOO_LARGE = -2,   /* a size exceeds what the handle was created for, or a hard limit */
    GR_ERR_HIP = -3,         /* a HIP runtime call failed */
    GR_ERR_NO_STATUS = -4,   /* gr_score_route before any gr_build_status / gr_risk_scan; a blend before gr_observe */
    GR_ERR_NOMEM = -5        /* host or device allocation failed in gr_create */
};

/* bits of gr_device_status */
enum {
    GR_DEV_LEN_CLAMPED = 1,   /* a length outside [0, max_len] was clamped */
    GR_DEV_ENTRIES_DROPPED = 2, /* an instance held more than max_entries_per_inst entries */
    GR_DEV_STALLED = 4         /* feedback routing gave up a wait inside the device after some two seconds (not expected to happen: all that
                                  it waits for is running).  The call had returned GR_OK; from some request on its outputs are
                                  what they were before, and the handle's tables and lists hold a part of what was routed: both
                                  are of no use until the next gr_build_status or gr_risk_scan. */
};

/*
 * Create a fleet handle on the current HIP device.
 *   n_inst, n_class           M instances of n_class GPU classes (n_class <= 64)
 *   delta, alpha, beta, gamma HOST, n_class doubles each, all >= 0: the model above
 *   inst_class                HOST, n_inst class ids in [0, n_class)
 *   max_entries_per_inst      upper bound of active + queued requests on one instance
 *   max_len                   upper bound of any remaining / predicted decode length
 *   max_requests              upper bound of n_req of one gr_score_route call
 * Hard limits: max_entries_per_inst <= 2048; max_len <= 32767.
 * Device memory held by the handle until gr_destroy, all of it allocated here: with
 * cap = max_entries_per_inst rounded up to 64, 128, .. 2048, M' = the instances of every class
 * rounded up to a multiple of 16 and added up, N = max(max_requests, n_inst * max_entries_per_inst) and
 * rows = min(max_len + 1, N) rounded up to a multiple of 256,
 *   18 * n_inst * cap bytes          instance tables and the lists of feedback routing,
 *   8 * n_inst * max_entries_per_inst bytes   per held request (its instance, a spare finish time),
 *   rows * (4 * M' + 4 * [M' / 16 rounded up to 16] + 128) bytes
 *                                    the per-(distinct length, instance) table of a scoring pass, its minima
 *                                    over runs, and the instances that can be least, reserved for the
 *                                    worst case whatever the batches turn out to be (295 MB for 4 096
 *                                    instances of 6 classes and max_len 16 384),
 *   8 * (max_len + 1) * [n_class rounded up to 2, 4, 8 or 16] bytes   the minima over classes, up to 16 classes (1 MB there),
 *   4 * rows * [M' / 16 rounded up to 16] bytes   the minima over runs once more (18 MB there), for max_requests of 131 072
 *                                    and more on fleets of up to 16 classes with M' of at least 1 024 and 64 * n_class,
 *   at most 64 MB, or 1 024 * n_inst bytes if that is more   rows of that table for out_T,
 *   (50 * cap + 1300) * n_inst bytes  feedback routing, up to 512 instances with cap of 128 and more: what they offer a chunk, sums
 *                                    behind the tables and of what is routed,
 *   0.4 MB                           selections of small batches on fleets of more than 4 096 instances,
 * plus a few arrays of n_inst, M' or max_len + 1 words.
 */
int gr_create(gr_fleet** out, int32_t n_inst, int32_t n_class,
              const double* delta, const double* alpha, const double* beta, const double* gamma,
              const int32_t* inst_class,
              int32_t max_entries_per_inst, int32_t max_len, int64_t max_requests);

/* Free the handle and its device memory (waits for the device first). NULL is allowed. */
int gr_destroy(gr_fleet* f);

/*
 * Step 1 (Eq. 2's per-instance terms; "expected finish time" of Sec. 3.4).
 * For every instance: q_g = delta * (sum of queued prompts); the requests it
 * holds are ordered by remaining length, which turns the step-by-step run of
 * its batch into a closed form; out come the finish time of every request,
 * d_g = duration of the instance's next decode step (alpha for an idle
 * instance), the capability rank used by Alg. 1's argmax d_g, and the
 * instance tables kept in the handle for gr_score_route.
 *
 *   act_off        DEVICE int32[n_inst+1]  CSR offsets of active requests by instance
 *   act_prompt     DEVICE int32[n_active]  prompt tokens
 *   act_gen        DEVICE int32[n_active]  tokens generated so far
 *   act_rem        DEVICE int32[n_active]  predicted remaining decode length
 *   q_off          DEVICE int32[n_inst+1]  CSR offsets of queued requests by instance
 *   q_prompt,q_len DEVICE int32[n_queued]  prompt tokens, predicted decode length
 *   n_active, n_queued                     array lengths (host values)
 *   out_act_finish DEVICE float[n_active]  expected finish time, same order as inputs
 *   out_q_finish   DEVICE float[n_queued]  may be NULL
 *   out_d          DEVICE double[n_inst]   may be NULL
 *   out_rank       DEVICE int32[n_inst]    may be NULL; 0 = largest d_g, ties by index
 */
int gr_build_status(gr_fleet* f,
                    const int32_t* act_off, const int32_t* act_prompt,
                    const int32_t* act_gen, const int32_t* act_rem, int64_t n_active,
                    const int32_t* q_off, const int32_t* q_prompt, const int32_t* q_len,
                    int64_t n_queued,
                    float* out_act_finish, float* out_q_finish,
                    double* out_d, int32_t* out_rank, void* hip_stream);

/*
 * Step 2 (Alg. 1 on a batch; every request is scored against the same
 * snapshot: the tables of the last gr_build_status / gr_risk_scan).
 * A request that goes to instance g waits q_g, prefills its ctx0 tokens
 * (no cached prefix), then decodes pred_len steps in g's batch:
 *   T(r,g) = q_g + delta*ctx0 + [time of g's next pred_len steps with r in the batch].
 * Feasible iff T <= budget.  Choice: the feasible instance with the largest
 * d_g (ties: lowest index); if none, the instance with the smallest T (ties:
 * lowest index).
 *
 *   n_req          number of requests (0 allowed)
 *   ctx0           DEVICE int32[n_req]  tokens to prefill (prompt; prompt+generated when migrating)
 *   pred_len       DEVICE int32[n_req]  predicted decode length
 *   budget         DEVICE float[n_req]  D_r, seconds from now
 *   exclude_inst   DEVICE int32[n_req]  instance a request may not go to, -1 none; may be NULL
 *   out_inst       DEVICE int32[n_req]  chosen instance (-1 if every instance is excluded)
 *   out_slack      DEVICE float[n_req]  budget - T(r, chosen)
 *   out_fallback   DEVICE uint8[n_req]  1 if no instance was feasible; may be NULL
 *   out_T          DEVICE float[n_req*n_inst], row-major; may be NULL. Every pair's
 *                  T, for checking; costs 4 bytes of traffic per pair.
 */
int gr_score_route(gr_fleet* f, int64_t n_req,
                   const int32_t* ctx0, const int32_t* pred_len, const float* budget,
                   const int32_t* exclude_inst,
                   int32_t* out_inst, float* out_slack, uint8_t* out_fallback,
                   float* out_T, void* hip_stream);

/*
 * gr_score_route for callers that want the same work queued whatever the batch: code under HIP
 * graph capture, tight serving loops.  Same inputs, outputs and answers as gr_score_route's
 * pair-by-pair pass (whatever gr_set_small_batch_pairs says; no out_T), for at most
 * GR_NOALLOC_MAX_REQUESTS requests per call; more is GR_ERR_TOO_LARGE.  (An infinite latency
 * always counts as one here: see gr_set_small_batch_pairs.)  The call queues one
 * kernel on the stream (two for fleets of more than 4 096 instances) and calls no hipMalloc,
 * hipFree, memset, copy or synchronisation.
 */
#define GR_NOALLOC_MAX_REQUESTS 4096
int gr_score_route_noalloc(gr_fleet* f, int64_t n_req,
                           const int32_t* ctx0, const int32_t* pred_len, const float* budget,
                           const int32_t* exclude_inst,
                           int32_t* out_inst, float* out_slack, uint8_t* out_fallback,
                           void* hip_stream);

/*
 * Step 2 with cached prefixes (Eq. 2's hit prefix token length H_{r,g};
 * Alg. 1's prefix-reuse lookup before T(r,g) is formed).  As gr_score_route,
 * but request r already has hit_len[k] of its ctx0 tokens cached on instance
 * hit_inst[k] for k = hit_off[r] .. hit_off[r+1]-1; those tokens are not
 * prefilled again (they still count as context while decoding):
 *   T(r,g) = q_g + delta*(ctx0 - H_{r,g}) + [decode time as in gr_score_route].
 * Pairs without an entry have H = 0.  An instance named more than once for a
 * request counts with its longest prefix; a prefix is cut to [0, ctx0].
 *
 *   hit_off    DEVICE int32[n_req+1]  CSR offsets by request, non-decreasing, hit_off[0] = 0
 *   hit_inst   DEVICE int32[n_hits]   instance of each cached prefix (entries outside [0, n_inst) are ignored)
 *   hit_len    DEVICE int32[n_hits]   its length in tokens
 *   n_hits     number of entries (0 allowed: same as gr_score_route)
 * out_T, when given, holds T with the prefixes applied.
 */
int gr_score_route_cached(gr_fleet* f, int64_t n_req,
                          const int32_t* ctx0, const int32_t* pred_len, const float* budget,
                          const int32_t* exclude_inst,
                          const int32_t* hit_off, const int32_t* hit_inst, const int32_t* hit_len,
                          int64_t n_hits,
                          int32_t* out_inst, float* out_slack, uint8_t* out_fallback,
                          float* out_T, void* hip_stream);

/*
 * Step 2 with the status kept up to date between decisions.  The paper's proxy
 * runs Alg. 1 request after request, refreshing the instances' status before
 * each decision, so that a request sees the ones routed before it; a batch
 * scored against one snapshot sends every similar request to the same
 * instance.  Here the batch is taken `chunk` requests at a time, in order: a
 * chunk is decided as by gr_score_route, then each of its requests joins the
 * queue of the instance it was sent to (prompt = ctx0, length = pred_len; it is
 * prefilled behind the queue and decodes with the batch), the status is
 * rebuilt, and the next chunk is decided.  chunk = 1 is the paper's order;
 * chunk >= n_req is gr_score_route.  On return the handle's tables hold the
 * status with all n_req requests in place; the next gr_build_status or
 * gr_risk_scan starts from the caller's arrays again.
 *
 * The arrays passed to the last gr_build_status / gr_risk_scan are read again
 * and must still be valid and unchanged.  An instance takes routed requests
 * while it holds fewer than max_entries_per_inst entries; beyond that the
 * request is still reported but no longer counted (GR_DEV_ENTRIES_DROPPED).
 * Cost: one scoring pass and one status rebuild per chunk; the rebuild leaves
 * instances that were given nothing in the chunk as they are (unless the blend
 * weight, the observations or the caps have changed since the tables were built:
 * then the first rebuild of the call takes every instance).  Chunks of up to 64 on
 * fleets of up to 512 instances, without caps and with max_entries_per_inst above 64,
 * that are scored pair by pair (see gr_set_small_batch_pairs) are one launch each, or all
 * of them are one: between a launch that builds every instance and one that rebuilds those that were
 * given any, what comes is added to sums behind the tables.  That takes at least four rounds (three on more than 64 instances), and more
 * the larger the chunks are for the fleet (rounds * (2.9 + n_inst / 64 - 0.08 * chunk) above 7, or 10 for three), and
 * compute units for all its workgroups (see gr_set_feedback_units).  The results are the same.
 *
 *   chunk      requests per decision round, >= 1 (cut to max_requests)
 * Other arguments as gr_score_route (no out_T).
 */
int gr_route_feedback(gr_fleet* f, int64_t n_req, int64_t chunk,
                      const int32_t* ctx0, const int32_t* pred_len, const float* budget,
                      const int32_t* exclude_inst,
                      int32_t* out_inst, float* out_slack, uint8_t* out_fallback, void* hip_stream);

/*
 * Step 3 (Sec. 3.4, periodic re-check).  Rebuilds the status from refreshed
 * remaining lengths (as gr_build_status, replacing the handle's tables), flags
 * every active request whose expected finish exceeds its budget
 * (finish > budget, compared in fp64), and for every flagged request runs
 * Alg. 1 over all other instances with ctx0 = prompt + generated (migration
 * moves token IDs, the target prefills them again), pred_len = its refreshed
 * remaining length and D = its budget.  Targets are scored against the
 * refreshed snapshot, the request still counted where it runs now.
 *
 *   act_budget       DEVICE float[n_active]  arrival + SLO - now (may be negative)
 *   out_flag         DEVICE uint8[n_active]
 *   out_finish       DEVICE float[n_active]
 *   out_target       DEVICE int32[n_active]  -1 if not flagged (or no other instance)
 *   out_target_slack DEVICE float[n_active]  0 if not flagged
 *   out_n_flagged    DEVICE int32[1]         may be NULL
 */
int gr_risk_scan(gr_fleet* f,
                 const int32_t* act_off, const int32_t* act_prompt,
                 const int32_t* act_gen, const int32_t* act_rem_refreshed, int64_t n_active,
                 const int32_t* q_off, const int32_t* q_prompt, const int32_t* q_len,
                 int64_t n_queued,
                 const float* act_budget,
                 uint8_t* out_flag, float* out_finish,
                 int32_t* out_target, float* out_target_slack, int32_t* out_n_flagged,
                 void* hip_stream);

/*
 * The paper's own status estimate (Sec. 3.3; Alg. 1 before it forms T(r,g)):
 * q_g, p_g, d_g taken black-box from what was recently observed on the
 * instance and smoothed by an exponential moving average,
 *   x_g <- weight * sample_g + (1 - weight) * x_g,
 * for each of the three terms that comes with a new sample (a term's first
 * sample is its estimate).  Samples: the average waiting time of instance g,
 * its prefill seconds per token, its decode seconds per token (TPOT).
 *
 *   weight       in [0, 1]
 *   obs_wait, obs_prefill, obs_decode   DEVICE float[n_inst] each; NULL = no new sample of that term
 * The estimates live in the handle, in double precision.  Tables and capability order of the
 * last gr_build_status / gr_risk_scan keep the estimates they were built with: new samples show
 * from the next build on.
 */
int gr_observe(gr_fleet* f, double weight, const float* obs_wait, const float* obs_prefill,
               const float* obs_decode, void* hip_stream);

/*
 * How much of that black-box estimate enters every figure the library
 * produces.  With weight w every estimate is
 *   (1 - w) * [white-box value] + w * [Eq. 2 with the smoothed q_g, p_g, d_g]:
 * T(r,g) = q_g + p_g*(ctx0 - H) + d_g*pred_len for a pair; d_g itself for
 * Alg. 1's argmax; d_g per remaining token for the finish time of a running
 * request, q_g + p_g*prompt + d_g*length for a queued one.  w = 0 (the state
 * after gr_create) is the white-box model alone, w = 1 the paper's estimator
 * alone.  Takes effect at the next gr_build_status / gr_risk_scan.  Host call.
 * GR_ERR_NO_STATUS if w > 0 before all three terms have been observed.
 */
int gr_set_blend(gr_fleet* f, double black_box_weight);

/*
 * The paper's second constraint (Sec. 3.1): the number of requests an instance
 * serves concurrently is bounded by its memory.  With a cap B_g, at most B_g
 * requests of instance g decode together: queued requests are admitted in
 * queue order whenever the batch has room (at time 0 and after every decode
 * step); an admission prefills the request, stalling the batch, and puts it
 * into the batch.  Requests already running keep running even if they
 * outnumber the cap.  A request that arrives now is last in the queue, so
 *   q_g = the time at which it would be admitted,
 * after which nobody else joins and T(r,g) = q_g + delta*(ctx0 - H) + [its
 * pred_len decode steps in the batch as it is then].  d_g is the duration of
 * the next decode step that runs.  Every call uses the caps from the next
 * gr_build_status / gr_risk_scan on.  With room for everybody and a newcomer
 * (B_g > entries of g) nothing changes.
 *
 *   cap   HOST int32[n_inst], each >= 1; NULL removes the caps.
 * Host call; waits for the device.
 *
 * With gr_route_feedback under caps, the requests of a chunk queue up on their instances in
 * the order of the batch, whatever the chunk size (without caps the order of a queue shows
 * in no output and is not kept).
 */
int gr_set_batch_cap(gr_fleet* f, const int32_t* cap);

/*
 * How a batch is scored.  Alg. 1 is the same either way; the work is laid out
 * differently.  For a large batch the decode term of Eq. 2 is tabulated once per
 * (distinct length, instance), with its minima over runs of instances, and a
 * request looks at the instances of a run only where the minimum of the run
 * leaves it in question.  A batch of a few requests (the paper routes one
 * arriving request at a time) skips the table: a thread per (request, instance)
 * pair searches the instance's own tables, and the whole call is one kernel.
 *
 *   max_pairs   gr_score_route, gr_route_feedback (its chunks) and gr_risk_scan (its running
 *               requests) score a batch pair by pair when n * (n_inst rounded up to
 *               128) is at most this and n <= 4096.  0: never.  If it is never set, the
 *               number of pairs decides (up to 524 288, with at least 16 per request, or up to
 *               786 432 with more than 32 instances rounded up to whole 64).
 * gr_score_route_cached always takes the table.
 * Equal latencies go to the lowest instance index either way.
 *
 * An infinite latency (an infinite observation, see gr_observe) is nobody's in the pass over the table and in
 * gr_risk_scan: where every latency of a request is infinite, its instance is -1.  It counts as a latency, no less
 * than any other, and the request goes to the lowest index, in gr_score_route_noalloc, and in gr_score_route and
 * gr_route_feedback for batches (chunks) that are scored pair by pair and either max_pairs is set or the batch is of
 * at most 4096 requests and n * (n_inst rounded up to 128) at most 262 144.
 */
int gr_set_small_batch_pairs(gr_fleet* f, int64_t max_pairs);

/*
 * How often the workgroups of a feedback routing that runs in one launch look for each other (about a microsecond
 * each) before those that have started share the work of all, several instances to each of their wavefronts in turn: `looks` times, 64 if it
 * is never set, divided by the share of them that has started.  The results are the same.  It takes about twice as long with
 * half of the workgroups, and 20 to 75 times as long with one of 64 or 128 (256 or 512 instances).
 */
int gr_set_feedback_wait(gr_fleet* f, int32_t looks);

/*
 * At most how many workgroups share that work, >= 1 (all that there are if it is never set).  The results are the same.
 * gr_feedback_team synchronises the device and says how many did in the last feedback routing that was one launch and has
 * ended (HOST int32 out; 0: there was none).  For tests and measurements.
 */
int gr_set_feedback_team(gr_fleet* f, int32_t workgroups);
int gr_feedback_team(gr_fleet* f, int32_t* out_workgroups);

/*
 * How many of the device's compute units a feedback routing may count on (others may have work that stays on the rest).  All
 * rounds are one launch only where its workgroups, one for every four instances, fit these and those that the
 * stream may use at once; else every round is a launch.  The results are the same.  As many as there are if it is never set.
 */
int gr_set_feedback_units(gr_fleet* f, int32_t units);

/*
 * Synchronises the device and returns the OR of the GR_DEV_* bits raised by
 * kernels since gr_create (HOST int32 out).  Not for the hot path.
 */
int gr_device_status(gr_fleet* f, int32_t* out_bits);

/*
 * Per-kernel timing, for benchmarks (not cited from the paper: a measuring aid).
 * gr_profile_enable(f, n) with n > 0 makes every kernel launch of the following
 * calls record a pair of HIP events on the call's stream, up to n launches
 * (events are created here, not in the calls); n = 0 switches timing off.
 * gr_profile_read synchronises the device, adds up the elapsed time and the
 * number of launches per kernel id since the last read into HOST arrays of
 * n_kernels entries, and forgets them.  Kernel ids run from 0 to
 * gr_profile_kernel_count() - 1; gr_profile_kernel_name gives a static name.
 * gr_profile_select restricts the timing to the kernel ids whose bit is set in
 * kernel_mask (all of them after gr_create): an event pair costs a few
 * microseconds of stream time, which adds up over a dozen short launches.
 * gr_profile_read_launches is gr_profile_read launch by launch, in launch order:
 * kernel id and elapsed milliseconds of up to max_launches recorded launches
 * into HOST arrays, their number into *n_launches (for medians and percentiles).
 */
int gr_profile_enable(gr_fleet* f, int32_t max_launches);
int gr_profile_select(gr_fleet* f, uint64_t kernel_mask);
int gr_profile_read(gr_fleet* f, int32_t n_kernels, double* total_ms, int64_t* launches);
int gr_profile_read_launches(gr_fleet* f, int32_t max_launches, int32_t* kernel_id, float* ms, int32_t* n_launches);
int32_t gr_profile_kernel_count(void);
const char* gr_profile_kernel_name(int32_t id);

/*
 * ---- Operators of a length predictor -------------------------------------------------------
 *
 * The routing above takes predicted lengths.  The paper's predictor of them (Sec. 3.2) is a
 * mixture of experts: a small network scores the experts of a request, each expert is a
 * multilayer network, and their results are added up by the scores.  The calls below are what
 * such a predictor is made of, forward and backward: the choice of experts, one layer of all
 * experts, the weighted sum, and the clipping of gradients by their global norm.
 *
 * T rows (requests) go to top_k experts each: S = T * top_k slots, slot r * top_k + j being
 * choice j of row r.  The layers work on positions: the slots in the order of experts, those of
 * expert e at positions off[e] .. off[e+1]-1, in the order of slots.  Slots without an expert
 * (expert -1) come behind all others.
 *
 * Conventions as above: DEVICE pointers, work queued on the stream and nothing else (the calls
 * can be recorded into a HIP graph), workspace in the handle, calls on one handle must not
 * overlap.  Arrays are dense and row-major, aligned to their element (rows that are whole 16 bytes on
 * 16-byte boundaries are faster).  dtype is GR_F32, GR_BF16 or GR_F16 for every `void` array of a call;
 * sums, softmax statistics and norms are held in 32 bits or more and results are rounded once, to nearest.
 * Outputs must not overlap inputs unless it is said.  Indexes on the device are not validated: kernels stay in
 * bounds whatever off, slot, pos and expert hold, and give results only for arrays as gr_expert_plan leaves them.
 * Results do not depend on the order in which workgroups run: the same call gives the same bits.
 * A call whose kernels would have 2^32 threads or more (of a layer: 2^24 tiles of 64 by 64 of its results or of its weights' gradient; else
 * some tens of gigabytes of results at the least) is GR_ERR_TOO_LARGE.
 */
typedef struct gr_experts gr_experts;

enum { GR_F32 = 0, GR_BF16 = 1, GR_F16 = 2 };                    /* dtype */
enum { GR_SCORE_SOFTMAX = 0, GR_SCORE_SIGMOID = 1 };             /* scoring */
#define GR_MAX_EXPERTS 512
#define GR_MAX_TOP_K 16
#define GR_MAX_GROUPS 32
#define GR_MAX_GRADIENTS 4096
#define GR_MAX_WIDTH 65536      /* features of a layer */

/*
 * Create the workspace of calls on up to n_expert experts, max_rows rows and max_top_k experts per row, on the
 * current HIP device.  max_rows * max_top_k <= 2^30.  Device memory held until gr_experts_destroy: 64 MB for the parts of long
 * sums, 4 * (n_expert + 1) bytes for each 1 024 slots or each 256 / l rows, whichever are more (l = 1, 2, 4, ... 32 lanes a row,
 * the least with 16 l >= n_expert), and 0.4 MB.
 */
int gr_experts_create(gr_experts** out, int32_t n_expert, int64_t max_rows, int32_t max_top_k);
int gr_experts_destroy(gr_experts* h);       /* waits for the device first; NULL is allowed */

/*
 * The choice of experts.  With s = softmax or sigmoid of a row's logits (softmax over all experts that are not
 * masked), bias b and c = s + b:
 *   a logit of -inf masks its expert: score 0, never chosen; so does a c of -inf;
 *   the experts are n_group groups of equal size, neighbours together; of these the n_group_kept with
 *   the largest sum of their two largest c stay (a single c where a group has no second);
 *   the top_k experts of those groups with the largest c are chosen, largest first;
 *   weight_j = scale * s_j, divided by the sum of the chosen s if `renormalise` (0 where that sum is 0 in single precision).
 * Ties go to the lowest index.  The bias enters the choice only.  Where fewer than top_k experts are left the last
 * slots have expert -1 and weight 0.  A c that is no number ranks below every number and above masked experts; its weight is what
 * the arithmetic gives (a row whose softmax is not defined has weights that are no numbers).
 *
 *   logits      DEVICE dtype[n_rows * n_expert]   n_expert is the handle's
 *   bias        DEVICE float[n_expert], may be NULL
 *   out_weight, out_expert      DEVICE float, int32 [n_rows * top_k]
 *   out_off, out_slot, out_pos  DEVICE, as gr_expert_plan; all three or none (NULL)
 * top_k <= n_expert; n_group divides n_expert, 1 <= n_group_kept <= n_group; scale is finite.
 */
int gr_expert_route(gr_experts* h, int64_t n_rows, int32_t top_k, const void* logits, int32_t dtype, const float* bias,
                    int32_t scoring, int32_t n_group, int32_t n_group_kept, int32_t renormalise, float scale,
                    float* out_weight, int32_t* out_expert, int32_t* out_off, int32_t* out_slot, int32_t* out_pos, void* hip_stream);

/*
 * Its gradient: of the loss by the logits, from that by the weights.  The choice is constant (`expert`, as it was given out; no
 * expert twice in a row); experts outside [0, n_expert) get nothing and give nothing, whatever dweight holds there.
 *   dweight     DEVICE float[n_rows * top_k]
 *   out_dlogits DEVICE dtype[n_rows * n_expert], written whole
 */
int gr_expert_route_backward(gr_experts* h, int64_t n_rows, int32_t top_k, const void* logits, int32_t dtype, int32_t scoring,
                             int32_t renormalise, float scale, const int32_t* expert, const float* dweight,
                             void* out_dlogits, void* hip_stream);

/*
 * The slots in the order of given experts (those of gr_expert_route, or a caller's own: the paper trains each
 * expert on a part of the data of its own).
 *   expert   DEVICE int32[n_rows * top_k]; outside [0, n_expert): none
 *   out_off  DEVICE int32[n_expert + 1]
 *   out_slot DEVICE int32[n_rows * top_k]   the slot at every position; -1 - slot behind off[n_expert]
 *   out_pos  DEVICE int32[n_rows * top_k]   the position of every slot, -1 for slots without an expert
 */
int gr_expert_plan(gr_experts* h, int64_t n_rows, int32_t top_k, const int32_t* expert, int32_t* out_off, int32_t* out_slot,
                   int32_t* out_pos, void* hip_stream);

/*
 * One layer of every expert: y[p] = act(W_e x[row] + b_e) for the positions p of expert e.
 *   n_pos    number of positions (S), and of rows of out_y; rows behind off[n_expert] are set to 0
 *   off      DEVICE int32[n_expert + 1]; NULL: one matrix for all (W and b are those of a single expert)
 *   slot     DEVICE int32[n_pos]: x is [ceil(n_pos / top_k), n_in], row = slot[p] / top_k.
 *            NULL: x is [n_pos, n_in], row = p
 *   x, w, bias, out_y   DEVICE dtype; w [n_expert, n_out, n_in], bias [n_expert, n_out] or NULL, out_y [n_pos, n_out]
 *   relu     0: act is the identity; 1: max(0, .) (a value that is no number stays one)
 */
int gr_expert_linear(gr_experts* h, int64_t n_pos, int32_t n_in, int32_t n_out, int32_t dtype, const int32_t* off,
                     const int32_t* slot, int32_t top_k, const void* x, const void* w, const void* bias, int32_t relu,
                     void* out_y, void* hip_stream);

/*
 * Its gradient, from dy:  dz = dy where y > 0, else 0 (dy itself without y);
 *   dx[p] = dz[p] W_e;  dW_e = sum over its positions of dz[p]^T x[row];  db_e = sum of dz[p].
 *   y        DEVICE, as gr_expert_linear gave it with relu; NULL: the layer had none
 *   out_dz   DEVICE [n_pos, n_out]: where dz goes; needed with y, NULL without (dy itself is allowed: it is then overwritten)
 *   out_dx   DEVICE [n_pos, n_in], by position: a row of x that several slots share has the sum of theirs
 *            (gr_expert_combine without weights); rows behind off[n_expert] are 0.  May be NULL
 *   out_dw, out_db   DEVICE [n_expert, n_out, n_in], [n_expert, n_out]; 0 for experts without a position; may be NULL
 */
int gr_expert_linear_backward(gr_experts* h, int64_t n_pos, int32_t n_in, int32_t n_out, int32_t dtype, const int32_t* off,
                              const int32_t* slot, int32_t top_k, const void* x, const void* w, const void* y, const void* dy,
                              void* out_dz, void* out_dx, void* out_dw, void* out_db, void* hip_stream);

/*
 * The weighted sum of a row's results: out[r] = sum over j of weight[r, j] * y[pos[r, j]].
 * Slots without an expert add nothing, whatever their weight holds.
 *   weight   DEVICE float[n_rows * top_k]; NULL: all 1
 *   pos      DEVICE int32[n_rows * top_k]
 *   y, out   DEVICE dtype; [n_rows * top_k, n_out], [n_rows, n_out]
 */
int gr_expert_combine(gr_experts* h, int64_t n_rows, int32_t top_k, int32_t n_out, int32_t dtype, const float* weight,
                      const int32_t* pos, const void* y, void* out, void* hip_stream);

/*
 * Its gradient, from dout [n_rows, n_out]: dy[p] = weight[slot] * dout[row], dweight[slot] = <dout[row], y[p]>, both 0 for slots
 * without an expert.
 *   slot        DEVICE int32[n_rows * top_k]
 *   out_dy      DEVICE dtype[n_rows * top_k, n_out]; may be NULL
 *   out_dweight DEVICE float[n_rows * top_k]; may be NULL (y is not read then, and may be NULL)
 */
int gr_expert_combine_backward(gr_experts* h, int64_t n_rows, int32_t top_k, int32_t n_out, int32_t dtype, const float* weight,
                               const int32_t* slot, const void* y, const void* dout, void* out_dy, float* out_dweight,
                               void* hip_stream);

/*
 * Clipping by the global norm: norm = the root of the sum of the squares of all elements of all gradients;
 * out_i = grad_i * min(1, max_norm / norm).  Gradients are given out as they are where the norm is not finite.  Squares are
 * summed and the norm is held in double precision: one past single precision clips as any other, and out_norm is infinite.
 *   grad, out HOST arrays of n_grad DEVICE pointers (read during the call); out[i] may be grad[i], NULL for an empty one
 *   count     HOST int64[n_grad], >= 0, at most 2^40
 *   dtype     HOST int32[n_grad], of gradient and output alike
 *   max_norm  >= 0, may be infinite
 *   out_norm  DEVICE float[1]; may be NULL
 */
int gr_clip_gradients(gr_experts* h, int32_t n_grad, const void* const* grad, void* const* out, const int64_t* count,
                      const int32_t* dtype, float max_norm, float* out_norm, void* hip_stream);

/*
 * ---- Operators that read a request's tokens -------------------------------------------------
 *
 * A length predictor takes features of requests.  The calls below make them from the tokens: rows of a
 * table by token, a gated recurrence over the tokens of every request, whose last state stands for the
 * request, and dropout while it is trained; forward, backward, and token by token while a request runs.
 *
 * Conventions as for the operators above, with these besides: `stride` is the number of elements from one row
 * to the next, at least the width and at most GR_MAX_STRIDE (the halves of one product's result are such arrays); arrays without one are
 * dense.  Indexes on the device are not validated: kernels stay in bounds whatever token and off hold.
 */
typedef struct gr_tokens gr_tokens;

#define GR_MAX_VOCAB (1 << 24)
#define GR_MAX_STRIDE (1 << 18)

/*
 * Create the workspace of calls on up to max_tokens tokens (<= 2^30) of up to max_vocab different ones and rows of up to max_width
 * elements, on the current HIP device (not inside a capture).  All of it is allocated here, whichever of the calls follow, and held until
 * gr_tokens_destroy; in bytes, with quotients rounded up, p = (max_tokens + max_vocab) / 1 024, and t = max_tokens / 96, or max_tokens / 64 up to 512
 * of those if that is more:
 *   16 * max_tokens + 2 048 * (max_tokens / 2 048 + 1)   the sort,
 *   8 * max_width * p, 2^24 at least                     parts of long sums (570 MB for 2^20 tokens of 2^24 and rows of 4 096),
 *   8 * p, 16 384 at least                               the rows whose sums have parts,
 *   8 * (2 * t + t / 16) * [max_width + 3, rounded up to a multiple of 128 if max_width is more than that]
 *                                                        what the recurrence's tiles tell each other (738 MB there),
 * and its counters, 2 * max_width + 400.
 */
int gr_tokens_create(gr_tokens** out, int64_t max_tokens, int32_t max_vocab, int32_t max_width);
int gr_tokens_destroy(gr_tokens* h);         /* waits for the device first; NULL is allowed */

/*
 * Rows by token: out[t] = scale * table[token[t]]; 0 where token[t] is outside [0, n_vocab) (padding).
 *   token       DEVICE int32[n_tokens]
 *   table, out  DEVICE dtype; [n_vocab, width], [n_tokens, width]
 *   scale       finite
 */
int gr_token_embed(gr_tokens* h, int64_t n_tokens, int32_t n_vocab, int32_t width, int32_t dtype, const int32_t* token,
                   const void* table, float scale, void* out, void* hip_stream);

/*
 * Its gradient: dtable[v] = scale * the sum of dout[t] over the t with token[t] = v, written whole (0 for a token that is not there).
 *   dout        DEVICE dtype[n_tokens, width]; rows of tokens outside [0, n_vocab) are not read
 *   out_dtable  DEVICE dtype[n_vocab, width]
 */
int gr_token_embed_backward(gr_tokens* h, int64_t n_tokens, int32_t n_vocab, int32_t width, int32_t dtype, const int32_t* token,
                            const void* dout, float scale, void* out_dtable, void* hip_stream);

/*
 * A gated recurrence along every sequence of tokens, channel by channel:
 *   f_t = sigmoid(gate_t),  h_t = f_t h_{t-1} + (1 - f_t) x_t,  y_t = h_t.
 * Sequence s has the tokens off[s] .. off[s+1]-1; off does not decrease.  States are held in single precision.  A state that is not
 * finite leaves the sequence's later ones not finite (an infinity may become no number); other sequences are not affected.
 *   off         DEVICE int32[n_seq + 1]; NULL: n_seq is n_tokens and every token is a sequence of its own (a step of running requests)
 *   gate, x     DEVICE dtype[n_tokens, width], rows gate_stride and x_stride apart
 *   h0          DEVICE float[n_seq, width], the states that sequences start from; NULL: 0
 *   out_y       DEVICE dtype[n_tokens, width]; rows of no sequence are left as they are.  May be NULL
 *   out_h       DEVICE float[n_seq, width], the states after the last tokens, h0 for a sequence of none.  May be NULL; may be h0 itself
 *               where off is NULL
 */
int gr_gated_scan(gr_tokens* h, int64_t n_tokens, int64_t n_seq, int32_t width, int32_t dtype, const int32_t* off,
                  const void* gate, int64_t gate_stride, const void* x, int64_t x_stride, const float* h0, void* out_y, float* out_h,
                  void* hip_stream);

/*
 * Its gradient, from dy (of y) and dh (of the last states), either of which may be NULL (0):
 *   D_t = dy_t + f_{t+1} D_{t+1}  (dh in the place of the last product after a sequence's last token)
 *   dx_t = (1 - f_t) D_t,  dgate_t = f_t (1 - f_t) D_t (h_{t-1} - x_t),  dh0 = f D of the first token, dh for a sequence of none.
 *   y           DEVICE dtype[n_tokens, width], as gr_gated_scan gave it; h_{t-1} is taken from it as it was rounded
 *   dy          DEVICE dtype[n_tokens, width];  dh DEVICE float[n_seq, width]
 *   out_dgate, out_dx   DEVICE dtype[n_tokens, width], rows dgate_stride and dx_stride apart; rows of no sequence are left as they are
 *   out_dh0     DEVICE float[n_seq, width]; may be NULL; may be dh itself where off is NULL
 */
int gr_gated_scan_backward(gr_tokens* h, int64_t n_tokens, int64_t n_seq, int32_t width, int32_t dtype, const int32_t* off,
                           const void* gate, int64_t gate_stride, const void* x, int64_t x_stride, const void* y, const float* h0,
                           const void* dy, const float* dh, void* out_dgate, int64_t dgate_stride, void* out_dx, int64_t dx_stride,
                           float* out_dh0, void* hip_stream);

/*
 * Dropout: out_i = residual_i + (u_i < m ? 0 : x_i * 65536 / (65536 - m)), m = rate * 65536 rounded to the nearest, ties to even.
 * u_i are 16 random bits of no memory: of a block of eight elements, the four words (lower halves first) that Philox 4x32 of ten
 * rounds (Salmon et al. 2011) makes of the counter (i / 8, offset) and the key seed, 64 bits each.  The gradient is the same call on
 * that of out, without a residual.
 *   x, residual, out  DEVICE dtype[n]; residual may be NULL; out may be x or residual itself.  n <= 2^40
 *   rate         >= 0, and m < 65536
 *   offset_add   DEVICE uint64[1], added to offset (modulo 2^64) when the kernel runs, so that the replays of a recorded call draw anew; may be NULL
 */
int gr_dropout(gr_tokens* h, int64_t n, int32_t dtype, const void* x, const void* residual, double rate, uint64_t seed,
               uint64_t offset, const uint64_t* offset_add, void* out, void* hip_stream);

/* Static, human-readable text for a return code. */
const char* gr_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* GOODROUTE_H */
