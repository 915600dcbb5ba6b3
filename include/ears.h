/*
 * ears.h -- C ABI of the EARS speculative-decoding verification step for
 * NVIDIA B200 (sm_100a).
 *
 * One call verifies K draft tokens for each of B independent sequences
 * ("Efficient Adaptive Rejection Sampling", arXiv 2512.13194):
 *
 *   1. every target and draft logits row becomes a temperature softmax
 *      (Sec. 3.1; temperature as discussed in Sec. 4.3);
 *   2. draft token x_k is accepted iff
 *          R_k >= max(U_k - Tolerance_k, 0),
 *          R_k = P_t(x_k) / max(P_d(x_k), 1e-10),
 *          Tolerance_k = beta * (1 - max_v P_t(v))
 *      (Sec. 3.2: uncertainty, tolerance equation, acceptance condition;
 *       Sec. 3.3 item 2: division guard and threshold clamp);
 *   3. the first rejected position n ends the accepted prefix (Sec. 3.1);
 *   4. position n receives a token drawn from normalize(max(0, P_t - P_d)) of
 *      that position, or, when all K were accepted (n = K), a token drawn from
 *      P_t of the extra target row.  The paper leaves this step to the target
 *      model ("generate ... starting from position i", Sec. 3.1); the rule used
 *      is the speculative-sampling one of its refs. [1], [2].
 *
 * Random numbers (not in the paper; fixed here so results are reproducible and
 * independent of how a batch is split): Philox4x32-10 with
 *     key     = (seed[31:0], seed[63:32])
 *     counter = (offset[31:0], offset[63:32], b_global, slot)
 *   slot k in [0,K): U_k = (word0 >> 8) * 2^-24              (exact in fp32)
 *   slot K         : u   = ((word0 << 32 | word1) >> 11) * 2^-53, the uniform of
 *                    the inverse-CDF draw in step 4 (token = smallest j with
 *                    u*S < C_j, C_j the running sum of the masses, S their total).
 * A caller advances `offset` by one per verification step.
 *
 * Conventions for every entry point unless stated otherwise:
 *   - logits are row-major and contiguous: target [B, K+1, V], draft [B, K, V],
 *     fp32, bf16 (bit pattern of the upper half of an fp32) or fp16 (IEEE binary16); draft tokens [B, K]
 *     int32.  -inf logits (masked vocabulary) are legal.
 *   - pointers are DEVICE pointers owned by the caller; the library neither
 *     retains nor frees them.  Logits must be aligned to their element size.
 *     When both logits bases are 16-byte aligned and V * elem_size is a multiple
 *     of 16 the rows are fetched with bulk asynchronous copies (TMA) or 16-byte
 *     vector loads, depending on the kernel the call's shape selects; otherwise
 *     slower element-wise loads are used with identical results.
 *   - `stream` is a cudaStream_t passed as void* (NULL = default stream).  Calls
 *     enqueue work and return; they do not synchronise.
 *   - outputs: out_accept_len[b] = n in [0, K]; out_tokens[b, 0:n] = the accepted
 *     draft tokens, out_tokens[b, n] = the resampled (n < K) or bonus (n = K)
 *     token, out_tokens[b, n+1:] = -1.
 *   - a sequence whose data cannot be verified (draft token outside [0, V); a NaN
 *     or +inf logit; a row with no finite logit) gets out_accept_len[b] = -1 and
 *     out_tokens[b, :] = -1, and bit EARS_DEV_INVALID_INPUT is set in the device
 *     status; other sequences are unaffected.  Nothing traps.
 *   - the return value reports host-detectable errors only (enum below); 0 = enqueued.
 */
#ifndef EARS_H
#define EARS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EARS_VERSION 100

enum {
    EARS_OK = 0,
    EARS_ERR_NULL = -1,      /* a required pointer is NULL */
    EARS_ERR_SHAPE = -2,     /* B, K or V < 1; K > EARS_MAX_K; V > 2^30; sizes overflow */
    EARS_ERR_PARAM = -3,     /* temperature not finite or <= 0; beta not finite or < 0; bad dtype */
    EARS_ERR_ALIGN = -4,     /* logits not aligned to their element size; workspace not 256-byte aligned */
    EARS_ERR_WORKSPACE = -5, /* caller workspace smaller than ears_workspace_bytes() */
    EARS_ERR_CUDA = -6,      /* a CUDA runtime call failed (see ears_last_cuda_error) */
    EARS_ERR_TIMEOUT = -7    /* a bounded device-side wait gave up (reported by ears_last_device_status) */
};

enum { EARS_DTYPE_F32 = 0, EARS_DTYPE_BF16 = 1, EARS_DTYPE_F16 = 2 };

/* bits of the device status word of a call */
enum { EARS_DEV_INVALID_INPUT = 1, EARS_DEV_TIMEOUT = 2 };

#define EARS_MAX_K 64

/*
 * The verification step as listed above, fp32 logits.  Uses a library-owned
 * workspace cached per (device, stream); calls sharing a stream are ordered,
 * calls on different streams are independent.
 */
int ears_verify_f32(const float* target_logits, const float* draft_logits,
                    const int32_t* draft_tokens, int B, int K, int V,
                    float temperature, float beta, uint64_t seed, uint64_t offset,
                    int32_t* out_accept_len, int32_t* out_tokens, void* stream);

/* Same, bf16 logits (pointer to 16-bit elements). */
int ears_verify_bf16(const void* target_logits, const void* draft_logits,
                     const int32_t* draft_tokens, int B, int K, int V,
                     float temperature, float beta, uint64_t seed, uint64_t offset,
                     int32_t* out_accept_len, int32_t* out_tokens, void* stream);

/* Same, fp16 (IEEE binary16) logits. */
int ears_verify_f16(const void* target_logits, const void* draft_logits,
                    const int32_t* draft_tokens, int B, int K, int V,
                    float temperature, float beta, uint64_t seed, uint64_t offset,
                    int32_t* out_accept_len, int32_t* out_tokens, void* stream);

/* Alias of ears_verify_f32 (the element type cannot be inferred from the arguments). */
int ears_verify(const void* target_logits, const void* draft_logits,
                const int32_t* draft_tokens, int B, int K, int V,
                float temperature, float beta, uint64_t seed, uint64_t offset,
                int32_t* out_accept_len, int32_t* out_tokens, void* stream);

/*
 * General form.  Beyond the arguments above:
 *   dtype       EARS_DTYPE_F32, EARS_DTYPE_BF16 or EARS_DTYPE_F16 (IEEE binary16).
 *   b_first     global index of local sequence 0; it enters the random counter so
 *               that a batch sharded across GPUs (Sec. 3.3 item 3 treats all active
 *               sequences independently) reproduces the unsharded result.
 *   out_pt_tok, out_pd_tok, out_max_pt   [B,K] double, optional (NULL to skip):
 *               P_t(x_k), P_d(x_k) and max_v P_t(v) of Sec. 3.2 step 1, for every
 *               position (also those after the first rejection).
 *   out_class   [B,K] uint8, optional: 0 reject, 1 direct accept (R >= U),
 *               2 accept via the pardon path (Sec. 3.2 step 5).
 *   out_resid_mass [B] double, optional: total mass S the final token was drawn
 *               from (the residual mass, or ~1 for a bonus token).
 *   workspace, workspace_bytes   caller-owned device scratch of at least
 *               ears_workspace_bytes(B,K,V) bytes, 256-byte aligned, contents
 *               arbitrary; or (NULL, 0) to use the library-owned one.  With a
 *               caller workspace the call allocates nothing.  Two calls that may
 *               overlap on the GPU must not share a workspace.
 */
int ears_verify_ex(int dtype, const void* target_logits, const void* draft_logits,
                   const int32_t* draft_tokens, int B, int K, int V,
                   float temperature, float beta, uint64_t seed, uint64_t offset,
                   int64_t b_first, int32_t* out_accept_len, int32_t* out_tokens,
                   double* out_pt_tok, double* out_pd_tok, double* out_max_pt,
                   uint8_t* out_class, double* out_resid_mass,
                   void* workspace, size_t workspace_bytes, void* stream);

/*
 * ears_verify_ex with a temperature and a base tolerance per sequence.  Sec. 3.3 item 3 verifies
 * all active sequences side by side and independently, and in a serving batch each request brings
 * its own sampling temperature (Sec. 4.3 discusses its effect on the tolerance) and possibly its
 * own beta (Sec. 3.2); the paper states both as scalars.
 *   seq_temperature, seq_beta   DEVICE arrays [B] of float, either may be NULL.  Where given,
 *               sequence b uses seq_temperature[b] / seq_beta[b] and the scalar argument of the
 *               same name is ignored; where NULL the scalar applies to every sequence.
 *   A value the scalar form would refuse (temperature not finite or <= 0, beta not finite or
 *   < 0) cannot be seen by the host: it marks that one sequence invalid (out_accept_len = -1,
 *   tokens -1, EARS_DEV_INVALID_INPUT), the others are unaffected.
 *   flags       0, EARS_FLAG_STOP_AT_FIRST_REJECT and / or EARS_FLAG_ENTROPY_UNCERTAINTY (for the latter
 *               see ears_verify_entropy).  Sec. 3.1: rejecting x_i discards every later
 *               draft token.  With the flag, what lies after a sequence's first rejected position
 *               (later rows and tokens, and the extra target row unless everything was accepted)
 *               is not part of the step: it is not validated and the optional per-position
 *               outputs are not written there; lengths and tokens are the same as without the
 *               flag on valid data.  Where a cluster kernel runs (the resident kernel for short
 *               rows, the cluster-streamed kernel from four sequences per SM on; see
 *               ears_set_path) those rows are not even read -- a cluster then walks a sequence
 *               position by position -- which saves their HBM traffic at the price of a longer
 *               chain per sequence; the other streaming kernels read them anyway and ignore them.
 * Everything else is as in ears_verify_ex.
 */
#define EARS_FLAG_STOP_AT_FIRST_REJECT 1u
#define EARS_FLAG_ENTROPY_UNCERTAINTY 2u   /* see ears_verify_entropy */
#define EARS_FLAGS_ALL (EARS_FLAG_STOP_AT_FIRST_REJECT | EARS_FLAG_ENTROPY_UNCERTAINTY)
int ears_verify_var(int dtype, const void* target_logits, const void* draft_logits,
                    const int32_t* draft_tokens, int B, int K, int V,
                    float temperature, float beta,
                    const float* seq_temperature, const float* seq_beta, unsigned flags,
                    uint64_t seed, uint64_t offset,
                    int64_t b_first, int32_t* out_accept_len, int32_t* out_tokens,
                    double* out_pt_tok, double* out_pd_tok, double* out_max_pt,
                    uint8_t* out_class, double* out_resid_mass,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * ears_verify_var with the entropy of the target distribution.  Sec. 3.2 measures the target
 * model's uncertainty at a position as 1 - max_v P_t(v); Sec. 5 (future work, item 1) names the
 * distribution's entropy as a more refined measure and gives no formula.  Here
 *     H = -sum_v P_t(v) ln P_t(v)   (nats; masked entries contribute nothing)
 * comes out of the same sweep over the target row that yields its normaliser (one more
 * multiply-add per logit), and
 *   out_entropy [B,K] double, optional (NULL to skip): H of target row k, for every position
 *               (with EARS_FLAG_STOP_AT_FIRST_REJECT: up to the first rejection);
 *   flags may include EARS_FLAG_ENTROPY_UNCERTAINTY: the tolerance of Sec. 3.2 becomes
 *               beta * H / ln V in place of beta * (1 - max P_t).  H / ln V lies in [0, 1] like
 *               the printed measure (1 for a flat row, 0 for a one-hot row or V = 1); dividing by
 *               ln V is this library's reading of "entropy as the uncertainty measure".
 * Without the flag and with out_entropy = NULL this is ears_verify_var.  Everything else
 * (arguments, outputs, errors, workspace) as there; out_entropy must be 8-byte aligned.
 */
int ears_verify_entropy(int dtype, const void* target_logits, const void* draft_logits,
                        const int32_t* draft_tokens, int B, int K, int V,
                        float temperature, float beta,
                        const float* seq_temperature, const float* seq_beta, unsigned flags,
                        uint64_t seed, uint64_t offset,
                        int64_t b_first, int32_t* out_accept_len, int32_t* out_tokens,
                        double* out_pt_tok, double* out_pd_tok, double* out_max_pt,
                        uint8_t* out_class, double* out_resid_mass, double* out_entropy,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * The temperature -> 0 limit of the step (Sec. 1 names temperature = 0 as the deterministic
 * regime; the entry points above refuse temperature <= 0 because their arithmetic divides by it).
 * In the limit every softmax is one-hot at its row's largest logit (the smallest index among
 * equal ones), max P_t = 1, the tolerance beta (1 - max P_t) of Sec. 3.2 is zero, and for a
 * greedily drafted token R_k is 1 or 0: x_k is accepted iff it is the top token of target row k.
 * The first mismatch n ends the accepted prefix (Sec. 3.1); out_tokens[b, n] is the top token of
 * target row n (row K if all K matched).  Draft logits, beta, seed and offset play no role.
 * Outputs, invalid-sequence marking (NaN, +inf, no finite logit in ANY of the K+1 target rows; a
 * draft token outside [0, V)), workspace rules and status words are those of ears_verify_ex.
 */
int ears_verify_greedy(int dtype, const void* target_logits, const int32_t* draft_tokens,
                       int B, int K, int V, int32_t* out_accept_len, int32_t* out_tokens,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * Verification with the VOCABULARY split across devices (tensor-parallel logits).  Device r of
 * n_shards holds the columns [v_first, v_first + Vs) of every row: target_shard [B, K+1, Vs],
 * draft_shard [B, K, Vs], row-major and contiguous; the devices' column ranges are disjoint,
 * cover [0, V) and ascend with r.  draft_tokens [B, K] (ids in [0, V)) are the same everywhere.
 * The step is the one of ears_verify_ex [Sec. 3.1-3.3] on the concatenated rows, computed in
 * three local phases with two small exchanges the CALLER performs (all-gathers of device
 * buffers, e.g. NCCL; logits never move):
 *
 *   ears_shard_stats   -> out_stats [B (2K+1)] x 4 floats per row of this device's columns:
 *                         (max m, sum of exp((l - m)/T), logit of the row's draft token if its
 *                         column lies here else 0, 1 or 0 saying which).  Rows of a sequence:
 *                         target 0..K, then draft 0..K-1.
 *   -- all-gather out_stats over devices into all_stats [n_shards][B (2K+1)][4] --
 *   ears_shard_decide  -> every device combines the statistics in device order (so decisions
 *                         are bitwise identical everywhere), applies the acceptance rule of
 *                         Sec. 3.2 per position with U_k from the counter stream of ears_verify,
 *                         writes out_accept_len [B] and the accepted prefix of out_tokens
 *                         [B, K+1] (-1 elsewhere), and out_mass [B]: the mass this device's
 *                         columns hold of the row to draw from, in units of 1/Z_t
 *                         (max(0, P_t - P_d) of the rejected position, P_t of row K after K
 *                         acceptances).  Invalid sequences (as in ears_verify, or a token whose
 *                         column no device or more than one device claimed): length -1, tokens -1.
 *   -- all-gather out_mass over devices into all_mass [n_shards][B] --
 *   ears_shard_pick    -> the device whose columns contain the point u S of the cumulative mass
 *                         (devices in order; u the final uniform of ears_verify, S the total)
 *                         writes the drawn token's id into out_tokens[b, n]; the others leave
 *                         -1 there.  An element-wise MAX of out_tokens over devices completes
 *                         the step on every device.
 *
 * All pointers are device memory.  `workspace` (256-byte aligned, at least
 * ears_shard_workspace_bytes(dtype, B, K, Vs) bytes, caller-owned) carries state from phase to
 * phase: pass the same buffer, untouched, to the three calls of one step.  Calls are enqueued
 * on `stream`; nothing synchronises.  temperature, seed, offset, b_first as in ears_verify_ex.
 * Errors: as ears_verify_ex; EARS_ERR_SHAPE also for v_first / Vs outside [0, V];
 * EARS_ERR_PARAM for n_shards outside [1, EARS_MAX_SHARDS] or shard outside [0, n_shards).
 */
#define EARS_MAX_SHARDS 64
size_t ears_shard_workspace_bytes(int dtype, int B, int K, int Vs);
int ears_shard_stats(int dtype, const void* target_shard, const void* draft_shard,
                     const int32_t* draft_tokens, int B, int K, int Vs, int V, int v_first,
                     float temperature, float* out_stats,
                     void* workspace, size_t workspace_bytes, void* stream);
int ears_shard_decide(int dtype, const void* target_shard, const void* draft_shard,
                      const int32_t* draft_tokens, int B, int K, int Vs, int V, int v_first,
                      int n_shards, const float* all_stats, float temperature, float beta,
                      uint64_t seed, uint64_t offset, int64_t b_first,
                      int32_t* out_accept_len, int32_t* out_tokens, double* out_mass,
                      void* workspace, size_t workspace_bytes, void* stream);
int ears_shard_pick(int dtype, const void* target_shard, const void* draft_shard,
                    const int32_t* draft_tokens, int B, int K, int Vs, int V, int v_first,
                    int n_shards, int shard, const float* all_stats, const double* all_mass,
                    float temperature, uint64_t seed, uint64_t offset, int64_t b_first,
                    int32_t* out_tokens, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Same step with HOST buffers: copies the inputs to library-owned device staging
 * buffers, runs the step, copies out_accept_len / out_tokens back and waits for
 * completion.  All pointers are host memory (pinned memory makes the copies
 * asynchronous and faster).  Returns a host error, or EARS_ERR_TIMEOUT if a device
 * wait gave up; invalid sequences are reported in the outputs as above.
 */
int ears_verify_host(int dtype, const void* target_logits, const void* draft_logits,
                     const int32_t* draft_tokens, int B, int K, int V,
                     float temperature, float beta, uint64_t seed, uint64_t offset,
                     int64_t b_first, int32_t* out_accept_len, int32_t* out_tokens,
                     void* stream);

/*
 * Verification step for callers that must not allocate device memory.
 * (The paper has no counterpart; this is a packaging variant of ears_verify_ex.)
 *
 * Some hosts of this library cannot call cudaMalloc at the moment they verify: code
 * running while a CUDA graph is being captured on the thread, a serving loop that gave
 * all device memory to its own pool at start-up and forbids later driver allocations,
 * or a latency-critical thread that must never take the allocator's device-wide lock.
 * ears_verify_ex allocates when it is given no workspace, and a caller workspace has
 * to come from somewhere.  This entry point instead keeps its scratch in a fixed
 * array of EARS_NOALLOC_SCRATCH_BYTES that is part of the library image: every GPU
 * that loads the library holds those bytes until the process exits, whether or not
 * this function is ever called.
 *
 * Arguments and results are those of ears_verify_ex without the optional outputs and
 * without a workspace; inputs and outputs are still the caller's device buffers.
 * The function calls no cudaMalloc, cudaFree or other allocating routine (keep the
 * ears_profile_* timing hooks off around it: they create events).
 *
 *   - Shapes whose scratch need, ears_workspace_bytes(B,K,V), exceeds
 *     EARS_NOALLOC_SCRATCH_BYTES are refused with EARS_ERR_WORKSPACE before anything
 *     is enqueued (B=512, K=3, V=256000 needs about 4.2 MB).
 *   - The first call on each device looks up the array's device address (and sets the
 *     kernels' shared-memory attribute); make that first call outside any stream
 *     capture.  The device must be current, as for every other entry point.
 *   - "Allocates nothing" holds once the code a call needs is resident: the CUDA driver loads
 *     a kernel when it is first launched (one kernel per element type and per launch plan:
 *     rows that stay in shared memory, long rows, 2- or 4-byte logits), and loading
 *     allocates.  Make one warm-up call per element type and kind of shape you will use,
 *     outside any capture, before the phase in which allocation is forbidden.
 *   - All calls on a device share the one array.  It keeps the previous call's
 *     contents; the counters that must start at zero are cleared at the start of every
 *     call, on the call's stream.  Calls that can overlap on the GPU (different streams
 *     without an ordering between them, or different host threads) race on it and
 *     give wrong results: serialise them, or use ears_verify_ex with separate workspaces.
 *   - out_device_status: optional DEVICE pointer to one int32; when not NULL the call's
 *     status word (EARS_DEV_* bits, 0 = clean) is copied there on `stream` after the
 *     kernels, for the caller to read once the stream has been waited for.
 */
#define EARS_NOALLOC_SCRATCH_BYTES (8u << 20)
int ears_verify_noalloc(int dtype, const void* target_logits, const void* draft_logits,
                        const int32_t* draft_tokens, int B, int K, int V,
                        float temperature, float beta, uint64_t seed, uint64_t offset,
                        int64_t b_first, int32_t* out_accept_len, int32_t* out_tokens,
                        int32_t* out_device_status, void* stream);

/* Upper bound of the scratch bytes a call with these sizes needs (either dtype). */
size_t ears_workspace_bytes(int B, int K, int V);

/*
 * Waits for `stream`, then returns the device status of the most recent call that
 * used the library-owned workspace of (current device, stream): an OR of EARS_DEV_*
 * bits (every call starts from 0), or a negative EARS_ERR_* if the wait itself failed.
 */
int ears_last_device_status(void* stream);

/* Same for a caller-owned workspace that was passed to ears_verify_ex on `stream`. */
int ears_workspace_device_status(void* workspace, void* stream);

/*
 * How the most recent call on the library-owned workspace of (current device, stream) decided its
 * positions -- the three-way decision of Sec. 3.2 step 5 as production telemetry, counted on the
 * device by the kernels themselves (no optional output is needed for it):
 *   out_counts[0] direct acceptances (R >= U), [1] acceptances by pardon (U - Tolerance <= R < U),
 *   [2] rejections, [3] sequences marked invalid.
 * A sequence contributes the positions it really decided: its accepted prefix and, if there is
 * one, its first rejection (so [2] is the number of sequences that ended in a rejection).  Waits
 * for `stream`; out_counts is a HOST array of four words.  The greedy form counts [3] only.
 */
int ears_last_decision_counts(void* stream, uint32_t out_counts[4]);

/* Same for a caller-owned workspace that was passed to a verification call on `stream`. */
int ears_workspace_decision_counts(void* workspace, void* stream, uint32_t out_counts[4]);

/*
 * Self-test of the kernels' bounded waits (every device-side wait in this library gives up
 * after a time limit, sets EARS_DEV_TIMEOUT and lets the kernel return; nothing can hang
 * the GPU).  Launches a tiny kernel that waits limit_ms (1..2000) on a barrier no thread ever
 * completes, waits for it and returns EARS_ERR_TIMEOUT when the wait gave up as designed
 * (EARS_OK would mean the limit did not work).  The context stays usable.
 */
int ears_selftest_bounded_wait(int limit_ms, void* stream);

/*
 * Test hook for the device random stream: out[i, 0:4] = Philox4x32-10 of counter
 * ctr_key[i, 0:4] and key ctr_key[i, 4:6]; both device pointers, n >= 0.
 */
int ears_philox_device(const uint32_t* ctr_key, uint32_t* out, int n, void* stream);

/*
 * Launch-plan override for tests (0 = automatic for every field):
 *   loader 1 = bulk-copy (TMA) loader where alignment allows, 2 = element-wise loader;
 *   parts  = number of pieces each row is split into for the statistics pass (clamped
 *   to what the row allows).
 * Results never depend on the plan except through floating-point summation order.
 */
int ears_set_plan(int loader, int parts);

/*
 * Choice among the four kernels, for tests and measurements (0 = automatic for both fields):
 *   path 1 = streaming kernel with a ring of shared-memory slots filled by bulk copies (the rows of
 *            a rejected position are read a second time);
 *        3 = streaming kernel whose warps read straight from global memory (same second pass);
 *        2 = resident kernel (the two rows of a position stay in the shared memory of a
 *            thread-block cluster; every logit is read once);
 *        4 = cluster-streamed kernel (the same clusters stream their slices instead of holding
 *            them; per sequence only the rows of the first rejected position are read again, in
 *            pieces that all CTAs of the launch serve; with EARS_FLAG_STOP_AT_FIRST_REJECT nothing
 *            after a first rejection is read).
 *            Forcing path 2 or 4 on a shape it cannot take (rows that do not fit a cluster's
 *            shared memory) makes the verification calls return EARS_ERR_SHAPE.  A non-zero
 *            `parts` of ears_set_plan also selects the ring kernel.
 *   cluster = CTAs per cluster of paths 2 and 4: 1, 2, 4, 8 or 16.
 * All kernels implement the same step (Sec. 3.1-3.3); results differ only through
 * floating-point summation order.  The initial values can also come from the environment,
 * read once when the library is loaded: EARS_PATH=streaming|resident|direct|cluster-streamed (or 1..4),
 * EARS_CLUSTER=1|2|4|8|16.
 */
int ears_set_path(int path, int cluster);

/*
 * Writes a one-line description of the launch plan a verification call with these sizes
 * would use on the current device (which kernel, cluster size and slices or pieces per row,
 * how many CTAs) into the HOST buffer `out` of `out_bytes` bytes (NUL-terminated, truncated
 * if short).  Launches nothing.
 */
int ears_describe_plan(int dtype, int B, int K, int V, char* out, size_t out_bytes);

/*
 * Device timing of the kernel for benchmarks.  After ears_profile_begin(max_calls) every
 * verification call (up to max_calls) records a CUDA event on its stream right before and
 * right after its kernel; nothing synchronises.  ears_profile_end waits for the last
 * recorded event, writes the per-call kernel durations in milliseconds into the host array
 * of `capacity` floats, stores the number of calls timed in *n_calls and releases the
 * events.  Not thread-safe against concurrent verification calls.
 */
int ears_profile_begin(int max_calls);
int ears_profile_end(float* kernel_ms, int capacity, int* n_calls);

/*
 * ---- Operators on rows of logits ----------------------------------------------------------------
 *
 * What a program that verifies drafts does with the same rows next to the verification: take the
 * target's top logits as a teacher for the draft (ears_top_logits), train the draft towards them
 * (ears_distill_*), score the emitted tokens (ears_token_logprobs*), and train a policy on sampled
 * tokens (ears_policy_*; `old` is their log probability under the law that they were drawn from.  For tokens
 * that a verification call emitted that is ln P_t, as ears_token_logprobs scores it on the target rows, only if
 * beta was 0: with beta > 0 they follow a wider law, whose probabilities no call here returns).
 *
 * Common arguments:
 *   logits        [B, R, V], entries of a row contiguous; row (b, k) starts at logits + b stride_b +
 *                 k stride_r (strides in entries, >= 0), so that the first K rows of a target
 *                 [B, K+1, V], or rows padded to a longer pitch, are used in place.  Any alignment of at
 *                 least the element size and any V serve; rows that share their start within 16 bytes with the
 *                 gradient's rows run at full speed, others store the gradient entry by entry, two to four
 *                 times slower where rows are long.  Per-row arrays are contiguous, row b R + k.
 *   temperature   l / temperature enters every softmax; seq_temperature [B] replaces it where not NULL.  It is
 *                 taken in 64 bits: rounding it to 32 would move logits of 20 by 1e-6.
 *   status        optional DEVICE word into which EARS_DEV_INVALID_INPUT is OR-ed when a row could not be
 *                 used, and EARS_DEV_TIMEOUT when a bounded wait gave up; the caller clears it.
 *   out_grad      [B, R, V] in the logits' type, with strides of its own; rows must not overlap.  It may be
 *                 the logits themselves (same pointer, same strides): the gradient then replaces them.
 *                 Any other overlap of the two address ranges is refused.
 *   out_saved     optional, 4 floats per row, 16-byte aligned: what the backward call of the same
 *                 operator needs (`saved`); logits and the other inputs must be unchanged until then.
 * -inf logits (masked vocabulary) are legal, and so are masks of the type's lowest value.  A row left out
 * (see each operator) is not read: its outputs are 0 and its gradient row is zeros.  A row that cannot be
 * used (NaN or +inf logit, no finite logit, index outside [0, V), unusable temperature) gives NaN outputs
 * and a gradient row of zeros, and sets the status bit.  Other rows are unaffected.
 * Sums and row scalars are kept in 32 bits and 64 bits; a gradient entry is rounded once, to its type, and what lies
 * below 2^-126 of its row's largest exponential is 0.
 * The calls use no workspace, allocate nothing and may be recorded into CUDA graphs and run side by side
 * on any streams (the driver loads a kernel at its first launch: make that one outside any capture).  The same call on
 * the same kind of device gives the same bits.  Which threads share a row, and with that the order of its sums, goes by
 * the number of rows, their length and type, the device's SM count, ears_set_row_cluster and the row's start within 16
 * bytes: the same row may come out with other last bits in a larger batch or at another address.
 */
#define EARS_MAX_TOP 128
#define EARS_MAX_DISTILL_V (1 << 20)
enum { EARS_DISTILL_FORWARD_KL = 0, EARS_DISTILL_REVERSE_KL = 1, EARS_DISTILL_JSD = 2 };

/*
 * The k largest logits of every row (1 <= k <= EARS_MAX_TOP) in descending order, equal ones by ascending
 * index: out_values, out_ids [B R, k]; and out_lse [B R] = ln sum_v exp(l_v / temperature).  Entries of
 * -inf are never listed: where fewer than k are finite the rest is id -1, value -inf.
 * accept_len [B], optional: the lengths a verification call reported.  Rows k > accept_len[b], which lie
 * behind the first rejection (all rows of an invalid sequence, -1), are left out: ids -1, values and lse -inf.
 * A row that cannot be used has ids -1, values -inf and a NaN lse.
 */
int ears_top_logits(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                    double temperature, const float* seq_temperature, const int32_t* accept_len, int k,
                    float* out_values, int32_t* out_ids, float* out_lse, int32_t* status, void* stream);

/*
 * Log probability of one token per row, and optionally the row's entropy (nats):
 *   out_logp = l_x / T - ln sum exp(l / T),   out_entropy = -sum q ln q.
 * tokens [B R] int32; -1 leaves the row out (out_tokens of a verification call serves as it is).
 * The backward call adds d_logp[r] (1[v = x] - q_v) / T - d_entropy[r] q_v (ln q_v + H) / T; d_entropy is
 * optional, and needs `saved` of a call that returned the entropy.  The step call does both at once for
 * upstream gradients that are known beforehand (d_logp = -weight is the cross entropy).
 */
int ears_token_logprobs(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                        double temperature, const float* seq_temperature, const int32_t* tokens,
                        float* out_logp, float* out_entropy, float* out_saved, int32_t* status, void* stream);
int ears_token_logprobs_backward(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                                 double temperature, const float* seq_temperature, const int32_t* tokens, const float* saved,
                                 const float* d_logp, const float* d_entropy, void* out_grad, int64_t grad_stride_b,
                                 int64_t grad_stride_r, int32_t* status, void* stream);
int ears_token_logprobs_step(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                             double temperature, const float* seq_temperature, const int32_t* tokens, const float* d_logp,
                             const float* d_entropy, float* out_logp, float* out_entropy, void* out_grad,
                             int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream);

/*
 * Clipped policy loss per token, with rho = exp(logp - old_logp), logp as above:
 *   loss = -min(rho A, clip(rho, 1 - clip_low, 1 + clip_high) A) + kl_coef kl - entropy_coef H,
 *   kl   = exp(ref_logp - logp) - (ref_logp - logp) - 1     (0 without ref_logp; kl_coef > 0 needs it; with kl_coef = 0
 *          it is reported and enters neither the loss nor the gradient, infinite or not).
 * tokens, old_logp, ref_logp, advantage [B R]; token -1 leaves the row out.  out_logp, out_kl and out_entropy
 * are optional (not differentiated).  Where the clipped branch is taken the ratio's gradient is 0; on a tie
 * it is the unclipped branch's.  The gradient is that of sum_r w_r loss_r with w = d_loss (backward) or
 * row_weight (step; NULL: 1).  A row whose loss or gradient is not finite counts as unusable.
 */
int ears_policy_loss(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                     double temperature, const float* seq_temperature, const int32_t* tokens, const float* old_logp,
                     const float* ref_logp, const float* advantage, double clip_low, double clip_high, double kl_coef,
                     double entropy_coef, float* out_loss, float* out_logp, float* out_kl, float* out_entropy,
                     float* out_saved, int32_t* status, void* stream);
int ears_policy_backward(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                         double temperature, const float* seq_temperature, const int32_t* tokens, const float* old_logp,
                         const float* ref_logp, const float* advantage, double clip_low, double clip_high, double kl_coef,
                         double entropy_coef, const float* saved, const float* d_loss, void* out_grad,
                         int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream);
int ears_policy_step(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                     double temperature, const float* seq_temperature, const int32_t* tokens, const float* old_logp,
                     const float* ref_logp, const float* advantage, double clip_low, double clip_high, double kl_coef,
                     double entropy_coef, const float* row_weight, float* out_loss, float* out_logp, float* out_kl,
                     float* out_entropy, void* out_grad, int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status,
                     void* stream);

/*
 * Divergence of a draft row's distribution q (at `temperature`) from a teacher given by its top logits:
 * values, ids [B R, k] and, optionally, lse [B R] (its log normaliser at the same temperature), as
 * ears_top_logits writes them.  With lse, p_j = exp(value_j / T - lse) for the listed entries and everything
 * else is one outcome of mass max(1 - sum p_j, 2^-20) (2^-20: what a 32-bit lse resolves; 0 if the draft has
 * no mass outside the list either); without it the listed entries are renormalised and the rest has mass 0.
 *   EARS_DISTILL_FORWARD_KL   sum p ln(p / q)
 *   EARS_DISTILL_REVERSE_KL   sum q ln(q / p)                     (needs lse: infinite otherwise)
 *   EARS_DISTILL_JSD          mix sum p ln(p / m) + (1 - mix) sum q ln(q / m), m = mix p + (1 - mix) q, 0 < mix < 1
 * over the k + 1 outcomes.  An entry is absent when its id is -1 or its value -inf; a row without any is left
 * out.  A list that names an id twice, an id outside [0, V), or a value of NaN or +inf make the row unusable.
 * V <= EARS_MAX_DISTILL_V.  The gradient is that of sum_r w_r loss_r with w = d_loss (backward) or row_weight
 * (step; NULL: 1); rows of weight 0 get zeros.
 */
int ears_distill_loss(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                      double temperature, const float* seq_temperature, int k, const float* values, const int32_t* ids,
                      const float* lse, int kind, double mix, float* out_loss, float* out_saved, int32_t* status, void* stream);
int ears_distill_backward(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                          double temperature, const float* seq_temperature, int k, const float* values, const int32_t* ids,
                          const float* lse, int kind, double mix, const float* saved, const float* d_loss, void* out_grad,
                          int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream);
int ears_distill_step(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                      double temperature, const float* seq_temperature, int k, const float* values, const int32_t* ids,
                      const float* lse, int kind, double mix, const float* row_weight, float* out_loss, void* out_grad,
                      int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream);

/*
 * CTAs per row of the operators above, for tests and measurements: 1, 2, 4, 8 or 16; 0 = automatic.
 * Results differ only through floating-point summation order.  (0 may give short rows to a warp or to 128 threads.)
 */
int ears_set_row_cluster(int cluster);

/*
 * ---- A key/value cache held in 4 bits -----------------------------------------------------------------
 *
 * What stands before a verification step and after it: the forward pass whose logits the step verifies writes the
 * K + 1 newest tokens of every sequence into the cache (ears_kv_write) and attends from them over it
 * (ears_kv_attention); of those tokens the step keeps accept_len + 1, so that `start` of the next pass is
 * start + accept_len + 1 (an unusable sequence, accept_len -1, stays where it is).  What was written behind is
 * overwritten by the next pass and never seen.  Serving only: nothing here has a gradient.
 *
 * The cache is a pool of pages of page_size tokens (a multiple of 16), keys and values of all heads:
 *   codes   uint8 [pages, 2, heads, page_size, head_dim / 2]: 0 keys, 1 values; two codes a byte, the even
 *           dimension's in the low half
 *   params  bfloat16 [pages, 2, heads, page_size, head_dim / EARS_KV_GROUP, 2]: scale s and minimum m of each group
 *           of EARS_KV_GROUP = 64 consecutive dimensions; a code c stands for m + s c
 * 4.5 bits a value; both 16-byte aligned and contiguous.  head_dim is 64, 128 or 256.
 * Writing a group x: m = min x rounded down to bfloat16; s = (max x - m) r in 32 bits, r the 32-bit number nearest
 * to 1 / 15 (it lies above), rounded up to bfloat16, at least 2^-126; c = (x - m) / s, the difference rounded to 32 bits, to the nearest whole number, ties to even.  A value comes back
 * within s / 2 of what was written.  A group with a NaN or an infinity, or whose range overflows 32 bits, reads back as NaN.
 *
 * Common arguments:
 *   page_table   [B, table_width] int32, rows table_stride apart: token t of sequence b lies in page
 *                page_table[b, t / page_size], place t % page_size.  Sequences may share pages that are only read; two
 *                tokens written to the same place by one call leave either there, or codes of one and scales of the other.
 *   start        [B] int32: position i of the call is token start[b] + i.
 *   counts       [B] int32 or NULL: positions i >= counts[b] are left out (NULL, or more than Q: none is).
 *   strides      in elements, >= 0; the head_dim elements of a head are contiguous.  Any alignment of at least the
 *                element size serves; starts on 16 bytes are fetched at full speed.
 *   status       as above: EARS_DEV_INVALID_INPUT where a position lies outside the table, or a page outside the pool.
 * Every address is formed in 64 bits.  A position outside is not written and reads as NaN.  In ears_kv_attention a page outside the pool
 * makes NaN of the rows that see one of its tokens; a position outside the table (start[b] < 0, or start[b] + counts[b] past its end) makes NaN
 * of ALL rows of its sequence: a pass whose last positions have no place leaves them out by counts.
 * The calls allocate nothing and may be recorded into CUDA graphs and run side by side on any streams, as long as calls
 * that overlap have workspaces of their own.
 */
#define EARS_KV_GROUP 64
typedef struct {
    void* codes;
    void* params;
    int pages;       /* in the pool */
    int heads;
    int page_size;   /* tokens, a multiple of 16 */
    int head_dim;
} ears_kv_cache;

/* Quantises keys and values [B, Q, heads, head_dim] of type `dtype` into the cache. */
int ears_kv_write(int dtype, const ears_kv_cache* cache, const void* k, const void* v, int B, int Q, int64_t k_stride_b, int64_t k_stride_q,
                  int64_t k_stride_h, int64_t v_stride_b, int64_t v_stride_q, int64_t v_stride_h, const int32_t* page_table,
                  int table_width, int64_t table_stride, const int32_t* start, const int32_t* counts, int32_t* status, void* stream);

/* The values m + s c of Q tokens per sequence, in 32 bits and rounded once to `dtype`: out_k, out_v [B, Q, heads, head_dim],
   contiguous, 16-byte aligned.  Positions that are left out are zeros.  A value that rounds past the type's largest is infinite: within s / 2
   of it, what is read can lie beyond where what was written did not (-65504 in half precision, stored as a minimum of -65536). */
int ears_kv_read(int dtype, const ears_kv_cache* cache, int B, int Q, const int32_t* page_table, int table_width, int64_t table_stride,
                 const int32_t* start, const int32_t* counts, void* out_k, void* out_v, int32_t* status, void* stream);

/*
 * Attention of Q positions per sequence, whose own tokens are in the cache already: position i, at p = start[b] + i, sees
 * the tokens t <= p, and of those, with window > 0, the last `window` (t > p - window) and the first `sinks` (t < sinks).
 *   out = sum_t softmax_t(scale q . k_t) v_t,    out_lse = ln sum_t exp(scale q . k_t)   (optional)
 * q [B, Q, heads_q, head_dim] bfloat16 or half precision; query head n reads head n / (heads_q / cache->heads).  out, of q's type,
 * [B, Q, heads_q, head_dim] contiguous, 16-byte aligned; out_lse [B, Q, heads_q].  They must not overlap the inputs.
 * Positions that are left out get zeros and -inf.  A NaN or infinity in a row of q, or a NaN (of values, an infinity too) read from a token
 * that it sees, makes that row and its out_lse NaN, in all dimensions, and no other.
 * Scores, their sums (n / 32 weights one after the other, for n tokens) and the results are kept in 32 bits; q is taken as it is, or, where its
 * row spans more than 2^25, to within 2^-26 of the row's largest element.  Weights times scales, p s, enter the second product in half precision,
 * whose range follows the row's and group's own products: of sum_t p_t s_t c_t that and the product lose at most 2^-11 of it and 2^-10 of
 * 7.5 sum_t p_t s_t, whatever scales there are in other groups or in tokens that weigh nothing or are not seen.  For half-precision q what
 * rounding loses is added back times the middle code: 2^-10 of 7.5 sum_t p_t s_t are left.  Values between 2^-86 and the type's largest; weights
 * below 2^-95 of a row's largest are none.
 * workspace: ears_kv_attention_workspace_bytes for the same arguments on the same device (0: they would be refused), 256-byte
 * aligned; its contents before and after mean nothing.  It does not grow with the lengths.  The same call on the same kind of
 * device gives the same bits; a row's may differ with what else is in the batch (the order of its sums).
 * Made for few positions (Q x heads_q / heads up to some tens): more are right, and read the cache once for every 8 to 32 rows.
 * How rows are cut into blocks, and how many CTAs there are, goes by table_width (or a window), not by the lengths, which the host does not
 * know: in a table much wider than its sequences small calls take longer (5 positions of one sequence, 32 / 8 heads of 128, in a
 * table for 131072 tokens: 1000 tokens 13.8 us instead of 12.3, 4000 tokens 20.6 instead of 14.9).
 */
size_t ears_kv_attention_workspace_bytes(int dtype, const ears_kv_cache* cache, int B, int Q, int heads_q, int table_width, int window, int sinks);
int ears_kv_attention(int dtype, const ears_kv_cache* cache, const void* q, int B, int Q, int heads_q, int64_t q_stride_b, int64_t q_stride_q,
                      int64_t q_stride_h, const int32_t* page_table, int table_width, int64_t table_stride, const int32_t* start,
                      const int32_t* counts, double scale, int window, int sinks, void* out, float* out_lse, void* workspace,
                      size_t workspace_bytes, int32_t* status, void* stream);

const char* ears_status_string(int status);
const char* ears_last_cuda_error(void); /* text of the last failing CUDA call on this thread, or "" */
int ears_version(void);

/* Frees every library-owned workspace and staging buffer (synchronises the devices used). */
void ears_shutdown(void);

#ifdef __cplusplus
}
#endif
#endif /* EARS_H */
