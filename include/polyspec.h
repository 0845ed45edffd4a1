/*
 * polyspec.h -- C ABI of libpolyspec: the chained speculative-sampling verification
 * step of polybasic speculative decoding, as CUDA kernels for sm_100a.
 *
 * Vocabulary of the paper (Section 3.1, Problem Formulation): a chain of models
 * M_1 (the target) ... M_n (the smallest drafter); p_i(x | x_<=t) is model i's
 * distribution over the vocabulary at a position; M_n drafts a block of tokens that is
 * checked bottom-up, by M_{n-1} first and M_1 last; the acceptance length of a
 * verifier (Eq. 1) is the number of consecutive block tokens it accepts.  A *level* is
 * one adjacent pair: verifier M_l checking the token stream handed up by M_{l+1}.
 *
 * The rule at a level (Algorithm 1: Verify in the inner loop with a break at the first
 * failure, then VerifyBlock / SampleOne for the level above; the rule itself is
 * speculative sampling, Sections 2 and 3.1):
 *   P_j = softmax(logits_p[j] / T), Q_j = softmax(logits_q[j] / T);
 *   position j is accepted iff  u_j * Q_j(x_j) <= P_j(x_j)   (u_j <= min(1, P/Q));
 *   accepted_len = a = number of accepted positions before the first rejection;
 *   next_token   = inverse CDF at the sampling uniform of
 *                    normalised max(0, P_{a+1} - Q_{a+1})   if a < block_len (residual)
 *                    P_{block_len+1}                         if a = block_len (bonus row),
 *                  in ascending vocabulary order, first v whose running sum exceeds u * total.
 * The emitted stream (x_1..x_a, next_token) is what the next level up verifies, with
 * that level's q = this level's verifier rows.
 *
 * Conventions for every call
 *   - All pointers are DEVICE pointers owned by the caller unless a parameter says
 *     "host".  Logits buffers must be 16-byte aligned and V must be a multiple of 8 (the
 *     kernels read logits eight at a time; other V return POLYSPEC_ERR_UNSUPPORTED).
 *     Row-major, innermost dimension = vocabulary.
 *   - Calls only enqueue work on `cuda_stream` (a cudaStream_t passed as void*; NULL is
 *     the default stream) and return; outputs are valid once the stream has synchronised.
 *   - The library allocates no device memory: the caller passes a workspace of at least
 *     the size the matching *_workspace call reports, 256-byte aligned.  Concurrent calls
 *     need distinct workspaces.
 *   - Uniforms are caller-supplied floats in the open interval (0, 1); the library draws
 *     no random numbers.  Outputs are a pure function of the inputs.
 *   - Problems visible on the host (NULL pointers, sizes out of range, misalignment,
 *     temperature <= 0 or not finite, workspace too small) return an error status and
 *     launch nothing.  Problems only visible on the device (a token outside [0, V), a row
 *     holding NaN / +inf or no finite logit) never trap: the affected sequence gets
 *     accepted_len = next_token = -1 (and -1 in every later level of a chain) and
 *     *device_status is set to POLYSPEC_ERR_BAD_INPUT_ON_DEVICE.
 *   - No kernel polls memory without a limit.  The kernels of the logits path wait on nothing but
 *     hardware barriers (block, cluster, grid dependency) that every participant reaches
 *     unconditionally.  The LM-head projection waits on its TMA copies and on the tensor core with
 *     bounded polls: should one ever run out, *device_status becomes POLYSPEC_ERR_TIMEOUT, the
 *     outputs of that call are undefined, and the kernel still returns.
 */
#ifndef POLYSPEC_H
#define POLYSPEC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define POLYSPEC_MAX_K       32   /* largest block a level may verify */
#define POLYSPEC_MAX_MODELS   8   /* largest chain */

typedef enum {
    POLYSPEC_OK = 0,
    POLYSPEC_ERR_INVALID_ARG = 1,
    POLYSPEC_ERR_UNSUPPORTED = 2,
    POLYSPEC_ERR_WORKSPACE = 3,
    POLYSPEC_ERR_CUDA = 4,
    POLYSPEC_ERR_TIMEOUT = 5,
    POLYSPEC_ERR_BAD_INPUT_ON_DEVICE = 6,
    POLYSPEC_ERR_SCRATCH_LIMIT = 7,     /* problem too large for the built-in scratch of a *_static call */
    POLYSPEC_ERR_NO_PAGES = 8           /* a cache pool has too few free pages (reported on the device) */
} polyspec_status;

typedef enum { POLYSPEC_F32 = 0, POLYSPEC_BF16 = 1 } polyspec_dtype;

/* Static strings; never NULL. */
const char* polyspec_status_string(polyspec_status s);
/* major * 10000 + minor * 100 + patch */
int polyspec_version(void);
/* The CUDA runtime's message for the most recent call that returned POLYSPEC_ERR_CUDA ("no error" if none did).
 * Static string; not synchronised between host threads. */
const char* polyspec_last_cuda_error(void);

/*
 * polyspec_verify_level -- one adjacent pair (verifier p, drafter-side q) over a batch of
 * independent sequences: Algorithm 1's Verify loop plus the replacement / bonus token.
 *
 *   logits_p      [B, k+1, V]  verifier logits; row j scores block position j, row k is the bonus row
 *   logits_q      [B, k,   V]  logits of the distribution the block tokens were drawn from
 *   draft_tokens  [B, k]       block tokens, each in [0, V)
 *   uniforms      [B, k+1]     [b, j<k] accept uniform of position j; [b, k] the sampling uniform
 *   block_len     [B] or NULL  tokens actually presented per sequence (0..k); NULL means k
 *   accepted_len  out [B]      0..block_len[b]
 *   next_token    out [B]      residual sample if accepted_len < block_len, else bonus sample
 *   p_at_draft, q_at_draft  out [B, k] or NULL: P_j(x_j), Q_j(x_j) for j < block_len, 0 elsewhere
 *   device_status out [1] or NULL: left untouched when all is well (zero it before the call)
 */
polyspec_status polyspec_verify_level_workspace(int B, int k, int V, polyspec_dtype dt, size_t* bytes /* host out */);
polyspec_status polyspec_verify_level(
    const void* logits_p, const void* logits_q, const int32_t* draft_tokens, const float* uniforms,
    const int32_t* block_len, int B, int k, int V, polyspec_dtype dt, float temperature,
    int32_t* accepted_len, int32_t* next_token, float* p_at_draft, float* q_at_draft,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * polyspec_verify_chain -- n models, n-1 levels, verified bottom-up in one call
 * (Section 3.1; Algorithm 1 is the n = 3 case).  Level index l = 0 .. n-2: verifier is
 * models[l]; models[0] = M_1 (target), models[n-1] = M_n (bottom drafter).
 *
 *   models        host array [n_models]: device pointer to [B, rows, V] logits and its row
 *                 count; rows >= k[l] + 1 for l < n-1, rows >= k[n-2] for the drafter
 *   k             host [n_models-1]; k[l] = largest block level l verifies; k[n-2] = draft length
 *   draft_tokens  [B, k[n-2]]
 *   uniforms      [n_models-1, B, kmax+1], kmax = max k[l]; level l uses [l, b, j < k[l]] for
 *                 its accept tests and [l, b, kmax] as its sampling uniform
 *   Level l verifies the first min(k[l], out_len[l+1]) tokens of the stream emitted by
 *   level l+1 against q = models[l+1]'s rows.
 *   accepted_len, block_len, out_len   out [n_models-1, B]; out_len = accepted_len + 1
 *   out_tokens    out [n_models-1, B, kmax+1]: stream emitted by each level, -1 past out_len;
 *                 level 0's stream is the committed output
 */
typedef struct {
    const void* logits;   /* device pointer, [B, rows, V] */
    int rows;
} polyspec_model_logits;

polyspec_status polyspec_verify_chain_workspace(int n_models, const int* k /* host */, const int* rows /* host [n_models] */,
                                                int B, int V, polyspec_dtype dt, size_t* bytes /* host out */);
polyspec_status polyspec_verify_chain(
    const polyspec_model_logits* models /* host */, int n_models, const int* k /* host */,
    const int32_t* draft_tokens, const float* uniforms, int B, int V, polyspec_dtype dt, float temperature,
    int32_t* accepted_len, int32_t* block_len, int32_t* out_tokens, int32_t* out_len,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The two halves of polyspec_verify_chain, for callers that want to time or overlap them:
 *   polyspec_chain_row_stats  the temperature-softmax normaliser of every row of every model
 *                             (the single pass over all logits; Section 3.1's p_i over the
 *                             vocabulary) written to the workspace;
 *   polyspec_chain_walk       everything after it (Algorithm 1's accept loop, first rejection,
 *                             replacement / bonus token, hand-off between levels), reading the
 *                             workspace the first half filled on the same stream.
 * Calling one after the other with the same arguments is exactly polyspec_verify_chain.
 */
polyspec_status polyspec_chain_row_stats(
    const polyspec_model_logits* models /* host */, int n_models, const int* k /* host */, int B, int V,
    polyspec_dtype dt, float temperature, int32_t* device_status, void* workspace, size_t workspace_bytes,
    void* cuda_stream);
polyspec_status polyspec_chain_walk(
    const polyspec_model_logits* models /* host */, int n_models, const int* k /* host */,
    const int32_t* draft_tokens, const float* uniforms, int B, int V, polyspec_dtype dt, float temperature,
    int32_t* accepted_len, int32_t* block_len, int32_t* out_tokens, int32_t* out_len,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * polyspec_verify_chain_host -- the same call for a caller whose buffers live in HOST
 * memory (pinned memory makes the copies asynchronous): logits, draft tokens and
 * uniforms are copied to a device staging area inside the caller's workspace, the chain
 * runs, and the four outputs are copied back, all on `cuda_stream`.  Every data pointer
 * here is a host pointer with the layouts above; `host_status` (host, [1], may be NULL)
 * receives the device status word.  Outputs are valid after the stream synchronises.
 */
polyspec_status polyspec_verify_chain_host_workspace(int n_models, const int* k, const int* rows, int B, int V,
                                                     polyspec_dtype dt, size_t* bytes /* host out */);
polyspec_status polyspec_verify_chain_host(
    const polyspec_model_logits* models_host /* host array of HOST logits pointers */, int n_models, const int* k,
    const int32_t* draft_tokens_host, const float* uniforms_host, int B, int V, polyspec_dtype dt, float temperature,
    int32_t* accepted_len_host, int32_t* block_len_host, int32_t* out_tokens_host, int32_t* out_len_host,
    int32_t* host_status, void* workspace /* device */, size_t workspace_bytes, void* cuda_stream);

/*
 * polyspec_verify_from_hidden -- polyspec_verify_level with the LM-head projection fused
 * in front (the last op of the model forwards in Algorithm 1, "p_{1:K} <- M_2(...)" and
 * "v <- M_1(...)"): logits[b, j, v] = sum_d hidden[b, j, d] * W[v, d], bf16 inputs,
 * fp32 accumulation on the tensor cores; logits are never passed in.
 *
 *   hidden_p [B, k+1, d_p] bf16, W_p [V, d_p] bf16 (row-major, d contiguous)
 *   hidden_q [B, rows_q, d_q] bf16 with rows_q = k or k + 1 (a row k is projected but not used), W_q [V, d_q] bf16
 *   d_p, d_q multiples of 64; V a multiple of 8; all four buffers 16-byte aligned
 *   the remaining arguments are those of polyspec_verify_level
 */
polyspec_status polyspec_verify_from_hidden_workspace(int B, int k, int V, int d_p, int d_q, size_t* bytes /* host out */);
polyspec_status polyspec_verify_from_hidden(
    const void* hidden_p, const void* W_p, const void* hidden_q, const void* W_q, int rows_q,
    const int32_t* draft_tokens, const float* uniforms, const int32_t* block_len,
    int B, int k, int V, int d_p, int d_q, float temperature,
    int32_t* accepted_len, int32_t* next_token, float* p_at_draft, float* q_at_draft,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * polyspec_verify_chain_greedy -- the chain under greedy matching, the other verification rule
 * Section 3.1 names and Section 4.5 compares with speculative sampling: a block token is accepted
 * iff it is the verifier's most likely token at its position (first index on ties), the loop breaks
 * at the first mismatch, and the token emitted after the accepted prefix is the verifier's most
 * likely token there (at the first mismatch, or in the bonus row after a fully accepted block).
 * No uniforms, no temperature; the emitted stream of a level is that verifier's own greedy text.
 *
 *   models, k, draft_tokens and the four outputs are those of polyspec_verify_chain; only the
 *   verifiers models[0 .. n_models-2] are read (rows >= k[l] + 1); models[n_models-1].logits may be
 *   NULL.  One pass over the verifiers' logits, no second pass.
 */
polyspec_status polyspec_verify_chain_greedy_workspace(int n_models, const int* k /* host */, const int* rows /* host [n_models] */,
                                                       int B, int V, polyspec_dtype dt, size_t* bytes /* host out */);
polyspec_status polyspec_verify_chain_greedy(
    const polyspec_model_logits* models /* host */, int n_models, const int* k /* host */, const int32_t* draft_tokens,
    int B, int V, polyspec_dtype dt,
    int32_t* accepted_len, int32_t* block_len, int32_t* out_tokens, int32_t* out_len,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The two halves of polyspec_verify_from_hidden, for callers that want to time or overlap them:
 *   polyspec_from_hidden_project  both LM-head projections (one launch): logits and, from the same
 *                                 accumulators, every row's softmax-normaliser partials into the workspace;
 *   polyspec_from_hidden_verify   everything after it, reading the workspace the first half filled
 *                                 on the same stream.
 * Calling one after the other with the same sizes and workspace is exactly polyspec_verify_from_hidden.
 */
polyspec_status polyspec_from_hidden_project(
    const void* hidden_p, const void* W_p, const void* hidden_q, const void* W_q, int rows_q,
    int B, int k, int V, int d_p, int d_q, float temperature, int32_t* device_status, void* workspace, size_t workspace_bytes,
    void* cuda_stream);
polyspec_status polyspec_from_hidden_verify(
    int rows_q, const int32_t* draft_tokens, const float* uniforms, const int32_t* block_len,
    int B, int k, int V, int d_p, int d_q, float temperature,
    int32_t* accepted_len, int32_t* next_token, float* p_at_draft, float* q_at_draft,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * polyspec_lm_head -- the projection of polyspec_verify_from_hidden on its own (the last op
 * of a model forward in Algorithm 1): logits[r, v] = sum_d hidden[r, d] * W[v, d].
 *
 *   hidden  [rows, d] bf16, W [V, d] bf16, both row-major and 16-byte aligned; d a multiple of 64,
 *           V a multiple of 4
 *   logits  out [rows, V] fp32, 16-byte aligned
 *   No workspace.  device_status as above (only POLYSPEC_ERR_TIMEOUT can be reported here).
 */
polyspec_status polyspec_lm_head(const void* hidden, const void* W, int rows, int V, int d, float* logits,
                                 int32_t* device_status, void* cuda_stream);

/*
 * polyspec_verify_level with the vocabulary sharded over n_ranks ranks (the layout a tensor-parallel
 * LM head leaves the logits in): rank r holds entries [r * V_local, (r + 1) * V_local) of every row,
 * as logits_p [B, k+1, V_local] and logits_q [B, k, V_local]; the rule is Algorithm 1's Verify loop
 * and replacement / bonus token over the whole vocabulary V = n_ranks * V_local, unchanged.
 * The normaliser, the accept tests and the inverse-CDF search need sums over all slices, so a level
 * is three calls per rank with two small exchanges and one reduction between them, which the caller
 * performs (all-gather, all-gather, max); the library itself never talks to another rank:
 *
 *   polyspec_sharded_level_stats   writes this rank's stats record (stats_record_bytes)
 *        -- all-gather the records into [n_ranks][stats_record_bytes], rank order --
 *   polyspec_sharded_level_decide  accept tests on every rank (identical results): accepted_len [B];
 *                                  writes this rank's mass record (mass_record_bytes)
 *        -- all-gather the mass records into [n_ranks][mass_record_bytes] --
 *   polyspec_sharded_level_pick    next_token [B]: the token (index in the whole vocabulary) on the one
 *                                  rank whose slice contains it, -1 on the others
 *        -- max over ranks of next_token --
 *
 *   draft_tokens [B, k] hold indices in the whole vocabulary; uniforms, block_len, accepted_len,
 *   p_at_draft, q_at_draft, temperature and device_status are those of polyspec_verify_level and must be
 *   the same on every rank.  The three calls of a level share one workspace, whose contents carry from
 *   call to call; records are opaque, 16-byte aligned device buffers.  V_local a multiple of 8,
 *   n_ranks <= 64.  An unusable input gives accepted_len = next_token = -1 on every rank.
 *   With n_ranks = 1 the result is bit-identical to polyspec_verify_level.
 */
polyspec_status polyspec_sharded_level_sizes(int B, int k, int V_local, polyspec_dtype dt, int n_ranks,
                                             size_t* workspace_bytes, size_t* stats_record_bytes,
                                             size_t* mass_record_bytes /* host out, all three */);
polyspec_status polyspec_sharded_level_stats(
    const void* logits_p, const void* logits_q, const int32_t* draft_tokens, int B, int k, int V_local, int rank, int n_ranks,
    polyspec_dtype dt, float temperature, void* stats_record /* out */, int32_t* device_status,
    void* workspace, size_t workspace_bytes, void* cuda_stream);
polyspec_status polyspec_sharded_level_decide(
    const void* logits_p, const void* logits_q, const int32_t* draft_tokens, const float* uniforms, const int32_t* block_len,
    int B, int k, int V_local, int rank, int n_ranks, polyspec_dtype dt, float temperature,
    const void* stats_records /* all ranks' */, int32_t* accepted_len, float* p_at_draft, float* q_at_draft,
    void* mass_record /* out */, int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);
polyspec_status polyspec_sharded_level_pick(
    const void* logits_p, const void* logits_q, const float* uniforms, int B, int k, int V_local, int rank, int n_ranks,
    polyspec_dtype dt, float temperature, const void* mass_records /* all ranks' */, int32_t* next_token,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * polyspec_verify_chain with the vocabulary sharded over n_ranks ranks: every model's logits as
 * [B, rows, V_local] slices (models[i].logits, models[i].rows as in polyspec_verify_chain), levels verified
 * bottom-up (Section 3.1).  One stats call covers every row of every model; each level then takes a
 * gather call (the logits at its block tokens, which only exist once the level below is done), decide
 * and pick as in the single-level calls, and a hand-off that turns (accepted length, token) into the
 * block of the level above.  Per chain: all-gather of the stats records; per level, for
 * level = n_models-2 down to 0: all-gather of the gather records, all-gather of the mass records, max of
 * next_token, then polyspec_sharded_chain_handoff on every rank.
 *
 *   block_tokens [B, kmax+1], block_len [B]: the block the current level verifies, the same on every
 *       rank; the caller fills them with the draft tokens and k[n_models-2] (or fewer) before the
 *       bottom level, the hand-off rewrites them for the level above (block_len -1: unusable input below)
 *   uniforms [n_models-1, B, kmax+1], accepted_len, block_len_out, out_tokens, out_len: those of
 *       polyspec_verify_chain (block_len_out is its block_len output); each call touches its level's part
 *   With n_ranks = 1 the four outputs are bit-identical to polyspec_verify_chain's.
 */
polyspec_status polyspec_sharded_chain_sizes(int n_models, const int* k /* host */, const int* rows /* host [n_models] */, int B,
                                             int V_local, polyspec_dtype dt, int n_ranks, size_t* workspace_bytes,
                                             size_t* stats_record_bytes, size_t* gather_record_bytes,
                                             size_t* mass_record_bytes /* host out, all four */);
polyspec_status polyspec_sharded_chain_stats(
    const polyspec_model_logits* models /* host */, int n_models, const int* k /* host */, int B, int V_local, int rank, int n_ranks,
    polyspec_dtype dt, float temperature, void* stats_record /* out */, int32_t* device_status,
    void* workspace, size_t workspace_bytes, void* cuda_stream);
polyspec_status polyspec_sharded_chain_gather(
    const polyspec_model_logits* models, int n_models, const int* k, int level, const int32_t* block_tokens, const int32_t* block_len,
    int B, int V_local, int rank, int n_ranks, polyspec_dtype dt, void* gather_record /* out */,
    void* workspace, size_t workspace_bytes, void* cuda_stream);
polyspec_status polyspec_sharded_chain_decide(
    const polyspec_model_logits* models, int n_models, const int* k, int level, const int32_t* block_tokens, const int32_t* block_len,
    const float* uniforms, int B, int V_local, int rank, int n_ranks, polyspec_dtype dt, float temperature,
    const void* stats_records /* all ranks' */, const void* gather_records /* all ranks' */, int32_t* accepted_len,
    int32_t* block_len_out, void* mass_record /* out */, int32_t* device_status, void* workspace, size_t workspace_bytes,
    void* cuda_stream);
polyspec_status polyspec_sharded_chain_pick(
    const polyspec_model_logits* models, int n_models, const int* k, int level, const float* uniforms, int B, int V_local, int rank,
    int n_ranks, polyspec_dtype dt, float temperature, const void* mass_records /* all ranks' */, int32_t* next_token /* [B] */,
    int32_t* device_status, void* workspace, size_t workspace_bytes, void* cuda_stream);
polyspec_status polyspec_sharded_chain_handoff(
    int n_models, const int* k, int level, int B, const int32_t* accepted_len, const int32_t* next_token /* after the max */,
    int32_t* block_tokens /* in/out */, int32_t* block_len /* in/out */, int32_t* out_tokens, int32_t* out_len, void* cuda_stream);

/*
 * Cost model of Section 3.2 (host arithmetic only; nothing is launched).
 *
 * polyspec_cost_total_time -- Lemma 3.1 (Eq. 3): the time to generate N tokens with n models,
 *     T = sum_{i=1}^{n-1} (N / L_i) T_i + beta (N / L_{n-1}) T_n,
 *   T[0..n-1] the forward-pass costs T_1..T_n, L[0..n-2] the acceptance lengths L_1..L_{n-1} (Eq. 1:
 *   what polyspec_verify_chain reports as accepted_len, averaged), beta the drafter's scaling factor.
 *   Returns NaN for n < 2, a NULL array or a non-positive L.
 * polyspec_cost_insertion -- Theorem 3.2, first condition, with the quantities of Table 1: inserting
 *   M_new between M_i and M_{i+1} pays off iff
 *     T_new / T_i  <  L_new (1 / L_i - 1 / L_{i-new}),
 *   L_i the acceptance length of the pair (M_i, M_{i+1}) before the insertion, L_{i-new} that of
 *   (M_i, M_new) and L_new that of (M_new, M_{i+1}) after it.  Writes both sides (either pointer may be
 *   NULL) and returns 1 if the condition holds, 0 if not, -1 on non-positive inputs.
 * polyspec_cost_insertion_drafter -- Theorem 3.2, second condition, as its proof derives it (the three-model
 *   case, M_new between M_i and the drafter M_{i+1}): the insertion also pays off if
 *     T_new / T_{i+1}  <  beta (L_new / L_i - 1),
 *   the sign of the last two terms of the difference of the two Lemma 3.1 totals; L_new and L_i as above,
 *   T_{i+1} the drafter's forward-pass cost, beta its scaling factor (Lemma 3.1).  The theorem's statement
 *   prints other subscripts for this condition; the proof's are used.  Same outputs and return values.
 */
double polyspec_cost_total_time(int n, const double* T /* host [n] */, const double* L /* host [n-1] */, double beta, double N);
int polyspec_cost_insertion(double T_new, double T_i, double L_new, double L_i, double L_i_new,
                            double* lhs /* host out */, double* rhs /* host out */);
int polyspec_cost_insertion_drafter(double T_new, double T_next, double L_new, double L_i, double beta,
                                    double* lhs /* host out */, double* rhs /* host out */);

/*
 * Staged verification with a threshold (Section 3.3, "Staged Verification"; Algorithm 1, three models)
 * for a batch of independent sequences.  Algorithm 1's loop: M_3 drafts K tokens, M_2 verifies them, what
 * M_2 hands on joins `accepted` (count `cnt`); once cnt >= mu, M_1 verifies the accumulated block in one
 * pass, the verified part is committed, t advances, `accepted` and cnt are reset.  Each M_2 round hands on
 * its whole emitted stream (accepted prefix plus the replacement or bonus token), which is distributed as
 * M_2's own samples, so the pass of M_1 verifies it against q = M_2's rows and the committed text keeps
 * M_1's distribution; a round therefore always adds a token.  Accumulation also stops when one more round
 * might not fit the largest block a level verifies (cnt + K + 1 > POLYSPEC_MAX_K).
 *
 * The two verifications of an iteration are ordinary polyspec_verify_level calls (per-sequence block_len);
 * these calls keep the loop's bookkeeping on the device, so that the loop needs no host read-back per step:
 *
 *   polyspec_staged_init          zeroes the state, remaining = B
 *   per iteration of Algorithm 1's loop, for all sequences at once:
 *     polyspec_staged_round_begin   -> pos2 [B] (= t + cnt), tokens2 [B, K] (M_3's drafts there), uniforms2 [B, K+1],
 *                                      block_len2 [B] (K, or 0 for a sequence that is finished)
 *       -- caller: logits of M_2 at positions pos2 .. pos2+K and of M_3 at pos2 .. pos2+K-1 (the model forwards),
 *          then polyspec_verify_level(M_2 rows, M_3 rows, tokens2, uniforms2, block_len2) -> accepted_len2, next_token2 --
 *     polyspec_staged_accumulate    appends each round's stream; where cnt >= mu (or the block is full): pos1 [B] (= t),
 *                                      tokens1 [B, kcap] (= accepted), uniforms1 [B, kcap+1], block_len1 [B] (= cnt);
 *                                      block_len1 = 0 elsewhere
 *       -- caller: logits of M_1 at pos1 .. pos1+kcap and of M_2 at pos1 .. pos1+kcap-1, then
 *          polyspec_verify_level(M_1 rows, M_2 rows, tokens1, uniforms1, block_len1) -> accepted_len1, next_token1 --
 *     polyspec_staged_commit        where block_len1 > 0: commits accepted[0 .. a1) and M_1's token, t += a1 + 1,
 *                                      cnt = 0; a sequence with n_tokens committed is finished
 *   *remaining (device) counts the sequences still running; a sequence needs at most mu iterations per pass of M_1,
 *   so reading it back once every mu iterations is at most one read-back per pass.
 *
 *   drafts [B, N] int32: M_3's proposal per position (synthetic stand-in: position-indexed);
 *   u2 [B, R, K+1]: row r serves a sequence's r-th round; u1 [B, C, POLYSPEC_MAX_K+1]: row c serves its c-th pass of
 *   M_1, slots 0..m-1 the accept tests, slot POLYSPEC_MAX_K the sampling uniform.
 *   State arrays (device, caller-owned): t, cnt, rounds, cycles, n_committed, done [B]; accepted [B, POLYSPEC_MAX_K];
 *   committed [B, cap] (-1 where nothing was committed); presented, per_cycle [B, C] (block length and tokens
 *   committed of each pass); remaining [1].  kcap >= min(POLYSPEC_MAX_K, mu + K).  done: 0 running, else a
 *   POLYSPEC_STAGED_* code (EXHAUSTED: out of positions N, of uniform rows R / C; BAD_INPUT: a level call reported -1).
 */
#define POLYSPEC_STAGED_FINISHED  1
#define POLYSPEC_STAGED_EXHAUSTED 2
#define POLYSPEC_STAGED_BAD_INPUT 3
typedef struct {
    int B, K, mu, kcap, N, R, C, cap, n_tokens;
    int32_t *t, *cnt, *rounds, *cycles, *n_committed, *done;
    int32_t *accepted, *committed, *presented, *per_cycle, *remaining;
} polyspec_staged_state;
polyspec_status polyspec_staged_init(const polyspec_staged_state* s /* host */, void* cuda_stream);
polyspec_status polyspec_staged_round_begin(const polyspec_staged_state* s /* host */, const int32_t* drafts, const float* u2,
                                            int32_t* pos2, int32_t* tokens2, float* uniforms2, int32_t* block_len2, void* cuda_stream);
polyspec_status polyspec_staged_accumulate(const polyspec_staged_state* s /* host */, const int32_t* tokens2, const int32_t* block_len2,
                                           const int32_t* accepted_len2, const int32_t* next_token2, const float* u1,
                                           int32_t* pos1, int32_t* tokens1, float* uniforms1, int32_t* block_len1, void* cuda_stream);
polyspec_status polyspec_staged_commit(const polyspec_staged_state* s /* host */, const int32_t* block_len1, const int32_t* accepted_len1,
                                       const int32_t* next_token1, void* cuda_stream);

/*
 * polyspec_lm_head_quantized -- polyspec_lm_head for a verifier whose LM head is held in 4 bits with group scales (the paper's M_2
 * is a 4-bit copy of M_1 with groups of 128, Section 4.1):
 *   logits[r, v] = sum_g scales[v, g] * sum_{k in group g} hidden[r, k] * (q[v, k] - z[v, g])
 *
 *   hidden       [rows, d] bf16, 16-byte aligned; any number of rows
 *   qweight      [V, d/8] 32-bit words, 16-byte aligned: word i of a row holds q[v, 8i .. 8i+7], weight 8i + e in the four
 *                bits from bit 4 * (e / 2) + 16 * (e % 2) on (polyspec_pack_quantized makes it from one code per byte)
 *   scales       [V, d/group] bf16; group 32, 64 or 128, d a multiple of group
 *   zero_points  [V, d/group] bytes, or NULL for 8 everywhere; the low four bits of a byte count
 *   logits       out [rows, V] fp32 or bf16 (logits_dt), 16-byte aligned; any V
 *   q - z is multiplied exactly, a group's sum and the sum over the groups are held in fp32; bf16 logits are rounded once.
 *   The result of a row does not depend on timing.  The order in which a logit's partial sums are added depends on the sizes: up to
 *   eight rows and above are two kernels, and up to eight rows it changes with V.  So a row in a larger batch, or a slice of the
 *   vocabulary, equals the whole within fp32 rounding, not bit for bit.
 *   No workspace; nothing outside [rows, V] is written.  device_status as in polyspec_lm_head.
 */
polyspec_status polyspec_pack_quantized(const void* codes /* [V, d] bytes, 16-byte aligned, low four bits count */, int V, int d /* a multiple of 32 */,
                                 void* qweight /* out [V, d/8] words */, void* cuda_stream);
polyspec_status polyspec_lm_head_quantized(const void* hidden, const void* qweight, const void* scales, const void* zero_points,
                                    int rows, int V, int d, int group, polyspec_dtype logits_dt, void* logits,
                                    int32_t* device_status, void* cuda_stream);

/*
 * polyspec_process_logits -- a request's sampling controls on the logits rows of a block, before they are verified: penalties
 * for repeated tokens, biases and allowed-token masks.  Every row of a block has a context of its own, the text so far and
 * the drafted tokens before the row, so row j of sequence b is controlled with history[b, 0 .. history_len) followed by
 * draft_tokens[b, 0 .. j); give the rows of every model of the chain the same controls, and the chain verifies controlled
 * distributions.  With n(v) the occurrences of v in that context behind the prompt:
 *     z1 = v occurs in the context ? (z > 0 ? z / repetition : z * repetition) : z
 *     z2 = n(v) > 0 ? z1 - frequency * n(v) - presence : z1
 *     z3 = z2 + the biases listed for v (a token listed twice counts twice)
 *     z4 = v allowed ? z3 : -inf            (whatever z3 is, NaN included)
 * in fp32, rounded once to the storage type.  Entries that no control touches keep their bits.  A row whose mask allows
 * nothing becomes -inf throughout, which the verification calls report as unusable.
 *
 *   logits [B, rows, V] fp32 or bf16, out [B, rows, V]: either the same buffer (in place) or one that does not overlap it;
 *   both 16-byte aligned, V a multiple of 8
 *   draft_tokens [B, k] or NULL (every row then has the history alone as its context), k <= POLYSPEC_MAX_K, rows <= k + 1
 *   controls (host struct of device pointers; a NULL pointer leaves that control out):
 *     history       [B, history_cap] token ids; history_len [B] (NULL: history_cap), prompt_len [B] (NULL: 0): the first
 *                   prompt_len tokens are the prompt, which counts for the repetition penalty only
 *     repetition, frequency, presence   [B] (NULL: 1, 0, 0); repetition > 0
 *     bias_tokens, bias_values          [B, n_bias]
 *     mask          [B, rows, ceil(V/32)] words: entry v is allowed iff bit v % 32 of word v / 32 is set
 *     vocab_begin, vocab_size           where the logits are one rank's slice of a sharded vocabulary: their first entry and
 *                   the whole size; token ids are always whole-vocabulary ids, mask bits are the slice's.  0, 0: not sharded
 *   A negative token id is padding and counts nowhere.  An id >= vocab_size, a length outside its bounds (it is clamped) or
 *   a repetition that is not > 0 (1 is used) sets *device_status to POLYSPEC_ERR_BAD_INPUT_ON_DEVICE.
 */
typedef struct {
    const int32_t* history;
    const int32_t* history_len;
    const int32_t* prompt_len;
    const float* repetition;
    const float* frequency;
    const float* presence;
    const int32_t* bias_tokens;
    const float* bias_values;
    const uint32_t* mask;
    int history_cap, n_bias, vocab_begin, vocab_size;
} polyspec_logit_controls;
polyspec_status polyspec_process_logits(const void* logits, const polyspec_logit_controls* controls /* host */, const int32_t* draft_tokens,
                                        int k, int B, int rows, int V, polyspec_dtype dt, void* out, int32_t* device_status,
                                        void* cuda_stream);

/*
 * Page tables of a model's cache around a verified block (Algorithm 1 commits a prefix and rolls the rest back), kept on the
 * device like the staged loop's state: no call is read back.
 *
 *   table [n_seqs, max_pages]  the pages a sequence holds, in order (-1 behind them); len [n_seqs] tokens held, in pages of
 *   page_tokens; refs [n_pages] table entries naming each page; free_bits [ceil(n_pages/32)] bit p % 32 of word p / 32 set iff
 *   refs[p] == 0, no bits set past n_pages.  Caller-owned device arrays, filled by polyspec_cache_init.
 *   n_pages <= 1048576, max_pages * page_tokens < 2^31.
 *   A pool is the contents: n_planes planes (layers, keys and values) of n_pages pages of page_bytes, page p of plane i at
 *   data + (i * n_pages + p) * page_bytes; page_bytes a multiple of 16, data 16-byte aligned.
 *   In reserve and rollback the target length of sequence b is base[b] + (extra ? extra[b] : 0) + plus; base or extra may be
 *   the staged loop's t and cnt, or len itself.
 *
 *   polyspec_cache_reserve   sequences whose target is above their length grow to it.  Pages are taken lowest number first,
 *        sequences in order; where the first new token falls into a last page that other sequences hold too, the page is
 *        replaced by a copy of its own first (in every pool given).  A sequence for which the free pages, counted off in
 *        order, do not suffice stays as it was, with all after it that need a page (POLYSPEC_ERR_NO_PAGES in *device_status);
 *        so does one whose target exceeds max_pages * page_tokens (POLYSPEC_ERR_BAD_INPUT_ON_DEVICE).  len tells what was granted.
 *        Where several sequences stay as they were, the status is the first one's.
 *   polyspec_cache_rollback  sequences whose target is below their length (and not negative) fall back to it; pages wholly
 *        behind it are given back.  Others stay as they are.
 *   polyspec_cache_fork      for n pairs: sequence dst[i], which holds nothing, becomes a copy of src[i] that shares its pages.
 *        Both negative: unused.  A pair is left out (POLYSPEC_ERR_BAD_INPUT_ON_DEVICE) if a number is out of range, dst holds
 *        tokens, src is a dst of the list, or an earlier pair has the same dst.
 *   polyspec_cache_compact   moves pages so that those in use are numbered 0 .. n_live-1: the i-th used page from n_live on
 *        goes to the i-th free page below n_live, its contents in every pool with it; tables follow.  moved_to [n_pages] (or
 *        NULL): the new number of every page in use, -1 for free ones.  Table words behind a sequence's pages stay as they are.
 *   Reserve and compact need a workspace of polyspec_cache_workspace bytes.  Calls on one state must be ordered by the
 *   caller (one stream); the outcome depends on the state alone.  A page number out of range or a reference too many found on
 *   the way is skipped and reported as POLYSPEC_ERR_BAD_INPUT_ON_DEVICE.
 */
#define POLYSPEC_CACHE_MAX_POOLS 8
typedef struct {
    int n_seqs, max_pages, n_pages, page_tokens;
    int32_t *table, *len, *refs;
    uint32_t* free_bits;
} polyspec_cache_pages;
typedef struct {
    void* data;
    int n_planes;
    size_t page_bytes;
} polyspec_cache_pool;
polyspec_status polyspec_cache_workspace(int n_seqs, int n_pages, size_t* bytes /* host out */);
polyspec_status polyspec_cache_init(const polyspec_cache_pages* s /* host */, void* cuda_stream);
polyspec_status polyspec_cache_reserve(const polyspec_cache_pages* s /* host */, const int32_t* base, const int32_t* extra, int plus,
                                       const polyspec_cache_pool* pools /* host */, int n_pools, int32_t* device_status,
                                       void* workspace, size_t workspace_bytes, void* cuda_stream);
polyspec_status polyspec_cache_rollback(const polyspec_cache_pages* s /* host */, const int32_t* base, const int32_t* extra, int plus,
                                        int32_t* device_status, void* cuda_stream);
polyspec_status polyspec_cache_fork(const polyspec_cache_pages* s /* host */, const int32_t* src, const int32_t* dst, int n,
                                    int32_t* device_status, void* cuda_stream);
polyspec_status polyspec_cache_compact(const polyspec_cache_pages* s /* host */, const polyspec_cache_pool* pools /* host */, int n_pools,
                                       int32_t* moved_to, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * A model's attention around the cache pages: what its pass over a prompt or a block needs between its projections and its LM head.
 * At most 2^24 rows, and in attention 1024 query heads.  All of it takes rows of heads in bf16: [rows, heads, head_dim] with the heads of a row behind one another and `stride` elements from
 * row to row (a multiple of 8, at least heads * head_dim), 16-byte aligned, so that queries, keys and values may be parts of the rows of
 * one fused projection.  Outputs of heads are contiguous.
 *
 * polyspec_rotate_heads -- norm of every query and key head and its rotation by position, in one pass:
 *     y = weight ? x / sqrt(mean(x^2) + eps) * weight : x
 *     (a, b) -> (a cos - b sin, a sin + b cos),  angle = positions[row] * frequencies[i],
 *   (a, b) the elements (i, i + rotary_dim/2), or (2i, 2i + 1) if interleaved, of the first rotary_dim of a head; the others stay.
 *   In fp32 (the angle's turns in fp64), rounded once to bf16.
 *   q [rows, q_heads, head_dim], k [rows, kv_heads, head_dim]; k may be NULL (kv_heads 0)
 *   positions [rows] (any int32), frequencies [rotary_dim/2] fp32, in radians per position
 *   q_weight, k_weight [head_dim] bf16, or NULL: no norm.  eps >= 0
 *   head_dim and rotary_dim multiples of 16, rotary_dim <= head_dim <= 256 (0: no rotation, positions and frequencies unread)
 *   q_out, k_out  out, row strides of their own; either the rows of q, k themselves (in place) or rows that overlap none of the inputs.
 *
 * polyspec_prompt_attention -- causal attention over whole prompts, packed one behind the other:
 *     out[i, h] = sum_{j <= i} softmax_j(scale * q[i, h] . k[j, h / (q_heads/kv_heads)]) v[j, .]   i, j rows of one prompt
 *   rows_at [n_seqs + 1]: prompt b is the rows rows_at[b] .. rows_at[b + 1]-1 (none if equal); rows outside all of them are neither read into
 *   a result nor written.  q_heads a multiple of kv_heads; head_dim 64 or 128; 0 <= scale <= 1e30
 *   out [rows, q_heads, head_dim]; lse out [rows, q_heads] fp32 or NULL: the natural logarithm of the softmax's denominator.
 *   Products of bf16, sums and softmax in fp32 (values are at most 2^64 in size); weights are rounded to bf16 for their product with the values.  Keys and values behind a
 *   row never reach it, NaN and infinities included.  Row numbers that decrease or lie outside 0 .. rows make the prompt empty
 *   (POLYSPEC_ERR_BAD_INPUT_ON_DEVICE in *device_status); POLYSPEC_ERR_TIMEOUT as in polyspec_lm_head.
 *
 * Caches held in 4 bits.  One plane of a pool holds one layer's keys or values; a token's head is head_dim codes with one scale and one
 * offset (bf16): value = scale * code + offset, scale a normal number > 0.  A page of polyspec_cache_pages (page_tokens a multiple of 8, at most 32768,
 * and max_pages * page_tokens at most 2^31 - 2^16) is [kv_heads, page_tokens / 8] units of 8 tokens; a unit is head_dim 32-bit words of codes, then 8 pairs (scale, offset):
 * page_bytes = kv_heads * (page_tokens / 8) * (4 head_dim + 32).  Code e of eight neighbours is in the four bits from bit
 * 4 * (e / 2) + 16 * (e % 2) on of their word.  Word w of token r lies at r * head_dim/8 + w in a unit of keys; in a unit of values, with
 * w = 8 h + g, at (8 g + r) * head_dim/64 + h (where the attention's matrix instructions want it).
 * A pool [2 * layers, n_pages, page_bytes] serves reserve, compact and evict as it is; the calls of one layer take its two
 * planes, keys then values.
 *
 * Which rows are whose in append, attention and weigh: sequence b has the rows rows_at[b] .., rows_at[b + 1] - rows_at[b] of them or the
 * first n_rows[b] (NULL: all); its row i stands at slot base[b] + (extra ? extra[b] : 0) + i of its cache.  Reserve comes first: a row
 * whose slot is not below len[b] is not written or attends to nothing (POLYSPEC_ERR_BAD_INPUT_ON_DEVICE), as are the rows of a sequence
 * whose len or base makes no sense, and all rows between the row numbers of one whose n_rows does not.  Row numbers that decrease or lie
 * outside 0 .. rows leave the sequence without rows.
 *
 * polyspec_cache_append -- keys and values of new rows into their slots:  offset = min(x), scale = the smallest normal bf16
 *   number >= (max(x) - offset) / 15 (1 if that is 0), code = (x - offset) / scale rounded to the nearest, ties to even, at most 15; differences and
 *   quotients in fp32.  Of x with NaN, infinities or a range past fp32: every value NaN.
 *   k_held, v_held  out [rows, kv_heads, head_dim] bf16 or NULL: the values the pages now stand for
 *   weights         [n_seqs, max_pages * page_tokens] fp32 or NULL: set to 0 at the new slots
 *   A page that other sequences hold too is not written (POLYSPEC_ERR_BAD_INPUT_ON_DEVICE).
 *
 * polyspec_cache_attention -- the rows of a block over the cache, each row over the slots up to its own:
 *     out[i, h] = sum_{j <= slot(i)} softmax_j(scale * q[i, h] . K[j, h / (q_heads/kv_heads)]) V[j, .]
 *   head_dim 64 or 128, any number of rows; -1e30 <= scale <= 1e30 (it may be negative here and in weigh); out, lse as in
 *   polyspec_prompt_attention; a row that attends to nothing, or to no page that can be read (POLYSPEC_ERR_BAD_INPUT_ON_DEVICE: pages that
 *   cannot be read are left out), gets zeros and -inf.  Codes are multiplied as whole numbers, scales and offsets applied to fp32 sums.
 *   Weights times the values' scales are rounded to fp16 for their product with the codes: each is off by 2^-11 of itself at most, or by
 *   2^-28 of its row's largest, heads of equal elements (all codes 0) aside (2^-20 where all its scales are below 2^-118).  lse, and with it
 *   the weights of polyspec_cache_weigh, depends on queries and keys alone.  Values are at most 2^64 in size: sums of weights times values
 *   stay within fp32.  The order of the sums depends on the lengths and on the batch.
 *   Workspace of polyspec_cache_attention_workspace bytes.
 *   POLYSPEC_ERR_TIMEOUT as in polyspec_lm_head.
 *
 * polyspec_cache_weigh -- adds to every cached token the attention weight that the rows gave it, over all heads:
 *     weights[b, j] = keep * weights[b, j] + sum_{i, h} exp(scale * q[i, h] . K[j, .] - lse[i, h])   for j < len[b]
 *   with lse of polyspec_cache_attention on the same rows (n_rows may be fewer: only the rows that were accepted).  The sum over rows and
 *   heads has a fixed order.
 *
 * polyspec_cache_evict -- sequences of more than budget[b] tokens (budget[b] >= 0) keep the first `first`, the last `recent` and, of those between, the ones of
 *   largest weight (the lower slot of equal ones; NaN below everything) until budget[b] are left.  What is kept moves together in
 *   every plane of the pool and in the weights, in order; pages wholly behind are given back, len follows.  What lies behind the kept tokens in
 *   a page or in the weights stays as it is.  A sequence stays as it was (POLYSPEC_ERR_BAD_INPUT_ON_DEVICE) if its budget is below first + recent,
 *   if one of its page numbers makes no sense, or if a page that keeps tokens from the first changed slot on is held by others too, as the
 *   holds were before the call.  (Pages wholly behind only lose the sequence's hold, and where the kept tokens are the first ones no slot changes.)
 *   kept_from  out [n_seqs, max_pages * page_tokens] or NULL: the slot each kept token of a shortened sequence had, -1 behind them;
 *              sequences that were not shortened get -1 throughout.
 *   Workspace of polyspec_cache_evict_workspace bytes.
 */
polyspec_status polyspec_rotate_heads(const void* q, long long q_stride, int q_heads, const void* k, long long k_stride, int kv_heads,
                                      int rows, int head_dim, int rotary_dim, int interleaved, const int32_t* positions,
                                      const float* frequencies, const void* q_weight, const void* k_weight, float eps,
                                      void* q_out, long long q_out_stride, void* k_out, long long k_out_stride, void* cuda_stream);
polyspec_status polyspec_prompt_attention(const void* q, long long q_stride, const void* k, long long k_stride, const void* v, long long v_stride,
                                          const int32_t* rows_at, int n_seqs, int rows, int q_heads, int kv_heads, int head_dim, float scale,
                                          void* out, float* lse, int32_t* device_status, void* cuda_stream);
typedef struct {
    const int32_t *rows_at, *n_rows, *base, *extra;     /* device; n_rows and extra may be NULL */
    int rows;                                           /* rows of the tensors of heads */
} polyspec_block_rows;
polyspec_status polyspec_cache_append(const polyspec_cache_pages* s /* host */, const polyspec_block_rows* r /* host */,
                                      const void* k, long long k_stride, const void* v, long long v_stride, int kv_heads, int head_dim,
                                      void* pool, void* k_held, void* v_held, float* weights, int32_t* device_status, void* cuda_stream);
polyspec_status polyspec_cache_attention_workspace(int q_heads, int kv_heads, int head_dim, size_t* bytes /* host out */);
polyspec_status polyspec_cache_attention(const polyspec_cache_pages* s /* host */, const polyspec_block_rows* r /* host */,
                                         const void* q, long long q_stride, int q_heads, int kv_heads, int head_dim, float scale,
                                         const void* pool, void* out, float* lse, int32_t* device_status,
                                         void* workspace, size_t workspace_bytes, void* cuda_stream);
polyspec_status polyspec_cache_weigh(const polyspec_cache_pages* s /* host */, const polyspec_block_rows* r /* host */,
                                     const void* q, long long q_stride, int q_heads, int kv_heads, int head_dim, float scale,
                                     const void* pool, const float* lse, float keep, float* weights, int32_t* device_status, void* cuda_stream);
polyspec_status polyspec_cache_evict_workspace(int n_seqs, int max_pages, int page_tokens, size_t* bytes /* host out */);
polyspec_status polyspec_cache_evict(const polyspec_cache_pages* s /* host */, const int32_t* budget, int first, int recent, float* weights,
                                     void* pool, int n_planes, int kv_heads, int head_dim, int32_t* kept_from, int32_t* device_status,
                                     void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * polyspec_verify_level_static -- polyspec_verify_level without a workspace argument.
 * (The paper has no counterpart to this call; it exists for integration reasons only.)
 *
 * Some callers cannot give the library a workspace because they cannot allocate device
 * memory at the point where they verify: a plugin invoked from inside a serving engine
 * that owns every byte of the device, code running under a fixed post-start-up memory
 * budget, a callback in which cudaMalloc is forbidden.  For them the row-statistics
 * partials live in a fixed array of POLYSPEC_STATIC_SCRATCH_BYTES inside the library image
 * (each GPU that loads the library holds that much until the process exits).  The call
 * allocates nothing, neither through CUDA nor through any library.
 *
 *   - Inputs and outputs are the caller's, exactly as in polyspec_verify_level.
 *   - Limit: the call needs polyspec_verify_level_workspace(B, k, V, dt) bytes; if that
 *     exceeds POLYSPEC_STATIC_SCRATCH_BYTES it returns POLYSPEC_ERR_SCRATCH_LIMIT and launches
 *     nothing.  (1 MiB covers e.g. B = 256, k = 8, V = 152064 in bf16.)
 *   - The device that owns `cuda_stream` must be current.  The first call on each device
 *     looks up the device address of the array (a one-time set-up step); make that first
 *     call before starting any stream capture.
 *   - All calls on a device share the one array.  A call overwrites every entry it later
 *     reads, so leftovers from earlier calls do not matter, but two calls whose kernels
 *     overlap on the GPU (different streams) race: serialise them.
 */
#define POLYSPEC_STATIC_SCRATCH_BYTES (1u << 20)
size_t polyspec_static_scratch_bytes(void);
polyspec_status polyspec_verify_level_static(
    const void* logits_p, const void* logits_q, const int32_t* draft_tokens, const float* uniforms,
    const int32_t* block_len, int B, int k, int V, polyspec_dtype dt, float temperature,
    int32_t* accepted_len, int32_t* next_token, float* p_at_draft, float* q_at_draft,
    int32_t* device_status, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* POLYSPEC_H */
