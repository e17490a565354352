/*
 * brisk.h - C ABI of the BRISK-DLM decoding hot path on MI355X (gfx950).
 *
 * One decoding step of the paper's prefix-conditioned proposal selection
 * (Section 3.3, Algorithm 1(b)) in three calls:
 *
 *   brisk_propose_block  LM-head projection of every masked position's hidden
 *                        state and its ordered top-K candidate set;
 *   brisk_rerank         the corrector that re-scores those candidates left to
 *                        right, conditioned on the tokens already selected;
 *   brisk_verify_accept  greedy verification: accepted-prefix length and the
 *                        correction token of each block.
 *
 * brisk_rerank_verify makes the last two in one call; brisk_rerank_hoist and
 * brisk_rerank_finish split the rerank at the candidates, so that its first
 * part can overlap the LM-head pass.
 *
 * Further down stand the operators around the step: attention over a shared
 * prefix and a paged cache, that cache's eviction, and verification of drafts
 * from given probabilities.
 *
 * Conventions shared by every entry point
 *   - Every pointer argument is a DEVICE pointer owned by the caller, except
 *     the brisk_corrector struct itself (host memory, read during the call)
 *     and the size out-parameters.  The library allocates nothing and is
 *     reentrant; calls on different streams are safe when their workspaces
 *     and outputs differ.  Its only global state is the fixed scratch of
 *     brisk_propose_block_noalloc (one array per GPU, and its address).
 *   - bf16 tensors are passed as uint16_t bit patterns; all matrices are
 *     row-major and densely packed (row stride = row length) where a call
 *     takes no strides.
 *   - Rows of a block are numbered r = b * L + (i - 1) for sequence b and
 *     in-block position i = 1..L.
 *   - `stream` is a hipStream_t (NULL = the default stream).  Work is queued
 *     on it asynchronously; nothing synchronises.
 *   - Every call returns a brisk_status.  Arguments are validated on the host
 *     before any HIP call: on an error return nothing has been launched and no
 *     output has been touched.  BRISK_ERR_HIP reports a failed launch.
 *   - Token ids read from device memory (candidate ids, anchor tokens) are
 *     clamped into [0, V) before they address a table, so a bad id cannot make
 *     a kernel read out of bounds; the results for such a row are unspecified.
 *   - Pointers must be 16-byte aligned and d a multiple of 8, otherwise
 *     BRISK_ERR_UNSUPPORTED.
 */
#ifndef BRISK_H_
#define BRISK_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  BRISK_OK = 0,
  BRISK_ERR_NULL = -1,        /* a required pointer is NULL                   */
  BRISK_ERR_SHAPE = -2,       /* a size is out of range or inconsistent        */
  BRISK_ERR_UNSUPPORTED = -3, /* alignment / divisibility the kernels need, or
                                 buffers that must not overlap and do         */
  BRISK_ERR_WORKSPACE = -4,   /* workspace missing or smaller than required    */
  BRISK_ERR_HIP = -5,         /* a HIP launch failed                           */
  BRISK_ERR_SCRATCH = -6      /* the shape needs more than the fixed scratch  */
} brisk_status;

/* Static, NUL-terminated description of a status code. */
const char* brisk_status_str(int status);

/* Library ABI version (bumped on any signature or struct change). */
int brisk_abi_version(void);

/*
 * Corrector parameters psi (Section 3.3 Eq. inference_head_state and
 * Eq. candidate_residual; Appendix "Candidate-Refinement Head Details",
 * Eq. head_residual_logits and the head configuration table).  All tensor
 * pointers are device bf16 bit patterns, row-major:
 *
 *   u_0      = tanh(A_h h_c + A_e E(x_0))
 *   x_hat_i  = [P_h m_i ; P_e E(x_{i-1}) ; pos_emb[i-1] ; P_phi phi_i]
 *   z        = sigmoid(W_z x_hat_i),  u_i = (1 - z) * u_{i-1} + z * (W_h x_hat_i)
 *   gamma_i  = sigmoid(alpha) * sigmoid(w_g . [u_i ; phi_i] + b_g)
 *   l~_{i,k} = l_{i,k} + gamma_i * <W_s u_i, W_c E_out(v_{i,k})>
 *
 * with phi_i = [top1-top2, top1-top4, 1[x_{i-1} = top1], 1[x_{i-1} in top4],
 * top1 - l_i(x_{i-1})] from the position's ordered candidates and E_out the
 * LM head.  Dimension limits: d_state in [1, 512], d_hproj, d_tproj, rank in
 * [1, 256], d_pos, d_feat in [1, 64], max_L >= 1.
 */
typedef struct brisk_corrector {
  int32_t d_state, d_hproj, d_tproj, d_pos, d_feat, rank, max_L;
  const uint16_t* A_h;      /* [d_state, d]                               */
  const uint16_t* A_e;      /* [d_state, d]                               */
  const uint16_t* P_h;      /* [d_hproj, d]                               */
  const uint16_t* P_e;      /* [d_tproj, d]                               */
  const uint16_t* pos_emb;  /* [max_L, d_pos]                             */
  const uint16_t* P_phi;    /* [d_feat, 5]                                */
  const uint16_t* W_z;      /* [d_state, d_in], d_in = d_hproj+d_tproj+d_pos+d_feat */
  const uint16_t* W_h;      /* [d_state, d_in]                            */
  const uint16_t* W_s;      /* [rank, d_state]                            */
  const uint16_t* W_c;      /* [rank, d]                                  */
  const uint16_t* w_g;      /* [d_state + 5]                              */
  float alpha;              /* gate scale logit (host value)               */
  float b_g;                /* gate bias (host value)                      */
  /* Optional per-token tables from brisk_corrector_prepare (NULL: none).
   * When set, the rerank calls read the lifts of candidate and anchor tokens
   * from them instead of projecting their embedding rows; tables_V must then
   * equal the call's V, and the tables must have been prepared from these
   * parameters and the same lm_head and tok_embed (not checked). */
  const float* tables;      /* [3][tables_V][max(256, d_state)] fp32       */
  int32_t tables_V;
} brisk_corrector;

/*
 * Per-token tables of the corrector (Section 3.3 Eq. inference_head_state and
 * Eq. candidate_residual; Appendix Eq. head_residual_logits).  Every map the
 * corrector applies to a token's embedding rows is linear and fixed once the
 * model is loaded: the token projection reaches the state update as
 * TZ(v) = W_z[:, t] P_e E(v) and TH(v) = W_h[:, t] P_e E(v), and the residual
 * re-associates to <u_i, EH(v)> with EH(v) = W_s^T W_c E_out(v) (t = the
 * d_tproj columns of W_z and W_h that read P_e E).  brisk_corrector_prepare
 * computes the three for every token (bf16 inputs, fp32 accumulation) into
 * tables [EH; TZ; TH], each [V][max(256, d_state)] fp32 with rows zero-padded
 * past d_state.  Preparing once per model replaces the per-step gathers of
 * whole E and E_out rows by gathers of table rows; the decoding results are
 * those of the per-step projections up to fp32 rounding.
 *
 *   c          corrector parameters (its tables field is ignored here)
 *   lm_head    [V, d] bf16  E_out;   tok_embed [V, d] bf16  E
 *   tables     out, table_bytes >= *table_bytes of brisk_corrector_tables_size
 *   ws         scratch of at least *ws_bytes bytes (V * (d_tproj + rank) fp32)
 *
 * Limits as brisk_rerank's for the corrector; 1 <= V <= 2^24, 8 <= d <= 65536,
 * d % 8 == 0, 16-byte aligned pointers.
 */
int brisk_corrector_tables_size(const brisk_corrector* c, int32_t V, size_t* table_bytes, size_t* ws_bytes);
int brisk_corrector_prepare(const brisk_corrector* c, const uint16_t* lm_head, const uint16_t* tok_embed,
                            int32_t V, int32_t d, float* tables, size_t table_bytes, void* ws,
                            size_t ws_bytes, void* stream);

/*
 * Workspace bytes brisk_propose_block needs for this shape (written to *bytes).
 * Returns BRISK_ERR_SHAPE / BRISK_ERR_NULL on bad arguments.
 */
int brisk_propose_workspace_size(int32_t rows, int32_t d, int32_t V, int32_t K, size_t* bytes);

/*
 * Candidate construction C_i = TopK(q_i, K) (Section 3.3; Appendix head
 * details; Algorithm 1(b) first step and loop head).  Computes the proposal
 * logits l[r, v] = sum_k hidden[r, k] * lm_head[v, k] (bf16 inputs, fp32
 * accumulation; the [rows, V] logits never reach memory) and returns the K
 * largest per row, ordered by logit descending and, among equal logits, by
 * token id ascending.  Top-K of the softmax q equals top-K of the logits.
 *
 *   hidden      [rows, d]  bf16   masked-position hidden states m_i
 *   lm_head     [V, d]     bf16   frozen LM head (output vocabulary rows)
 *   cand_logit  [rows, K]  fp32   out: candidate logits, descending
 *   cand_id     [rows, K]  int32  out: candidate token ids
 *   ws          device scratch of at least brisk_propose_workspace_size bytes
 *
 * Limits: 1 <= rows <= 2^20, 8 <= d <= 65536, 1 <= K <= 64, K <= V; V*d*2 and
 * rows*d*2 below 2^32 bytes (BRISK_ERR_UNSUPPORTED otherwise).
 */
int brisk_propose_block(const uint16_t* hidden, const uint16_t* lm_head,
                        int32_t rows, int32_t d, int32_t V, int32_t K,
                        float* cand_logit, int32_t* cand_id,
                        void* ws, size_t ws_bytes, void* stream);

/*
 * brisk_propose_block without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc).  Same arguments, results, limits and errors as
 * brisk_propose_block, minus ws and ws_bytes: the key lists live in a fixed
 * array of BRISK_NOALLOC_SCRATCH_BYTES (16 MiB) that the library holds on
 * each GPU it runs on until the process ends.  A shape whose
 * brisk_propose_workspace_size exceeds that returns BRISK_ERR_SCRATCH (the
 * five decoding workloads need 0.5-8 MiB).  The call allocates nothing; its
 * first call on a device looks up that device's copy of the array (with the
 * stream's device made current for the lookup), and BRISK_ERR_HIP reports a
 * failed lookup.  Every call on one GPU uses the same array: calls that
 * overlap in time on one GPU (on different streams, or from different host
 * threads) race and their results are undefined; serialise them.
 */
#define BRISK_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)
int brisk_propose_block_noalloc(const uint16_t* hidden, const uint16_t* lm_head,
                                int32_t rows, int32_t d, int32_t V, int32_t K,
                                float* cand_logit, int32_t* cand_id, void* stream);

/*
 * The two launches of brisk_propose_block, one call each (same section of the
 * paper, same arguments, limits and workspace).  brisk_propose_lmhead is the
 * LM-head pass: it leaves in ws, for every row and vocabulary share, the
 * ordered keys of that share's K largest logits.  brisk_propose_merge reduces
 * those keys to the candidates.  brisk_propose_block is exactly the two in
 * order on one stream; calling them separately lets a caller time or
 * schedule each launch on its own.  A merge reads the workspace of the pass
 * before it on the same stream, which must have used the same rows, V and K
 * (the layout depends on them); it does not check that.
 */
int brisk_propose_lmhead(const uint16_t* hidden, const uint16_t* lm_head, int32_t rows, int32_t d,
                         int32_t V, int32_t K, void* ws, size_t ws_bytes, void* stream);
int brisk_propose_merge(int32_t rows, int32_t V, int32_t K, float* cand_logit, int32_t* cand_id,
                        const void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes brisk_rerank needs (written to *bytes). */
int brisk_rerank_workspace_size(const brisk_corrector* c, int32_t B, int32_t L, int32_t K,
                                size_t* bytes);

/*
 * Prefix-conditioned rerank of the candidates (Section 3.3; Appendix head
 * details; Algorithm 1(b) loop): steps the corrector over i = 1..L for every
 * sequence, feeding the token selected at i-1 (x_0 at i = 1) into step i, and
 * selects x_i = the candidate with the largest refined logit (the smallest
 * candidate index on ties).
 *
 *   c           host struct of device parameter pointers (see above)
 *   hidden      [B*L, d] bf16   m_i
 *   ctx_hidden  [B, d]   bf16   h_c
 *   anchor_tok  [B]      int32  x_0, the token preceding each block
 *   lm_head     [V, d]   bf16   E_out (the same matrix brisk_propose_block used)
 *   tok_embed   [V, d]   bf16   E, the input token embedding
 *   cand_logit, cand_id [B*L, K] the candidate sets from brisk_propose_block
 *   selected    [B, L]   int32  out: x_{1..L}
 *   refined     [B*L, K] fp32   out, nullable: refined logits l~
 *   gamma       [B*L]    fp32   out, nullable: gate gamma_i
 *   resid       [B*L, K] fp32   out, nullable: residual <W_s u_i, W_c E_out(v)>
 *
 * Limits: 4 <= K <= 64 (the features read the top-4), 1 <= L <= max_L,
 * B*L <= 2^20, and one sequence's step blocks L*(2+3K)*max(256, d_state)*4
 * below 2^31 bytes (each step vector is padded to at least 256 floats);
 * beyond that the call returns BRISK_ERR_UNSUPPORTED.
 */
int brisk_rerank(const brisk_corrector* c, const uint16_t* hidden, const uint16_t* ctx_hidden,
                 const int32_t* anchor_tok, const uint16_t* lm_head, const uint16_t* tok_embed,
                 const float* cand_logit, const int32_t* cand_id,
                 int32_t B, int32_t L, int32_t K, int32_t d, int32_t V,
                 int32_t* selected, float* refined, float* gamma, float* resid,
                 void* ws, size_t ws_bytes, void* stream);

/*
 * Greedy verification (Section 2.2 accepted prefix; Section 3.3 speculative
 * acceptance, temperature-zero case; Algorithm 1(b) verify and commit):
 * accept_len[b] = number of leading positions i with proposal[b, i] ==
 * verifier[b, i], in [0, L]; correction[b] = verifier[b, accept_len[b]] when
 * accept_len[b] < L, else -1.
 *
 *   proposal    [B, L] int32   proposed tokens x_{1..L}
 *   verifier    [B, L] int32   the verifier's argmax tokens
 *   accept_len  [B]    int32   out
 *   correction  [B]    int32   out, nullable
 */
int brisk_verify_accept(const int32_t* proposal, const int32_t* verifier, int32_t B, int32_t L,
                        int32_t* accept_len, int32_t* correction, void* stream);

/*
 * brisk_rerank followed by brisk_verify_accept on its selections, in one call
 * (Algorithm 1(b): select, then verify).  Same arguments as brisk_rerank plus
 *
 *   verifier    [B, L] int32  the verifier's token at every position
 *   accept_len  [B] int32 out, correction [B] int32 out (nullable), as in
 *               brisk_verify_accept
 *
 * When the single-wavefront scan runs (d_state <= 256, K <= 16) the scan
 * itself compares each selection with the verifier's token, so no separate
 * launch follows; otherwise the verification kernel runs after the scan.
 * Results equal the two calls made one after the other.
 */
int brisk_rerank_verify(const brisk_corrector* c, const uint16_t* hidden, const uint16_t* ctx_hidden,
                        const int32_t* anchor_tok, const uint16_t* lm_head, const uint16_t* tok_embed,
                        const float* cand_logit, const int32_t* cand_id, const int32_t* verifier,
                        int32_t B, int32_t L, int32_t K, int32_t d, int32_t V, int32_t* selected,
                        float* refined, float* gamma, float* resid, int32_t* accept_len,
                        int32_t* correction, void* ws, size_t ws_bytes, void* stream);

/*
 * brisk_rerank (or brisk_rerank_verify) in two parts, so that the first can
 * run while the LM-head pass that makes the candidates streams (same section
 * of the paper).  brisk_rerank_hoist queues the work that does not read the
 * candidates: the projections P_h m_i, A_h h_c and A_e E(x_0), the sums of
 * their split reductions, and their lifts into the step vectors together
 * with the position and feature terms.  brisk_rerank_finish queues the rest
 * on a workspace that a brisk_rerank_hoist call filled and nothing has
 * written since: with verifier NULL it completes brisk_rerank, otherwise
 * brisk_rerank_verify (then accept_len is required; correction is nullable).
 *
 * Both calls take brisk_rerank's arguments (brisk_rerank_hoist only those it
 * reads) with the same c, hidden, ctx_hidden, anchor_tok, tok_embed, B, L,
 * K, d, V and workspace, and the same limits and errors; the library does
 * not check that the two calls agree.  The caller orders them: on one
 * stream, or the finishing call's stream waits on an event recorded after
 * the hoist.  The results are bitwise those of the single call.
 */
int brisk_rerank_hoist(const brisk_corrector* c, const uint16_t* hidden, const uint16_t* ctx_hidden,
                       const int32_t* anchor_tok, const uint16_t* tok_embed, int32_t B, int32_t L,
                       int32_t K, int32_t d, int32_t V, void* ws, size_t ws_bytes, void* stream);
int brisk_rerank_finish(const brisk_corrector* c, const uint16_t* hidden, const uint16_t* ctx_hidden,
                        const int32_t* anchor_tok, const uint16_t* lm_head, const uint16_t* tok_embed,
                        const float* cand_logit, const int32_t* cand_id, const int32_t* verifier,
                        int32_t B, int32_t L, int32_t K, int32_t d, int32_t V, int32_t* selected,
                        float* refined, float* gamma, float* resid, int32_t* accept_len,
                        int32_t* correction, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes brisk_propose_verify needs (written to *bytes). */
int brisk_propose_verify_workspace_size(int32_t rows_prop, int32_t rows_ver, int32_t d, int32_t V,
                                        int32_t K, size_t* bytes);

/*
 * One LM-head pass for both kinds of rows a self-verifying decoding step
 * produces (Section 2.1 introspective strided decoding, where proposal and
 * causal verification come from the same model evaluation; Section 3.3;
 * Algorithm 1(b) first step and verify): the proposal rows of the next block
 * get their ordered top-K candidates, exactly as brisk_propose_block, and the
 * verifier rows of the block under verification get their argmax token (the
 * largest logit, the lower id on ties), without a second pass over lm_head.
 *
 *   hidden      [rows_prop + rows_ver, d] bf16: proposal rows first, then
 *               verifier rows
 *   lm_head     [V, d] bf16
 *   cand_logit, cand_id  [rows_prop, K] out (may be NULL when rows_prop == 0)
 *   ver_token   [rows_ver] int32 out (may be NULL when rows_ver == 0)
 *   ws          device scratch of brisk_propose_verify_workspace_size bytes
 *
 * Limits as brisk_propose_block with rows = rows_prop + rows_ver >= 1.
 */
int brisk_propose_verify(const uint16_t* hidden, const uint16_t* lm_head, int32_t rows_prop,
                         int32_t rows_ver, int32_t d, int32_t V, int32_t K, float* cand_logit,
                         int32_t* cand_id, int32_t* ver_token, void* ws, size_t ws_bytes,
                         void* stream);

/*
 * Greedy verification and commit (Algorithm 1(b): verify, then commit the
 * accepted prefix and the correction; Section 2.2 accepted prefix).  For
 * block b with a = accept length (as brisk_verify_accept):
 *   committed[b, 0..a-1] = proposal[b, 0..a-1];
 *   committed[b, a]      = verifier[b, a]        when a < L;
 *   the rest of the L + 1 slots = -1;  n_committed[b] = a + (a < L).
 *
 *   proposal, verifier  [B, L] int32
 *   accept_len          [B] int32 out, nullable
 *   committed           [B, L + 1] int32 out
 *   n_committed         [B] int32 out
 */
int brisk_verify_commit(const int32_t* proposal, const int32_t* verifier, int32_t B, int32_t L,
                        int32_t* accept_len, int32_t* committed, int32_t* n_committed,
                        void* stream);

/* Workspace bytes brisk_spec_verify needs (written to *bytes). */
int brisk_spec_verify_workspace_size(int32_t B, int32_t L, int32_t V, int32_t K, size_t* bytes);

/*
 * Stochastic speculative verification (Section 3.3; Algorithm 1(b) verify
 * and commit).  Position i of block b (row r = b * L + i) accepts its
 * proposal x_r with probability min{1, p_r(x_r) / pi_r(x_r)}, where p_r is
 * the verifier's softmax at temperature T over the whole vocabulary (logits
 * <lm_head[v], ver_hidden[r]>, one fused LM-head pass with an online
 * log-sum-exp) and pi_r the proposal law over the position's candidates.
 * Each row also draws y_r from the normalised positive part [p_r - pi_r]_+,
 * which keeps the committed token distributed as p_r; the block stops at its
 * first rejection a and commits y at position a.
 *
 *   ver_hidden  [B*L, d] bf16    verifier hidden states
 *   lm_head     [V, d]   bf16
 *   proposal    [B, L]   int32   x
 *   cand_id     [B*L, K] int32   distinct candidate ids of each position
 *   cand_prob   [B*L, K] fp32    pi over those ids (tokens outside have pi = 0);
 *               nullable: NULL means the greedy proposer, pi = point mass at
 *               x (when x is among the candidates)
 *   u_accept    [B*L]    fp32    uniforms in [0, 1) for the accept tests
 *   seed        key of the Philox4x32-10 generator of the residual draws
 *               (Gumbel variate of token v at row r from word v mod 4 of
 *               counter (v / 4, r, 0, 0))
 *   accept_len  [B] int32 out;  correction [B] int32 out, nullable (-1 when
 *               the block is fully accepted)
 *   row_accept, row_resample  [B*L] int32 out, nullable: every position's
 *               accept decision (1/0) and residual draw
 *   ws          device scratch of brisk_spec_verify_workspace_size bytes
 *
 * Limits: 1 <= K <= 64, K < V, temperature > 0, B*L <= 2^20, and the LM-head
 * limits of brisk_propose_block.
 */
int brisk_spec_verify(const uint16_t* ver_hidden, const uint16_t* lm_head, const int32_t* proposal,
                      const int32_t* cand_id, const float* cand_prob, const float* u_accept,
                      uint64_t seed, float temperature, int32_t B, int32_t L, int32_t K, int32_t d,
                      int32_t V, int32_t* accept_len, int32_t* correction, int32_t* row_accept,
                      int32_t* row_resample, void* ws, size_t ws_bytes, void* stream);

/*
 * Corrector training loss, forward (Appendix "Candidate-Refinement Head
 * Details", Eq. head_training_loss).  For position j of block b (row
 * r = b * L + j) with candidates v_{r,k}:
 *   p_S = softmax_k <lm_head[v_{r,k}], ver_hidden[r]>   (verifier, restricted)
 *   q_S = softmax_k cand_logit[r, k]                     (base proposal, restricted)
 *   r   = softmax_k refined[r, k]                        (corrector)
 *   loss_pos[r] = CE(p_S, r) + beta * KL(q_S || r)  on reached positions
 *                 (j <= accept_len[b]: the accepted prefix and the first
 *                 rejection), 0 elsewhere
 *   loss_mean   = {mean of loss_pos over reached positions, their count}
 *
 *   ver_hidden  [B*L, d] bf16   the verifier's hidden states
 *   lm_head     [V, d]   bf16
 *   cand_id, cand_logit, refined  [B*L, K] (from brisk_propose_block and
 *               brisk_rerank)
 *   accept_len  [B] int32      (from brisk_verify_accept)
 *   loss_pos    [B*L] fp32 out;  ce, kl [B*L] fp32 out, nullable
 *   loss_mean   [2]   fp32 out
 *
 * Limits: 1 <= K <= 64, d % 8 == 0 with 16-byte aligned bf16 pointers, B*L
 * <= 2^20.  Deterministic (fixed-order sums).
 */
int brisk_corrector_loss(const uint16_t* ver_hidden, const uint16_t* lm_head, const int32_t* cand_id,
                         const float* cand_logit, const float* refined, const int32_t* accept_len,
                         int32_t B, int32_t L, int32_t K, int32_t d, int32_t V, float beta,
                         float* loss_pos, float* ce, float* kl, float* loss_mean, void* stream);

/* Workspace bytes brisk_accept_profile needs (written to *bytes). */
int brisk_accept_profile_workspace_size(int32_t n_blocks, int32_t M, size_t* bytes);

/*
 * Acceptance profile and efficiency statistics of verified blocks (Section
 * 3.2 Eq. nonuniform_tpf and Eq. brisk_weighting; Appendix "Brisk Backbone",
 * Eq. idlm_tpf_instantiation and the rejection-rate estimate of a_i).  From
 * the accepted-prefix lengths of n_blocks blocks of M proposal positions
 * (block b reaches positions 1..L_b + 1 and is rejected at L_b + 1 when
 * L_b < M):
 *   a[i]      = 1 - rejected_i / reached_i   (1 for a position no block reaches)
 *   w_raw[i]  = -dFPT/dz_i, z_i = log(a_i / (1 - a_i)), FPT = 1 / TPF with the
 *               ISD instantiation TPF = (2 + sum_{k=1}^{M-1} A_k) / (2 - A_M),
 *               A_k = prod_{j<=k} a_j
 *   w[i]      = M w_raw[i] / (sum_j w_raw[j] + eps)
 *   tpf_fpt   = {TPF, FPT}
 *
 *   accept_len  [n_blocks] int32   accepted-prefix lengths (e.g. the output of
 *                                  brisk_verify_accept); values outside [0, M]
 *                                  are clamped into it; may be NULL when
 *                                  n_blocks == 0
 *   a, w_raw, w [M] fp64 out;  tpf_fpt [2] fp64 out
 *   ws          device scratch of brisk_accept_profile_workspace_size bytes
 *
 * Limits: 1 <= M <= 1024, 0 <= n_blocks <= 2^30.  Deterministic: the counts
 * are integers and every floating-point sum runs in a fixed order.
 */
int brisk_accept_profile(const int32_t* accept_len, int32_t n_blocks, int32_t M, double eps,
                         double* a, double* w_raw, double* w, double* tpf_fpt,
                         void* ws, size_t ws_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * Operators around the step: the attention that makes a block's hidden states
 * from a shared prefix and a paged cache, the weights and the eviction that
 * keep that cache short, and verification from given probabilities (Section
 * 2.1 strided decoding, Section 3.3 verification, Algorithm 1(b)).  Where a
 * call does not say otherwise, its outputs must not overlap its inputs.
 * ---------------------------------------------------------------------------
 */
typedef enum { BRISK_BF16 = 0, BRISK_F16 = 1 } brisk_dtype;

/*
 * A paged key/value cache (host struct of device pointers and sizes).  Slot j
 * of sequence b lies in page block_table[b, j / page_size] at place
 * j % page_size; its key for key/value head h starts at element
 *   page * page_stride + place * slot_stride + h * head_stride
 * of k_pages, its value at the same element of v_pages, and the d_head
 * elements of both are contiguous.  Offsets are computed in 64 bits.  Page
 * ids are clamped into [0, n_pages), lengths into what the table addresses.
 *
 * Limits: 1 <= n_kv_heads <= 1024; d_head a multiple of 8 in [8, 128];
 * page_size a power of two in [1, 65536]; n_pages, max_pages >= 1; max_pages *
 * page_size <= 2^30; strides non-negative multiples of 8; k_pages and v_pages
 * 16-byte aligned.
 */
typedef struct brisk_kv_cache {
  int32_t dtype;             /* brisk_dtype of keys, values, queries, outputs */
  int32_t n_kv_heads, d_head, page_size, n_pages, max_pages;
  int64_t page_stride, slot_stride, head_stride;   /* in elements             */
  uint16_t* k_pages;
  uint16_t* v_pages;
  const int32_t* block_table;  /* [B, max_pages]                              */
  const int32_t* seq_len;      /* [B] slots held, the block's own included    */
} brisk_kv_cache;

/* Keys and values that every sequence of a batch shares, held once: key j of
 * head h starts at element j * slot_stride + h * head_stride of k, its value
 * at the same element of v.  Type, heads and d_head are the cache's; strides
 * and alignment as there; 0 <= len <= 2^30. */
typedef struct brisk_kv_prefix {
  int32_t len;
  int64_t slot_stride, head_stride;
  const uint16_t* k;
  const uint16_t* v;
} brisk_kv_prefix;

/* Workspace bytes brisk_block_attention needs (written to *bytes). */
int brisk_block_attention_workspace_size(int32_t B, int32_t L, int32_t n_heads, int32_t n_kv_heads,
                                         int32_t d_head, int32_t prefix_len, int32_t max_seq_len,
                                         size_t* bytes);

/*
 * Attention of every sequence's block over the shared prefix and its own
 * cache.  The rows are the L positions of each block (L = 1: single-token
 * decoding) times n_heads query heads; query head h reads key/value head
 * h / (n_heads / n_kv_heads).  The block's own keys are the last L slots of
 * its sequence (already written to the cache): with n = seq_len[b], position
 * i sees every prefix key, every slot below n - L, and slot n - L + t when
 * bit t of block_mask[b, i] is set (all of them when block_mask is NULL).
 *   out = sum_j softmax_j(scale * <q, k_j>) v_j,   lse = log sum_j exp(scale * <q, k_j>)
 * over the visible keys.  A row that sees no key gets out = 0, lse = -inf.
 * What lies in slots that a row does not see has no effect on it, infinities
 * and NaN included.  The prefix is read once for all sequences.
 *
 *   q           element (b * L + i) * q_row_stride + h * q_head_stride starts
 *               the d_head contiguous elements of a row; strides multiples of 8
 *   block_mask  [B, L] uint64, nullable
 *   max_seq_len host bound of the lengths (longer ones are cut to it); 0 when
 *               no sequence holds a key.  The split of long caches over the
 *               GPU follows from it, so a bound near the real lengths is faster
 *   out         [B*L, n_heads, d_head], the cache's type
 *   lse         [B*L, n_heads] fp32, nullable
 *   ws          device scratch of brisk_block_attention_workspace_size bytes
 *
 * Limits: 1 <= L <= 64, B >= 1, n_heads a multiple of n_kv_heads with
 * B * L * n_heads <= 2^24, 0 <= max_seq_len <= max_pages * page_size,
 * 0 < scale <= 1e30.  Sums, maxima and partial outputs are held in fp32;
 * probabilities are rounded to the cache's type where they meet the values
 * (in f16 a weight is off by at most 2^-37 of the row's largest besides: less
 * than that rounding for up to 2^25 weak keys beside a strong one).
 * Deterministic.
 */
int brisk_block_attention(const brisk_kv_cache* cache, const brisk_kv_prefix* prefix, const uint16_t* q,
                          int64_t q_row_stride, int64_t q_head_stride, const uint64_t* block_mask,
                          int32_t B, int32_t L, int32_t n_heads, int32_t max_seq_len, float scale,
                          uint16_t* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Attention weight received by every cached key (the measure by which
 * brisk_cache_evict chooses).  For n = seq_len[b] and slots j < n:
 *   score_out[b, h, j] = decay * score_in[b, h, j] + sum over the rows (i, query heads of group h)
 *                        that see j of exp(scale * <q, k_j> - lse)
 * and 0 for n <= j < cap.  q, block_mask, lse and L as given to and left by
 * brisk_block_attention (so the weights are those over prefix and cache
 * together); a row with lse = -inf adds nothing.  A weight carries the rounding
 * of its row's lse in fp32: a factor within about 1 +- 2^-22 |lse|.
 *
 *   lse         [B*L, n_heads] fp32
 *   score_in, score_out  [B, n_kv_heads, cap] fp32; they may be the same array,
 *               but score_out may not overlap score_in otherwise, nor the other
 *               inputs (BRISK_ERR_UNSUPPORTED where the call can tell)
 *
 * Limits as brisk_block_attention; 1 <= cap <= 2^30, and the launch holds fewer
 * than 2^24 workgroups: B * n_kv_heads * ceil(cap / 1024) < 2^24; lengths are
 * cut to cap.
 * Deterministic (fixed-order sums, no atomics).
 */
int brisk_cache_score(const brisk_kv_cache* cache, const uint16_t* q, int64_t q_row_stride,
                      int64_t q_head_stride, const uint64_t* block_mask, const float* lse, int32_t B,
                      int32_t L, int32_t n_heads, float scale, float decay, const float* score_in,
                      float* score_out, int32_t cap, void* stream);

/* Workspace bytes brisk_cache_evict needs (written to *bytes). */
int brisk_cache_evict_workspace_size(int32_t B, int32_t n_kv_heads, int32_t cap, int32_t budget,
                                     size_t* bytes);

/*
 * Eviction to at most `budget` slots a sequence, each key/value head keeping
 * its own keys.  For a sequence of n > budget slots, head h keeps first the
 * slots with pos >= next_pos[b] - recent (the latest tokens), then those of
 * the largest score; equal ones go to the lower slot, and a NaN score counts
 * as the smallest.  Of the kept slots, those below budget stay where they
 * are; the i-th kept slot at or above budget (ascending) moves, with its key,
 * value, score and position, into the i-th evicted slot below budget
 * (ascending).  A sequence of n <= budget slots keeps all.
 *   new_len[b] = min(n, budget);
 *   score_out, pos_out [b, h, j] = those of the slot now at j, for j < new_len; 0 and -1 beyond
 * The slots' order carries no meaning for brisk_block_attention (keys hold
 * their positions), so only moved slots are copied; the sources are left
 * unchanged.  seq_len is not updated: the caller takes new_len, and releases
 * the pages past it.
 *
 *   score_in, score_out  [B, n_kv_heads, cap] fp32;  pos_in, pos_out the same
 *               in int32
 *   next_pos    [B] int32  position of the next token (tokens seen so far)
 *   new_len     [B] int32 out; not seq_len itself (copy it there afterwards)
 *   ws          device scratch of brisk_cache_evict_workspace_size bytes
 *
 * No output, nor ws, may overlap another output or an input (next_pos, seq_len
 * and block_table among them), and no two places of the pages one another (as
 * where heads are one expanded head): BRISK_ERR_UNSUPPORTED.
 * Limits: the cache's; B >= 1, B * n_kv_heads <= 2^20, 1 <= cap <= 2^24,
 * B * n_kv_heads * cap <= 2^36, budget >= 1, 0 <= recent <= budget, and what
 * a launch holds: B * n_kv_heads * ceil(min(budget, cap - budget) / 64) < 2^24
 * and, past 32768 slots, B * n_kv_heads * ceil(cap / 4096) < 2^22 (at most 64
 * counted of the last quotient).  Lengths are cut to cap.  Two sequences must
 * not share a page that holds slots below budget of either.
 */
int brisk_cache_evict(const brisk_kv_cache* cache, int32_t B, const float* score_in,
                      const int32_t* pos_in, int32_t cap, const int32_t* next_pos, int32_t budget,
                      int32_t recent, float* score_out, int32_t* pos_out, int32_t* new_len, void* ws,
                      size_t ws_bytes, void* stream);

/* Workspace bytes brisk_draft_verify needs (written to *bytes). */
int brisk_draft_verify_workspace_size(int32_t B, int32_t V, size_t* bytes);

/*
 * Verification of drafted tokens against the target's probabilities, with the
 * random numbers given (Section 3.3, speculative acceptance; Algorithm 1(b)
 * verify and commit).  brisk_spec_verify is the form for a verifier's hidden
 * states and a law over K candidates; this one takes laws over the whole
 * vocabulary, as sampled or filtered by the caller.
 *   position i of block b accepts x = draft_tok[b, i] when
 *     u_accept[b, i] * draft_prob[b, i, x] < target_prob[b, i, x]   (fp32 product);
 *   a = accept_len[b] = the positions before the first one that does not, at
 *       most n = draft_len[b] (L when draft_len is NULL);
 *   w = [target_prob[b, a] - draft_prob[b, a]]_+ when a < n, or
 *       target_prob[b, a] when a = n or when that difference is positive nowhere;
 *   token[b] = argmax_v w_v / noise[b, v] over the v with w_v > 0, the lower
 *       id on ties; -1 when no such ratio is positive (in fp32: one that
 *       underflows to 0, or is NaN, is not).
 * With noise drawn from Exp(1), token follows the law w / sum w, so committed
 * tokens keep the target's law.
 *
 *   target_prob [B, L + 1, V] fp32, rows target_stride elements apart
 *   draft_prob  [B, L, V]     fp32, rows draft_stride elements apart
 *   draft_tok   [B, L] int32;  draft_len [B] int32, nullable (values are
 *               clamped into [0, L]);  u_accept [B, L] fp32
 *   noise       [B, V] fp32, rows noise_stride elements apart
 *   accept_len, token  [B] int32 out
 *   ws          device scratch of brisk_draft_verify_workspace_size bytes
 *
 * With L = 0 the draft's arrays may be NULL (a plain draw from the target).
 * Limits: B >= 1, 0 <= L <= 1024, B * (L + 1) <= 2^20, 1 <= V <= 2^24, row
 * strides >= V; 4-byte aligned pointers.
 */
int brisk_draft_verify(const float* target_prob, int64_t target_stride, const float* draft_prob,
                       int64_t draft_stride, const int32_t* draft_tok, const int32_t* draft_len,
                       const float* u_accept, const float* noise, int64_t noise_stride, int32_t B,
                       int32_t L, int32_t V, int32_t* accept_len, int32_t* token, void* ws,
                       size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BRISK_H_ */
