/*
 * gr.h -- C interface of the B200 (sm_100a) global-resolution library.
 *
 * For a batch of decode positions the library turns target logits, draft logits
 * and the number n of i.i.d. drafts into the optimal-transport verification rule
 * of "Global Resolution" (optimal multi-draft speculative sampling) and then
 * draws the emitted token for the n drafted tokens.
 *
 * Letters.  The paper writes p for the target distribution and q for the draft
 * distribution; this interface uses the opposite letters, as serving stacks do:
 *   q_logits = TARGET model logits,  p_logits = DRAFT model logits.
 * In the comments below "tgt" is the target distribution after temperature and
 * "drf" the single-token draft distribution after temperature, top-k truncation
 * and renormalisation (App. A, first paragraph; App. N).
 *
 * Conventions shared by every call
 *   - every pointer named below is a DEVICE pointer owned by the caller unless
 *     it is marked "host"; the library never allocates or frees device memory;
 *   - calls only enqueue work on `stream` (a cudaStream_t passed as void*) and
 *     return without synchronising;
 *   - the int return value is 0 (GR_OK) when the work was enqueued, or a negative
 *     GR_E_* code when the arguments were rejected on the host (nothing enqueued);
 *   - data-dependent outcomes are reported per instance in the status arrays.
 */
#ifndef GR_H_
#define GR_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* element type of the logits */
#define GR_F32  0
#define GR_BF16 1
/* further element types of caches, and of what goes in and comes out of them */
#define GR_F16  2
#define GR_Q4   3

/* per-instance status values (status arrays, device memory) */
#define GR_OK                    0
#define GR_NOT_CONVERGED         1  /* iteration cap reached; the rule is usable, its gradient norm is in params */
#define GR_SUPPORT_TOO_LARGE     2  /* support larger than GR_MAX_SUPPORT: no rule was solved; gr_verify falls
                                       back to sampling the target distribution (still lossless), the paper's
                                       "early termination" convention (Sec. 6.2 last paragraph, App. K)   */
#define GR_BAD_LOGITS            3  /* a NaN or infinite logit in the row                                 */
#define GR_DRAFT_OUT_OF_SUPPORT  4  /* a drafted token does not belong to the draft support               */
#define GR_STALE_PARAMS          5  /* params block was not written by gr_solve for this shape            */
#define GR_PARTIAL_RULE          6  /* params written by gr_solve_verify: only the system its drafted tuple
                                       selects was solved; gr_verify refuses such a block (token -1)       */
#define GR_CHECK_FAILED          7  /* bounds-checked build of the library only: a kernel skipped an access
                                       outside an array's extent while it worked on this instance          */
#define GR_NO_BLOCKS             8  /* gr_block_plan: the pool has too few free blocks for the row         */
#define GR_ROW_FULL              9  /* gr_block_plan: more tokens than the row's table or the slot map hold */
#define GR_BAD_ROW              10  /* gr_block_plan: a negative count, a length beyond the table, a parent outside
                                       the group, or a block id outside the pool; gr_cache_attend: a position
                                       beyond the table, or a block id outside the pool                     */

/* host-side argument errors (return values) */
#define GR_E_INVALID   (-1)  /* a size, temperature or option is out of range */
#define GR_E_NULL      (-2)  /* a required pointer is NULL                    */
#define GR_E_ALIGN     (-3)  /* a logits base pointer is not 16-byte aligned  */
#define GR_E_LAUNCH    (-4)  /* the CUDA runtime refused a launch             */
#define GR_E_TOO_LARGE (-5)  /* beyond a stated capacity                      */

/* capacities */
#define GR_MAX_SUPPORT 128   /* largest draft support for which the convex programs are solved */
#define GR_MAX_DRAFTS  32    /* largest n                                                     */
#define GR_MAX_BEAMS   32    /* largest number of hypotheses in a group                       */
#define GR_MAX_SELECT  128   /* most continuations gr_beam_select returns for a group, alternatives gr_token_logprobs returns */
#define GR_MAX_GIVEN   64    /* most tokens a row of gr_token_logprobs                        */
#define GR_MAX_HEADS   1024  /* most heads of a cache, and of queries                         */
#define GR_MAX_DIM     512   /* largest dim of a head in a 16- or 32-bit cache                */
#define GR_MAX_DIM_Q4  256   /* in a 4-bit cache                                              */

/*
 * Solver options (host struct, read during the call).  NULL selects the defaults.
 *   tol        stop when the L1 norm of the gradient of the convex function
 *              (Theta for the inner system, Phi restricted to a block for the outer
 *              system; Sec. 6.2) is <= tol.                      default 3e-7
 *              (The default sits just below the ~4.5e-7 that fp32 summation over a
 *              128k-token row leaves in the target's log-sum-exp, i.e. below the
 *              accuracy to which the target distribution itself is known; the emitted
 *              token's law then differs from that target by at most tol in L1.  Smaller
 *              values are honoured down to the quadrature floor of a few 1e-9 at the
 *              default quad_step.)
 *              The kernels also stop after a Newton step taken from a point evaluated
 *              on the full quadrature grid when the residual r' that step leaves is
 *              predicted below tol, in one of two ways.  By the step: from its second-order
 *              size s2 = sum_i g_i (delta alpha_i)^2 (r' stayed within 8.5 s2 + 3e-9 on every
 *              shape measured) and, in the faster kernel, where the Newton system is solved
 *              with a Hessian in half precision that may belong to an earlier point, from
 *              lin = (0.02 + 2 x the distance to that point) x the residual: stop when
 *              10 s2 + 3 lin < tol, reported 3 s2 + lin.  By the ratio (faster kernel only):
 *              after a step that contracted the residual to r by rho < 0.1, stop when
 *              3 c r < tol and 1.5 h r < tol, with c the larger of rho and the step's length and h (with such a
 *              Hessian) 0.02 + 2 x the distance, reported max(c, h) r.  On 28 kinds of rows at tolerances of 1e-8,
 *              3e-7 and 1e-5 a stop left at most 0.44 of what it reported, beyond the floor of 3e-9.  Neither
 *              is used when the Newton system is too close to singular in fp32: less than 2 %
 *              of a diagonal entry left as the factorisation's pivot, or of the Hessian's trace
 *              as the slope along the common scale of the weights.
 *   max_iters  cap on gradient evaluations per system.            default 40
 *   quad_step  accuracy of the rule by which the gradient integral is evaluated, as the step of
 *              a trapezoid rule in the log-time variable; smaller is more accurate and
 *              slower (largest relative error of a tuple's term at 0.25 2e-13, 0.3 3e-13, 0.35
 *              2e-11, 0.39 3e-10, 0.4 6e-10, 0.5 7e-8, 0.8 9e-5).  From 0.4 up the faster kernel
 *              takes rules with fewer nodes and a relative error of 2e-10 where the weights of an
 *              instance allow it, whatever the step: a larger one saves it nothing then.  (Evaluations
 *              that cannot end the iteration are fp32 by rules of 5e-7.)      default 0.4
 *   scan_done_event  optional cudaEvent_t (as void*) recorded on `stream` between
 *              the streaming kernel and the solve kernel, so that a caller can
 *              time the two separately; NULL records nothing.      default NULL
 *   force_robust  non-zero sends every shape to the general (slower) solve kernel;
 *              by default supports of at most 128 tokens with n >= 2 take a faster
 *              kernel that computes the same rule.  For an untruncated draft on a
 *              vocabulary beyond GR_MAX_SUPPORT (optimal acceptance only) it selects the
 *              whole-row sort instead of the bucketed search.         default 0
 *   tau        error threshold of Algorithm 1 (Sec. 6.2 "tunable errors", Sec. 6.3).  0 solves the
 *              convex programs on the whole support (the default: both tunable errors are 0 and `tol`
 *              is the stopping rule).  tau in (0, 1] selects the truncated variant: the inner system
 *              is solved on the fewest tokens T of H* with gamma_T = drf(H*)^n - drf(T)^n <= tau, every
 *              outer block on the fewest outer tokens T with epsilon_T = 1 - (drf(H*) + drf(T))^n <= tau
 *              (largest drf first), each to gradient norm 5 tau (`tol` is then not used); tokens outside
 *              the sets keep weight 0 (a tuple served only by such tokens of an outer block is shared
 *              equally among them).  The emitted token then follows the target within 15 tau in L1 and
 *              the acceptance is within 10 tau of alpha* (Lemma "Approximation Guarantee").     default 0
 */
typedef struct gr_options {
    double tol;
    int    max_iters;
    double quad_step;
    void*  scan_done_event;
    int    force_robust;
    double tau;
} gr_options;

/*
 * Bytes of the opaque per-batch `params` block that gr_solve writes and
 * gr_verify reads, and of the scratch `workspace` gr_solve needs while it runs.
 * Both depend only on the shape.  Return 0 when the shape is invalid.
 */
size_t gr_params_bytes(int V, int n, int topk, int batch);
size_t gr_workspace_bytes(int V, int n, int topk, int batch);

/*
 * gr_solve -- steps 1-3 of Algorithm 1 for every instance of the batch.
 *
 * Per instance (one decode position):
 *   tgt = softmax(q_logits / temp_target) over the whole vocabulary;
 *   support = the `topk` largest draft logits (equal logits: the smaller id is
 *   kept), drf = softmax(p_logits / temp_draft) over the support (App. N);
 *   H* and the optimal acceptance alpha* = 1 + min_H psi(H) by ordering the
 *   support by decreasing drf/tgt and scanning prefixes (Eq. "subset-select",
 *   Sec. 5.1; ties: smaller id first, shortest minimising prefix);
 *   outer residuals by cumulative minima of psi along the increasing-ratio
 *   chain (Sec. 6.1, Thm "polymatroid", Lemma "q-convex");
 *   softmax parameters exp(alpha_i) of the inner system on H* (Thm "Inner
 *   Convex Solver") and of every block of the outer system (Thm "Outer Convex
 *   Solver" restricted to the tokens between two consecutive tight prefixes),
 *   with the full truncation set T (tunable errors epsilon_T = gamma_T = 0).
 *
 * Arguments
 *   q_logits, p_logits  [batch, V] row-major, dtype GR_F32 (float) or GR_BF16;
 *                       base pointers 16-byte aligned; read only.
 *   V >= 1, 1 <= n <= GR_MAX_DRAFTS, batch >= 0.
 *   topk                1..V-1 truncates the draft; 0 or >= V keeps every id.
 *   temp_target, temp_draft   > 0.
 *   opt                 host pointer or NULL.
 *   params              out, gr_params_bytes() bytes, 16-byte aligned.  It records
 *                       the address of q_logits: gr_verify re-reads at most one
 *                       1024-element chunk of a target row on the resample branch,
 *                       so q_logits must stay unchanged until gr_verify has run.
 *   workspace           scratch, gr_workspace_bytes() bytes, 16-byte aligned;
 *                       contents are meaningless after the call completes.
 *   alpha_star          out [batch] float, optimal acceptance probability (also produced when the support
 *                       exceeds GR_MAX_SUPPORT and no rule is solved: by a bucketed search over the whole row,
 *                       or a sort where the buckets do not separate it).
 *   status              out [batch] int, GR_OK / GR_NOT_CONVERGED /
 *                       GR_SUPPORT_TOO_LARGE / GR_BAD_LOGITS.
 */
int gr_solve(const void* q_logits, const void* p_logits, int dtype, int V, int n, int topk,
             float temp_target, float temp_draft, int batch, const gr_options* opt,
             void* params, void* workspace, float* alpha_star, int* status, void* stream);

/*
 * gr_solve_static -- gr_solve without the `workspace` argument, for callers that cannot
 * allocate device memory.  (The paper has no counterpart: this is an interface variant.)
 *
 * Who needs it: a serving loop that has handed all free device memory to its own pool
 * (KV cache, activation arena) and therefore must not call cudaMalloc at steady state --
 * the call may fail there and it synchronises the whole device -- or a host that is not
 * allowed to allocate at all once it is running (latency-bounded control loops).  Such a
 * caller still owns `params` and the outputs, but has nowhere to take scratch from.
 *
 * The scratch is a fixed array inside the library's device image, GR_STATIC_MAX_BATCH
 * instances large (about 0.4 MB, held by every GPU that loads the library until exit).
 *   - batch > GR_STATIC_MAX_BATCH returns GR_E_TOO_LARGE and launches nothing; split the batch.
 *     So does an untruncated draft on a vocabulary larger than GR_MAX_SUPPORT (its alpha* needs a
 *     per-row sort buffer the built-in scratch does not have).
 *   - The first call on each device looks the array's device address up (that device must
 *     be current, as for any launch); make that first call before any stream capture.
 *   - The call itself allocates and frees nothing.
 *   - All calls share the one array and it keeps the previous call's contents.  Nothing in it
 *     needs clearing (each call rewrites all it reads), but two calls whose kernels overlap on
 *     the GPU -- different streams, or different host threads -- race on it: serialise them.
 * Every other argument, the outputs and the statuses are exactly those of gr_solve, and
 * gr_verify / gr_read_rule take the resulting `params` unchanged.
 */
#define GR_STATIC_MAX_BATCH 256
int gr_solve_static(const void* q_logits, const void* p_logits, int dtype, int V, int n, int topk,
                    float temp_target, float temp_draft, int batch, const gr_options* opt,
                    void* params, float* alpha_star, int* status, void* stream);

/*
 * gr_verify -- step 4 of Algorithm 1 (the slice pi(.|omega), Eqs. "cases" and
 * "approx-c", normalised) and the draw of App. A steps 3-4.
 *
 * Per instance, U = distinct drafted tokens in order of first occurrence.
 * If U lies in H*: pi(i) = w_i / (1 + sum_U w) and the rest, 1 / (1 + sum_U w), goes
 * to the resample distribution (residuals / (1 - alpha*)); otherwise only the
 * tokens of the lowest-ratio block met by U share the mass, pi(i) = w_i / sum w.
 * The emitted token is the first segment (U's tokens in order, then the resample
 * segment) whose cumulative probability exceeds u0; inside the resample segment
 * it is the first id (ascending) whose cumulative residual exceeds u1 times the
 * total residual.
 *
 *   params        written by gr_solve for the same batch; read only.
 *   draft_tokens  [batch, n] int32 (n as given to gr_solve).
 *   uniforms      [batch, 2] float in [0,1): (u0, u1).
 *   out_token     out [batch] int32 emitted id, -1 on a per-instance error.
 *   out_accepted  out [batch] 1 iff the emitted token is one of the drafts.
 *   status        out [batch] GR_OK / GR_DRAFT_OUT_OF_SUPPORT / GR_STALE_PARAMS /
 *                 GR_BAD_LOGITS, or the solve status when it was not GR_OK.
 */
int gr_verify(const void* params, const int* draft_tokens, const float* uniforms, int batch,
              int* out_token, unsigned char* out_accepted, int* status, void* stream);

/*
 * gr_solve_verify -- gr_solve and gr_verify in one call for drafts known beforehand:
 * the solve kernel of every instance looks at its drafted tuple, solves only the
 * system that tuple selects (Eq. "cases": the inner system when every drafted token
 * lies in H*, else the lowest-ratio outer block the tuple meets; Algorithm 1 does the
 * same) and finishes with the draw itself, so no separate verification launch and no
 * second read of the rule.  Arguments as for gr_solve and gr_verify; `status` holds
 * what gr_verify would report.  alpha_star is written as by gr_solve.  The params block
 * is still written (for gr_read_rule); instances where a system was skipped carry
 * GR_PARTIAL_RULE in it and must not be given to gr_verify with other drafts.
 * Same return values as gr_solve.
 */
int gr_solve_verify(const void* q_logits, const void* p_logits, int dtype, int V, int n, int topk,
                    float temp_target, float temp_draft, int batch, const gr_options* opt,
                    const int* draft_tokens, const float* uniforms, void* params, void* workspace,
                    float* alpha_star, int* out_token, unsigned char* out_accepted, int* status,
                    void* stream);

/*
 * gr_alpha_star -- the optimal acceptance alpha* = 1 + min_H psi(H) alone (Eq. "subset-select"), for up to
 * GR_MAX_ALPHA_N draft counts at once: one pass over the logits (the same streaming kernel as gr_solve) and a
 * prefix scan along the ratio order, which all the draft counts share.  No rule is solved and no params block
 * is written; this is what an acceptance-versus-(n, k) sweep needs.
 *   n_list      HOST array of n_count draft counts, each in 1..GR_MAX_DRAFTS.
 *   workspace   scratch of gr_workspace_bytes(V, 1, topk, batch) bytes, 16-byte aligned.
 *   alpha_star  out [batch, n_count] float, row-major; NaN where status is not GR_OK.
 *   status      out [batch]: GR_OK or GR_BAD_LOGITS.
 * Supports: top-k up to GR_MAX_SUPPORT, or the whole vocabulary of any size (beyond GR_MAX_SUPPORT tokens
 * the minimum of psi is searched per draft count without sorting the row, as in gr_solve); a top-k beyond
 * GR_MAX_SUPPORT on a larger vocabulary returns GR_E_TOO_LARGE.
 * Other return values as gr_solve.
 */
#define GR_MAX_ALPHA_N 8
int gr_alpha_star(const void* q_logits, const void* p_logits, int dtype, int V, const int* n_list, int n_count,
                  int topk, float temp_target, float temp_draft, int batch, void* workspace,
                  float* alpha_star, int* status, void* stream);

/*
 * gr_read_rule -- copies the rule of every instance out of `params` into plain
 * arrays (for inspection and tests); all outputs are optional (NULL skips).
 * Per-support arrays have `kcap` entries per instance and are filled in ratio
 * order (position 0 = largest drf/tgt); unused entries are set to -1 / 0.
 *   ids    [batch,kcap] int   token id          w   [batch,kcap] double exp(alpha_i)
 *   block  [batch,kcap] int   -1 on H*, else block number counted from the lowest ratio
 *   resid  [batch,kcap] double outer residual r_i (0 on H*)
 *   flow   [batch,kcap] double p_i = tgt_i - r_i
 *   header [batch,8] double: k, jstar, nblocks, alpha_star, gnorm, iterations, lse of the target row, status
 *          (iterations = gradient evaluations spent, plus 65536 when the gradient norm of at least one of the
 *          instance's convex programs is a prediction from its last Newton step rather than an evaluation)
 */
int gr_read_rule(const void* params, int batch, int kcap, int* ids, int* block, double* w,
                 double* resid, double* flow, double* header, void* stream);

/*
 * gr_read_slice -- the slice pi(.|omega) of every instance for its drafted tuple (Eq. "cases" and Eq. "approx-c",
 * "normalized" as in Algorithm 1), computed by the same device code gr_verify draws from, for inspection and tests:
 * what gr_verify compares u0 with, without the draw.
 *   params        written by gr_solve (not by gr_solve_verify) for the same batch; read only.
 *   draft_tokens  [batch, n] int32, n as given to gr_solve.
 *   U    out [batch, n] int32: U[b, s] = drafted token s of instance b, or -1 when it repeats an earlier one.
 *   pi   out [batch, n] double: probability that token is emitted (0 for repeats, and for tokens outside the
 *        block that serves the tuple); the accepted segments of the draw are these, in this order.
 *   rho  out [batch] double: mass of the resample segment (1 / (1 + sum of the weights) when every drafted token
 *        lies in H*, else 0).
 *   status out [batch]: GR_OK / GR_NOT_CONVERGED (slice given), or GR_DRAFT_OUT_OF_SUPPORT /
 *        GR_SUPPORT_TOO_LARGE / GR_BAD_LOGITS / GR_PARTIAL_RULE / GR_STALE_PARAMS (no slice: U = -1, pi = 0).
 */
int gr_read_slice(const void* params, const int* draft_tokens, int batch, int n, int* U, double* pi,
                  double* rho, int* status, void* stream);

/*
 * ------------------------------------------------------------------------------------------------
 * Around the decoding step: beam search's selection (the other rule that turns logit rows into emitted
 * tokens), and what a serving loop does with the outcome of either rule -- hypotheses, drafted or searched,
 * go on from a parent's state, in dense states (gr_reorder_states) or in a paged cache (gr_block_plan,
 * gr_copy_blocks).  (The paper has no counterpart.)  Conventions as above.
 * A workspace is scratch of one call: calls that may run at the same time (other streams, captured graphs) need one each.
 * ------------------------------------------------------------------------------------------------
 *
 * gr_beam_select -- the best continuations of every group of `beams` hypotheses.
 *
 * Of group b, hypothesis w and token v, with x = logits[b, w, v]:
 *   total = scores[b, w] + x / temperature - log sum_v' exp(x' / temperature),
 *   key   = total / L^length_penalty,  L = max(1, lengths[b, w] + 1)   (key = total without `lengths`);
 * a finished hypothesis (done[b, w] != 0) has the one continuation `eos`, with total = scores[b, w] and
 * L = max(1, lengths[b, w]); its logits are not read.  The `select` largest keys are returned in descending
 * order; equal keys: the smaller w first, then the larger logit, then the smaller v.  Keys are compared as
 * 64-bit values (of temperature and length_penalty as the call takes them, rounded to float); where two hypotheses'
 * continuations come closer than the bounds of the streaming pass's errors, their rows' sums are taken again in 64 bits.
 *   logits   [batch, beams, V], dtype GR_F32 or GR_BF16: row (b, w) begins (b * beams + w) * ld elements after
 *            the base pointer (aligned to the element), ld >= V.  -infinity masks a token: it is never returned, and
 *            a row may be masked as a whole.  NaN or +infinity in a row that is read: GR_BAD_LOGITS.
 *   scores   [batch, beams] float.  -infinity: there is no such hypothesis, its logits are not read.
 *            NaN or +infinity: GR_BAD_LOGITS.
 *   lengths  [batch, beams] int or NULL; |length_penalty| <= 32 (0 without lengths).
 *   done     [batch, beams] bytes or NULL (no hypothesis is finished).  With `done`, eos must be a token id;
 *            without, eos may be -1 (no token finishes a hypothesis).
 *   1 <= beams <= GR_MAX_BEAMS, 1 <= select <= GR_MAX_SELECT, V <= 2^21, temperature > 0.
 *   workspace   gr_beam_workspace_bytes() bytes, 16-byte aligned.
 *   out_token, out_parent [batch, select] int; out_score [batch, select] float (total); out_length [batch,
 *            select] int (L) or NULL; out_done [batch, select] bytes: the parent was finished or the token is
 *            eos.  Places that no continuation is left for: token -1, parent -1, score -infinity, length 0,
 *            done 0; all places of a group with GR_BAD_LOGITS.  None of them may be an input of the same call.
 *   status   out [batch] GR_OK or GR_BAD_LOGITS.
 */
size_t gr_beam_workspace_bytes(int V, int beams, int select, int batch);
int gr_beam_select(const void* logits, int dtype, int V, long long ld, int beams, int batch, float temperature,
                   const float* scores, const int* lengths, const unsigned char* done, int eos,
                   float length_penalty, int select, void* workspace, int* out_token, int* out_parent,
                   float* out_score, int* out_length, unsigned char* out_done, int* status, void* stream);

/*
 * gr_reorder_states -- state j of group b becomes a copy of state parents[b, j] of that group, in `count`
 * tensors of one layout (the layers' caches, recurrent states, drafted hidden states).
 *
 * A state is `parts` pieces (heads, say) of part_bytes bytes.  Piece p of state w of group b begins
 * b * src_group + w * src_beam + p * src_part bytes after src[i], and likewise for dst[i].
 *   src, dst   HOST arrays of `count` device pointers.  dst[i] == src[i] with equal strides reorders in place (any
 *              mapping, cycles and repeated parents included); otherwise no dst may meet a src (from the first byte of its
 *              pieces to the last: GR_E_INVALID).  Two dst that share a byte are GR_E_INVALID (one may lie between the pieces
 *              of another), and so are strides that make the pieces of a dst overlap.  Within src, groups, states and
 *              pieces may coincide (stride 0), unless it is reordered in place.
 *   parents    [batch, beams_out] int.  -1, or any number outside 0 .. beams_in - 1: that state is left as it was.
 *   lengths    [batch, beams_in] int or NULL.  With it a piece is a run of tokens of token_bytes bytes each and only the
 *              first lengths[b, parent] tokens of each piece are copied (clamped to what the piece holds); the
 *              rest of dst stays as it was.  token_bytes must divide part_bytes.
 *   1 <= beams_in, beams_out <= GR_MAX_BEAMS; in place beams_out <= beams_in.
 * No workspace.  Any alignment works; pointers, strides and part_bytes that are multiples of 16 are fastest.
 */
typedef struct gr_state_layout {
    int       batch, beams_in, beams_out, parts;
    long long src_group, src_beam, src_part;
    long long dst_group, dst_beam, dst_part;
    long long part_bytes;
    long long token_bytes;
} gr_state_layout;
int gr_reorder_states(const void* const* src, void* const* dst, int count, const gr_state_layout* layout,
                      const int* parents, const int* lengths, void* stream);

/*
 * gr_block_plan -- block tables and slots of a paged cache for the next step, built on the device.
 *
 * A pool of num_blocks blocks of block_size tokens serves `rows` rows, each with a table of `width` block ids and
 * a number of tokens: token t of row r lies in block table[r, t / block_size] at t % block_size.  Blocks may be
 * shared between rows; refs[i] counts the rows that hold block i (0: free).  Rows form groups of `beams`.
 * Per row r of a group, in one call:
 *   1. it goes on from row parents[r] of its group (NULL: from itself; -1: from nothing, it holds no tokens then),
 *      of which it keeps base = min(lengths[parent], keep[r]) tokens (keep NULL: all of them), and the blocks
 *      they lie in; what it held otherwise is released.  Parents are read before any row changes.
 *   2. append[r] tokens are added.  Where the first of them lands in a partly filled block that another row
 *      holds too, the row gets a block of its own for it and the pair (copy_src, copy_dst) is listed, to be
 *      copied (gr_copy_blocks) before the new tokens are written.  If every holder of the block is about to write to it,
 *      the one with the most tokens in it (the lowest row of several) keeps it and only the others copy.
 *   3. new blocks are the free ones with the smallest ids, taken in the order of the rows (the copy's first), those that
 *      were released in this call among them.
 * Rows that cannot be served keep their `base` tokens and blocks and get no new ones; status says why:
 *   GR_ROW_FULL   more tokens than width * block_size, or more appended tokens up to and with this row than max_tokens;
 *   GR_NO_BLOCKS  the row needs blocks, and up to and with it (counting all rows that are not GR_ROW_FULL or GR_BAD_ROW)
 *                 more are needed than are free;
 *   GR_BAD_ROW    append[r] < 0 (taken as 0), lengths[parent] outside 0 .. width * block_size (clamped), a parent outside
 *                 -1 .. beams - 1 (taken as -1), or a held block id outside the pool, where the call meets one: it looks at
 *                 all blocks of a row that goes on from another, and at the partly filled one that is to be written to.
 *   keep[r] < 0 counts as 0.
 *   table     in/out [rows, width] int.  Entries that a row no longer holds become -1.  (Start with -1 everywhere.)
 *   lengths   in/out [rows] int;  refs in/out [num_blocks] int.   (Start with 0.)
 *   slots     out [max_tokens] long long: slot (block * block_size + offset) of every appended token, row after row;
 *             -1 for the tokens of rows that were not served and behind the last one.
 *   positions out [max_tokens] int: index of the token within its row, -1 where slots is.
 *   offsets   out [rows + 1] int: row r's tokens are offsets[r] .. offsets[r + 1] - 1 (by append as given, cut at max_tokens).
 *   copy_src, copy_dst  out [rows] int, -1 where nothing is copied.
 *   status    out [rows].
 *   workspace gr_block_workspace_bytes() bytes, 16-byte aligned.
 *   rows a multiple of beams, 1 <= beams <= GR_MAX_BEAMS (beams only matters with parents), rows <= 2^20,
 *   rows * width < 2^31, num_blocks <= 2^26, width * block_size < 2^31.  The arrays must not overlap one another (but keep
 *             may be lengths).
 */
size_t gr_block_workspace_bytes(int rows, int num_blocks);
int gr_block_plan(int* table, int rows, int width, int beams, int block_size, int* lengths, int* refs, int num_blocks,
                  const int* parents, const int* keep, const int* append, int max_tokens, void* workspace,
                  long long* slots, int* positions, int* offsets, int* copy_src, int* copy_dst, int* status,
                  void* stream);

/*
 * gr_copy_blocks -- block copy_dst[i] of every cache becomes a copy of block copy_src[i], for the listed pairs.
 *   caches      HOST array of `count` device pointers; block k of a cache begins k * block_stride bytes after it and
 *               is block_bytes long (block_stride >= block_bytes).  Two caches that share a byte are GR_E_INVALID (one may
 *               lie between the blocks of another).
 *   copy_src, copy_dst  [pairs] int, as gr_block_plan writes them: a pair with an index outside 0 .. num_blocks - 1 (-1:
 *               nothing to copy) is skipped.  Blocks that are copied to must be distinct and none may be copied from.
 *   pairs <= 2^24 - 256; blocks up to 2^22 x 1024 bytes times the power of two (up to 16) that divides pointers, stride and size.
 * No workspace.  Any alignment works; multiples of 16 are fastest.
 */
int gr_copy_blocks(void* const* caches, int count, int num_blocks, long long block_stride, long long block_bytes,
                   const int* copy_src, const int* copy_dst, int pairs, void* stream);

/*
 * ------------------------------------------------------------------------------------------------
 * Filling and reading a paged cache: what gr_block_plan's slots, positions and offsets are for.
 *
 * A cache holds keys and values of `heads` heads of `dim` elements for num_blocks blocks of block_size tokens; slot
 * z is token z % block_size of block z / block_size.
 *   format GR_F32, GR_BF16, GR_F16: two arrays, in each of which (block, token, head) begins block * block_stride + token * token_stride +
 *       head * head_stride elements after the pointer.  dim even, <= GR_MAX_DIM.  No two places may share an element.
 *   format GR_Q4: one array (`keys`; `values` is not looked at), aligned to 16 bytes; block b begins b * block_stride BYTES after it (a
 *       multiple of 16; the other strides are not looked at) and holds, for each head, block_size / 8 octets of 9 dim bytes,
 *       one after another.  dim a multiple of 32, <= GR_MAX_DIM_Q4, block_size a multiple of 8.
 *       Groups of 32 dims share a 16-bit scale s; a number x is held as a code u of 4 bits that stands for s (u - 8):
 *       s = fp16(-x* / 8), x* the group's element of largest magnitude (of +a and -a the positive one; beyond 524032: clamped), u = 8 + x / s
 *       rounded to the nearest whole number (ties to even), from 0 to 15.  4.5 bits an element.  A group with a NaN or an infinity
 *       has the scale NaN.  With J = dim / 32, an octet (eight tokens of a head) holds, one after another,
 *         keys' codes    [8 tokens][4][J] words: word (t, j): dims 32 j + 8 t .. + 7, the first in its lowest bits
 *         keys' scales   [8 tokens][J] fp16
 *         values' codes  [8][4 pairs of tokens][J][2 tokens] 16-bit words: word (g, ., j, .): dims 32 j + 4 g .. + 3
 *         values' scales [4 pairs of tokens][J][2 tokens] fp16
 *       A block is whole bytes of its own, as gr_copy_blocks wants it; bytes of different tokens are different bytes.
 *   heads <= GR_MAX_HEADS.
 */
typedef struct gr_cache_layout {
    int       format, heads, dim, block_size, num_blocks;
    long long block_stride, token_stride, head_stride;
} gr_cache_layout;

/*
 * gr_cache_append -- new tokens' keys and values go to their slots, keys and queries rotated by the tokens' positions on the way.
 *
 * Token i with slot z = slots[i] (outside the cache, -1 say: nothing is written to the cache) and position p = positions[i]:
 * of the first `rot` dims of a key or query, pair c is turned by the angle p * frequencies[c],
 *   a' = a cos - b sin,  b' = b cos + a sin,
 * with (a, b) dims (c, c + rot / 2), or (2 c, 2 c + 1) if `interleaved`.  The angle is a 64-bit number, its cosine and sine are rounded to
 * 32 bits, products and sums are rounded to 32 bits one by one, the result once more, to what holds it.  Cosine and sine of angles of 2^50 and
 * more in magnitude, next to which 64-bit numbers are a fifth apart and more, are NaN, as they are where an angle is no number.
 *   k, v      [tokens, heads, dim] of type dtype (GR_F32, GR_BF16, GR_F16): (i, h) begins i * k_token + h * k_head elements after k.
 *   q, q_out  [tokens, q_heads, dim] likewise, of the same type; q_heads 0: there are none.  Queries of tokens with a negative position
 *             are left as they were in q_out.  q_out may be q, with equal strides; no other array that is written may share a byte with one that
 *             is read or another that is written, and no two places of q_out may share one.
 *   slots     [tokens], no slot twice.     positions [tokens]; without frequencies, that is rot 0, they may be NULL, and all queries are then written.
 *   rot       even, 0 .. dim.              frequencies [rot / 2] double.
 *   Strides of k, v and q below 2^31.
 * Any alignment to the element works; pointers and strides that are multiples of 16 bytes are fastest.
 */
typedef struct gr_cache_tokens {
    const void *k, *v, *q;
    void*     q_out;
    int       dtype, q_heads;
    long long k_token, k_head, v_token, v_head, q_token, q_head, out_token, out_head;
} gr_cache_tokens;
int gr_cache_append(void* keys, void* values, const gr_cache_layout* layout, const gr_cache_tokens* in, int tokens,
                    const long long* slots, const int* positions, const double* frequencies, int rot, int interleaved,
                    void* stream);

/*
 * gr_cache_read -- keys and values of listed slots, as numbers: k[i], v[i] become what slot slots[i] holds, rounded once to dtype (GR_F32,
 * GR_BF16, GR_F16); zeros for a slot outside the cache.  A slot may be listed any number of times.
 *   k, v   [tokens, heads, dim]: (i, h) begins i * k_token + h * k_head elements after k, and likewise for v.  No two places of them may share a
 *          byte, nor one with the cache or the slots (k and v may lie between one another's places).
 */
int gr_cache_read(const void* keys, const void* values, const gr_cache_layout* layout, const long long* slots, int tokens,
                  int dtype, void* k, long long k_token, long long k_head, void* v, long long v_token, long long v_head,
                  void* stream);

/*
 * gr_cache_attend -- attention of each row's query tokens over the row's tokens in a 4-bit cache.
 *
 * Query tokens offsets[r] .. offsets[r + 1] - 1 of row r have the positions positions[offsets[r]], + 1, + 2, ... (only the first is
 * read; negative: all of them see nothing), as gr_block_plan leaves its appended tokens: one for a decoding step, a run of drafted ones, a
 * prompt's.  The query of head i of a token at position p becomes
 *   out = sum_t w_t v_t / sum_t w_t,   w_t = exp(scale q . k_t),   over the row's tokens t with p - window < t <= p  (window 0: t <= p),
 * k_t, v_t those of key head i / (q_heads / heads) that slot table[r, t / block_size] * block_size + t % block_size holds.
 * What is held in other places does not tell, whatever it is.  A query that sees nothing gets zeros.  One that sees a NaN gets no number anywhere, be the
 * NaN in one group of a value alone (a token whose weight is nothing beside the largest may be left out).
 * Weights and their products with the values' scales are rounded to 11 bits each, those far below the largest to 2^-35 of that.
 *   q, out    [tokens, q_heads, dim], GR_BF16 or GR_F16: (i, h) begins i * q_token + h * q_head elements after q, i * out_token + h * out_head after out.
 *             out must not meet q or the cache in memory, and no two of its places may share an element; out, workspace and status share no byte with one
 *             another or with what is read.  What lies behind the last row's tokens is left as it was.
 *   cache     of format GR_Q4, as in gr_cache_append.
 *   table     [rows, width] int;  offsets [rows + 1] int, ascending, 0 .. tokens;  positions [tokens] int.
 *   heads divides q_heads.  Strides of q below 2^31.  window >= 0.  |scale| < 1.7e38.  rows <= 2^20, rows * width < 2^31, width * block_size < 2^31 - 256,
 *             tokens * (q_heads / heads) < 2^31 - 256.
 *             The kernel is chosen by tokens / rows, room behind the last row's tokens included: give it the tokens that there are, and prompts in a
 *             call of their own, not among rows of one token.
 *   workspace gr_attend_workspace_bytes() bytes, aligned to 32.
 *   status    out [rows]: GR_OK; GR_BAD_ROW where offsets are none, a position is beyond the table, or a block id of a token that is looked at is outside the
 *             pool (such tokens are left out); GR_CHECK_FAILED in all rows when a copy did not arrive in two seconds (out is then not to be used).
 */
size_t gr_attend_workspace_bytes(int heads, int q_heads, int dim, int rows, int tokens);
int gr_cache_attend(const void* q, int dtype, int q_heads, long long q_token, long long q_head, const void* cache,
                    const gr_cache_layout* layout, const int* table, int width, int rows, const int* offsets,
                    const int* positions, int tokens, float scale, int window, void* workspace, void* out,
                    long long out_token, long long out_head, int* status, void* stream);

/*
 * ------------------------------------------------------------------------------------------------
 * gr_token_logprobs -- log probabilities of given tokens under logit rows, the rows' entropies and their likeliest tokens.
 *
 * Of row i, with x = logits[i, v] / temperature and lse = log sum_v exp(x_v):
 *   logprob[i, j] = x_t - lse for t = tokens[i, j] (-infinity for one outside 0 .. V - 1),
 *   entropy[i]    = - sum_v p_v log p_v,  p_v = exp(x_v - lse),
 *   top_token[i]  the `top` tokens of largest logits in descending order (equal logits: the smaller id first), top_logprob[i] theirs.
 *   logits   [rows, V], dtype GR_F32 or GR_BF16: row i begins i * ld elements after the pointer (aligned to the element), ld >= V.
 *            -infinity masks a token: its log probability is -infinity and it is not among the likeliest; so are all of a row that is masked as a
 *            whole, whose entropy is 0.  NaN or +infinity: GR_BAD_LOGITS, log probabilities and entropy NaN, no likeliest.
 *   tokens   [rows, given] int, given 0 .. GR_MAX_GIVEN (0: NULL, as logprob may be).
 *   top      0 .. GR_MAX_SELECT (0: top_token and top_logprob may be NULL).  Places that no token is left for: -1, -infinity.
 *   logprob [rows, given], entropy [rows] (or NULL), top_token, top_logprob [rows, top], status [rows]: out, apart from one another and from
 *            what is read.  status: GR_OK or GR_BAD_LOGITS.
 *   V <= 2^21, rows <= 2^26, temperature > 0.  No workspace.
 */
int gr_token_logprobs(const void* logits, int dtype, int V, long long ld, int rows, float temperature, const int* tokens,
                      int given, int top, float* logprob, float* entropy, int* top_token, float* top_logprob, int* status,
                      void* stream);

/* Text for a GR_* / GR_E_* code (host pointer to a static string). */
const char* gr_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* GR_H_ */
