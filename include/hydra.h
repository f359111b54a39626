/*
 * hydra.h -- C ABI of the Hydra-PPO hot path on MI355X (gfx950).
 *
 * The operations follow "Efficient RLHF: Reducing the Memory Usage of PPO"
 * (arXiv 2309.00754):
 *   - LoRA on every linear layer of the actor and critic (Sec. 2, Stage 3);
 *   - Dynamic LoRA: the reference / reward model is the same network with the
 *     LoRA parameters ignored, LO(.) (Sec. 3, "Dynamic LoRA");
 *   - Hydra-PPO: one frozen base and two adapter sets, actor and critic; the
 *     active set is the one whose (A, B) pair is passed (Sec. 3, "Stage 2");
 *   - pi^hydra's two heads: a causal-LM head and a scalar reward head on the
 *     same input (Sec. 3, opening paragraph);
 *   - reward and reference log-probabilities from the LoRA-off model
 *     (App. A, Alg. 1 and Alg. 2).
 *
 * Conventions shared by every entry point
 *   - All tensor arguments are DEVICE pointers (hipMalloc'd or equivalent),
 *     row-major and contiguous.  bf16 values are passed as uint16_t bit
 *     patterns.  Operands read with 16-byte vector loads (x, W, A, h, W_lm,
 *     the fp32 logits and the workspace) must be 16-byte aligned; fp32 and
 *     int32 arrays 4-byte aligned; B and w_rm 2-byte aligned.
 *   - A linear layer's frozen weight W is stored output-major [N x K] (the
 *     nn.Linear.weight layout), LoRA-down A is [r x K], LoRA-up B is [N x r]:
 *         y_off = x W^T                     (LoRA off)
 *         y_on  = x W^T + s (x A^T) B^T     (LoRA on)
 *     Products are bf16 x bf16 with fp32 accumulation; outputs are fp32.
 *   - Ownership: the caller owns every buffer.  The library allocates no
 *     device memory and keeps no mutable global state; calls on different
 *     streams are independent.
 *   - Asynchrony: each call validates its arguments on the host, enqueues its
 *     kernels on `stream` (a hipStream_t; NULL = the default stream) and
 *     returns.  Inputs must stay valid until the stream reaches that point.
 *   - Errors: argument errors are detected on the host before any HIP call and
 *     returned as a negative status with nothing enqueued.  A failed launch
 *     returns HYDRA_ERR_HIP.  Data errors found on the device (a token id
 *     outside [0, V)) produce NaN in that token's outputs and OR 1 into
 *     *err_flag when err_flag is non-NULL.  NaN / Inf inputs propagate.
 *   - Results are deterministic: no floating-point atomics; every reduction
 *     runs in a fixed order, and the LoRA-on and LoRA-off log-softmax use
 *     identical reduction trees, so KL is exactly 0 wherever the two logit
 *     rows are equal (e.g. r = 0, s = 0 or B = 0).
 */
#ifndef HYDRA_H_
#define HYDRA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HYDRA_OK = 0,
  HYDRA_ERR_NULL = -1,        /* a required pointer is NULL                         */
  HYDRA_ERR_SHAPE = -2,       /* a size is out of range or inconsistent             */
  HYDRA_ERR_ALIGN = -3,       /* a pointer is not aligned as required               */
  HYDRA_ERR_UNSUPPORTED = -4, /* a valid request the library does not handle        */
  HYDRA_ERR_WORKSPACE = -5,   /* the workspace is missing or too small              */
  HYDRA_ERR_HIP = -6          /* the HIP runtime reported an error at launch        */
} hydra_status;

/* Element type of a tensor that a call takes in either. */
typedef enum {
  HYDRA_BF16 = 0, /* bf16 bit patterns, 2-byte aligned */
  HYDRA_F32 = 1   /* fp32, 4-byte aligned              */
} hydra_dtype;

/* Largest LoRA rank accepted. */
#define HYDRA_MAX_RANK 128

/*
 * hydra_lora_linear -- the LoRA-switchable linear layer.
 * Defined by: Sec. 2 Stage 3 (LoRA on all linears), Sec. 3 "Dynamic LoRA"
 * (LO(.) = LoRA off on the same W) and "Stage 2: Hydra-PPO" (the adapter set
 * in use is the (A, B) passed).
 *
 *   x     [M x K] bf16   input rows (tokens)
 *   W     [N x K] bf16   frozen base weight, read once for both outputs
 *   A     [r x K] bf16   LoRA down projection (may be NULL iff r == 0)
 *   B     [N x r] bf16   LoRA up projection   (may be NULL iff r == 0)
 *   s     fp32           LoRA scale
 *   y_off [M x N] fp32   out: x W^T                  (NULL: not written)
 *   y_on  [M x N] fp32   out: x W^T + s (x A^T) B^T  (NULL: not written)
 * At least one output must be non-NULL.  Requires 1 <= M <= 2^20, 1 <= N <= 2^21,
 * K >= 1, K % 8 == 0, K <= 2^21, 0 <= r <= HYDRA_MAX_RANK, and
 * ceil(M / 128) * ceil(N / 256) < 2^23 (the GEMM's tile grid fits one
 * dispatch; roughly M * N < 2^38).  With r == 0, y_on equals y_off.  M <= 8
 * (with y_on and r > 64 M <= 16) selects the bandwidth-bound (decode) kernels,
 * larger M the MFMA GEMM; both compute the same function.  At M > 16 with y_on
 * and r > 64 the update needs the pre-pass workspace of hydra_lora_linear_ws:
 * this call then returns HYDRA_ERR_WORKSPACE and launches nothing.
 */
hydra_status hydra_lora_linear(const uint16_t* x, const uint16_t* W, const uint16_t* A, const uint16_t* B,
                               float s, int64_t M, int64_t N, int64_t K, int64_t r,
                               float* y_off, float* y_on, void* stream);

/*
 * hydra_lora_linear_workspace_bytes -- device workspace that hydra_lora_linear_ws
 * needs for M rows, N outputs and rank r (0 when none is needed: r == 0).
 * Writes *bytes.  HYDRA_ERR_NULL for a NULL `bytes`, HYDRA_ERR_SHAPE for M
 * outside [1, 2^20], N outside [1, 2^21] or r outside [0, HYDRA_MAX_RANK].
 */
hydra_status hydra_lora_linear_workspace_bytes(int64_t M, int64_t N, int64_t r, size_t* bytes);

/*
 * hydra_lora_linear_ws -- hydra_lora_linear with a caller-provided workspace,
 * which lets the MFMA GEMM (M > 16) take the LoRA update from a pre-pass:
 * s x A^T is computed once per row (instead of once per column tile) as bf16
 * hi and lo parts, and added with B as 2 RP more k values of the GEMM (RP = r
 * rounded up to 16, 32, 64 or 128).  This is the path for the paper's rank 128
 * (App. B), and on the GEMM's largest tile (128 x 256) the faster one above
 * rank 16, where the in-tile product of hydra_lora_linear adds RP / 256 of the
 * base GEMM's work; at rank 16 the pre-pass costs about what the GEMM saves.
 * On the smaller tiles, which small M * N take, ranks up to 64 are formed in
 * the tile as by hydra_lora_linear (rank 64 in several rounds of 128 x 192
 * tiles excepted) and the workspace is checked and not used.  Defined by: the
 * same passages as hydra_lora_linear.
 *
 *   workspace, workspace_bytes   device memory of at least
 *       hydra_lora_linear_workspace_bytes(M, N, r) bytes, 16-byte aligned,
 *       contents ignored and overwritten; NULL allowed when that size is 0 or
 *       when no GEMM update runs (M <= 16, no y_on, or r == 0).
 * Other arguments and rules as in hydra_lora_linear; HYDRA_ERR_WORKSPACE for a
 * workspace that is needed and too small, HYDRA_ERR_ALIGN for a misaligned one.
 * y_off has the bits of hydra_lora_linear's; y_on agrees with it to the
 * rounding of T (different summation order).
 */
hydra_status hydra_lora_linear_ws(const uint16_t* x, const uint16_t* W, const uint16_t* A, const uint16_t* B,
                                  float s, int64_t M, int64_t N, int64_t K, int64_t r, float* y_off, float* y_on,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* Largest number of linears in one hydra_lora_linear_group call. */
#define HYDRA_MAX_GROUP 8

/*
 * hydra_lora_linear_group -- G independent LoRA-switchable linears that share
 * M, N, K and r, in one launch (for instance the q/k/v/o projections of one
 * decode step, App. A Alg. 2, generation step; each with its own adapter).
 * Defined by: the same passages as hydra_lora_linear.
 *
 *   G                     1 <= G <= HYDRA_MAX_GROUP
 *   x, W, A, B, y_off, y_on   HOST arrays of G device pointers with the meaning,
 *                         layout and alignment of hydra_lora_linear's arguments;
 *                         A, B, y_off, y_on may be NULL arrays (all members NULL)
 *                         or hold NULL entries
 *   s                     HOST array of G scales
 * Member i computes exactly what hydra_lora_linear(x[i], W[i], A[i], B[i], s[i],
 * M, N, K, r, y_off[i], y_on[i]) computes (to rounding where M is 9 to 16,
 * r > 64 and only other members have y_on: the member's own call would take
 * the GEMM).  Each member needs at least one output.  M <= 8 runs one launch
 * for the whole group; larger M one launch too where the GEMM takes its smaller
 * tiles, else the GEMM once per member.  Errors as in hydra_lora_linear;
 * HYDRA_ERR_SHAPE for G out of range.
 */
hydra_status hydra_lora_linear_group(int64_t G, const uint16_t* const* x, const uint16_t* const* W,
                                     const uint16_t* const* A, const uint16_t* const* B, const float* s,
                                     int64_t M, int64_t N, int64_t K, int64_t r,
                                     float* const* y_off, float* const* y_on, void* stream);

/*
 * hydra_lora_linear_group_workspace_bytes -- device workspace that
 * hydra_lora_linear_group_ws needs for G linears of M rows, N outputs and
 * rank r (writes *bytes).  HYDRA_ERR_NULL for a NULL `bytes`, HYDRA_ERR_SHAPE
 * for G, M, N or r outside the limits of hydra_lora_linear_group.
 */
hydra_status hydra_lora_linear_group_workspace_bytes(int64_t G, int64_t M, int64_t N, int64_t r, size_t* bytes);

/* Control area at the start of a hydra_lora_linear_group_ws workspace, its caller-owned wait-bound word, the size
 * of the region of published T values that follows it, and the size of the region of published LoRA-off outputs
 * after that. */
#define HYDRA_GROUP_WS_CONTROL_BYTES 4352
#define HYDRA_GROUP_WS_BOUND_WORD 8
#define HYDRA_GROUP_WS_T_BYTES 65536
#define HYDRA_GROUP_WS_Y_BYTES 2097152

/*
 * hydra_lora_linear_group_ws -- hydra_lora_linear_group with a caller
 * workspace, which lets a decode step (M <= 8 rows, App. A Alg. 1 / Alg. 2,
 * generation step) run as a single launch: the first workgroups form
 * T = x A^T of every member once and publish it in the workspace; up to
 * padded rank 64 (when G x N x M, with M rounded up to 1, 2, 4 or 8, is at
 * most HYDRA_GROUP_WS_Y_BYTES / 8) the workgroups that stream the rows of W
 * publish their LoRA-off outputs there too, and workgroups at the end of the
 * launch add s T B^T to them to form y_on; otherwise the workgroups that stream W add
 * s T B^T to their own rows of y_on (no second launch, no T recomputed per
 * column block).  Defined by: the same passages as hydra_lora_linear.
 *
 *   G, x, W, A, B, s, M, N, K, r, y_off, y_on   as in hydra_lora_linear_group
 *   workspace, workspace_bytes   device, 16-byte aligned, at least
 *                         hydra_lora_linear_group_workspace_bytes(G, M, N, r)
 *                         bytes.  Fill the whole buffer with zeros once after
 *                         allocating it; after that the library keeps its
 *                         state there (HYDRA_GROUP_WS_CONTROL_BYTES of control
 *                         words holding a call generation, then
 *                         HYDRA_GROUP_WS_T_BYTES of published T values and
 *                         HYDRA_GROUP_WS_Y_BYTES of published LoRA-off outputs,
 *                         each tagged with it), so the buffer is reused as it
 *                         is and serves calls of any shape.  To reset it, zero all of
 *                         it (the control words alone are not enough), and
 *                         zero it again before its next use here after lending
 *                         it to another entry point.  One workspace serves one
 *                         stream at a time: calls that overlap in time must
 *                         not share it.  The 32-bit word
 *                         HYDRA_GROUP_WS_BOUND_WORD of the control area is the
 *                         caller's: 0 selects the default bounds of the
 *                         launch's waits (for T and for a published LoRA-off
 *                         output, about 10 ms each; for every workgroup to
 *                         have read the generation, about 1 s); another value
 *                         bounds each to that many polls.  A workgroup that
 *                         gives up waiting for T or for an output forms it
 *                         itself, with the same bits; if the last wait runs
 *                         out, every later call forms them where they are used
 *                         (same bits, slower) until the workspace is zeroed.
 * By rows: M <= 8 one launch; 8 < M <= 16 as hydra_lora_linear_group, but at
 * rank above 64 the two row halves each take the single launch; M > 16 as
 * hydra_lora_linear_group, and at rank above 64 each member runs the pre-pass
 * GEMM of hydra_lora_linear_ws over a pre-pass workspace of its own (one per
 * member, after the regions above); when every member's B has rows of exactly
 * the padded rank and is 16-byte aligned, the members' pre-passes share one
 * pair of launches before the GEMMs (rank 128 is accepted at every M).  Errors as in hydra_lora_linear_group, plus
 * HYDRA_ERR_NULL for a NULL workspace, HYDRA_ERR_WORKSPACE when it is too
 * small, HYDRA_ERR_ALIGN when it is not 16-byte aligned.  Results: the
 * oracle's tolerances; the bits may differ from hydra_lora_linear_group's in
 * y_on (another summation order of the LoRA update); repeated calls give the
 * same bits.
 */
hydra_status hydra_lora_linear_group_ws(int64_t G, const uint16_t* const* x, const uint16_t* const* W,
                                        const uint16_t* const* A, const uint16_t* const* B, const float* s,
                                        int64_t M, int64_t N, int64_t K, int64_t r,
                                        float* const* y_off, float* const* y_on,
                                        void* workspace, size_t workspace_bytes, void* stream);

/* Largest number of LoRA-on inputs in one hydra_lora_linear_multi call. */
#define HYDRA_MAX_ADAPTERS 4

/*
 * hydra_lora_linear_multi -- one frozen W serving a LoRA-off input and up to
 * HYDRA_MAX_ADAPTERS LoRA-on inputs, each with its own adapter.
 * Defined by: App. A, Alg. 2 (in each PPO iteration the same base weights run
 * the actor pass with the actor adapter, the critic pass with the critic
 * adapter, and the reference / reward passes with LoRA turned off, over the
 * same sequences), Sec. 3 "Dynamic LoRA" (LO(.) on the same W).  In a
 * multi-layer model the passes' activations differ after the first layer, so
 * every pass brings its own input.
 *
 *   x_off  [M x K] bf16 or NULL     input of the LoRA-off pass
 *   W      [N x K] bf16             frozen base weight
 *   n_on   0 <= n_on <= HYDRA_MAX_ADAPTERS
 *   x_on, A, B, y_on   HOST arrays of n_on device pointers: x_on[a] [M x K] bf16,
 *                      A[a] [r x K] bf16, B[a] [N x r] bf16, y_on[a] [M x N] fp32
 *                      (A and B may be NULL arrays iff r == 0)
 *   s      HOST array of n_on scales (NULL iff n_on == 0)
 *   y_off  [M x N] fp32  out: x_off W^T (NULL iff x_off is NULL)
 *   y_on[a]              out: x_on[a] W^T + s[a] (x_on[a] A[a]^T) B[a]^T
 * Shape, rank and alignment rules as in hydra_lora_linear; the outputs must be
 * distinct buffers (HYDRA_ERR_SHAPE otherwise) and at least one input given.
 * At M <= 8 the inputs' rows are stacked, at most 8 rows per pass, and each
 * pass reads W from HBM once for all its rows (M = 4 with the off input and
 * one adapter: one read of W instead of two); larger M runs one GEMM per input.
 * Every output has the bits of the corresponding hydra_lora_linear call.
 * Above M = 16 with adapters, a padded rank above 64 (r > 64) returns
 * HYDRA_ERR_WORKSPACE before anything is launched (hydra_lora_linear_multi_ws
 * serves that rank).
 */
hydra_status hydra_lora_linear_multi(const uint16_t* x_off, const uint16_t* W, int64_t n_on,
                                     const uint16_t* const* x_on, const uint16_t* const* A,
                                     const uint16_t* const* B, const float* s, int64_t M, int64_t N, int64_t K,
                                     int64_t r, float* y_off, float* const* y_on, void* stream);

/*
 * hydra_lora_linear_multi_workspace_bytes -- device workspace that
 * hydra_lora_linear_multi_ws needs for M rows, N outputs and rank r (writes
 * *bytes): the workspace of hydra_lora_linear_ws, shared by the adapters in
 * turn.  HYDRA_ERR_NULL / HYDRA_ERR_SHAPE as hydra_lora_linear_workspace_bytes.
 */
hydra_status hydra_lora_linear_multi_workspace_bytes(int64_t M, int64_t N, int64_t r, size_t* bytes);

/*
 * hydra_lora_linear_multi_ws -- hydra_lora_linear_multi with a caller
 * workspace, so that the paper's rank 128 (App. B) runs at every M.  Defined
 * by: the same passages as hydra_lora_linear_multi.
 *
 *   arguments as hydra_lora_linear_multi, plus
 *   workspace, workspace_bytes   device, 16-byte aligned, at least
 *                         hydra_lora_linear_multi_workspace_bytes(M, N, r)
 *                         bytes; its contents need not be anything in
 *                         particular, and the call overwrites them.
 * Above M = 16 with adapters at a padded rank above 64, the LoRA-off input runs
 * as hydra_lora_linear without an adapter and each adapter's input as
 * hydra_lora_linear_ws (the pre-pass GEMM), in turn over the workspace: every
 * output has the bits of that call.  Otherwise the call is
 * hydra_lora_linear_multi (the workspace is not used).  Errors as in
 * hydra_lora_linear_multi, plus HYDRA_ERR_NULL for a NULL workspace,
 * HYDRA_ERR_WORKSPACE when it is too small for the rank-128 case,
 * HYDRA_ERR_ALIGN when it is not 16-byte aligned; all before any launch.
 */
hydra_status hydra_lora_linear_multi_ws(const uint16_t* x_off, const uint16_t* W, int64_t n_on,
                                        const uint16_t* const* x_on, const uint16_t* const* A,
                                        const uint16_t* const* B, const float* s, int64_t M, int64_t N, int64_t K,
                                        int64_t r, float* y_off, float* const* y_on, void* workspace,
                                        size_t workspace_bytes, void* stream);

/*
 * hydra_score_workspace_bytes -- device workspace that hydra_score needs for
 * M = n_seq * seq_len token rows and a vocabulary of V.  Writes *bytes.
 * Returns HYDRA_ERR_NULL for a NULL `bytes`, HYDRA_ERR_SHAPE for M outside
 * [1, 2^20] or V outside [1, 2^21].
 */
hydra_status hydra_score_workspace_bytes(int64_t M, int64_t V, size_t* bytes);

/*
 * hydra_score -- fused two-head PPO scoring pass.
 * Defined by: Sec. 3 (pi^hydra's CLM head and reward head on the same input),
 * App. A Alg. 1 / Alg. 2 (the LoRA-off scoring step that yields the reward
 * and the reference log-probabilities; the actor log-probability is the
 * LoRA-on pass), App. B
 * (the KL penalty weight beta is applied by the caller, not here).
 *
 *   h        [M x K] bf16   final hidden states, M = n_seq * seq_len, sequence-major
 *   W_lm     [V x K] bf16   CLM head weight (output-major)
 *   A, B     [r x K], [V x r] bf16   LoRA of the CLM head (NULL iff r == 0)
 *   s        fp32           LoRA scale
 *   tokens   [M] int32      sampled token scored at each row (the caller applies
 *                           the usual next-token shift)
 *   w_rm     [K] bf16       reward head weight (no bias); NULL: reward not computed
 *   lp_on    [M] fp32       out: log softmax(z_on)[token],  z_on  = h W^T + s (h A^T) B^T
 *   lp_off   [M] fp32       out: log softmax(z_off)[token], z_off = h W^T
 *   kl       [M] fp32       out: lp_on - lp_off (per-token sampled KL estimate)
 *   reward   [n_seq] fp32   out: <h[b*seq_len + seq_len - 1], w_rm> (NULL: skipped)
 *   lse_on, lse_off [M] fp32  out, optional: log-sum-exp of each logit row
 *   workspace, workspace_bytes  device scratch of at least
 *                           hydra_score_workspace_bytes(M, V) bytes, 16-byte aligned
 *   err_flag [1] int32      optional device flag; 1 is OR-ed in for an out-of-range token
 * The [M x V] logits are never written to memory.  Requires K % 8 == 0,
 * K <= 2^21, 0 <= r <= HYDRA_MAX_RANK, 1 <= M <= 2^20, 1 <= V <= 2^21 and
 * ceil(M / 256) * ceil(V / 256) < 2^24 (the GEMM's tile grid fits one dispatch).
 */
hydra_status hydra_score(const uint16_t* h, const uint16_t* W_lm, const uint16_t* A, const uint16_t* B, float s,
                         const int32_t* tokens, const uint16_t* w_rm,
                         int64_t n_seq, int64_t seq_len, int64_t K, int64_t V, int64_t r,
                         float* lp_on, float* lp_off, float* kl, float* reward, float* lse_on, float* lse_off,
                         void* workspace, size_t workspace_bytes, int32_t* err_flag, void* stream);

/*
 * hydra_score_two_input -- the scoring pass when the actor pass and the
 * LoRA-off pass have their own final hidden states, as in a multi-layer model
 * (their activations differ after the first layer).
 * Defined by: App. A Alg. 2 (the actor pass runs with the actor's adapter, the
 * reference / reward pass with LoRA off, over the same sequences), Sec. 3
 * "Dynamic LoRA" (the reward model is the LoRA-off network), Sec. 3 (the two
 * heads of pi^hydra).
 *
 *   h_act    [M x K] bf16   final hidden states of the actor pass
 *   h_off    [M x K] bf16   final hidden states of the LoRA-off pass
 *   lp_on    [M] fp32       out: log softmax(z_on)[token],  z_on  = h_act W^T + s (h_act A^T) B^T
 *   lp_off   [M] fp32       out: log softmax(z_off)[token], z_off = h_off W^T
 *   kl       [M] fp32       out: lp_on - lp_off
 *   reward   [n_seq] fp32   out: <h_off[b*seq_len + seq_len - 1], w_rm> (NULL: skipped)
 *   every other argument    as in hydra_score (the same workspace size:
 *                           hydra_score_workspace_bytes(M, V))
 * One launch covers both inputs: the LoRA-off tile and the actor tile of a row
 * block run next to each other, so each block of W_lm is read from HBM once
 * for both.  The [M x V] logits are never written.  Errors as in hydra_score
 * (h_act is checked like h), plus HYDRA_ERR_SHAPE when
 * 2 * ceil(M / 256) * ceil(V / 256) >= 2^24.  With h_act and h_off equal the
 * results have the bits of hydra_score.
 */
hydra_status hydra_score_two_input(const uint16_t* h_act, const uint16_t* h_off, const uint16_t* W_lm,
                                   const uint16_t* A, const uint16_t* B, float s, const int32_t* tokens,
                                   const uint16_t* w_rm, int64_t n_seq, int64_t seq_len, int64_t K, int64_t V,
                                   int64_t r, float* lp_on, float* lp_off, float* kl, float* reward, float* lse_on,
                                   float* lse_off, void* workspace, size_t workspace_bytes, int32_t* err_flag,
                                   void* stream);

/* Largest workspace that hydra_score_noalloc serves from its own device scratch (48 MiB). */
#define HYDRA_SCORE_NOALLOC_MAX_BYTES (48u << 20)

/*
 * hydra_score_noalloc -- hydra_score without a caller workspace, for callers
 * that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  The call itself allocates
 * nothing (no hipMalloc, hipFree or allocating library routine): the
 * workspace lives in a file-scope device array of the library,
 * HYDRA_SCORE_NOALLOC_MAX_BYTES long, one copy on each GPU the library runs
 * on, held until the process ends.  Its device address is looked up once per
 * device (on the first call there) and kept.
 *
 * Arguments, outputs and errors as in hydra_score, less `workspace` and
 * `workspace_bytes`; the caller still passes every input and output.
 * Returns HYDRA_ERR_WORKSPACE (before any HIP call) when
 * hydra_score_workspace_bytes(n_seq * seq_len, V) exceeds
 * HYDRA_SCORE_NOALLOC_MAX_BYTES (for example M = 2048, V = 32000 needs 21.5 MB
 * and fits; M = 4096, V = 50272 needs 44.6 MB and fits), and HYDRA_ERR_HIP if
 * the scratch's address cannot be found.  Results have the bits of hydra_score.
 * Every call on one GPU shares that GPU's scratch: calls that overlap in time
 * on one GPU (two streams, two host threads) race and give undefined results;
 * serialise them.  The scratch keeps the last call's contents; no call needs
 * it cleared.
 */
hydra_status hydra_score_noalloc(const uint16_t* h, const uint16_t* W_lm, const uint16_t* A, const uint16_t* B,
                                 float s, const int32_t* tokens, const uint16_t* w_rm,
                                 int64_t n_seq, int64_t seq_len, int64_t K, int64_t V, int64_t r,
                                 float* lp_on, float* lp_off, float* kl, float* reward, float* lse_on,
                                 float* lse_off, int32_t* err_flag, void* stream);

/*
 * hydra_score_logits -- the scoring epilogue alone, from materialised logits.
 * Defined by: App. A Alg. 2 (reference log-probabilities), Sec. 2 Stage 3
 * (the PPO policy ratio uses the same sampled-token log-probabilities).
 *
 *   logits_on, logits_off [M x V] fp32   logits of the LoRA-on and LoRA-off passes
 *   tokens   [M] int32                   sampled token per row
 *   lp_on, lp_off, kl [M] fp32           out (as in hydra_score)
 *   lse_on, lse_off [M] fp32             out, optional (NULL: not written)
 *   err_flag [1] int32                   optional, as in hydra_score
 * Requires 1 <= M <= 2^20 and 1 <= V <= 2^21.
 */
hydra_status hydra_score_logits(const float* logits_on, const float* logits_off, const int32_t* tokens,
                                int64_t M, int64_t V, float* lp_on, float* lp_off, float* kl,
                                float* lse_on, float* lse_off, int32_t* err_flag, void* stream);

/*
 * hydra_value_head -- the critic's scalar head on every token row.
 * Defined by: Sec. 2 Stage 3 (V(x, y) of the critic, used by generalized
 * advantage estimation), App. A Alg. 2 (the critic-LoRA pass over the
 * generated sequences that yields the values; h is that pass's final hidden
 * state).  No bias.
 *
 *   h       [M x K] bf16   hidden states, row-major, 16-byte aligned
 *   w_v     [K] bf16       value head weight, 16-byte aligned
 *   values  [M] fp32       out: values[m] = sum_k h[m][k] * w_v[k] (fp32 accumulation)
 * Requires 1 <= M <= 2^20, 1 <= K <= 2^21, K % 8 == 0.  Buffers are the caller's.
 */
hydra_status hydra_value_head(const uint16_t* h, const uint16_t* w_v, int64_t M, int64_t K, float* values,
                              void* stream);

/*
 * hydra_ppo_advantages -- per-token PPO reward and generalized advantage
 * estimates for n_seq sequences of seq_len tokens (M = n_seq * seq_len,
 * sequence-major).
 * Defined by: Sec. 2 Stage 3 (GAE builds the advantage estimates from the
 * reward using V; V is trained on the returns), App. A Alg. 2 (the advantage
 * step that combines the reward and the reference log-probabilities), App. B
 * (KL beta = 0.02,
 * GAE gamma = 1.0, lambda = 0.95).
 *
 *   kl      [M] fp32       per-token KL estimate lp_on - lp_off (hydra_score)
 *   reward  [n_seq] fp32   sequence reward (hydra_score), credited to the last token
 *   values  [M] fp32       critic values (hydra_value_head)
 *   start                  first response position, 0 <= start < seq_len
 *   beta, gamma, lam       KL weight and GAE discount / lambda
 *   rewards [M] fp32       out, optional: r_t = -beta * kl_t (t >= start) + (t == T-1) * reward
 *   advantages [M] fp32    out: A_t = delta_t + gamma * lam * A_{t+1},
 *                          delta_t = r_t + gamma * V_{t+1} - V_t, V_T = A_T = 0
 *   returns [M] fp32       out: A_t + V_t
 * Positions before `start` get advantage and return 0 (and reward 0).  No
 * output may be one of the inputs or another output (HYDRA_ERR_SHAPE);
 * partial overlaps are not detected and are not allowed.  Requires
 * n_seq, seq_len >= 1 and M = n_seq * seq_len <= 2^20 (HYDRA_ERR_SHAPE
 * otherwise, as for the other entry points' rows); buffers 4-byte aligned.
 */
hydra_status hydra_ppo_advantages(const float* kl, const float* reward, const float* values, int64_t n_seq,
                                  int64_t seq_len, int64_t start, float beta, float gamma, float lam, float* rewards,
                                  float* advantages, float* returns, void* stream);

/*
 * hydra_ppo_loss -- the PPO update stage's losses for n_seq sequences of
 * seq_len tokens (M = n_seq * seq_len, sequence-major), with their per-token
 * gradients.
 * Defined by: Sec. 2 Stage 3 (the clipped surrogate objective on the
 * probability ratio of the new and old policy; V trained with squared-error
 * loss on the returns).
 *
 *   lp_new, lp_old [M] fp32   sampled-token log-probabilities under the policy
 *                             being trained and under the one that sampled
 *   advantages, values, returns [M] fp32   A-hat (hydra_ppo_advantages), the
 *                             critic's current values, the returns
 *   start                     first response position, 0 <= start < seq_len
 *   eps                       clip range, 0 <= eps < 1 (the paper leaves it open)
 *   losses [3] fp32           out: policy loss -(1/n) sum min(rho A, clip(rho, 1-eps, 1+eps) A),
 *                             rho = exp(lp_new - lp_old); value loss (1/n) sum (V - R)^2 / 2;
 *                             the fraction of tokens where the clipped term is the smaller;
 *                             n = n_seq * (seq_len - start), the response tokens
 *   d_lp [M] fp32             out, optional: d policy loss / d lp_new (-rho A / n where the
 *                             unclipped term is the minimum, else 0; 0 before start)
 *   d_v [M] fp32              out, optional: d value loss / d V ((V - R) / n; 0 before start)
 * One workgroup per loss sums in a fixed order (deterministic), beside others
 * that write the gradients: no output may be an input or another output
 * (HYDRA_ERR_SHAPE).  Buffers 4-byte aligned; 16-byte aligned ones are faster.
 * Requires n_seq, seq_len >= 1 and M = n_seq * seq_len <= 2^20.
 */
hydra_status hydra_ppo_loss(const float* lp_new, const float* lp_old, const float* advantages, const float* values,
                            const float* returns, int64_t n_seq, int64_t seq_len, int64_t start, float eps,
                            float* losses, float* d_lp, float* d_v, void* stream);

/*
 * hydra_transpose_bf16 -- dst = src^T for a bf16 matrix: src [R x C]
 * row-major, dst [C x R] row-major (dst[c * R + q] = src[q * C + c]).  The
 * update stage's backward reads the frozen base weight as W^T [K x N]; the
 * caller makes that copy once with this call (W does not change during
 * training) and keeps it beside W.
 *   src, dst   device, 2-byte aligned, not overlapping (HYDRA_ERR_SHAPE if equal)
 *   R, C       1 ... 2^21, ceil(R / 64) * ceil(C / 64) < 2^24
 * Bit-exact (a copy).
 */
hydra_status hydra_transpose_bf16(const uint16_t* src, int64_t R, int64_t C, uint16_t* dst, void* stream);

/*
 * hydra_lora_linear_backward_workspace_bytes -- device workspace that
 * hydra_lora_linear_backward needs for M rows, N outputs, K inputs and rank r
 * (0 for r == 0).  HYDRA_ERR_NULL for a NULL `bytes`, HYDRA_ERR_SHAPE for
 * sizes outside the limits of hydra_lora_linear_backward.
 */
hydra_status hydra_lora_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t r, size_t* bytes);

/*
 * hydra_lora_linear_backward -- gradients of the LoRA-on output
 * y = x W^T + s (x A^T) B^T with the base weight W frozen (the update stage
 * trains only the adapter: Sec. 3 and App. A, Alg. 2; LoRA as in Sec. 2):
 *   dx = dy W + s (dy B) A,   dA = s (dy B)^T x,   dB = s dy^T (x A^T).
 *
 *   x [M x K] bf16           the layer's input (device, 16-byte aligned)
 *   Wt [K x N] bf16          W transposed (hydra_transpose_bf16 of W [N x K]);
 *                            16-byte aligned; only read when dx is wanted
 *   A [r x K], B [N x r] bf16   the adapter (A 16-byte aligned, B 2-byte)
 *   s                        LoRA scale
 *   dy [M x N] bf16          gradient of the loss with respect to y (16-byte aligned)
 *   1 <= M <= 2^20; N, K >= 1, multiples of 8, at most 2^21;
 *   ceil(M / 128) * ceil(K / 256) < 2^23; 0 <= r <= HYDRA_MAX_RANK
 *   dx [M x K] fp32          out, optional
 *   dA [r x K] fp32          out, optional (ignored for r == 0)
 *   dB [N x r] fp32          out, optional (ignored for r == 0)
 *   workspace, workspace_bytes   device memory of at least
 *       hydra_lora_linear_backward_workspace_bytes(M, N, K, r) bytes, 16-byte
 *       aligned, contents ignored and overwritten (NULL allowed for r == 0)
 * dx comes from the MFMA GEMM of hydra_lora_linear_ws run on (dy, W^T) with
 * s (dy B) as its pre-pass; dA and dB are fp32 sums of outer products over
 * the M rows.  Every sum has a fixed order: repeated calls give the same bits.
 * At least one output is required (HYDRA_ERR_NULL); outputs 4-byte aligned
 * and distinct (HYDRA_ERR_SHAPE); HYDRA_ERR_WORKSPACE for a workspace that is
 * too small.  Calls that share a workspace on different streams race.
 */
hydra_status hydra_lora_linear_backward(const uint16_t* x, const uint16_t* Wt, const uint16_t* A, const uint16_t* B,
                                        float s, const uint16_t* dy, int64_t M, int64_t N, int64_t K, int64_t r,
                                        float* dx, float* dA, float* dB, void* workspace, size_t workspace_bytes,
                                        void* stream);

/*
 * hydra_layer_norm -- layer normalisation of M rows of K values (OPT's layers
 * put one before the attention projections, one before fc1, one before the
 * heads):
 *   mean = sum x / K,  var = sum (x - mean)^2 / K,  rstd = 1 / sqrt(var + eps),
 *   y = (x - mean) rstd weight + bias.
 *
 *   x       [M x K] bf16 or fp32 (x_type)
 *   weight, bias [K] bf16 or fp32 (w_type, both), optional (NULL: ones / zeros)
 *   eps     > 0, finite
 *   y       [M x K] bf16 or fp32 (y_type): out; may be x where the types are
 *           the same
 *   mean, rstd [M] fp32   out, optional: what the backward takes
 * Statistics and products are fp32 (the variance from the centred values),
 * y is rounded once, to nearest even.  A row that holds NaN or an infinity
 * becomes NaN; the squares of values from about 1e19 on leave the range of fp32.
 * Requires 1 <= M <= 2^20, 1 <= K <= 2^21; K need be no multiple of anything,
 * and buffers need their element's alignment only (16-byte aligned ones with
 * K % 8 == 0 are faster).  Outputs distinct (HYDRA_ERR_SHAPE); partial overlaps
 * are not detected and are not allowed.
 */
hydra_status hydra_layer_norm(const void* x, hydra_dtype x_type, const void* weight, const void* bias,
                              hydra_dtype w_type, float eps, int64_t M, int64_t K, void* y, hydra_dtype y_type,
                              float* mean, float* rstd, void* stream);

/*
 * hydra_layer_norm_backward_workspace_bytes -- device workspace that
 * hydra_layer_norm_backward needs for M rows of K values (writes *bytes).
 * HYDRA_ERR_NULL for a NULL `bytes`, HYDRA_ERR_SHAPE for M outside [1, 2^20]
 * or K outside [1, 2^21].
 */
hydra_status hydra_layer_norm_backward_workspace_bytes(int64_t M, int64_t K, size_t* bytes);

/*
 * hydra_layer_norm_backward -- gradients of hydra_layer_norm for an upstream
 * gradient dy.  With g = dy weight and xh = (x - mean) rstd:
 *   dx = rstd (g - sum g / K - xh sum (g xh) / K),
 *   dweight = sum over the rows of dy xh,  dbias = sum over the rows of dy.
 *
 *   dy      [M x K] bf16 or fp32 (dy_type; hydra_lora_linear_backward's dx is fp32)
 *   x       [M x K] bf16 or fp32 (x_type): the forward's input
 *   weight  [K] bf16 or fp32 (w_type), optional (NULL: ones)
 *   mean, rstd [M] fp32   the forward's
 *   dx      [M x K] bf16 or fp32 (dx_type; bf16 is the dy of the linear
 *           before), optional; may be dy or x where the types are the same
 *   dweight, dbias [K] fp32   out, optional; overwritten, not added to
 *   workspace, workspace_bytes  device, 16-byte aligned, at least
 *           hydra_layer_norm_backward_workspace_bytes(M, K) bytes, contents
 *           ignored and overwritten
 * At least one output (HYDRA_ERR_NULL).  Products and sums are fp32, every sum
 * in a fixed order: repeated calls give the same bits.  Sizes, alignment and
 * overlaps as in hydra_layer_norm.  Calls that share a workspace on different
 * streams race.
 */
hydra_status hydra_layer_norm_backward(const void* dy, hydra_dtype dy_type, const void* x, hydra_dtype x_type,
                                       const void* weight, hydra_dtype w_type, const float* mean, const float* rstd,
                                       int64_t M, int64_t K, void* dx, hydra_dtype dx_type, float* dweight,
                                       float* dbias, void* workspace, size_t workspace_bytes, void* stream);

/* Most alternatives per token of hydra_token_logprobs. */
#define HYDRA_MAX_TOP 32

/*
 * hydra_token_logprobs_workspace_bytes -- device workspace that
 * hydra_token_logprobs needs for M rows, a vocabulary of V and `top`
 * alternatives (writes *bytes; 0 when none is needed).  HYDRA_ERR_NULL for a NULL `bytes`,
 * HYDRA_ERR_SHAPE for M outside [1, 2^20], V outside [1, 2^21], M V above 2^38
 * or top outside [0, min(V, HYDRA_MAX_TOP)].
 */
hydra_status hydra_token_logprobs_workspace_bytes(int64_t M, int64_t V, int64_t top, size_t* bytes);

/*
 * hydra_token_logprobs -- log-probabilities of given tokens under one set of
 * logits, with the distribution's entropy and the most likely alternatives
 * (the update stage's new log-probabilities of Sec. 2 Stage 3, over logits
 * that the program keeps for the backward; and what a generation step reports).
 *
 *   logits  [M x V] bf16 or fp32 (logits_type), row m at logits + m * ld
 *           elements, ld >= V; -inf marks a masked-out entry
 *   tokens  [M] int32, optional (NULL iff lp is)
 *   lp      [M] fp32   out: z[token] - lse
 *   lse     [M] fp32   out, optional: ln sum_j e^z_j
 *   entropy [M] fp32   out, optional: -sum_j p_j ln p_j, p_j = e^(z_j - lse)
 *   top     alternatives per row, 0 <= top <= min(V, HYDRA_MAX_TOP)
 *   top_ids [M x top] int32   out: indices of the row's `top` largest logits,
 *           the largest first, the lowest index first among equals (+0 and -0
 *           are equal); NULL iff top == 0
 *   top_lp  [M x top] fp32    out, optional: their log-probabilities
 *   workspace, workspace_bytes  device, 16-byte aligned, at least
 *           hydra_token_logprobs_workspace_bytes(M, V, top) bytes (NULL
 *           allowed when that is 0), contents ignored and overwritten
 *   err_flag [1] int32  optional: 1 is OR-ed in for a token outside [0, V),
 *           whose lp is NaN
 * At least one output (HYDRA_ERR_NULL).  Masked-out entries have probability 0
 * and log-probability -inf; a row of nothing else has lse -inf and NaN lp,
 * entropy and top_lp (top_ids 0, 1, ...).  In a row that holds NaN or +inf lp,
 * lse, entropy and top_lp are NaN (top_ids then take NaN first, then +inf).
 * Sums and maxima are fp32, in an order that depends on M, V, the type and how
 * the rows lie to 16-byte boundaries alone.
 * Requires 1 <= M <= 2^20, 1 <= V <= 2^21, M V <= 2^38, ld <= 2^31 - 1; logits
 * need their element's alignment only.  Outputs distinct (HYDRA_ERR_SHAPE).
 * Calls that share a workspace on different streams race.
 */
hydra_status hydra_token_logprobs(const void* logits, hydra_dtype logits_type, int64_t ld, const int32_t* tokens,
                                  int64_t M, int64_t V, int64_t top, float* lp, float* lse, float* entropy,
                                  int32_t* top_ids, float* top_lp, void* workspace, size_t workspace_bytes,
                                  int32_t* err_flag, void* stream);

/*
 * hydra_token_logprobs_backward -- gradient of hydra_token_logprobs' lp and
 * entropy H with respect to the logits, for upstream gradients d_lp (that of
 * hydra_ppo_loss) and d_entropy:
 *   dz_j = d_lp ([j == token] - p_j) - d_entropy p_j (ln p_j + H),  p_j = e^(z_j - lse).
 *
 *   logits, logits_type, ld, tokens, M, V   as in hydra_token_logprobs
 *   lse     [M] fp32   the forward's
 *   entropy [M] fp32   the forward's (needed and read with d_entropy alone)
 *   d_lp    [M] fp32   optional (NULL: zeros; tokens may then be NULL too)
 *   d_entropy [M] fp32 optional (NULL: zeros)
 *   d_logits [M x V] bf16 or fp32 (d_type), row m at d_logits + m * ld_d
 *           elements, ld_d >= V: out (bf16 and ld_d == V is the dy of
 *           hydra_lora_linear_backward for the head); may be logits where types
 *           and strides are the same.  Elements between V and ld_d are left as they are.
 *   err_flag [1] int32  optional: 1 is OR-ed in for a token outside [0, V) of
 *           a row whose d_lp is not 0; that row's gradient is NaN
 * At least one of d_lp and d_entropy (HYDRA_ERR_NULL).  A row whose upstream
 * gradients are both 0 (a prompt token, padding) gets zeros, whatever its
 * logits, token and statistics hold; another row of -inf alone gets NaN.  p_j
 * goes by the lse given, one fp32: half a step of it, up to 2^-24 |lse|, makes
 * every p_j of the row larger or smaller by the factor e^(2^-24 |lse|) at most
 * (2.4e-4 at 4096, 6% at 2^20) and shifts ln p_j by as much; where it has lost
 * ln V (a row of logits near the type's lowest value alone) the p_j are not
 * probabilities any more.  Logits with such an offset in common are to be shifted
 * before both calls.  Products are fp32, each gradient rounded once, to
 * nearest even.  Sizes, alignment and overlaps as in hydra_token_logprobs.
 */
hydra_status hydra_token_logprobs_backward(const void* logits, hydra_dtype logits_type, int64_t ld,
                                           const int32_t* tokens, const float* lse, const float* entropy,
                                           const float* d_lp, const float* d_entropy, int64_t M, int64_t V,
                                           void* d_logits, hydra_dtype d_type, int64_t ld_d, int32_t* err_flag,
                                           void* stream);

/* Most tensors of one hydra_grad_norm or hydra_grad_clip call. */
#define HYDRA_MAX_GRADS 4096

/* hydra_grad_norm_workspace_bytes -- device workspace that hydra_grad_norm and
 * hydra_grad_clip need, whatever the tensors (writes *bytes; HYDRA_ERR_NULL for NULL). */
hydra_status hydra_grad_norm_workspace_bytes(size_t* bytes);

/*
 * hydra_grad_norm -- the norm over all gradients of an update (the dA and dB
 * of every linear's hydra_lora_linear_backward):
 *   norm = sqrt(sum over the tensors of sum g^2).
 *
 *   n       1 <= n <= HYDRA_MAX_GRADS
 *   grads   HOST array of n device pointers (an entry may be NULL where its numel is 0)
 *   types   HOST array of n hydra_dtype values
 *   numels  HOST array of n element counts, 0 <= numel <= 2^40
 *   norm    [1] fp32   out
 *   workspace, workspace_bytes  device, 16-byte aligned, at least
 *           hydra_grad_norm_workspace_bytes() bytes, contents ignored and overwritten
 * Squares and sums are 64-bit floats, in a fixed order: gradients whose
 * squares leave the range of fp32 count, and repeated calls give the same bits.
 * Tensors need their element's alignment only.  NaN and infinities propagate.
 * Calls that share a workspace on different streams race.
 */
hydra_status hydra_grad_norm(int64_t n, const void* const* grads, const int32_t* types, const int64_t* numels,
                             float* norm, void* workspace, size_t workspace_bytes, void* stream);

/*
 * hydra_grad_clip -- hydra_grad_norm, and the gradients scaled to a norm of
 * at most max_norm:
 *   out = g c,  c = max_norm / norm where norm > max_norm, else 1.
 *
 *   n, grads, types, numels, norm, workspace   as in hydra_grad_norm
 *   max_norm  >= 0 (infinity: never scaled)
 *   outs      HOST array of n device pointers, outs[i] of grads[i]'s size (it
 *             may be grads[i] itself where the types are the same); NULL: the
 *             gradients are scaled in place
 *   out_types HOST array of n hydra_dtype values (NULL iff outs is)
 *   err_flag  [1] int32, optional: 1 is OR-ed in when the norm is not finite;
 *             c is 1 then, so that a program can leave the step out
 * c is formed in 64 bits and rounded to fp32; each product is rounded once.
 * Where c is 1, gradients in place are not written.  A tensor that is
 * written may not overlap another tensor that is written or read
 * (HYDRA_ERR_SHAPE): neither may a gradient that is scaled in place stand in the
 * list twice.  `norm` and `err_flag` may not lie in a tensor that is written or
 * read (HYDRA_ERR_SHAPE).
 */
hydra_status hydra_grad_clip(int64_t n, const void* const* grads, const int32_t* types, const int64_t* numels,
                             float max_norm, float* norm, void* const* outs, const int32_t* out_types,
                             void* workspace, size_t workspace_bytes, int32_t* err_flag, void* stream);

/*
 * hydra_fp8_quantize -- a matrix in 8 bits: e4m3 values (OCP: 1 sign, 4 exponent
 * and 3 fraction bits, largest 448, no infinities) with a power-of-two scale for
 * each block of 128 consecutive values of a row (block_rows 1: activations), or of
 * 128 x 128 values (block_rows 128: a frozen weight).  In 8 bits the base takes
 * half the memory of bf16, which is what Hydra-PPO keeps once for all its roles
 * (Sec. 3).  Per block, a its largest finite magnitude:
 *   e = the least integer >= -127 with a <= 448 2^e,  q = the e4m3 value nearest
 *   to x 2^-e (ties to even),  scale = e + 127, one byte (E8M0).
 *
 *   x        [M x K] bf16 or fp32 (x_type)
 *   q        [M x K] e4m3    out
 *   scale    [M or ceil(M / 128) x ceil(K / 128)] bytes   out
 *   qt       [K x M] e4m3    out, optional, block_rows 128 only: q transposed, which
 *            hydra_fp8_lora_linear_backward reads
 *   scale_t  [ceil(K / 128) x ceil(M / 128)] bytes   out, NULL iff qt is: scale transposed
 * Values below 2^-10 of the scale become 0; NaN and infinities become NaN and
 * do not count for the scale.  Requires 1 <= M, K <= 2^21 (no multiple of
 * anything) and M ceil(K / 128) <= 2^28 - 16, or ceil(M / 128) ceil(K / 128) < 2^24;
 * x at its element's alignment (K % 8 == 0 and 16-byte aligned: faster).
 * HYDRA_ERR_UNSUPPORTED for another block_rows, or qt with block_rows 1.
 */
hydra_status hydra_fp8_quantize(const void* x, hydra_dtype x_type, int64_t M, int64_t K, int64_t block_rows, uint8_t* q,
                                uint8_t* scale, uint8_t* qt, uint8_t* scale_t, void* stream);

/* hydra_fp8_lora_linear_workspace_bytes -- device workspace that hydra_fp8_lora_linear
 * needs at most for up to M rows, N outputs, K inputs and rank r (writes *bytes; less is
 * never asked for more rows, so the largest call's workspace serves all).  HYDRA_ERR_NULL
 * for a NULL `bytes`, HYDRA_ERR_SHAPE for sizes outside that call's limits. */
hydra_status hydra_fp8_lora_linear_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t r, size_t* bytes);

/*
 * hydra_fp8_lora_linear -- hydra_lora_linear over a frozen weight in 8 bits:
 *   y_off = xh Wh^T,  y_on = xh Wh^T + s (xa A^T) B^T,
 * xh and Wh what the bytes of the quantized x and W stand for, xa the adapter's
 * input in bf16 (x, or x after dropout).
 *
 *   x         [M x K] bf16   input rows; quantized by the call as hydra_fp8_quantize
 *             with block_rows 1 does (NULL allowed where xq is given)
 *   x_adapter [M x K] bf16   the adapter's own input, optional (NULL: x)
 *   xq, x_scale   x already quantized (several linears may share an input), optional
 *   Wq, w_scale   [N x K] and [ceil(N / 128) x ceil(K / 128)]: W quantized with block_rows 128
 *   A, B, s   as in hydra_lora_linear
 *   y_off, y_on  [M x N] bf16 or fp32 (y_type, both)   out, each optional, at least one
 *   workspace, workspace_bytes  device, 16-byte aligned, contents ignored and
 *             overwritten; hydra_fp8_lora_linear_workspace_bytes(M, N, K, r) bytes are
 *             always enough
 * x, x_adapter, xq, Wq and A 16-byte aligned, B 2-byte, outputs at their element's
 * alignment.  Into fp32 outputs, and up to 16 rows, every product is exact and
 * added in fp32; into bf16 outputs of more rows the 8-bit matrix instructions run,
 * which keep of every eight products with consecutive k what lies above 2^-12 of the
 * largest: typical sums are 2e-5 off (a step of bf16 is 8e-3), a sum whose products
 * cancel keeps more of its digits in fp32 outputs.  The update takes all that fp32
 * holds of s x A^T, but into bf16 outputs of more than 16 rows, where it takes two
 * bf16 parts (2^-17 of it).  Outputs are rounded once, to nearest even.  A scale byte
 * 255 stands for NaN; a value whose bytes stand for 2^128 (above 1.94 2^127 in x)
 * counts as infinite where products are exact.  NaN and infinities in x make their
 * row's outputs NaN; in x_adapter alone they go through the update as fp32 takes them.
 * With r == 0 y_on equals y_off.  Requires 1 <= M <= 2^20, 1 <= N <= 2^21, 16 <= K <= 2^21,
 * K % 16 == 0, 0 <= r <= HYDRA_MAX_RANK, ceil(M / 128) ceil(N / 256) < 2^23; outputs distinct
 * (HYDRA_ERR_SHAPE).  Repeated calls give the same bits.  Calls that share a
 * workspace on different streams race.
 */
hydra_status hydra_fp8_lora_linear(const uint16_t* x, const uint16_t* x_adapter, const uint8_t* xq,
                                   const uint8_t* x_scale, const uint8_t* Wq, const uint8_t* w_scale,
                                   const uint16_t* A, const uint16_t* B, float s, int64_t M, int64_t N, int64_t K,
                                   int64_t r, void* y_off, void* y_on, hydra_dtype y_type, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* hydra_fp8_lora_linear_backward_workspace_bytes -- device workspace that
 * hydra_fp8_lora_linear_backward needs (writes *bytes); errors as above. */
hydra_status hydra_fp8_lora_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t r, size_t* bytes);

/*
 * hydra_fp8_lora_linear_backward -- gradients of hydra_fp8_lora_linear's y_on, with
 * W frozen in 8 bits and dropout of probability p on the adapter's input
 * (xa = m x, m the mask of hydra_dropout over [M x K] with the same p and rng):
 *   dx = q(dy) Wh + m (s (dy B) A),  dA = s (dy B)^T xa,  dB = s dy^T (xa A^T),
 * q(dy) what dy stands for after quantizing (block_rows 1).
 *
 *   x        [M x K] bf16   the adapter's input xa of the forward
 *   Wqt, wt_scale   [K x N] and [ceil(K / 128) x ceil(N / 128)]: W's transpose in 8 bits
 *            (qt and scale_t of hydra_fp8_quantize); only read when dx is wanted
 *   A, B, s, dy   as in hydra_lora_linear_backward
 *   p, rng   as in hydra_dropout (p == 0: no dropout, rng may be NULL)
 *   dx       [M x K] bf16 or fp32 (dx_type)   out, optional
 *   dA, dB   [r x K], [N x r] fp32            out, optional (ignored for r == 0)
 *   workspace, workspace_bytes  device, 16-byte aligned, at least
 *            hydra_fp8_lora_linear_backward_workspace_bytes(M, N, K, r) bytes,
 *            contents ignored and overwritten
 * dx: into fp32 every product of the base is exact and added in fp32, into bf16 the
 * 8-bit matrix instructions run (but with r == 0 up to 16 rows, where products are exact
 * too); its update takes all that fp32 holds of s (dy B), into bf16 two bf16 parts (2^-17
 * of it).  dA and dB take 24 bits of s (dy B) and s (xa A^T).  What a NaN or an infinity
 * reaches is NaN or infinite.
 * The quantized x of the forward's base product counts as x itself (its
 * rounding has no gradient).  Requires N and K multiples of 16, other limits as in
 * hydra_fp8_lora_linear with N and K exchanged.  At least one output
 * (HYDRA_ERR_NULL).  Every sum has a fixed order.
 */
hydra_status hydra_fp8_lora_linear_backward(const uint16_t* x, const uint8_t* Wqt, const uint8_t* wt_scale,
                                            const uint16_t* A, const uint16_t* B, float s, const uint16_t* dy, int64_t M,
                                            int64_t N, int64_t K, int64_t r, double p, const uint64_t* rng, void* dx,
                                            hydra_dtype dx_type, float* dA, float* dB, void* workspace,
                                            size_t workspace_bytes, void* stream);

/*
 * hydra_dropout -- dropout whose mask is never stored (on the input of an
 * adapter; on a layer's output before it joins the residual stream):
 *   y = residual + m x,  m = 65536 / (65536 - d) where the element is kept, else 0,
 * d = p 65536 rounded to the nearest whole number: what is kept is scaled for the
 * probability d / 65536 that is in force, so y's mean is x.
 *
 *   x        [n] bf16 or fp32 (x_type)
 *   residual [n] bf16 or fp32 (residual_type), optional
 *   p        0 <= p <= 1 (1: everything dropped)
 *   rng      [2] 64-bit numbers in DEVICE memory, 8-byte aligned: seed and offset.  A
 *            program (or a captured graph) changes the offset from call to call; the
 *            same two numbers give the same mask.
 *   y        [n] bf16 or fp32 (y_type): out; may be x or residual where the types are the same
 * Element i is dropped iff its sixteen bits of Philox4x32-10 are below d: key =
 * seed, counter = (i / 8, offset), low 64 bits first; of the block's four words element
 * i takes word (i % 8) / 2, its lower half where i is even.  The gradient with
 * respect to x is this call on the upstream gradient, without (or with another) residual.
 * A dropped element does not count, be it NaN or infinite.  fp32 inside, rounded
 * once.  Requires 1 <= n <= 2^34; element's alignment (16-byte aligned: faster).
 */
hydra_status hydra_dropout(const void* x, hydra_dtype x_type, const void* residual, hydra_dtype residual_type, double p,
                           const uint64_t* rng, int64_t n, void* y, hydra_dtype y_type, void* stream);

/* Most drafted tokens per sequence of hydra_verify_drafts. */
#define HYDRA_MAX_DRAFTS 128

/* hydra_verify_drafts_workspace_bytes -- device workspace that hydra_verify_drafts needs
 * for n sequences, up to k drafts and a vocabulary of V (writes *bytes).  HYDRA_ERR_NULL
 * for a NULL `bytes`, HYDRA_ERR_SHAPE for sizes outside that call's limits. */
hydra_status hydra_verify_drafts_workspace_bytes(int64_t n, int64_t k, int64_t V, size_t* bytes);

/*
 * hydra_verify_drafts -- drafted tokens of a rollout against the target's
 * probabilities, and the next token (App. A, Alg. 1 and 2, the generation step; a
 * decode step of up to 8 rows costs one read of the weights, so the k drafts of a
 * sequence are scored in the step that its next token needs anyway).
 * With p_j = softmax(target row j / temperature), q_j = softmax(draft row j / temperature):
 *   draft t_j is accepted iff u_j q_j(t_j) < p_j(t_j) and all before it are;
 *   at the first position a that is not accepted the next token is drawn from
 *   max(p_a - q_a, 0), after the last draft from p_a; with draft == NULL (tokens
 *   looked up, no distribution) q_j is 1 at t_j.
 * Drawn means: the lowest v where the running sum over 0 ... v exceeds u_k times the
 * total.  For uniform u the tokens are distributed as the target's own samples.
 *
 *   target  n (k + 1) rows of V, bf16 or fp32 (target_type), row i at target + i * ld elements,
 *           ld >= V: for sequence b rows b (k + 1) ... b (k + 1) + k, the logits of the positions
 *           of its drafts and of the one after; -inf marks a masked-out entry
 *   draft   n k rows of V (draft_type, ld_draft): the logits that the drafts were drawn from; optional
 *   drafts  [n x k] int32    (NULL allowed for k == 0: one sample of each sequence's row)
 *   lens    [n] int32, optional: how many of the k drafts a sequence has (NULL: all); rows past them are not read
 *   u       [n x (k + 1)] fp32   random numbers in [0, 1): one for each draft, the last for the next token
 *   temperature   > 0
 *   accepted [n] int32           out: how many drafts are accepted
 *   tokens  [n x (k + 1)] int32  out: the accepted drafts, the next token, then -1
 *   lp      [n x (k + 1)] fp32   out, optional: ln p_j of those tokens (lp_old of hydra_ppo_loss at
 *           temperature 1), 0 past the next token
 *   workspace, workspace_bytes   device, 16-byte aligned, at least
 *           hydra_verify_drafts_workspace_bytes(n, k, V) bytes, contents ignored and overwritten
 *   err_flag [1] int32   optional: 1 is OR-ed in for a target row (of an accepted draft or the next token)
 *           without a distribution (NaN, +inf, or -inf alone: the next token there is -1, its lp
 *           NaN); for a draft outside [0, V) or with such a draft row, if the drafts before it are accepted
 *           (it counts as no draft: the next token is drawn from p_j); for a length outside [0, k] (the nearest is taken)
 * Exponentials and sums are 64-bit, in a fixed order (e^-700 of the largest of a row and
 * less count as 0); where rounding leaves nothing of p_a - q_a, the next token is drawn
 * from p_a.  Requires n >= 1, 0 <= k <= HYDRA_MAX_DRAFTS,
 * n (k + 1) <= 2^20, 1 <= V <= 2^21, n (2 k + 1) ceil(V / 2048) < 2^24, ld <= 2^31 - 1; logits at their
 * element's alignment; outputs distinct (HYDRA_ERR_SHAPE).  Calls that share a workspace on
 * different streams race.
 */
hydra_status hydra_verify_drafts(const void* target, hydra_dtype target_type, int64_t ld, const void* draft,
                                 hydra_dtype draft_type, int64_t ld_draft, const int32_t* drafts, const int32_t* lens,
                                 const float* u, int64_t n, int64_t k, int64_t V, double temperature, int32_t* accepted,
                                 int32_t* tokens, float* lp, void* workspace, size_t workspace_bytes, int32_t* err_flag,
                                 void* stream);

/* A static, human-readable name for a status code. */
const char* hydra_status_string(hydra_status status);

/* ABI version of this header (incremented on any incompatible change). */
int hydra_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* HYDRA_H_ */
