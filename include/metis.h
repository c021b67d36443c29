/*
 * metis.h -- C ABI of the MI355X-native Metis hot path (spectral split + NVFP4
 * quantization + FP4 GEMMs of one linear layer; Metis, arXiv 2509.00404).
 *
 * Conventions that hold for every entry point
 *   - Every matrix pointer is DEVICE memory owned by the caller, row-major.
 *     Scalars and the structs themselves are HOST memory, read before return.
 *   - `stream` is a hipStream_t passed as void*; all work is enqueued on it and
 *     the call returns without synchronising.  Nothing is allocated or freed.
 *   - Return value: METIS_OK (0) or a negative metis_status.  Argument and shape
 *     errors are detected on the host before anything is enqueued.
 *   - Layout of one linear layer (PyTorch convention): X[L,K] activations,
 *     W[N,K] weight, Y = X W^T [L,N], G = dL/dY [L,N].  The paper's W (Sec. 3.2)
 *     is the transpose of this W.
 */
#ifndef METIS_H
#define METIS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    METIS_OK = 0,
    METIS_INVALID_ARG = -1,      /* null pointer, k < 1, rho outside (0,1], unknown dtype */
    METIS_BAD_SHAPE = -2,        /* quantized axis not a multiple of 16, k+p too large, mismatched operands */
    METIS_WORKSPACE_TOO_SMALL = -3,
    METIS_HIP_ERROR = -4,        /* a launch failed; hipGetLastError() has the reason */
    METIS_UNSUPPORTED = -5,      /* size outside what the kernels are built for (e.g. k+p > 96) */
    METIS_SCRATCH_TOO_SMALL = -6 /* the input needs more than the library's built-in scratch array holds */
} metis_status;

enum { METIS_BF16 = 0, METIS_F32 = 1 };

/* Dense device matrix, row-major, leading dimension `ld` in elements. */
typedef struct {
    void*   ptr;
    int64_t rows, cols, ld;
    int     dtype;               /* METIS_BF16 or METIS_F32 */
} metis_mat;

/*
 * NVFP4-quantized device matrix (Sec. 2.3; value set in App. C.1).
 *   codes  [rows, cols/2]  two E2M1 codes per byte, low nibble = even column,
 *                          nibble = sign<<3 | magnitude code (0..7 -> 0,.5,1,1.5,2,3,4,6)
 *   scales [rows, cols/16] one FP8-E4M3 bit pattern (0x00..0x7E) per block of 16
 *                          consecutive columns
 *   tscale                 per-tensor power-of-two scale g; element value =
 *                          grid[code] * e4m3(scale) * g.  g = 1 is the paper's text verbatim.
 * Blocks always run along `cols` (the contiguous axis).  A matrix that must be
 * blocked along its rows is stored transposed.
 */
typedef struct {
    uint8_t* codes;
    uint8_t* scales;
    float    tscale;
    int64_t  rows, cols;
} metis_fp4;

/*
 * Split-quantized operand A[M,N] ~ U diag(S) V^T + R  (Sec. 3.2: Q_b is applied to
 * U, V and R separately, S stays in high precision).
 *   Ut  Q(U^T) [k,M]   each left singular vector contiguous, blocks along M
 *   Vt  Q(V^T) [k,N]
 *   R   Q(R)   [M,N]   blocks along N (for a GEMM contracting over A's columns)
 *   Rt  Q(R^T) [N,M]   blocks along M (for a GEMM contracting over A's rows); may be
 *                      all-null if the caller does not need that orientation
 *   S   fp32 [k]
 * k = 0: not split; R (and Rt) hold Q(A), Ut/Vt/S are ignored.
 */
typedef struct {
    metis_fp4 Ut, Vt, R, Rt;
    float*    S;
    int       k;
} metis_split;

const char* metis_status_string(int status);
int metis_version(void);

/*
 * Per-tensor scale of a metis_fp4 for data whose largest magnitude is `amax` (host-only helper, no
 * GPU work): the smallest power of two g with 6 * 448 * g >= amax, so that the largest block scale
 * still fits FP8-E4M3.  The paper's text has no such scale (g = 1); this build's reading adds it so
 * that small-magnitude tensors (singular vectors, gradients) do not fall into E4M3's subnormals,
 * and keeps it a power of two so that every quantizer comparison stays exact.  amax <= 0 or not
 * finite returns 1.  Callers typically take amax from a previous step (metis_decompose's amax_out).
 */
float metis_tensor_scale(float amax);

/* ---- random draws of the decomposition (Sec. 3.1) ------------------------------------- */

/* Number of sampled rows l_k = min(M, max(k+p, ceil(rho*M))). Host-only helper. */
int64_t metis_sample_count(int64_t M, int k, int p, double rho);

/*
 * Row sample (Sec. 3.1, sparse random sampling): idx[Ms] (device, uint32), ascending,
 * distinct, one row per stratum [floor(j*M/Ms), floor((j+1)*M/Ms)), offset = word j of
 * Philox4x32-10 stream 1 under `seed`, modulo the stratum length.
 */
int metis_sample_rows(void* stream, uint64_t seed, int64_t M, int64_t Ms, uint32_t* idx);

/*
 * Sequence-granular sample (Sec. 3.1 speaks of sampling sequences, i.e. runs of consecutive token rows): the M
 * rows are M / group sequences of `group` consecutive rows (M % group == 0); whole sequences are drawn exactly as
 * metis_sample_rows draws rows -- one sequence per stratum of sequences, offset = word j of Philox stream 1 modulo
 * the stratum length -- and each contributes its rows in order.  metis_sample_count_sequences gives the number of
 * sampled ROWS: ceil(rho * M / group) sequences, at least ceil((k+p) / group), at most M / group, times group
 * (0 on invalid arguments); group = 1 is metis_sample_count / metis_sample_rows.  idx: device uint32 [Ms].
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE (M or Ms not a multiple of group, Ms > M).
 */
int64_t metis_sample_count_sequences(int64_t M, int k, int p, double rho, int64_t group);
int metis_sample_sequences(void* stream, uint64_t seed, int64_t M, int64_t Ms, int64_t group, uint32_t* idx);

/*
 * Gaussian test matrix (Sec. 3.1, random projection): omega[N,r] (device, bf16 bits as
 * uint16, row-major).  Entry e = n*r+c: Box-Muller on words 2e, 2e+1 of Philox stream 2,
 * u1 = ((w0>>9)+0.5)*2^-23, u2 = (w1>>8)*2^-24, z = sqrt(-2 ln u1) cos(2 pi u2), rounded
 * to bf16 (nearest even).
 */
int metis_gaussian_omega(void* stream, uint64_t seed, int64_t N, int r, uint16_t* omega);

/* ---- decomposition (Sec. 3.1 + the split of Sec. 3.2) ---------------------------------- */

/* Bytes of device workspace metis_decompose needs for an M x N input. */
size_t metis_decompose_workspace_bytes(int64_t M, int64_t N, int k, int p, double rho);

/*
 * A[M,N] (bf16) -> U[M,k], S[k], V[N,k] (all fp32, row-major, device) such that
 * U diag(S) V^T = A V V^T, U^T U = V^T V = I, S descending; span(V) is the top-k right
 * singular subspace of the sampled, sketched matrix:
 *   sample l_k rows -> Z = A_s Omega -> thin QR (CholeskyQR2) Z = H R -> B = H^T A_s ->
 *   top-k right singular vectors V0 of B -> broadcast C = A V0 over ALL rows ->
 *   SVD of C = U S W^T, V = V0 W.
 * No power iteration.  `amax_out` (device fp32[1], optional) receives max|A|.
 * `idx` / `omega` (optional, device): explicit draws replacing the seeded ones (n_idx rows;
 * omega is [N, k+p] bf16); pass NULL/0 to draw from `seed`.
 * `info` (device int32[1], optional): set non-zero if a Cholesky pivot was not positive
 * (rank-deficient sketch); the outputs are then unspecified.
 * The result is a function of the arguments alone: split contractions write partial products that are added in a
 * fixed order (no floating-point atomics), so two calls give the same bits.
 * Errors: INVALID_ARG, BAD_SHAPE (k+p > min(l_k, N)), UNSUPPORTED (k+p > 96, dtype not
 * bf16), WORKSPACE_TOO_SMALL.
 */
int metis_decompose(void* stream, const metis_mat* A, int k, int oversample, double sample_rate,
                    uint64_t seed, float* U, float* S, float* V, float* amax_out,
                    void* workspace, size_t workspace_bytes,
                    const uint32_t* idx, int64_t n_idx, const uint16_t* omega, int32_t* info);

/*
 * Decomposition and split in one call, with one pass over A in HBM (Sec. 3.2's residual A - U S V^T equals
 * A - (A V0) V0^T, V0 being the subspace found on the sampled rows, so it does not have to wait for the
 * singular-value form of the factors).  A is processed in bands of rows small enough to stay in the
 * last-level cache (64 MiB of A): a band's C = A V0 is formed, then the band is read again -- from cache -- for
 * the residual and its quantization into out->R (and out->Rt when its codes pointer is non-null).  Afterwards
 * U, S, V are brought to singular-value form as in metis_decompose and Q(U^T), Q(V^T), S go to out.
 * Arguments as for metis_decompose and metis_split_quantize (out->R.tscale etc. are read as the tensor
 * scales); workspace: metis_decompose_split_workspace_bytes.  U, S, V equal those of metis_decompose; the
 * residual differs from the two-call form only by fp32 rounding (both subtract the same product in different
 * factorizations), so quantization codes may differ where a value sits within rounding of a decision threshold.
 * Errors: those of metis_decompose and metis_split_quantize.
 */
size_t metis_decompose_split_workspace_bytes(int64_t M, int64_t N, int k, int p, double rho);
int metis_decompose_split_quantize(void* stream, const metis_mat* A, int k, int oversample, double sample_rate,
                                   uint64_t seed, float* U, float* S, float* V, float* amax_out, metis_split* out,
                                   float* R_debug, void* workspace, size_t workspace_bytes,
                                   const uint32_t* idx, int64_t n_idx, const uint16_t* omega, int32_t* info);

/*
 * Several decompositions in one call (Sec. 3.2: activations and output gradients are re-decomposed at every
 * step, so one training step decomposes many matrices; they are independent of each other).  Each job has
 * the arguments of metis_decompose; results are what n_jobs separate calls would give.  The stages that
 * run on a single workgroup (Cholesky factorizations, the two eigen-decompositions) are launched once for
 * all jobs of the same k + oversample (resp. k), so they cost one problem's latency instead of n_jobs
 * times it; the stages that stream the matrices are enqueued job after job.  Jobs may differ in every
 * argument; their workspaces and outputs must not overlap.  The array is host memory, read before return.
 * Errors: those of metis_decompose, for the first offending job, before anything is enqueued.
 */
typedef struct {
    const metis_mat* A;
    int      k, oversample;
    double   sample_rate;
    uint64_t seed;
    float*   U;
    float*   S;
    float*   V;
    float*   amax_out;          /* optional */
    void*    workspace;
    size_t   workspace_bytes;
    const uint32_t* idx;        /* optional explicit draws, as for metis_decompose */
    int64_t  n_idx;
    const uint16_t* omega;
    int32_t* info;              /* optional */
    metis_split* split;         /* optional: also split-quantize A as metis_decompose_split_quantize does; the
                                   workspace is then metis_decompose_split_workspace_bytes */
    float*   R_debug;           /* optional, with split: fp32 [M,N] dump of the quantizer's input */
    int64_t  sample_group;      /* 0 or 1: rows are sampled; > 1: whole sequences of that many consecutive rows
                                   (metis_sample_sequences; needs M % sample_group == 0) */
} metis_decompose_job;
int metis_decompose_batch(void* stream, int n_jobs, const metis_decompose_job* jobs);

/* ---- quantization (Sec. 2.3) and split (Sec. 3.2) -------------------------------------- */

/*
 * Plain NVFP4 quantization of A[M,N] (bf16 or fp32): per block of 16 along the columns,
 * scale = smallest E4M3 s with 6*s*g >= block amax (saturating at 448), codes = nearest
 * E2M1 value of e/(s*g), ties to the even code.  `out` (blocks along N, may be NULL) and
 * `out_t` (A^T [N,M], blocks along M, may be NULL) are filled from the same input; their
 * tscale members are read as g.
 */
int metis_quantize(void* stream, const metis_mat* A, metis_fp4* out, metis_fp4* out_t);

/*
 * Stochastically rounded variant (Sec. 4, "FP4 Training": stochastic rounding is the default of
 * every FP4 run).  Block scales as above.  With y = e/(s*g) (fp32 quotient, |y| clipped at 6)
 * between the neighbouring E2M1 magnitudes lo <= |y| <= hi, the element goes to hi with
 * probability (|y| - lo)/(hi - lo), else to lo; values on the grid do not move.  The draw of an
 * element is u = (w >> 8) * 2^-24, w = Philox4x32-10 word under `seed` whose index is the
 * element's row-major position in the output it belongs to (stream 3 for `out`, stream 4 for
 * `out_t`; word w = lane w%4 of the block with counter (w/4 low, w/4 high, stream, 0)); it goes
 * up iff u < t.  Same arguments, layouts and errors as metis_quantize; results are
 * reproducible bit for bit from (A, g, seed).
 */
int metis_quantize_sr(void* stream, const metis_mat* A, uint64_t seed, metis_fp4* out, metis_fp4* out_t);

/*
 * The recipe the paper compares with (Sec. 4.3, "Comparison with Nvidia's Recipe"; Sec. 5, "Hadamard
 * transformations"): a random Hadamard rotation in front of the stochastically rounded quantizer.  The paper
 * gives no definition; this build's reading: every block of 16 consecutive columns is rotated,
 * z = (x * d) H_16 / 4 (H_16 the Sylvester Hadamard matrix in natural order, d_i = -1 iff the top bit of word i of
 * Philox stream 5 under `seed` is set, the same 16 signs for every block), evaluated in fp32 by the radix-2
 * butterfly in natural order (h = 1, 2, 4, 8: pairs (i, i + h) -> (a + b, a - b)), then z is quantized as
 * metis_quantize_sr does (draws: `seed`, stream 3).  H_16 / 4 is orthogonal, so two operands rotated along their
 * common contraction axis with the same seed keep their product.  A: device bf16 [M,N], N % 16 == 0, 16-byte
 * aligned rows; out as for metis_quantize (blocks along N).
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_UNSUPPORTED (A not bf16).
 */
int metis_quantize_rht_sr(void* stream, const metis_mat* A, uint64_t seed, metis_fp4* out);

/*
 * Split + quantize: R = A - U diag(S) V^T in fp32 (unquantized factors, Sec. 3.2), then
 * Q(R) into out->R (and Q(R^T) into out->Rt when its codes pointer is non-null), Q(U^T)
 * into out->Ut, Q(V^T) into out->Vt, S copied to out->S.  out->k must equal k.
 * `R_debug` (device fp32 [M,N], optional) receives the exact quantizer input.
 * `workspace`: metis_split_workspace_bytes(M, N, k) bytes of device scratch.
 * Errors: INVALID_ARG, BAD_SHAPE (N % 16, or M % 16 when Rt is requested, mismatched out),
 * UNSUPPORTED (A not bf16, k > 128), WORKSPACE_TOO_SMALL.
 */
size_t metis_split_workspace_bytes(int64_t M, int64_t N, int k);
int metis_split_quantize(void* stream, const metis_mat* A, const float* U, const float* S,
                         const float* V, int k, metis_split* out, float* R_debug,
                         void* workspace, size_t workspace_bytes);

/*
 * metis_split_quantize for callers that cannot allocate device memory or hand over a workspace (code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): same arguments minus
 * the workspace, same kernels, same results bit for bit.  The factor staging (-U S and V as bf16 pairs,
 * metis_split_workspace_bytes(M, N, k) bytes) lives in an array built into the library,
 * METIS_SPLIT_STATIC_SCRATCH_BYTES per GPU, held until the process ends; an input that needs more
 * returns METIS_SCRATCH_TOO_SMALL before anything is enqueued ((M + N) * 4 * k' <= 8 MiB with k' = k
 * rounded up to 16/32/64/128: e.g. 16384 x 14336 at k = 64 fits).  The call itself allocates nothing
 * and never synchronises.  All calls on one GPU share that GPU's array: calls that may overlap on one
 * GPU (different streams, concurrent graph branches) race on it and must be serialised by the caller;
 * calls on one stream are ordered and safe.  Nothing in the array needs clearing between calls (every
 * byte read is rewritten first by the same call).
 */
#define METIS_SPLIT_STATIC_SCRATCH_BYTES (8u << 20)
int metis_split_quantize_static(void* stream, const metis_mat* A, const float* U, const float* S,
                                const float* V, int k, metis_split* out, float* R_debug);

/*
 * Stochastically rounded split (Sec. 4, "FP4 Training"): as metis_split_quantize, with every
 * quantizer replaced by the rule of metis_quantize_sr.  Draws: R from `seed` (stream 3), R^T from
 * `seed` (stream 4), Q(U^T) from `seed + 1` and Q(V^T) from `seed + 2` (stream 4 each), the word
 * index being the element's row-major position in the tensor it is written to.
 */
int metis_split_quantize_sr(void* stream, const metis_mat* A, const float* U, const float* S,
                            const float* V, int k, uint64_t seed, metis_split* out, float* R_debug,
                            void* workspace, size_t workspace_bytes);

/*
 * Split of a weight whose parts are stored, not recomputed (Sec. 3.2: for parameters the low-rank
 * factors and the residual are separate trainable variables, updated independently).  Q_b on
 * U, V and W_R as given; S copied to out->S; no subtraction and no workspace.
 *   W_R  device, bf16 or fp32, [M,N] row stride ld >= N (N % 16 == 0; M % 16 == 0 when out->Rt is wanted)
 *   U [M,k], S [k], V [N,k]  device fp32, contiguous; 1 <= k <= 128, k == out->k
 *   out  as for metis_split_quantize (Rt all-null: that orientation is skipped)
 * The _sr form rounds stochastically with the keys of metis_split_quantize_sr
 * (W_R: seed, U: seed+1, V: seed+2).  Asynchronous on `stream`.
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE (as metis_quantize).
 */
int metis_split_from_parts(void* stream, const metis_mat* W_R, const float* U, const float* S,
                           const float* V, int k, metis_split* out);
int metis_split_from_parts_sr(void* stream, const metis_mat* W_R, const float* U, const float* S,
                              const float* V, int k, uint64_t seed, metis_split* out);

/* ---- FP4 GEMMs on split operands (Eq. 2, Eq. 3, and the W_R gradient after Eq. 3) ------ */

/* Bytes of device workspace the three GEMM calls need (max over them) for operands of ranks up to k, equal or not. */
size_t metis_linear_workspace_bytes(int64_t L, int64_t N, int64_t K, int k);

/* Y[L,N]  = Xbar Wbar^T   uses X.R [L,K], W.R [N,K]                       (Eq. 2) */
int metis_fp4_linear_fwd(void* stream, const metis_split* X, const metis_split* W, metis_mat* Y,
                         void* workspace, size_t workspace_bytes);
/* dX[L,K] = Gbar Wbar     uses G.R [L,N], W.Rt [K,N]                      (Eq. 3) */
int metis_fp4_linear_dgrad(void* stream, const metis_split* G, const metis_split* W, metis_mat* dX,
                           void* workspace, size_t workspace_bytes);
/* dW[N,K] = Gbar^T Xbar   uses G.Rt [N,L], X.Rt [K,L]   (dL/dW_R of Sec. 3.2, transposed) */
int metis_fp4_linear_wgrad(void* stream, const metis_split* G, const metis_split* X, metis_mat* dW,
                           void* workspace, size_t workspace_bytes);

/*
 * The same three products in two phases, for callers that want to run the pre-pass of several products side by
 * side (it is a handful of small kernels: the skinny products with the factors and the assembly of the low-rank
 * columns, Sec. 3.3's extra terms) and their main kernels back to back afterwards:
 *   product  METIS_LINEAR_FWD (a = X, b = W), METIS_LINEAR_DGRAD (a = G, b = W), METIS_LINEAR_WGRAD (a = G, b = X)
 *   phase    METIS_LINEAR_PREPARE writes only the workspace; METIS_LINEAR_APPLY reads what PREPARE of the same
 *            product, operands and workspace left there and writes `out`; METIS_LINEAR_ALL = both, which is what
 *            the three calls above do.  `out` may be null for PREPARE.
 * The factors (Ut, Vt, S) are read by PREPARE alone; APPLY reads the residuals and the workspace, given with the same
 * workspace_bytes.  Between PREPARE and APPLY the workspace must not be used by anything else (one workspace per product in
 * flight).
 * Same argument rules, workspace size and errors as the three calls above; METIS_INVALID_ARG for an unknown
 * product or phase.  Asynchronous on `stream`.
 */
enum { METIS_LINEAR_FWD = 0, METIS_LINEAR_DGRAD = 1, METIS_LINEAR_WGRAD = 2 };
enum { METIS_LINEAR_ALL = 0, METIS_LINEAR_PREPARE = 1, METIS_LINEAR_APPLY = 2 };
int metis_fp4_linear_phase(void* stream, int product, int phase, const metis_split* a, const metis_split* b,
                           metis_mat* out, void* workspace, size_t workspace_bytes);

/* ---- gradients of the weight's low-rank factors (Sec. 3.2, backward formulas after Eq. 3) --- */

/* Bytes of device workspace metis_fp4_factor_grads needs for W[N,K] split at rank k. */
size_t metis_factor_grads_workspace_bytes(int64_t N, int64_t K, int k);

/*
 * Gradients with respect to the factors of W[N,K] = U diag(S) V^T + W_R, given the dense
 * dW[N,K] = Gbar^T Xbar that metis_fp4_linear_wgrad wrote (which is also dL/dW_R).  The
 * paper's sums over the split terms of X and of the output gradient collect into dW:
 *     dU[N,k] = dW Vbar diag(S)      dS[k,k] = Ubar^T dW Vbar      dV[K,k] = dW^T Ubar diag(S)
 * Ubar, Vbar are the dequantized W->Ut [k,N], W->Vt [k,K]; S = W->S stays fp32.  (This
 * build's U [N,k] holds the paper's V_k and its V [K,k] the paper's U_k, because W is stored
 * [out, in].)  dS is the full k x k matrix, row-major; a diagonal S takes its diagonal.
 *   dW   device, fp32 or bf16, [N,K] with row stride ld >= K
 *   W    only Ut, Vt, S and k are read; 1 <= k <= 128; N, K multiples of 16
 *   dU, dS, dV   device fp32, caller-owned, contiguous row-major, overwritten
 *   workspace    device, 16-byte aligned, >= metis_factor_grads_workspace_bytes(N, K, k)
 * Products accumulate in fp64 and round once to fp32.  Asynchronous on `stream`.
 * Errors: METIS_INVALID_ARG (null pointer, dtype, k out of range, misaligned workspace),
 * METIS_BAD_SHAPE (factor shapes do not match dW), METIS_WORKSPACE_TOO_SMALL.
 */
int metis_fp4_factor_grads(void* stream, const metis_mat* dW, const metis_split* W,
                           float* dU, float* dS, float* dV,
                           void* workspace, size_t workspace_bytes);

/* ---- MXFP4 variant (the microscaling block format named in Sec. 2.3 beside NVFP4) ------------ */

/*
 * MXFP4-quantized device matrix (OCP Microscaling Formats v1.0):
 *   codes  [rows, cols/2]   two E2M1 codes per byte, same nibble layout as metis_fp4
 *   scales [rows, cols/32]  one E8M0 byte per block of 32 consecutive columns, value 2^(byte - 127)
 * element value = grid[code] * 2^(scale - 127).  Blocks run along `cols`.
 */
typedef struct {
    uint8_t* codes;
    uint8_t* scales;
    int64_t  rows, cols;
} metis_mxfp4;

/*
 * Quantize A (device, bf16 or fp32, [rows, cols], cols % 32 == 0, rows 16-byte aligned) to MXFP4:
 * per block X = 2^(floor(log2 amax) - 2) (the specification's conversion rule), elements round to the
 * nearest E2M1 value of e / X, ties to the even code, magnitudes above 6 saturate; an all-zero block
 * stores scale byte 0.  out's buffers are caller-owned and overwritten.  Asynchronous on `stream`.
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE (shape mismatch or misaligned rows).
 */
int metis_quantize_mx(void* stream, const metis_mat* A, metis_mxfp4* out);

/*
 * C[M,N] = A[M,K] B[N,K]^T on the block-scaled FP4 matrix instruction (the scales are applied by
 * the hardware, fp32 accumulation).  K % 32 == 0 (whole blocks); C device, bf16 or fp32, row stride ld >= N.
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_UNSUPPORTED (an operand larger than 4 GiB of codes).
 */
int metis_mxfp4_gemm_nt(void* stream, const metis_mxfp4* A, const metis_mxfp4* B, metis_mat* C);

/* ---- mixture of experts: routing --------------------------------------------------------------- */

/*
 * Routing of T tokens to experts.  x = logits [T, experts] (bf16 or fp32), evaluated in fp32:
 *   score    softmax over the row's experts, or sigmoid(x) = 1 / (1 + exp(-x)) of each expert
 *   key      what the selection compares: x + bias (softmax: the order of p * exp(bias), not that of p + bias), score + bias (sigmoid).  bias (device fp32
 *            [experts], optional) balances the load; it enters the selection alone, not the weights.  An expert whose logit is
 *            -inf or NaN, or whose key is -inf, is not available; a token with valid[t] == 0 (device uint8 [T], optional) has no
 *            expert at all.
 *   groups   the experts form `groups` equal runs.  A group's score is its highest key (softmax) or the sum of its two highest
 *            (sigmoid; of its highest alone where only one expert is available).  The top_groups best stay in the selection.
 *   top-k    the k highest keys in descending order -> idx [T, k] (int32).  Ties go to the lowest index, among groups as well.  Where
 *            fewer than k experts are available the rest of the row is idx -1, weight 0.
 *   weights  fp32 [T, k]: scale * score, or with renorm scale * score / (sum of the chosen scores), for softmax evaluated as
 *            a softmax over the chosen logits (0 where that sum is 0).
 * Limits: 1 <= experts <= 512, 1 <= k <= 16, groups divides experts, 1 <= top_groups <= groups, k <= top_groups * experts / groups.
 * Errors: METIS_INVALID_ARG (null pointer, dtype, unknown scores, parameters outside these rules), METIS_BAD_SHAPE (logits->cols !=
 * experts, ld < cols, more than 2^31 - 1 choices), METIS_UNSUPPORTED (experts > 512, k > 16, 2^28 - 15 tokens or more).
 * T = 0 is no work and no error.
 */
enum { METIS_SCORES_SOFTMAX = 0, METIS_SCORES_SIGMOID = 1 };
typedef struct {
    int   experts, k;
    int   scores;               /* METIS_SCORES_SOFTMAX or METIS_SCORES_SIGMOID */
    int   groups, top_groups;   /* 1, 1: no groups */
    int   renorm;
    float scale;
} metis_router;
int metis_route(void* stream, const metis_mat* logits, const metis_router* router, const float* bias, const uint8_t* valid,
                int32_t* idx, float* weights);

/*
 * dlogits [T, experts] (bf16 or fp32) from dweights [T, k] (fp32) for the choices idx [T, k] that metis_route made.  The selection has
 * no gradient.  With p the scores, v_j = scale * dweights_j (0 where idx_j is -1, or outside the experts):
 *   softmax             dx_e = p_e (sum of v_j over idx_j = e  -  sum_j v_j p_j)          dense: every available expert has one
 *   softmax, renorm     dx_j = q_j (v_j - sum_l v_l q_l), q the softmax over the chosen logits, 0 elsewhere
 *   sigmoid             dx_j = v_j p_j (1 - p_j), 0 elsewhere
 *   sigmoid, renorm     dx_j = (v_j - sum_l v_l p_l / Z) / Z * p_j (1 - p_j), Z = sum of the chosen p; 0 where Z is 0, and elsewhere
 * router->groups, top_groups are not looked at.  Errors as for metis_route.
 */
int metis_route_grads(void* stream, const metis_mat* logits, const metis_router* router, const int32_t* idx, const float* dweights,
                      metis_mat* dlogits);

/*
 * The plan of a batch: its S = tokens * k choices sorted into slots, expert by expert and within an expert in the order of the choices
 * (a stable counting sort of whole numbers: the same bits every time).  Expert e has the slots offsets[e] .. offsets[e + 1) - 1.
 *   offsets  device int32 [experts + 1]
 *   token    device int32 [S]: the token that a slot serves; -1 for the slots at and behind offsets[experts], which serve none
 *   slot     device int32 [tokens, k]: the slot of a choice, -1 where idx is -1 (or outside the experts)
 * Everything stays on the device: no call waits to learn how many tokens an expert has.
 * workspace: metis_dispatch_workspace_bytes bytes, 16-byte aligned (may be null where that is 0).
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE (more than 2^31 - 1 choices), METIS_UNSUPPORTED (experts > 512, k > 16),
 * METIS_WORKSPACE_TOO_SMALL.
 */
typedef struct {
    int32_t* offsets;
    int32_t* token;
    int32_t* slot;
    int64_t  tokens;
    int      experts, k;
} metis_expert_plan;
size_t metis_dispatch_workspace_bytes(int64_t tokens, int experts, int k);
int metis_dispatch(void* stream, const int32_t* idx, metis_expert_plan* plan, void* workspace, size_t workspace_bytes);

/* ---- mixture of experts: products in MXFP4 ------------------------------------------------------ */

/*
 * C [S, N] = the slots' rows times their experts' weights: C[s, :] = Q(A[r, :]) W_e^T, S = tokens * k, e the expert of slot s, r = token[s]
 * with gather (A [tokens, K]), r = s without (A [S, K]).  W: the experts' weights [N, K] quantized by metis_quantize_mx, one below the
 * other (rows = experts * N, cols = K).  A (bf16 or fp32) is quantized to MXFP4 on the way, as metis_quantize_mx does; the products are exact
 * and accumulate in fp32.  C: bf16 or fp32; its rows of slots that serve no choice become 0.  With W of metis_quantize_mx_t this is the input gradient.
 * The plan is read on the device: its offsets, and token and slot with gather.
 * Offsets that do not ascend are read as their running maximum, held to 0 .. S, and tokens and slots outside the rows are not followed: no plan,
 * whatever is in it, leads outside the operands.
 *   K % 32 == 0; A's rows 16-byte aligned; W's codes 16-byte, scales 8-byte aligned; workspace 256-byte aligned, metis_experts_workspace_bytes(A->rows, S, ...) bytes.
 * No tokens is no work.  Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_WORKSPACE_TOO_SMALL, METIS_UNSUPPORTED (experts > 512, k > 16,
 * K > 2^28, or a launch of 2^32 threads and more: A->rows * K of 2^35, rows of W of 2^30, and, where few slots an expert go straight from memory,
 * (S / 32 + experts) * N of some 2^31).
 */
size_t metis_experts_workspace_bytes(int64_t rows, int64_t slots, int experts, int64_t N, int64_t K);
int metis_experts_product(void* stream, const metis_mat* A, const metis_mxfp4* W, const metis_expert_plan* plan, int gather, metis_mat* C,
                          void* workspace, size_t workspace_bytes);

/*
 * MXFP4 with blocks along the rows: A [groups * M, cols] (bf16 or fp32) is `groups` matrices [M, cols], each of which is transposed and
 * quantized along its M.  out [groups * cols, M].  For the input gradient the experts' stacked weights [experts * N, K] become [experts * K, N].
 * M % 32 == 0, cols % 8 == 0, A's rows and out's codes 16-byte aligned.  Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_UNSUPPORTED (2^30
 * columns or 2^31 rows and more).
 */
int metis_quantize_mx_t(void* stream, const metis_mat* A, int groups, metis_mxfp4* out);

/*
 * The experts' weight gradients dW [experts * N, K] (bf16 or fp32): dW_e = Q(G_e^T) Q(X_e^T)^T over the slots of expert e, G [S, N] by slot,
 * X by slot ([S, K]) or, with gather, by token ([tokens, K]).  Both (bf16 or fp32) are quantized to MXFP4 in blocks of 32 consecutive
 * slots of one expert, from its first; what its last block lacks is zeros.  An expert without slots gets 0.
 *   N, K multiples of 8; G's and X's rows 16-byte aligned; workspace 256-byte aligned, metis_experts_wgrad_workspace_bytes(S, ...) bytes.
 * Errors: as for metis_experts_product, and METIS_UNSUPPORTED for more than 2^25 slots or 2^28 rows or columns.
 */
size_t metis_experts_wgrad_workspace_bytes(int64_t slots, int experts, int64_t N, int64_t K);
int metis_experts_wgrad(void* stream, const metis_mat* G, const metis_mat* X, const metis_expert_plan* plan, int gather, metis_mat* dW,
                        void* workspace, size_t workspace_bytes);

/* ---- mixture of experts: rows back to tokens ----------------------------------------------------- */

/*
 * y [tokens, D] = sum over j of weights[t, j] * rows[slot[t, j], :], in fp32, the choices in their order, rounded once.  Choices without a
 * slot add nothing.  weights: device fp32 [tokens, k], or null for ones (the input gradient of gathered rows).  rows [tokens * k, D]
 * and y: bf16 or fp32 each; any D and row strides (whole 16-byte units where both allow them).  plan->slot is read alone.
 * No tokens is no work.  Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_UNSUPPORTED (k > 16, more than 2^28 columns,
 * or y of some 2^35 elements and more).
 */
int metis_combine(void* stream, const metis_mat* rows, const metis_expert_plan* plan, const float* weights, metis_mat* y);

/*
 * Gradients of metis_combine from dy [tokens, D]: drows[slot[t, j], :] = weights[t, j] * dy[t, :], zeros in the slots that serve no
 * choice; dweights [tokens, k] (fp32) = <dy[t, :], rows[slot[t, j], :]>, 0 without a slot; the sums in fp32, in an order that depends on D
 * alone.  plan->slot and offsets are read.  rows and drows share a type, dy has its own.  drows must not overlap rows.  Errors as above; METIS_UNSUPPORTED for 2^24 tokens and more (up to
 * 1024 columns 2^25, up to 512 2^26).
 */
int metis_combine_grads(void* stream, const metis_mat* dy, const metis_mat* rows, const metis_expert_plan* plan, const float* weights,
                        metis_mat* drows, float* dweights);

/* ---- 8-bit checkpoints and the gated activation --------------------------------------------------- */

/*
 * A device matrix held in 8 bits for the backward pass (1.03 bytes an element):
 *   codes  [rows, cols]     one FP8-E4M3 bit pattern each
 *   scales [rows, cols/32]  one E8M0 byte per block of 32 consecutive columns, value 2^(byte - 127)
 * A block's scale is the smallest power of two 2^t, t >= -127, that keeps its largest magnitude within 448 * 2^t, so that nothing
 * saturates; elements are the nearest E4M3 value of e / 2^t, ties to the even code (relative error at most 2^-4 down to 2^-6 * 2^t).  A block
 * of zeros has scale byte 0 and keeps its signs; a block with an infinity or a NaN is NaN throughout (byte 255, codes 0x7F).
 */
typedef struct {
    uint8_t* codes;
    uint8_t* scales;
    int64_t  rows, cols;
} metis_mx8;

/*
 * Save A [rows, cols] (bf16 or fp32) into out; restore A into out.  cols % 32 == 0; the dense matrix's rows 16-byte aligned, codes 8-byte
 * aligned.  No rows is no work.  Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_UNSUPPORTED (rows of more than 2^28
 * columns, or some 2^35 elements and more).
 */
int metis_quantize_mx8(void* stream, const metis_mat* A, metis_mx8* out);
int metis_dequantize_mx8(void* stream, const metis_mx8* A, metis_mat* out);

/*
 * Gated activation of a product whose output holds gate and up side by side: gate_up [S, 2 F] = (g | u), act [S, F] = g * sigmoid(g) * u in
 * fp32, rounded once.  saved (optional, [S, 2 F]): the 8-bit checkpoint of gate_up, made on the way; with it the backward pass keeps 2.06
 * bytes per gate-up pair where the bf16 gate, up and activation take 6.
 *
 * metis_swiglu_grads reads that checkpoint alone: with g, u its values and p = sigmoid(g),
 *   dgate_up [S, 2 F] = (dact u p (1 + g (1 - p)) | dact g p),     act (optional, [S, F]) = g p u, recomputed for the gradient of the
 * weight behind it.
 * F % 32 == 0; gate_up, act, dact, dgate_up share a type (bf16 or fp32) and have 16-byte aligned rows; codes 8-byte aligned.
 * No rows is no work.  Errors: as for metis_quantize_mx8.
 */
int metis_swiglu(void* stream, const metis_mat* gate_up, metis_mat* act, metis_mx8* saved);
int metis_swiglu_grads(void* stream, const metis_mx8* saved, const metis_mat* dact, metis_mat* dgate_up, metis_mat* act);

/* ---- around the products of a block: dropout, epilogues, layer norm ------------------------------ */

/*
 * A dropout mask that is computed wherever it is needed and never stored.  Element (i, j) of a matrix has the 16-bit number j % 8 (low halves
 * first) of the Philox4x32-10 block with counter (j / 8, i, 16, step mod 2^32) and key `seed`.  It is dropped where that number is below
 * t = floor(65536 p + 1/2), so with a probability within 2^-17 of p, and multiplied by 65536 / (65536 - t) elsewhere.  A dropped element is 0 whatever
 * it was.  The mask goes by an element's row and column alone: strides, types and the kernel that applies it change nothing, and the backward pass
 * computes it again.
 *   p     0 <= p < 1, and t < 65536; 0 drops nothing
 *   seed  a layer's own; masks share no numbers with the library's other draws under the same seed
 *   step  device memory, 8-byte aligned, or null (0): read when the work runs, so that a captured graph draws another mask on every replay
 *         once the program counts it up in between
 */
typedef struct {
    double         p;
    uint64_t       seed;
    const int64_t* step;
} metis_dropout_mask;

/*
 * y = residual + m x, m the mask's factors (residual optional); dx = m dy is the same call.  x, residual, y: [rows, cols], one type (bf16 or fp32),
 * any row strides and alignments of elements; y may be x or residual itself, and must not overlap them otherwise.  The sum is formed in fp32 and
 * rounded once.  No rows is no work.  Errors: METIS_INVALID_ARG (null pointer, types, a mask outside these rules), METIS_BAD_SHAPE,
 * METIS_UNSUPPORTED (more than 2^28 columns, or some 2^35 elements and more).
 */
int metis_dropout(void* stream, const metis_mat* x, const metis_dropout_mask* mask, const metis_mat* residual, metis_mat* y);

/*
 * Y [rows, N] = residual + m act(Q(X) W^T + bias): metis_mxfp4_gemm_nt with an epilogue.  The products are exact and accumulate in fp32; the
 * epilogue is fp32 too, and its result is rounded once.
 *   X, Xq      exactly one of them: X [rows, K] (bf16 or fp32, rows 16-byte aligned), quantized to MXFP4 on the way as metis_quantize_mx does, or
 *              Xq, quantized already
 *   W          [N, K]; K % 32 == 0
 *   e          null: no epilogue.  bias: device fp32 [N], or null.  act: see below.  pre: null, or an output of Y's shape and type: Q(X) W^T + bias,
 *              rounded (the activation is applied to what is not rounded yet).  mask: null, or a dropout.  residual: null, or a matrix of Y's
 *              shape and type, which may be Y itself; Y, pre and residual must not overlap otherwise.
 *              Neither Y nor pre may overlap W, Xq or the bias.  Either may overlap X where the workspace's size is not 0: X is then quantized before the first
 *              output; where it is 0, such calls are refused (METIS_INVALID_ARG).
 *   workspace  with X: metis_mxfp4_linear_workspace_bytes bytes, 256-byte aligned (may be null where that is 0); with Xq, optional:
 *              metis_mxfp4_linear_quantized_workspace_bytes bytes (0 for most sizes) let a product of more than 64 rows and few outputs run faster, and a call
 *              without is right too.  Calls that may run at the same time have workspaces of their own.
 *   act        relu max(z, 0); gelu z Phi(z), Phi the normal distribution; gelu_tanh z sigmoid(2 sqrt(2 / pi) (z + 0.044715 z^3)); silu
 *              z sigmoid(z).  For bf16 outputs their exponentials are the hardware's: results are within 4e-5, relatively.
 * Any strides of Y, pre, residual, and alignments of their elements.  No rows is no work.
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_WORKSPACE_TOO_SMALL (with X), METIS_UNSUPPORTED (an operand larger than 4 GiB of codes).
 */
enum { METIS_ACT_NONE = 0, METIS_ACT_RELU = 1, METIS_ACT_GELU = 2, METIS_ACT_GELU_TANH = 3, METIS_ACT_SILU = 4 };
typedef struct {
    const float*              bias;
    int                       act;
    const metis_mat*          pre;
    const metis_dropout_mask* mask;
    const metis_mat*          residual;
} metis_epilogue;
size_t metis_mxfp4_linear_workspace_bytes(int64_t rows, int64_t N, int64_t K);
size_t metis_mxfp4_linear_quantized_workspace_bytes(int64_t rows, int64_t N, int64_t K);
int metis_mxfp4_linear(void* stream, const metis_mat* X, const metis_mxfp4* Xq, const metis_mxfp4* W, const metis_epilogue* epilogue, metis_mat* Y,
                       void* workspace, size_t workspace_bytes);

/*
 * Gradient of that epilogue: dZ = act'(pre) m dY, of what the activation is applied to, and dbias (device fp32 [cols]) = the sum of dZ's rows,
 * of its values before they are rounded, in an order that depends on shape and type alone.  (The residual's gradient is dY itself.)  relu' (0) = 0.  A dropped element's is 0 whatever dY and
 * `pre` hold in its place.
 *   pre        as the forward pass left it; not looked at for METIS_ACT_NONE
 *   mask       the forward pass's, or null
 *   dZ, dbias  either may be null; dZ may be dY or pre itself
 *   workspace  metis_linear_grads_workspace_bytes bytes where dbias is wanted, 256-byte aligned (may be null where that is 0)
 * dY, pre, dZ: [rows, cols], one type (bf16 or fp32), any strides and alignments of elements.  Without rows dbias becomes 0.
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_WORKSPACE_TOO_SMALL, METIS_UNSUPPORTED (more than 2^28 columns or 2^32 - 1 rows).
 */
size_t metis_linear_grads_workspace_bytes(int64_t rows, int64_t cols);
int metis_linear_grads(void* stream, const metis_mat* dY, const metis_mat* pre, int act, const metis_dropout_mask* mask, metis_mat* dZ, float* dbias,
                       void* workspace, size_t workspace_bytes);

/*
 * Layer norm of the rows of x [rows, cols]: y = (x - mean) rstd weight + bias, the mean from a sum in 64 bits and to twice fp32's places, the variance from the
 * differences to it, rstd = 1 / sqrt(variance + eps).  weight, bias: device fp32 [cols], each may be null (ones, zeros).  stats: null, or device fp32
 * [rows, 2], 8-byte aligned: mean and rstd, rounded, for the backward pass.  x, y: one type (bf16 or fp32), any strides and alignments of elements; y may be x
 * itself.  eps >= 0: a row of equal elements is its bias, exactly, and NaN with eps = 0.  No rows is no work.
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_UNSUPPORTED (more than 2^28 columns or 2^32 - 1 rows).
 */
int metis_layernorm(void* stream, const metis_mat* x, const float* weight, const float* bias, float eps, metis_mat* y, float* stats);

/*
 * Its gradients, with xh = (x - mean) rstd from `stats` and g = dy weight:
 *   dx = add + rstd (g - mean of g - xh * mean of g xh)    add: null, or the gradient that reaches x past the norm
 *   dweight, dbias (device fp32 [cols], each may be null) = sums over the rows of dy xh and of dy, in an order that depends on shape and type alone
 * dy, x, add, dx: one type (bf16 or fp32), any strides and alignments of elements; dx may be dy, x or add itself.
 * workspace: metis_layernorm_grads_workspace_bytes bytes where dweight or dbias is wanted, 256-byte aligned (may be null where that is 0).  Without rows
 * both become 0.
 * Errors: METIS_INVALID_ARG, METIS_BAD_SHAPE, METIS_WORKSPACE_TOO_SMALL, METIS_UNSUPPORTED (as above).
 */
size_t metis_layernorm_grads_workspace_bytes(int64_t rows, int64_t cols);
int metis_layernorm_grads(void* stream, const metis_mat* dy, const metis_mat* x, const float* stats, const float* weight, const metis_mat* add,
                          metis_mat* dx, float* dweight, float* dbias, void* workspace, size_t workspace_bytes);

/* ---- measurement aid ---------------------------------------------------------------------- */

/*
 * Bracket every launch of one hot kernel with caller-owned HIP events (hipEvent_t passed as
 * void*), recorded on the stream the kernel is launched on: launch i uses start[i % n] and
 * stop[i % n].  kernel_id: 0 main FP4 GEMM kernel of the three linear calls (the kernel that
 * writes Y / dX / dW), 1 broadcast C = A V0 (a launch serves all jobs of a batch whose ranks
 * round up to the same multiple of 32), 2 fused residual + quantize, 3 plain row
 * quantizer.  n = 0 switches it off.  The arrays (host memory) must stay valid while set.
 * Host-side state, not thread-safe; for benchmarks only.
 */
int metis_profile_events(int kernel_id, void** start, void** stop, int n);

/*
 * Measured ceilings of the GPU the library runs on, for quoting roofline fractions against what the chip
 * sustains as well as against its datasheet peaks.  Asynchronous on `stream`; the caller times them.
 *   metis_ceiling_copy   dst[0..bytes) = src[0..bytes) (device, 16-byte aligned, bytes % 16 == 0): a plain
 *                        streaming copy, 2 * bytes of traffic.
 *   metis_ceiling_read   streams src once; sink: device uint32[2048], normally left untouched.
 *   metis_ceiling_mfma   512 workgroups x 4 waves issue iters x 8 independent 32x32x16 fp16 matrix instructions
 *                        from registers; *flops_out (host, optional) = floating-point operations of the launch;
 *                        sink: device float[512 * 256], normally left untouched.
 *   metis_ceiling_mfma_mix  the FP4 GEMM's instruction mix without its memory system: one workgroup of four
 *                        waves per CU and per `waves_per_simd` (1 or 2), every wave issuing iters x 4 matrix
 *                        instructions (accumulators in the accumulation registers), each followed by
 *                        `valu_per_mfma` (0, 2, 4, 5, 6 or 8) independent packed fp16 multiplies on registers; shows
 *                        what the chip sustains when a wave has to issue that much vector work per matrix
 *                        instruction.  With valu_per_mfma = METIS_MIX_GEMM_EXPANSION (waves_per_simd 1) a wave
 *                        runs `iters` (rounded up to even) steps of the GEMM's own stage loop on registers instead:
 *                        eight fragments expanded from raw words (4 FP4 -> fp16 conversions + 4 packed multiplies
 *                        each), then the 16 matrix instructions of a 128 x 128 wave tile, in the compiler's order --
 *                        the GEMM without LDS traffic, global loads, waits and barrier.  METIS_MIX_GEMM_EXPANSION_FP6
 *                        is that loop with the codes in 6-bit containers, expanded by the 32-wide FP6 converter (two
 *                        instructions per step instead of 32): what a wider container format would buy.
 *                        *flops_out as above; sink as above.
 * Errors: METIS_INVALID_ARG.
 */
#define METIS_MIX_GEMM_EXPANSION (-1)
#define METIS_MIX_GEMM_EXPANSION_FP6 (-2)
int metis_ceiling_mfma_mix(void* stream, int iters, int valu_per_mfma, int waves_per_simd, float* sink, double* flops_out);
int metis_ceiling_copy(void* stream, const void* src, void* dst, size_t bytes);
int metis_ceiling_read(void* stream, const void* src, size_t bytes, uint32_t* sink);
int metis_ceiling_mfma(void* stream, int iters, float* sink, double* flops_out);

#ifdef __cplusplus
}
#endif
#endif /* METIS_H */
