/*
 * approxifer.h -- C ABI of the ApproxIFER coding layer for AMD MI355X (gfx950).
 *
 * ApproxIFER (arXiv 2109.09868) serves K queries of a group with N workers that all
 * host the same model f: the K queries are encoded into N coded queries, every worker
 * runs f on one coded query, and the K predictions are rebuilt from whichever workers
 * answer, after workers that answered wrongly have been located and dropped.
 *
 * Naming.  N here is the NUMBER OF WORKERS.  The paper indexes its workers 0..N and so
 * has N+1 of them (Section 2, "System Architecture"); this library's N is the paper's
 * N+1.  S is the number of stragglers, A the number of Byzantine workers (the paper's E).
 * alpha[K] are the query nodes, beta[N] the worker nodes (Section 3, "ApproxIFER
 * Encoding").
 *
 * Conventions common to all entry points
 *   - d_* arguments are DEVICE pointers owned by the caller; h_* arguments are HOST
 *     pointers that are read before the call returns and may be freed afterwards.
 *   - All tensors are dense, row-major, with the last index contiguous.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Work is
 *     enqueued on it and the call returns without synchronising.  The library allocates
 *     no device memory and keeps no state between calls; the one kind of scratch memory
 *     it uses (the Byzantine decoders' workspace) is the caller's.
 *   - Return value: APPROXIFER_OK when the kernels were enqueued; a negative
 *     APPROXIFER_ERR_* code otherwise.  Every code but APPROXIFER_ERR_LAUNCH is decided on
 *     the host before anything is enqueued: no output is touched.  APPROXIFER_ERR_LAUNCH is
 *     the HIP runtime's refusal of a launch; a call that consists of two launches (see the
 *     individual entry points) may then have enqueued the first.  approxifer_strerror()
 *     turns a code into text.
 *   - G = 0, D = 0 or C = 0 is a valid empty call: nothing is enqueued, OK is returned.
 *   - Limits: 1 <= K <= APPROXIFER_MAX_K, 2 <= N <= APPROXIFER_MAX_N; the Byzantine
 *     decoder additionally needs N - S <= APPROXIFER_MAX_AVAIL_BYZ.
 *   - Nodes must be finite and pairwise distinct within each set.  A query node may
 *     coincide with a worker node; the interpolant then passes through the data there.
 */
#ifndef APPROXIFER_H
#define APPROXIFER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define APPROXIFER_MAX_K 64
#define APPROXIFER_MAX_N 128
#define APPROXIFER_MAX_AVAIL_BYZ 64

#define APPROXIFER_OK 0
#define APPROXIFER_ERR_NULL_POINTER (-1)   /* a required pointer is NULL */
#define APPROXIFER_ERR_BAD_SHAPE (-2)      /* negative size, K < 1, N < 2, S < -1, S >= N, A < 1 ... */
#define APPROXIFER_ERR_LIMIT (-3)          /* K, N or N-S above the compiled limits */
#define APPROXIFER_ERR_BAD_NODES (-4)      /* a node is not finite, or two nodes of one set are equal */
#define APPROXIFER_ERR_TOO_FEW_WORKERS (-5)/* N - S < 2 (K + A): Algorithm 2's system would be under-determined */
#define APPROXIFER_ERR_BAD_SIGN_MODE (-6)  /* sign_mode is neither 0 nor 1 */
#define APPROXIFER_ERR_LAUNCH (-7)         /* the HIP runtime refused the launch */
#define APPROXIFER_ERR_WORKSPACE_LIMIT (-8)/* approxifer_decode_byzantine_static(): the built-in workspace is too small */
#define APPROXIFER_ERR_BAD_DTYPE (-9)      /* dtype is none of APPROXIFER_F32, APPROXIFER_F16, APPROXIFER_BF16 */
#define APPROXIFER_ERR_ALIGNMENT (-10)     /* a pointer or stride is not aligned as the call asks */
#define APPROXIFER_ERR_BAD_CACHE (-11)     /* sizes of a cache, of its sequences or of its heads that do not fit together */
#define APPROXIFER_ERR_WORKSPACE (-12)     /* a call that cannot do without a workspace was given none, or too small a one */

/* Decoder sign conventions, see approxifer_decode(). */
#define APPROXIFER_SIGN_WORKER_INDEX 0
#define APPROXIFER_SIGN_SURVIVOR_RANK 1

/* Passed as S to the decoders: every group has its own number of stragglers, read off its mask. */
#define APPROXIFER_S_FROM_MASK (-1)

/* Per-group status values written to d_status. */
#define APPROXIFER_GROUP_OK 0
#define APPROXIFER_GROUP_BAD_MASK 1        /* the group's mask does not hold an acceptable number of ones */

/*
 * Chebyshev nodes of Section 3, "ApproxIFER Encoding":
 *   h_alpha[j] = cos((2j+1) pi / (2K)), j = 0..K-1   (first kind, query nodes)
 *   h_beta[i]  = cos(i pi / (N-1)),     i = 0..N-1   (second kind, worker nodes)
 * Both arrays are host memory written by the call.  Returns OK, ERR_NULL_POINTER or
 * ERR_BAD_SHAPE (K < 1 or N < 2).
 */
int approxifer_chebyshev_nodes(int K, int N, double *h_alpha, double *h_beta);

/*
 * Encoder (Section 3, "ApproxIFER Encoding").  For every group g and worker i
 *     d_coded[g][i][:] = u_g(beta_i) = sum_j l_j(beta_i) d_queries[g][j][:],
 *     l_j(z) = ((-1)^j / (z - alpha_j)) / sum_j' ((-1)^j' / (z - alpha_j')),
 * Berrut's rational interpolant through the K queries, read at the worker nodes.
 * If beta_i equals some alpha_j exactly, coded query i is query j.
 *
 *   d_queries  [G][K][D] float32, device, read only
 *   d_coded    [G][N][D] float32, device, written; must not overlap d_queries
 *   h_alpha    [K] float64, host;  h_beta [N] float64, host
 * The basis functions are evaluated in float64 on the device and rounded to float32;
 * the contraction over j accumulates in float32.
 */
int approxifer_encode(const float *d_queries, float *d_coded,
                      int64_t G, int K, int N, int64_t D,
                      const double *h_alpha, const double *h_beta, void *stream);

/*
 * Forming groups out of a stream of queries (Section 2, "System Architecture": the K queries of a group are
 * encoded together).  With the [G][K][D] layout of approxifer_encode() a stream of Q queries stored row by row,
 * [Q][D], IS its groups: queries g K .. g K + K - 1 are group g, no copy is made.  approxifer_group_count()
 * returns G = ceil(Q / K) (-1 for Q < 0 or K < 1).  When K does not divide Q the last group is short; the paper
 * has no rule for it, this library completes it by repeating the stream's last query (the interpolant then passes
 * through that query at every added node -- for a group of one query this is the replication the encoder reduces
 * to at K = 1 -- and the added answers are simply not read back).
 *
 * approxifer_pad_last_group(): d_queries is a device buffer of at least G K rows of D floats whose first Q rows
 * hold the stream; rows Q .. G K - 1 are overwritten with copies of row Q - 1.  Nothing is enqueued when K
 * divides Q, or when Q = 0 or D = 0.  Ungrouping needs no call: row q of the decoded [G][K][C] tensor (of the
 * [G][K] top-1 tensor) is query q's answer, rows Q and up belong to the repeated query.
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_SHAPE (Q < 0, D < 0, K < 1), ERR_LIMIT (K > APPROXIFER_MAX_K) or ERR_LAUNCH.
 */
int64_t approxifer_group_count(int64_t Q, int K);
int approxifer_pad_last_group(float *d_queries, int64_t Q, int K, int64_t D, void *stream);

/*
 * Decoder (Section 3, "ApproxIFER Decoding", step 2).  For every group g, with F the
 * set of workers whose mask byte is non-zero, in ascending order,
 *     d_out[g][j][:] = r_g(alpha_j)
 *                    = sum_{i in F} w_i d_preds[g][i][:] / sum_{i in F} w_i,
 *     w_i = s_i / (alpha_j - beta_i).
 * sign_mode APPROXIFER_SIGN_WORKER_INDEX takes s_i = (-1)^i with i the worker index,
 * as that formula is printed; APPROXIFER_SIGN_SURVIVOR_RANK takes s_i = (-1)^rank(i in F),
 * which is Berrut's interpolant (Section 3, eq. (2)) on the surviving nodes.  The two are
 * equal when no worker is missing.
 *
 *   d_preds   [G][N][C] float32, device; rows of workers with mask 0 are never read
 *   d_mask    [G][N] uint8, device; non-zero = the worker returned
 *   d_out     [G][K][C] float32, device, written
 *   d_status  [G] int32, device, written, or NULL.  A group whose mask does not hold
 *             exactly N-S non-zero bytes gets APPROXIFER_GROUP_BAD_MASK and its d_out
 *             rows are left untouched; every other group gets APPROXIFER_GROUP_OK.
 *   S         number of stragglers of every group, 0 <= S < N, or APPROXIFER_S_FROM_MASK:
 *             groups may then differ in how many workers returned (the formula of Section 3
 *             holds for any non-empty F); only a group with no survivor at all is a bad mask.
 * Weights and accumulation are float64; each output is rounded to float32 once.
 */
int approxifer_decode(const float *d_preds, const uint8_t *d_mask, float *d_out, int32_t *d_status,
                      int64_t G, int K, int N, int S, int64_t C,
                      const double *h_alpha, const double *h_beta, int sign_mode, void *stream);

/*
 * Byzantine decoder (Section 3, "ApproxIFER Decoding", steps 1-2, Algorithm 2).
 * For every group: among the N-S available workers locate A adversaries, drop them,
 * decode over the rest as approxifer_decode() does.
 * Location, per class c = 0..C-1 (Algorithm 2): with M = K + A and x_i = beta_i,
 * y_i = d_preds[g][i][c] for the available i, find P (degree M-1) and
 * Q = 1 + Q_1 x + .. + Q_{M-1} x^{M-1} minimising sum_i (P(x_i) - y_i Q(x_i))^2
 * (ordinary least squares, orthogonal elimination in float64), set a_i = Q(x_i), and note the A
 * workers of smallest |a_i| (equal magnitudes: smaller worker index first).  The A workers
 * noted most often over the C classes (equal counts: smaller worker index first) are the
 * adversaries.
 *
 *   d_adv     [G][A] int32, device, written: located workers in ascending order
 *   d_workspace, workspace_bytes
 *             device scratch memory owned by the caller, 8-byte aligned, or NULL / 0; contents on entry and exit
 *             are meaningless, the call initialises what it uses.  Two things live there.
 *             (1) The vote of Algorithm 2's return step is the one place where the classes of a group meet.  With
 *             many classes the library spreads a group's over several workgroups, which pool their per-class
 *             picks in N vote counters and an arrival counter per group.
 *             (2) Without stragglers (S = 0, the setting of the paper's Byzantine experiments, or
 *             APPROXIFER_S_FROM_MASK) every group whose mask is full fits the same node set: the part of
 *             Algorithm 2's system that does not depend on the predictions is then factorised once per call
 *             instead of once per group, and kept in the workspace.  On the Chebyshev worker nodes with S = 0 most
 *             shapes need no factorisation; the bytes are asked for all the same, for nodes of the caller's own.
 *             approxifer_workspace_bytes() gives the size that allows both.  With NULL, fewer bytes or a
 *             misaligned pointer the call uses what fits and is just as correct: d_out, d_adv and d_status hold
 *             the same bits; only time is lost (every group stays with one workgroup and repeats the
 *             factorisation).  Nothing but the workspace is ever used as scratch: output rows are written
 *             once, with their final values.  The workspace must not be shared with a call that may run
 *             concurrently.
 *   other arguments as approxifer_decode(); groups with a bad mask leave d_out and
 *   d_adv rows untouched.
 * On APPROXIFER_ERR_LAUNCH the kernels that prepare the workspace may have been enqueued; no output
 * is touched.
 * Requires A >= 1, N - S >= 2 (K + A) (Section 3, eq. (3), the decoding condition) and
 * N - S <= APPROXIFER_MAX_AVAIL_BYZ.  With S = APPROXIFER_S_FROM_MASK a group is decoded when its
 * own number of available workers n satisfies 2 (K + A) <= n <= APPROXIFER_MAX_AVAIL_BYZ and gets
 * APPROXIFER_GROUP_BAD_MASK otherwise.  A worker whose node is exactly 0 can never be
 * located, since Q(0) = 1 by construction; the Chebyshev worker nodes contain 0 only
 * when N is odd.
 */
int approxifer_decode_byzantine(const float *d_preds, const uint8_t *d_mask, float *d_out,
                                int32_t *d_adv, int32_t *d_status,
                                int64_t G, int K, int N, int S, int A, int64_t C,
                                const double *h_alpha, const double *h_beta, int sign_mode,
                                void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Size in bytes of the workspace with which approxifer_decode_byzantine() and
 * approxifer_decode_byzantine_homogeneous() run fastest for this shape (Algorithm 2, return step: the
 * per-class picks of a group are pooled there when its classes are spread over several workgroups).
 * 0 when the shape needs none -- a fixed number S > 0 of stragglers with enough groups to fill the GPU with one
 * workgroup each, or few classes -- and for shapes the decoders refuse.  Host arithmetic only; at most
 * 4 (N + 1) bytes per group plus 13 KiB, each part rounded up to a multiple of 256.
 */
size_t approxifer_workspace_bytes(int64_t G, int K, int N, int S, int A, int64_t C);

/*
 * approxifer_decode_byzantine() for callers that cannot allocate device memory, not even a workspace:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The same call with
 * the workspace arguments left out; the scratch memory is an array of APPROXIFER_STATIC_WORKSPACE_BYTES
 * bytes built into the library's device code (every GPU the library runs on holds one copy until the
 * process ends).  The call allocates and frees nothing and calls no allocating routine; inputs and outputs
 * are still the caller's.
 *   - A shape for which approxifer_workspace_bytes() exceeds APPROXIFER_STATIC_WORKSPACE_BYTES is refused
 *     with APPROXIFER_ERR_WORKSPACE_LIMIT before anything is enqueued (4 (N + 1) G bytes are needed when
 *     few groups bring hundreds of classes or more, up to 13 KiB when no stragglers are asked for; shapes
 *     that need no workspace are never refused, nor are more groups than fill the GPU with one workgroup each:
 *     their votes are counted without the workspace where it has no room for them).
 *   - The device of `stream` must be the current device.  The first call on a device looks up the address
 *     of that device's copy of the array (no allocation, no synchronisation).
 *   - All calls on one GPU share that GPU's array.  Each call clears the part it uses with a kernel of
 *     its own, so what an earlier call left there does not matter; two calls whose work OVERLAPS on one
 *     GPU (different streams, or graphs replayed concurrently) race on it and give undefined results.
 *     Calls on one stream, one after the other, are safe.
 * Results, other arguments, requirements and error codes are those of approxifer_decode_byzantine().
 */
#define APPROXIFER_STATIC_WORKSPACE_BYTES 65536
int approxifer_decode_byzantine_static(const float *d_preds, const uint8_t *d_mask, float *d_out,
                                       int32_t *d_adv, int32_t *d_status,
                                       int64_t G, int K, int N, int S, int A, int64_t C,
                                       const double *h_alpha, const double *h_beta, int sign_mode, void *stream);

/*
 * Byzantine decoder with the locator of Section 2, Algorithm 1, in place of Algorithm 2: the
 * same call, the same picks, vote and decode, but per class the fit leaves Q_0 free.  With
 * M = K + A, P and Q both of degree M-1, the coefficient vector (P_0..P_{M-1}, Q_0..Q_{M-1})
 * is the unit vector minimising sum_i (P(x_i) - y_i Q(x_i))^2 over the available workers: the
 * right singular vector of the smallest singular value of the n x 2M matrix of the
 * homogeneous system (orthogonal elimination in float64, then inverse iteration on the triangular
 * factor and, for a class whose iteration does not settle, one-sided Jacobi rotations
 * until every pair of its columns is orthogonal to rounding).  a_i = Q(x_i) is
 * defined up to one factor, which the order of the |a_i| does not see.  Unlike Algorithm 2
 * this locator can find a worker whose node is exactly 0.  It costs a singular value
 * decomposition per class where Algorithm 2 costs a least-squares solve.
 * The iterations are bounded (24 or 64 rounds of inverse iteration, then at most 30 Jacobi sweeps); a
 * class whose columns are still not orthogonal to rounding after that -- not observed on finite
 * data -- votes with the shortest column found so far, best effort, and no status reports it.
 * Arguments, requirements and error behaviour as approxifer_decode_byzantine().
 */
int approxifer_decode_byzantine_homogeneous(const float *d_preds, const uint8_t *d_mask, float *d_out,
                                            int32_t *d_adv, int32_t *d_status,
                                            int64_t G, int K, int N, int S, int A, int64_t C,
                                            const double *h_alpha, const double *h_beta, int sign_mode,
                                            void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Decoder by rational reconstruction (Appendix A, Algorithm 3 and Theorem 2).  For every group, class c and
 * query j: with (P, Q) the least-squares fit of Algorithm 2 (degrees K + A - 1, Q_0 = 1) to the class's
 * values on the available workers,
 *     d_out[g][j][c] = P(alpha_j) / Q(alpha_j).
 * No worker is located or dropped and Berrut's interpolant is not used: when the hosted model makes the
 * coded predictions exactly rational in the node and at most A workers lie, P / Q is that rational function
 * (Theorem 2).  The paper sets this decoder aside because the quotient is fragile under round-off -- P and Q
 * share the error-locator factor -- and so does this library: it is here to make the comparison possible,
 * approxifer_decode_byzantine() is the decoder to use.  On float32 data of the paper's sizes single groups lose
 * several digits; the fit's condition number, not the arithmetic (float64 Householder QR), bounds the accuracy.
 *   arguments, requirements, status values and error codes as approxifer_decode_byzantine(), without
 *   d_adv, sign_mode and workspace; groups with a bad mask leave their d_out rows untouched.  Q can vanish
 *   at a query node only by accident of the data; the quotient is then non-finite.
 */
int approxifer_decode_rational(const float *d_preds, const uint8_t *d_mask, float *d_out, int32_t *d_status,
                               int64_t G, int K, int N, int S, int A, int64_t C,
                               const double *h_alpha, const double *h_beta, void *stream);

/*
 * Fused decoder + top-1 (Section 4.1, "Performance metric": the paper scores the class of the
 * largest decoded soft label).  Decodes exactly as approxifer_decode() does, in float64, and for
 * every group g and query j writes only
 *     d_top1[g][j]  = argmax_c r_g(alpha_j)[c]      (equal values: the smallest c)
 *     d_score[g][j] = that largest decoded value, rounded to float32 (d_score may be NULL)
 * The [G][K][C] prediction tensor is never written.  The argmax is taken on the float64
 * accumulators, before any rounding.  NaN never wins against a number; a query whose values are all NaN gets class 0,
 * and one that has nothing above -inf a class all the same: 0 <= d_top1 < C, with a score that is NaN or -inf.
 *
 *   d_top1    [G][K] int32, device, written
 *   d_score   [G][K] float32, device, written, or NULL
 *   other arguments, status values and errors as approxifer_decode(); groups with a bad mask
 *   leave their d_top1 / d_score rows untouched.
 */
int approxifer_decode_top1(const float *d_preds, const uint8_t *d_mask, int32_t *d_top1, float *d_score,
                           int32_t *d_status, int64_t G, int K, int N, int S, int64_t C,
                           const double *h_alpha, const double *h_beta, int sign_mode, void *stream);

/*
 * Top-1 of an already decoded tensor (Section 4.1, "Performance metric"): for every row of d_values [rows][C]
 * the class of the largest value (equal values: the smallest class) and, optionally, that value.  For the
 * outputs of approxifer_decode_byzantine(), whose [G][K][C] tensor is [G K][C] row by row;
 * approxifer_decode_top1() fuses the same decision into the plain decoder.  The decision is taken on the
 * float32 values as stored.  NaN never wins; a row without any ordinary value gives class 0.
 *   d_values  [rows][C] float32, device, read only
 *   d_top1    [rows] int32, device, written;  d_score [rows] float32, device, written, or NULL
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_SHAPE (rows < 0 or C < 0), ERR_LIMIT (C >= 2^31) or ERR_LAUNCH.
 */
int approxifer_top1(const float *d_values, int32_t *d_top1, float *d_score, int64_t rows, int64_t C, void *stream);

/*
 * Wait rule (Section 3, "ApproxIFER Decoding", step 1: the decoder waits for the results of the
 * fastest workers -- K of them without adversaries, 2 (K + E) with E of them).  Turns arrival times
 * into the survivor mask the decoders take: for every group g the `wait_for` workers with the
 * smallest arrival time get mask 1, all others 0.  Equal times: the smaller worker index first.
 * A time that is not finite (NaN, +-inf) means the worker never answers; a group in which fewer
 * than `wait_for` workers answer has all of those marked, and its count says so.
 *
 *   d_arrival  [G][N] float32, device, read only: arrival time of every worker's result, any unit
 *   d_mask     [G][N] uint8, device, written (0 or 1)
 *   d_count    [G] int32, device, written, or NULL: number of ones in the group's mask
 *   wait_for   1 <= wait_for <= N
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_SHAPE (G < 0, N < 1, wait_for out of range) or ERR_LIMIT
 * (N > APPROXIFER_MAX_N).
 */
int approxifer_wait_mask(const float *d_arrival, uint8_t *d_mask, int32_t *d_count,
                         int64_t G, int N, int wait_for, void *stream);

/*
 * Sequences kept by the workers.
 *
 * A hosted model that reads sequences keeps the keys and values of the tokens it has seen.  The code's weights sum to
 * one (Section 3, "ApproxIFER Encoding"), so what all queries of a group have in common, a prompt for one, is coded
 * into itself: its keys and values are computed once and shared by the N workers' sequences, which go apart with the
 * first token that differs.  They therefore live in pages that sequences can share.
 *
 *   pool    [P][Hkv][page][Dh] of one dtype: P pages of `page` tokens for Hkv heads of Dh values.  A layer has two, one
 *           of keys and one of values; page p is the same place in all of them.  16-byte aligned.
 *   table   [B][M] int32: place t of sequence b lives in page table[b][t / page], slot t % page
 *   lens    [B] int32: tokens of each sequence; a sequence holds its first ceil(lens / page) table entries, the
 *           entries behind them mean nothing
 *   refs    [P] int32: how many holders each page has, 0: free
 *   starts  [B + 1] int32: the calls below work on T rows, one per NEW token; rows starts[b] .. starts[b + 1] - 1 are
 *           the last tokens of sequence b.  With n of them, row i of the sequence is at place lens[b] - n + i.
 *           Sequences without new tokens have n = 0.
 *
 * All sizes and indices that the device holds are checked there before they are used; what is wrong with a sequence
 * is told in d_status [B] (int32, written, or NULL), and a bad sequence does not disturb the others:
 *   APPROXIFER_GROUP_OK
 *   APPROXIFER_SEQUENCE_BAD        its rows lie outside 0 .. T, or its length outside 0 .. M page: nothing is written.  (starts
 *                                  must not fall: where it does, rows of other sequences may stay unwritten too.)
 *   APPROXIFER_SEQUENCE_BAD_PAGE   a table entry that the call needs is not in 0 .. P - 1: see the calls
 *   APPROXIFER_SEQUENCE_NO_PAGES, APPROXIFER_SEQUENCE_SHARED_PAGE   see the calls that take pages
 *
 * Sizes: page a power of two up to 4096; Dh a multiple of 8 up to 256; Hq a multiple of Hkv, Hq <= 1024; T up to 2^24, B up
 * to 2^20, T Hq up to 2^30, B Hkv up to 2^22, P and M page up to 2^30 (pools may be larger than that), M and P at least 1.
 * APPROXIFER_ERR_BAD_CACHE, or APPROXIFER_ERR_LIMIT for sizes that are merely too large.
 */
#define APPROXIFER_F32 0
#define APPROXIFER_F16 1
#define APPROXIFER_BF16 2

#define APPROXIFER_SEQUENCE_BAD 1
#define APPROXIFER_SEQUENCE_BAD_PAGE 2
#define APPROXIFER_SEQUENCE_NO_PAGES 3
#define APPROXIFER_SEQUENCE_SHARED_PAGE 4

#define APPROXIFER_MAX_HEAD_DIM 256
#define APPROXIFER_MAX_HEADS 1024
#define APPROXIFER_MAX_PAGE 4096
#define APPROXIFER_MAX_AXES 4
#define APPROXIFER_MAX_ROWS (1 << 24)
#define APPROXIFER_MAX_SEQUENCES (1 << 20)
#define APPROXIFER_MAX_PAGES (1 << 30)
#define APPROXIFER_MAX_TOKENS (1 << 30)

typedef struct approxifer_sequences {   /* host memory, read before the call returns */
    const int32_t *d_table;             /* [B][M] device */
    const int32_t *d_lens;              /* [B] device */
    const int32_t *d_starts;            /* [B + 1] device */
    int64_t T, B, M, P;
    int32_t page;
} approxifer_sequences;

/* Rotation frequencies h_freq[i] = base^(-i / pairs), i = 0..pairs-1, in radians per position (host memory, written).
 * Returns OK, ERR_NULL_POINTER or ERR_BAD_SHAPE (pairs < 1, base not finite or not positive). */
int approxifer_rotary_frequencies(int pairs, double base, double *h_freq);

/*
 * Appends the T new tokens to the cache: norm of every head of the queries and keys, rotation by position, and keys
 * and values written into their pages, in one pass.  For one head's vector x of a token,
 *     y = x w / sqrt(mean(x^2) + eps)      (w the weight; without one y = x)
 *     angle_i = position[axis_i] freq_i,   i < pairs
 *     (a, b) -> (a cos - b sin, a sin + b cos)   for (a, b) = (y_i, y_{i + pairs}), or (y_{2i}, y_{2i+1}) if interleaved;
 * values of y behind the first 2 pairs stay as they are.
 *
 *   d_q [T][Hq][Dh], d_k, d_v [T][Hkv][Dh]   read only; a token's heads are contiguous, tokens q_stride, k_stride, v_stride
 *                     values apart (so slices of one projection's output need no copy; any alignment, 16 bytes is fastest)
 *   d_q_out           [T][Hq][Dh] written, contiguous, 16-byte aligned; may be d_q itself if that is contiguous
 *   d_k_pool, d_v_pool   one layer's pools; the new tokens' slots are written, nothing else.  No two of the sequences
 *                     may hold the page that a new token goes to (approxifer_cache_reserve() sees to it).
 *   d_q_weight, d_k_weight   [Dh] of the same dtype, device, or NULL: no norm
 *   d_positions       [T][axes] int32, device, or NULL: the token's place in its sequence (axes must be 1)
 *   h_freq            [pairs] float64, host; h_axis [pairs] int32, host, 0 <= h_axis[i] < axes, or NULL: all 0
 *   pairs             0 <= 2 pairs <= Dh;  1 <= axes <= APPROXIFER_MAX_AXES
 * Angles are reduced in float64, norms and rotations computed in float32, each output rounded once.  A new token whose place
 * is negative (more rows than the length) or whose page is bad is written to d_q_out, but not to the pools.
 * The rows of a sequence that is APPROXIFER_SEQUENCE_BAD are not written at all.
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_SHAPE (pairs, axes, strides, eps), ERR_BAD_CACHE, ERR_LIMIT, ERR_BAD_DTYPE,
 * ERR_BAD_NODES (a frequency that is not finite), ERR_ALIGNMENT or ERR_LAUNCH.
 */
int approxifer_append(const approxifer_sequences *h_seq, int Hq, int Hkv, int Dh, int dtype,
                      const void *d_q, int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_v, int64_t v_stride,
                      void *d_q_out, void *d_k_pool, void *d_v_pool,
                      const void *d_q_weight, const void *d_k_weight, double eps,
                      const int32_t *d_positions, int axes, const double *h_freq, const int32_t *h_axis, int pairs,
                      int interleaved, int32_t *d_status, void *stream);

/*
 * Attention of the T new tokens to what their sequences hold, themselves included (append first).  For the row at place t,
 * query head h and the cache's head h / (Hq / Hkv),
 *     out = sum_j softmax_j(scale q . k_j) v_j   over the visible places j <= t:
 *           all of them if window = 0, else those with j > t - window or j < sinks.
 * A row that sees nothing (its place is negative) gets zeros.  What a row does not see has no effect on it, whatever it
 * holds (infinities and NaN included); neither has what lies behind a sequence's length.
 *
 *   d_q     [T][Hq][Dh], tokens q_stride values apart, read only;  d_out [T][Hq][Dh] written, contiguous, 16-byte aligned,
 *           must not overlap d_q
 *   max_rows, max_len   bounds of the sequences' numbers of new tokens and lengths: a sequence beyond one is
 *           APPROXIFER_SEQUENCE_BAD.  The work is laid out for them, so close bounds are faster.
 *   window >= 0, sinks >= 0, |scale| <= 2^126 (it is used in float32)
 *   d_workspace, workspace_bytes   scratch of the caller's, 16-byte aligned, or NULL / 0, as for
 *           approxifer_decode_byzantine(): long sequences with few rows are split over the GPU, and the parts meet there.
 *           approxifer_attend_workspace_bytes() gives the size with which the call is fastest; with less it is split
 *           less, and as correct.
 * Rows that see a place in a bad page are NaN.  Scores, softmax and sums are float32; for 16-bit types the weights are
 * rounded before they multiply the values, for many rows to the type (which adds about a third to the error that the
 * output's own rounding makes), for few (up to 16 of a sequence and head of the cache) to twice its length.  Each output
 * is rounded once.
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_SHAPE, ERR_BAD_CACHE, ERR_LIMIT, ERR_BAD_DTYPE, ERR_ALIGNMENT or ERR_LAUNCH; the
 * call may consist of two launches.
 */
int approxifer_attend(const approxifer_sequences *h_seq, int Hq, int Hkv, int Dh, int dtype,
                      const void *d_q, int64_t q_stride, const void *d_k_pool, const void *d_v_pool, void *d_out,
                      int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks, double scale,
                      int32_t *d_status, void *d_workspace, size_t workspace_bytes, void *stream);
size_t approxifer_attend_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows,
                                         int64_t max_len, int64_t window, int64_t sinks);

/*
 * approxifer_attend() for sequences that begin alike, as forks of one prompt do: what a group of them has in common is read once for all of
 * its rows, not once for every sequence.
 *
 *   d_groups    [C + 1] int32, must not fall: sequences d_groups[c] .. d_groups[c + 1] - 1 are group c.  Others are in none.
 *   d_shared    [C] int32: the first d_shared[c] places of all sequences of group c, as far as they have them, hold the same keys and
 *               values, in the same pages or in copies (approxifer_cache_fork() shares the full ones and copies the last).  From whose
 *               pages they are read is the call's choice.
 *   max_shared  bound of d_shared.  Sequences of a group that reaches outside 0 .. B, or whose d_shared is not in 0 .. max_shared, are
 *               attended to as if they shared nothing.
 *   d_workspace as for approxifer_attend(), of approxifer_attend_shared_workspace_bytes(); without one, or with too small a one, and
 *               where the sequences have so many rows each that reading is not what they wait for, or hardly more than one is in a
 *               group, the call is approxifer_attend()
 * How long the common places are does not decide here: behind few of them the call takes longer than approxifer_attend() would.
 * approxifer_attend_shared_pays() says which one to call.
 * Common places' weights are rounded to the type once where a group has many rows, as those of many rows are in approxifer_attend().
 * Where d_groups or d_starts falls, any row may be unwritten or wrong.  A page that is not in 0 .. P - 1 of the sequence that a group's places are read from
 * makes the rows of the others that see it NaN too, and their statuses APPROXIFER_SEQUENCE_BAD_PAGE.
 * Others, and what is returned, as approxifer_attend(), with ERR_BAD_SHAPE also for a negative C or max_shared and ERR_LIMIT for a C beyond
 * 2^20; the call consists of up to three launches.
 */
int approxifer_attend_shared(const approxifer_sequences *h_seq, int Hq, int Hkv, int Dh, int dtype,
                             const void *d_q, int64_t q_stride, const void *d_k_pool, const void *d_v_pool, void *d_out,
                             const int32_t *d_groups, const int32_t *d_shared, int64_t C, int64_t max_rows, int64_t max_len,
                             int64_t max_shared, int64_t window, int64_t sinks, double scale, int32_t *d_status, void *d_workspace,
                             size_t workspace_bytes, void *stream);
size_t approxifer_attend_shared_workspace_bytes(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows,
                                                int64_t max_len, int64_t max_shared, int64_t window, int64_t sinks);
/* 1 where approxifer_attend_shared() is expected to take less time than approxifer_attend(), both with workspaces of the sizes that are
 * asked for, if about all C groups have max_shared places in common; else 0, also for sizes that the calls refuse.  Host arithmetic only. */
int approxifer_attend_shared_pays(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int page, int64_t max_rows,
                                  int64_t max_len, int64_t max_shared, int64_t window, int64_t sinks);

/*
 * approxifer_attend(), which also adds up the weights that it gives: for every place j of sequence b
 *     d_mass[b][j] += sum over the rows of b and the Hq query heads of softmax_j(scale q . k_j),
 * the measure by which approxifer_cache_evict() chooses.  Places that no row sees get nothing added; a call for each layer adds the
 * layers up.  Where a row's scores are no numbers (a NaN in its query or in a key that it sees, a score of +infinity, a page that is not in
 * 0 .. P - 1), so is the mass of all that it sees; what is in the values does not matter.
 *
 *   d_mass      [B][mass_stride] float32; places of a sequence's length and behind it are left as they are.  A sequence longer than
 *               mass_stride is APPROXIFER_SEQUENCE_BAD, as one beyond max_len is.
 *   d_workspace 16-byte aligned, at least 8 T Hq bytes rounded up to 256.  approxifer_attend_mass_workspace_bytes() gives the size with
 *               which the call is fastest; with less its work is split less, or scores are formed twice.  Where few rows' scores are kept it
 *               is 4 bytes for every row, head and place up to max_len, in all up to 2 GiB: a max_len near the lengths asks for less.
 * Others as approxifer_attend().  Weights and their sums are float32; a key's weights are added in an order that the sizes and the
 * workspace fix, so the same call gives the same bits.
 * Returns what approxifer_attend() does, or ERR_WORKSPACE; ERR_BAD_SHAPE for a negative mass_stride, ERR_ALIGNMENT for a d_mass that is not
 * at a multiple of 4.  The call consists of up to four launches.
 */
int approxifer_attend_mass(const approxifer_sequences *h_seq, int Hq, int Hkv, int Dh, int dtype,
                           const void *d_q, int64_t q_stride, const void *d_k_pool, const void *d_v_pool, void *d_out,
                           float *d_mass, int64_t mass_stride, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks,
                           double scale, int32_t *d_status, void *d_workspace, size_t workspace_bytes, void *stream);
size_t approxifer_attend_mass_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows,
                                              int64_t max_len, int64_t window, int64_t sinks);

/*
 * Room for d_add[b] >= 0 more tokens of every sequence: lens[b] += add[b], and the pages this takes are the free ones of
 * lowest index, given out in the order of the sequences; their refs become 1.  All in place.
 *   APPROXIFER_SEQUENCE_SHARED_PAGE   the sequence's last page is not full and has another holder: fork the sequence first
 *   APPROXIFER_SEQUENCE_NO_PAGES      the free pages end before this sequence; later ones that want any end so too
 *   APPROXIFER_SEQUENCE_BAD           add[b] < 0, lens[b] < 0, or more tokens than M page
 *   APPROXIFER_SEQUENCE_BAD_PAGE      the last page, which is not full, is not in 0 .. P - 1
 * A sequence with any of these stays as it is; it takes no pages (one without free pages keeps those behind it
 * from taking any).  The same holders are seen by all calls: several calls of one cache must not overlap.
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_CACHE, ERR_LIMIT or ERR_LAUNCH.
 */
int approxifer_cache_reserve(int32_t *d_table, int32_t *d_lens, int32_t *d_refs, const int32_t *d_add, int32_t *d_status,
                             int64_t B, int64_t M, int64_t P, int page, void *stream);

/*
 * New sequences out of old ones: forks, reorders, shortens and ends sequences.  New sequence i (0 <= i < B_out) continues
 * old sequence d_parents[i], all of it or its first d_keep[i] tokens; d_parents[i] = -1 is an empty sequence, and an old
 * sequence that nobody continues gives its pages back.  Full pages are shared.  A last page that is not full is taken over if
 * no other holder is left and i is the first to want it, else its copy is the free page of lowest index, in the order of i:
 * `page_bytes` bytes of each of the `planes` pools [planes][P][page_bytes] are copied.
 * d_refs_out = d_refs - what the old sequences held + what the new ones hold: holders that are no sequence stay counted.
 *   d_keep      [B_out] int32, device, or NULL: as many tokens as there are
 *   d_table_out [B_out][M], d_lens_out [B_out], d_refs_out [P]  written; must not overlap the inputs.  Entries of d_table_out
 *               behind a sequence's pages are -1.
 *   d_pools     16-byte aligned, page_bytes a multiple of 16; may be NULL with planes = 0
 *   d_status    [B_out]: APPROXIFER_SEQUENCE_BAD (parent outside -1 .. B - 1, keep < 0, or a parent's length outside 0 .. M page),
 *               APPROXIFER_SEQUENCE_BAD_PAGE (of the parent), APPROXIFER_SEQUENCE_NO_PAGES: the new sequence is empty
 *   d_workspace at least approxifer_cache_workspace_bytes(B, B_out, P) bytes, 16-byte aligned
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_SHAPE (planes, page_bytes), ERR_BAD_CACHE, ERR_LIMIT, ERR_ALIGNMENT, ERR_WORKSPACE or
 * ERR_LAUNCH; the call consists of several launches.
 */
int approxifer_cache_fork(const int32_t *d_table, const int32_t *d_lens, const int32_t *d_refs, const int32_t *d_parents,
                          const int32_t *d_keep, int32_t *d_table_out, int32_t *d_lens_out, int32_t *d_refs_out,
                          int32_t *d_status, void *d_pools, int64_t planes, int64_t page_bytes, int64_t B, int64_t B_out,
                          int64_t M, int64_t P, int page, void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Moves the live pages together: with L of them, the ones at L and above go to the free places below L, both in ascending
 * order, in all pools; d_table and d_refs follow, in place.  Afterwards pages 0 .. L - 1 are live, the others free.
 *   d_moved     [P] int32, written: where each page that was live is now, -1 for the others (for holders that are no
 *               sequence)
 *   d_live      [1] int32, written: L
 *   others as approxifer_cache_fork().  Table entries that are no live page stay as they are.
 */
int approxifer_cache_compact(int32_t *d_table, const int32_t *d_lens, int32_t *d_refs, int32_t *d_moved, int32_t *d_live,
                             void *d_pools, int64_t planes, int64_t page_bytes, int64_t B, int64_t M, int64_t P, int page,
                             void *d_workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace that approxifer_cache_fork() (with B_out new sequences) and approxifer_cache_compact() need; 0 for sizes
 * that they refuse.  Host arithmetic only. */
size_t approxifer_cache_workspace_bytes(int64_t B, int64_t B_out, int64_t P);

/*
 * Eviction: every sequence of more than `budget` tokens keeps that many.  Its `first` first and `recent` last tokens stay, and of
 * those between them the ones with the largest masses (approxifer_attend_mass() adds them up; equal ones: the lower place; NaN is
 * less than any number).  What stays keeps its order and closes up: the token that was at the i-th kept place is at place i, in all
 * pools.  Keys keep the rotation that they were appended with, so new tokens' positions are then the caller's to give.
 * Sequences of at most `budget` tokens stay as they are.
 *   d_mass      [B][mass_stride] float32, one for each place; of a sequence that is cut they close up too, and the places that it
 *               gives up get 0.  mass_stride >= 0; a sequence longer than that is bad.
 *   d_kept      [B][budget] int32, written: the places that are kept, ascending, then -1 (all of them -1 where the status is not OK)
 *   d_pools     [planes][P][heads][page][row_bytes], 16-byte aligned, row_bytes a multiple of 16 up to 1024; may be NULL with
 *               planes = 0.  Only places below `budget` are written, and of these none before the first page that changes.
 * Pages that a sequence holds alone are written in place.  One that has other holders too, and of which a token moves (or that is the
 * last one and not full), is left to them, and a free page takes its place: lowest index first, in the order of the sequences, as
 * they were free when the call began.  Pages behind the budget are given back, and their table entries become -1.
 *   1 <= budget <= 2^30, first >= 0, recent >= 0, first + recent <= budget
 *   d_status    [B]: APPROXIFER_SEQUENCE_BAD (length outside 0 .. M page, or beyond mass_stride), APPROXIFER_SEQUENCE_BAD_PAGE (it is
 *               to be cut, and a page of it is not in 0 .. P - 1, or has no holder), APPROXIFER_SEQUENCE_NO_PAGES (the free pages end
 *               before this sequence; later ones that want any end so too): the sequence stays as it is
 *   d_workspace at least approxifer_cache_evict_workspace_bytes(B, budget, P, page) bytes, 16-byte aligned
 * Returns OK, ERR_NULL_POINTER, ERR_BAD_SHAPE (planes, heads, row_bytes, mass_stride, budget, first, recent), ERR_BAD_CACHE, ERR_LIMIT,
 * ERR_ALIGNMENT, ERR_WORKSPACE or ERR_LAUNCH; the call consists of several launches.
 */
int approxifer_cache_evict(int32_t *d_table, int32_t *d_lens, int32_t *d_refs, float *d_mass, int64_t mass_stride, int32_t *d_kept,
                           int32_t *d_status, void *d_pools, int64_t planes, int64_t heads, int64_t row_bytes, int64_t B, int64_t M,
                           int64_t P, int page, int64_t budget, int64_t first, int64_t recent, void *d_workspace, size_t workspace_bytes,
                           void *stream);
size_t approxifer_cache_evict_workspace_bytes(int64_t B, int64_t budget, int64_t P, int page);

/* Text for a return code; never NULL.  The string is static. */
const char *approxifer_strerror(int code);

/* Library version, major*10000 + minor*100 + patch. */
int approxifer_version(void);

#ifdef __cplusplus
}
#endif
#endif /* APPROXIFER_H */
