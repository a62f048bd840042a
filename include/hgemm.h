/*
 * hgemm.h -- C ABI of the MI355X (gfx950) half-precision GEMM library.
 *
 * The operation (paper Section 2.1, "HGEMM"): C = alpha*A*B + beta*C with
 * alpha = 1, beta = 0, i.e. C = A*B, where A is M x K, B is K x N, C is M x N,
 * all stored as IEEE binary16.  Products are accumulated in fp32 (one of the
 * two accumulator choices Section 1 names as valid for fp16 inputs) and each
 * result is rounded once, to nearest even, to fp16.
 *
 * Layouts (Section 2.2.2): "NN" = A, B, C all row-major; "TN" = B stored
 * column-major (an N x K row-major array).  A and C are always row-major.
 *
 * One plan per (M,N,K,layout): the paper's premise (Abstract, Section 5) is
 * that every shape wants its own kernel configuration; hgemm_plan() looks the
 * shape up in a table of measured choices (one table per layout of B; a shape
 * tuned only with row-major B uses that row for column-major B too) and falls
 * back to a fitted cost model.
 *
 * Threading: functions are thread-compatible (no global mutable state apart
 * from a read-only table and two per-device caches behind mutexes: whether a
 * device is a gfx950, and the address of hgemm_run_static's scratch array); a
 * single plan must not be run on two streams at once because split-K,
 * stream-K and padded plans own a workspace.
 * The library never prints, never throws, never synchronises the device, and
 * launches only on the stream it is given (Section 2.4.1 forbids a kernel
 * under test from using extra streams).  A plan whose workspace holds
 * counters (a split of K joined in one launch, the routing of up to 128
 * tokens) clears them in the null stream when it is made; its first run waits
 * for that stream unless it goes there itself.
 */
#ifndef HGEMM_H
#define HGEMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hgemm_plan_s* hgemm_plan_t;      /* opaque; owned by the library */

typedef enum {
    HGEMM_OK              = 0,
    HGEMM_ERR_INVALID_ARG = 1,   /* null pointer, negative size, bad enum, bad spec string */
    HGEMM_ERR_UNSUPPORTED = 2,   /* layout / leading dimension / alignment not implemented */
    HGEMM_ERR_ALLOC       = 3,   /* workspace allocation failed                            */
    HGEMM_ERR_LAUNCH      = 4,   /* the HIP runtime reported a launch error                */
    HGEMM_ERR_ARCH        = 5,   /* current device is not gfx950                           */
    HGEMM_ERR_WORKSPACE   = 6    /* hgemm_run_static: the plan needs more scratch than the
                                    static buffer holds                                    */
} hgemm_status_t;

typedef enum { HGEMM_ROW_MAJOR = 0, HGEMM_COL_MAJOR = 1 } hgemm_layout_t;

/* Storage of the three matrices.  ld* are leading dimensions in ELEMENTS;
 * 0 means packed (lda = K, ldb = N for row-major B or K for column-major B,
 * ldc = N).  a and c must be HGEMM_ROW_MAJOR.                               */
typedef struct {
    hgemm_layout_t a, b, c;
    int64_t lda, ldb, ldc;
} hgemm_layouts_t;

/*
 * hgemm_plan -- choose a kernel specialisation for one shape (Section 5: tile
 * sizes BM/BN/BK, stage count, block swizzle and the rest are picked per
 * (M,N,K)).  Host only: no kernel is launched.
 *   out      receives the plan (host pointer, written on HGEMM_OK only)
 *   M,N,K    >= 0.  M, N or K equal to 0 is valid (K = 0 gives C = 0).
 *   layouts  host pointer; NULL means NN, packed
 * Allocates the plan's device workspace (split-K partial sums, stream-K
 * partial tiles, padded copies of unaligned A and B) on the CURRENT device,
 * if the choice needs one.
 * Size: the matrix-core kernels address an operand with 32-bit byte offsets,
 * i.e. up to 2 GiB of it.  A problem with a larger A, B or C (dimensions and
 * leading dimensions multiples of 8) is planned as a grid of blocks -- row
 * blocks of A and C by column panels of B and C, each a plan of its own run
 * on offset pointers, one after the other on the stream; a row-major B of
 * that size is first copied, transposed, into the workspace (2*K*N bytes
 * more), because only a K-contiguous B can be cut into panels of less than
 * 2 GiB.  hgemm_plan_describe() then starts with "blocks,rows=R,cols=C".
 * Only hgemm_plan() does this: an explicit spec returns UNSUPPORTED for
 * such a problem, and hgemm_run_static() runs it on the generic kernel.
 * Errors: INVALID_ARG, UNSUPPORTED, ALLOC, ARCH.
 */
hgemm_status_t hgemm_plan(hgemm_plan_t* out, int64_t M, int64_t N, int64_t K,
                          const hgemm_layouts_t* layouts);

/*
 * hgemm_plan_override -- as hgemm_plan, but with the specialisation given by
 * `spec` instead of the dispatch table; used by the autotuner and by tests
 * that must cover every kernel.  `spec` is a host string of the form
 *   "<family>[,key=value]..."    e.g.  "mfma,bm=256,bn=256,bk=64,st=2,sk=1"
 * Families and keys are listed by hgemm_spec_help().  One key changes the
 * arithmetic rather than the schedule: "ac=16" asks for a 16-bit accumulator
 * (Section 1: fp16 and fp32 accumulators are both valid for fp16 inputs;
 * Section 2.3.2's exact-match test is built for the former): the running
 * sums are rounded to fp16 after every 16 products.  hgemm_plan() never
 * chooses it.  A spec that cannot run
 * the shape as it lies in memory (alignment, tile larger than the limits)
 * returns UNSUPPORTED: an explicit spec never pads.
 */
hgemm_status_t hgemm_plan_override(hgemm_plan_t* out, int64_t M, int64_t N, int64_t K,
                                   const hgemm_layouts_t* layouts, const char* spec);

/*
 * hgemm_run -- enqueue C = A*B on `hip_stream` (Section 2.1; the call shape
 * kernel(a, b, out) of Section 2.4.1's timing listing).
 *   A, B, C     DEVICE pointers to fp16, owned by the caller, non-overlapping.
 *               The matrix-core kernels read A and B in aligned 16-byte chunks
 *               and store C at any address and width.  When K, N or a leading
 *               dimension is not a multiple of 8, hgemm_plan() reserves room
 *               in the plan's workspace for zero-padded packed copies of A and
 *               B (Section 5.2's zero padding) and the run makes, in one launch
 *               before the GEMM on the same stream, those that are needed: of
 *               an operand whose rows are not whole aligned chunks, or whose
 *               base is not 16-byte aligned; smaller problems (",di=1" in the
 *               description) are read where they lie.  (Room that only
 *               such a base would need is left out where the device has no
 *               memory for it; the generic kernel serves such a base then.)  A C whose rows are
 *               2^31 elements apart or more is stored in the workspace and
 *               copied into place by one more launch.  Problems below 2^20
 *               multiply-adds with such sizes take a generic
 *               one-thread-per-element kernel, as do calls on aligned sizes
 *               whose A or B is not 16-byte aligned.  C is write-only: every
 *               element is overwritten (beta = 0), earlier contents never
 *               leak, and nothing outside the M x N elements of C is written.
 *   hip_stream  a hipStream_t passed as void*; NULL = the default stream.
 * Asynchronous; allocates nothing; all kernels (main, split-K reduction,
 * stream-K fix-up, the optional transposing copy of B) go to hip_stream in
 * order.
 * Errors: INVALID_ARG (null plan / null pointer with a non-empty problem),
 * LAUNCH.
 */
hgemm_status_t hgemm_run(hgemm_plan_t plan, const void* A, const void* B, void* C,
                         void* hip_stream);

/*
 * hgemm_run_many -- enqueue `count` calls of one plan back to back on
 * `hip_stream` (Section 2.4.2's offline mode: the same kernel executed
 * consecutively, without pauses).  Call i works on operand set j = (first + i)
 * % sets, C[j] = A[j] * B[j]; the result is that of `count` calls of hgemm_run
 * in a loop, bit for bit.  The
 * loop runs inside the library so that a caller in an interpreted language
 * pays its per-call overhead once per batch: kernels of 2-3 us are otherwise
 * enqueued more slowly than the GPU executes them.  Consecutive small calls of
 * which none writes what another reads or writes share one launch.
 *   count       number of calls, >= 0
 *   sets        number of operand sets, >= 1
 *   first       set of the first call, 0 <= first < sets (a caller that cycles
 *               through sets larger than the caches continues where its last
 *               batch stopped)
 *   A, B, C     HOST arrays of `sets` DEVICE pointers each (read during the
 *               call only); the operands they point to are as in hgemm_run
 *   hip_stream  as hgemm_run
 * Errors: as hgemm_run; stops at the first call that fails (calls already
 * enqueued stay enqueued).
 */
hgemm_status_t hgemm_run_many(hgemm_plan_t plan, int64_t count, int64_t sets, int64_t first,
                              const void* const* A, const void* const* B, void* const* C,
                              void* hip_stream);

/*
 * hgemm_run_static -- plan and enqueue C = A*B in one call that allocates
 * nothing, for callers that cannot allocate: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same operation,
 * argument meaning and kernels as hgemm_plan() + hgemm_run(); the difference
 * is where the workspace lives.  Split-K planes, stream-K partial tiles and
 * the padded copies of unaligned operands go to a static device array of
 * HGEMM_STATIC_SCRATCH_BYTES inside the library (one copy per GPU, held until
 * the process ends) instead of a hipMalloc'ed buffer, and the plan itself
 * lives on the call's stack.  A problem whose chosen specialisation needs more
 * scratch than that, arrival counters aside, returns HGEMM_ERR_WORKSPACE and
 * launches nothing.  An unaligned problem counts with padded copies of A, B and
 * C, whether they are made or not; aligned problems that need no workspace are
 * never refused.  The kernels overwrite every
 * scratch element they later read, so nothing has to be cleared between calls.
 * All calls on one GPU share that GPU's array: calls whose kernels may overlap
 * in time (different streams, no dependency between them) race on it, and so
 * does a call overlapping nothing but itself replayed concurrently from two
 * graphs.  Calls on one stream are safe.
 *   M,N,K,layouts   as hgemm_plan (host values); A,B,C,hip_stream as hgemm_run
 * Errors: INVALID_ARG, UNSUPPORTED, ARCH, WORKSPACE, LAUNCH.
 */
#define HGEMM_STATIC_SCRATCH_BYTES (64u << 20)
hgemm_status_t hgemm_run_static(int64_t M, int64_t N, int64_t K, const hgemm_layouts_t* layouts,
                                const void* A, const void* B, void* C, void* hip_stream);

/* hgemm_destroy -- free the plan and its workspace.  NULL is accepted.
 * (Housekeeping of this interface; the paper has no passage to cite for it,
 * nor for hgemm_status_string and hgemm_plan_describe below.)               */
hgemm_status_t hgemm_destroy(hgemm_plan_t plan);

/* ---- products of 8-bit floats and what an expert layer needs beside them ----------------------
 *
 * Not in the paper.  8-bit floats are the OCP formats: e4m3 (4 exponent bits, largest value 448, no
 * infinity) and e5m2 (largest value 57344).  A matrix of them carries one scale for every block of
 * HGEMM_SCALE_BLOCK = 128 consecutive elements of a row, or for every 128 x 128 block: the value an
 * element stands for is element * scale.  Scales are fp32 or e8m0 (one byte, the biased exponent of a
 * power of two: 0 stands for 2^-127, 255 for NaN).
 *
 * Scales by row lie block-major: that of row r and block b at [b * ld + r], so that the scales a tile
 * needs for one block of K are one run of memory.  Scales of 128 x 128 blocks lie at
 * [row block * ld + column block].
 *
 * All calls are asynchronous on `hip_stream`, allocate nothing but in the _plan calls, and follow the
 * threading rules above.  Pointers are device pointers.                                           */
#define HGEMM_SCALE_BLOCK 128

typedef enum { HGEMM_E4M3 = 0, HGEMM_E5M2 = 1 } hgemm_byte_t;
typedef enum { HGEMM_F16 = 0, HGEMM_BF16 = 1, HGEMM_F32 = 2 } hgemm_type_t;
typedef enum { HGEMM_SCALE_F32 = 0, HGEMM_SCALE_E8M0 = 1 } hgemm_scale_type_t;
typedef enum { HGEMM_GROUPS_NONE = 0, HGEMM_GROUPS_ROWS = 1, HGEMM_GROUPS_DEPTH = 2 } hgemm_groups_t;

/*
 * hgemm_scaled_* -- C = A * B^T over 8-bit operands with block scales:
 *   C[m][n] = sum over blocks b of K of  sa(m, b) * sb(n, b) * sum over k in b of A[m][k] * B[n][k].
 * A is M x K and B is N x K, both K-contiguous; C is M x N.  The sum over a block is taken by the
 * matrix cores, scaled, and added to an fp32 sum in the order of the blocks; one rounding to the type of
 * C.  For a 16-bit C the 8-bit instructions take the sums, which drop what lies more than 13 bits below
 * the largest of eight products: 1.6e-5 of the result over normal values, and at most 2^-10 of the sum of
 * the products' magnitudes, which shows where large products cancel.  For an fp32 C the fp16 instructions do, on
 * bytes widened to fp16, in fp32 throughout: a caller that needs such sums asks for an fp32 C.  Scales of A are
 * by row.  Scales of B are by 128 x 128 block (a weight) or by row (the right operand of a weight gradient).
 *
 *   forward        Y  = X * W^T             A = X by rows,     B = W by blocks
 *   data gradient  dX = dY * W              A = dY by rows,    B = the transposed form of W, by blocks
 *   weight gradient dW = dY^T * X           A = dY^T by rows,  B = X^T by rows (quantised along the tokens)
 * hgemm_quantise() writes all of these.
 *
 * Groups, for experts (`groups` of them, boundaries in `offsets`, groups + 1 int32 on the device):
 *   ROWS   rows offsets[g] .. offsets[g + 1] - 1 of A and C belong to group g and meet B[g]; B is
 *          groups x N x K, its scales groups x ceil(N / 128) x ceil(K / 128) (packed by the leading dimensions).
 *          Rows of C that no group holds become zero.  With a_rows > 0 row m of the problem is row
 *          index[m] of an A of a_rows rows (its scales likewise); an index outside [0, a_rows) is a row of zeros.
 *   DEPTH  columns offsets[g] .. offsets[g + 1] - 1 of A and B give C[g]; C is groups x M x N.
 *          Offsets are multiples of 128, or K (other values count rounded down).  An empty group gives zeros.
 * offsets[0] counts as 0, the others are clamped to the problem; they stay on the device, no call waits for them.
 *
 * A and B start on 16 bytes and have leading dimensions that are multiples of 16; of the last 16-byte
 * chunk of a row, elements past K are not used.  One row of A and of B takes less than 2^23 bytes, one
 * group's B less than 2 GiB, and an indexed A less than 2 GiB; scales of 128 x 128 blocks have a leading
 * dimension below 2^28, and a launch has fewer than 2^24 tiles.  Otherwise sizes are not limited.  C may
 * start at any element and have any leading dimension; every element is overwritten.  A plan with a workspace (a
 * split of K; hgemm_scaled_workspace_bytes()) runs on one stream at a time.
 */
typedef struct {
    hgemm_byte_t a;                  /* B is e4m3 */
    hgemm_type_t c;
    hgemm_scale_type_t scale;        /* of A and of B */
    int32_t b_block_rows;            /* rows of B that share a scale: 128 or 1 */
    hgemm_groups_t group;
    int32_t groups;                  /* 1 .. 1024; 0 with HGEMM_GROUPS_NONE */
    int64_t a_rows;                  /* ROWS: rows of an indexed A; 0 = not indexed */
    int64_t lda, ldb, ldc;           /* elements; 0 = packed (K rounded up to 16 for A and B) */
    int64_t ld_scale_a, ld_scale_b;  /* scales; 0 = packed */
} hgemm_scaled_t;

typedef struct hgemm_scaled_plan_s* hgemm_scaled_plan_t;

/* Chooses the kernel for one problem and allocates the plan's workspace, if any, on the current device.
 * Errors: INVALID_ARG, UNSUPPORTED (alignment, sizes), ALLOC, ARCH.                               */
hgemm_status_t hgemm_scaled_plan(hgemm_scaled_plan_t* out, int64_t M, int64_t N, int64_t K, const hgemm_scaled_t* desc);
/* As hgemm_plan_override: a kernel named by the caller ("tile,bm=128,bn=128", ...; hgemm_scaled_describe()
 * shows the form): "rows,bm=16|32,bn=16[,wv=]" (up to bm rows), "tile,bm=,bn=[,st=][,wv=][,gm=][,sk=]" or
 * "phased,bm=128|256,bn=128|256[,wv=][,gm=]" (K a multiple of 16); gm: rows of tiles that share columns of B in
 * a cache (0: the library chooses), sk: ranges that K is split into (without groups).  UNSUPPORTED if it cannot run the problem.     */
hgemm_status_t hgemm_scaled_plan_override(hgemm_scaled_plan_t* out, int64_t M, int64_t N, int64_t K,
                                          const hgemm_scaled_t* desc, const char* spec);
/* offsets: with groups only, else ignored; index: with a_rows > 0 only.
 * Errors: INVALID_ARG (null pointers, alignment of A, B and their scales), LAUNCH.                */
hgemm_status_t hgemm_scaled_run(hgemm_scaled_plan_t plan, const void* A, const void* scale_a, const void* B,
                                const void* scale_b, void* C, const int32_t* offsets, const int32_t* index, void* hip_stream);
hgemm_status_t hgemm_scaled_destroy(hgemm_scaled_plan_t plan);
size_t hgemm_scaled_workspace_bytes(hgemm_scaled_plan_t plan);
hgemm_status_t hgemm_scaled_describe(hgemm_scaled_plan_t plan, char* buf, size_t n);

/*
 * hgemm_quantise -- an M x K matrix X to 8-bit floats with block scales, in one pass.
 * For a block with the largest finite magnitude a' and a = max(a', 2^-96), largest = 448 or 57344:
 *   f32 scales   scale = a / largest,  q = X * (largest / a) rounded to nearest even (two fp32 roundings before it)
 *   e8m0 scales  scale = the smallest power of two with a / scale <= largest,  q = X / scale rounded to nearest even
 * NaN and infinities become NaN (e5m2: an infinity stays one) and do not enter the scale.
 *   Q, S     by rows of X: Q[M][ldq] with S[ceil(K / 128)][lds >= M], or, block_rows = 128,
 *            S[ceil(M / 128)][lds >= ceil(K / 128)]
 *   QT, ST   transposed, quantised along M: QT[K][ldqt] with ST[ceil(M / 128)][ldst >= K], or, block_rows = 128,
 *            ST[ceil(K / 128)][ldst >= ceil(M / 128)] (the same scales)
 * Either pair may be null (not both).  ldq and ldqt are multiples of 16; columns from K (M) up to the next
 * multiple of 16 are written as zeros.  ld 0 = packed (ldq, ldqt rounded up to 16).
 * With x_rows > 0 row m is row index[m] of an X of x_rows rows; an index outside [0, x_rows) is a row of zeros.
 * M is at most 16 * 65535.
 */
typedef struct {
    hgemm_type_t x;
    hgemm_byte_t q;
    hgemm_scale_type_t scale;
    int32_t block_rows;              /* 1 or 128 */
    int64_t M, K;
    int64_t x_rows;
    int64_t ldx, ldq, lds, ldqt, ldst;
} hgemm_quantise_t;

hgemm_status_t hgemm_quantise(const hgemm_quantise_t* desc, const void* X, const int32_t* index, void* Q, void* S,
                              void* QT, void* ST, void* hip_stream);

/*
 * hgemm_route_* -- the choice of k experts for each of `tokens` rows of logits, and the order of the rows.
 *   s = softmax(x) or sigmoid(x) in fp32;  key = s + bias (bias null: 0);  with softmax, no bias and
 *   top2 = 0 the keys are the logits themselves, which order the same.
 *   groups > 1: the experts form `groups` equal groups; a group scores its largest key, or the sum of its
 *   two largest (top2 = 1); the `keep` best groups stay.  The k largest keys are chosen, descending; equal keys
 *   and scores go to the lower index.  A logit or key that is -infinity or NaN is never chosen (a softmax over +infinity
 *   is NaN throughout).
 *   weights[t][j] = factor * s, or, renormalise = 1, factor * s / (sum of the chosen s + 1e-20).
 *   Slots without an expert hold expert -1 and weight 0.
 * The order of rows (offsets, rows and tokens; all three or none): rows by expert, within an expert by token.
 *   offsets[experts + 1]   first row of each expert, a multiple of `align`
 *   rows[tokens][k]        the row of each choice, -1 for none
 *   tokens_of[capacity]    the token of each row, -1 for rows of padding; capacity = tokens * k +
 *                          experts * (align - 1) rounded up to align (hgemm_route_capacity())
 * hgemm_route_backward: dlogits from dweights, given the logits and the choice (through the weights only: the
 * choice itself has no gradient); in the type of the logits.
 * A plan has a workspace and runs on one stream at a time.  Fewer than 2^26 tokens, at most 2^30 choices.
 * The time of the order grows with the square of the tokens from some 100000 on.
 */
typedef struct {
    int64_t tokens;
    int32_t experts, k;              /* 1 .. 1024 experts, 1 .. min(experts, 32) */
    hgemm_type_t logits;
    int64_t ld;                      /* of the logits and their gradient; 0 = experts */
    int32_t sigmoid;                 /* 0: softmax */
    int32_t groups, keep, top2;
    int32_t renormalise;
    float factor;
    int32_t align;                   /* 1 .. 1024 */
} hgemm_route_t;

typedef struct hgemm_route_plan_s* hgemm_route_plan_t;

hgemm_status_t hgemm_route_plan(hgemm_route_plan_t* out, const hgemm_route_t* desc);
hgemm_status_t hgemm_route_run(hgemm_route_plan_t plan, const void* logits, const float* bias, float* weights,
                               int32_t* experts, int32_t* offsets, int32_t* rows, int32_t* tokens_of, void* hip_stream);
hgemm_status_t hgemm_route_backward(hgemm_route_plan_t plan, const void* logits, const int32_t* experts,
                                    const float* dweights, void* dlogits, void* hip_stream);
hgemm_status_t hgemm_route_destroy(hgemm_route_plan_t plan);
int64_t hgemm_route_capacity(const hgemm_route_t* desc);

/*
 * hgemm_combine -- out[t] = sum over j of weights[t][j] * Y[rows[t][j]], in fp32 in the order of j; a row
 * outside [0, y_rows) adds nothing.  weights null: ones (the gradient of a gather of rows).
 * hgemm_combine_backward: dY[rows[t][j]] = weights[t][j] * dout[t], zero for rows r with tokens_of[r] < 0, and
 * dweights[t][j] = sum over n of dout[t][n] * Y[rows[t][j]][n] (0 for a row outside).  dY or dweights may be null.
 * dout and dY have the types of out and Y.
 */
typedef struct {
    int64_t tokens, N, y_rows;
    int32_t k;                       /* 1 .. 32 */
    hgemm_type_t y, out;
    int64_t ldy, ldo;                /* of Y and dY; of out and dout; 0 = N */
} hgemm_combine_t;

hgemm_status_t hgemm_combine(const hgemm_combine_t* desc, const int32_t* rows, const float* weights, const void* Y,
                             void* out, void* hip_stream);
hgemm_status_t hgemm_combine_backward(const hgemm_combine_t* desc, const int32_t* rows, const int32_t* tokens_of,
                                      const float* weights, const void* Y, const void* dout, void* dY,
                                      float* dweights, void* hip_stream);

/* ---- helpers (not on the hot path) --------------------------------------- */

/* Static, NUL-terminated description of a status code.                      */
const char* hgemm_status_string(hgemm_status_t status);

/* Writes the chosen specialisation as a spec string (same grammar as
 * hgemm_plan_override accepts) into buf[0..n), always NUL-terminated.
 * Returns INVALID_ARG when buf is NULL, n is 0, or the text does not fit.   */
hgemm_status_t hgemm_plan_describe(hgemm_plan_t plan, char* buf, size_t n);

/* Device workspace bytes owned by the plan (0 for single-pass kernels).     */
size_t hgemm_plan_workspace_bytes(hgemm_plan_t plan);

/* Number of workgroups of the plan's main kernel and its LDS bytes per
 * workgroup; for reports.  Either out pointer may be NULL.                  */
hgemm_status_t hgemm_plan_launch_info(hgemm_plan_t plan, int64_t* workgroups,
                                      int64_t* lds_bytes, int64_t* threads);

/* Static text listing the kernel families and the keys a spec may carry.    */
const char* hgemm_spec_help(void);

/* Candidate specs worth timing for a shape (the autotuner's search space,
 * seeded by the trends of Section 6: tiles grow with M and N, stages with K).
 * Fills buf with specs separated by '\n'; returns INVALID_ARG if it does not
 * fit.                                                                      */
hgemm_status_t hgemm_candidates(int64_t M, int64_t N, int64_t K,
                                const hgemm_layouts_t* layouts, char* buf, size_t n);

/* What hgemm_plan() would choose for a problem, and why, without a device
 * (host only; nothing is allocated or launched): buf receives one of
 *   "table: SPEC"      the row of the layout's dispatch table (Section 5: one
 *                      configuration per (M,N,K), here from timed runs)
 *   "neighbour: SPEC"  a large problem the table does not hold: the kernel
 *                      tuned for the nearest shape it does hold
 *   "model: SPEC"      the fitted cost model's pick, or with few rows of A
 *                      that of the nearest measured problem, or strips of
 *                      B for every compute unit;  "rules: SPEC"  its last
 *                      resort
 *   "blocks,rows=R,cols=C[,bt=1]"   operands of 2 GiB and more
 *   "generic"          unaligned and too small to pad;  "empty"  M, N or K = 0
 * with ",pad=1" appended when N, K or a leading dimension is not a multiple
 * of 8 (zero-padded copies, or with ",di=1" none).
 * hgemm_plan() then still has to set the choice up on the device; where that
 * fails (a kernel this build lacks, no memory) it falls back as documented
 * there.  Errors: INVALID_ARG (also when buf is too small), UNSUPPORTED.    */
hgemm_status_t hgemm_plan_choice(int64_t M, int64_t N, int64_t K,
                                 const hgemm_layouts_t* layouts, char* buf, size_t n);

/* The planner's cost model: predicted microseconds of one call of `spec` (an "mfma" spec without
 * tb/sm, or a "skinny" one without mr/ra) on an M x N x K problem.  hgemm_plan() picks the compiled configuration and split factor
 * with the smallest prediction when its measured table has no row for the shape (Section 6 reads
 * such trends -- tile size against M and N, stages against K -- off the paper's winners; here they
 * are a fitted model of one launch).  The model does not know the phased schedule: a spec with ph=1
 * counts like the best schedule of its tile that the model knows, and is not what the planner
 * weighs phased kernels by (it has a model of their own for problems of 3e10 flop and more).
 * Host only.  Errors: INVALID_ARG, UNSUPPORTED.                                                */
hgemm_status_t hgemm_predict_us(int64_t M, int64_t N, int64_t K, const char* spec, double* us);

/* Tile-count arithmetic of the zero-padding technique (Section 5.2): number
 * of tiles along a dimension of size `dim` with tile size `tile`, and the
 * padded size tiles*tile.  Out-of-range rows/columns are read as zeros and
 * never stored, so no tile size needs to divide the dimension.              */
int64_t hgemm_tiles(int64_t dim, int64_t tile);
int64_t hgemm_padded(int64_t dim, int64_t tile);

/* Tile -> workgroup mapping (Section 5.3 "block swizzle", Section 6.3),
 * re-thought for 8 XCDs with private L2 caches: maps the linear workgroup id
 * the hardware dispatches round-robin over XCDs to a (tile_m, tile_n) pair so
 * that the workgroups resident on one XCD cover a compact block of tiles.
 * Host-side mirror of the device function, exported for tests.
 * Returns tile_m * tiles_n + tile_n, or -1 for bad arguments.               */
int64_t hgemm_tile_of_workgroup(int64_t wg, int64_t tiles_m, int64_t tiles_n,
                                int64_t swizzle);

/* Calibration kernels for the roofline (not part of any GEMM): run `iters`
 * dependent-free MFMA instructions per wave on every CU / stream `bytes`
 * bytes from `src` (device pointer) and return the elapsed milliseconds
 * measured with events on `hip_stream`.  These two calls synchronise.       */
hgemm_status_t hgemm_calibrate_mfma(int64_t iters, void* hip_stream, double* ms, double* flop);
hgemm_status_t hgemm_calibrate_hbm_read(const void* src, size_t bytes, void* hip_stream, double* ms);

#ifdef __cplusplus
}
#endif
#endif /* HGEMM_H */
