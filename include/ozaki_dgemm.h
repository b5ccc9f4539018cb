/*
 * ozaki_dgemm.h -- C ABI of the MI355X (gfx950) Ozaki-scheme DGEMM library, libozaki.so.
 *
 * The library computes C = A B for FP64 matrices without any FP64 multiply-add in the product,
 * following "DGEMM without FP64 Arithmetic -- Using FP64 Emulation and FP8 Tensor Cores with
 * Ozaki Scheme" (D. Mukunoki): Section 3 (slicing, Eq. 1-8; error-free product expansion,
 * Eq. 9-11), Section 4.1 (FP8 E4M3 and FP16 slices with FP32 accumulation), Section 4.2 (FP64
 * addition emulated with integer instructions) and Section 4.3 (inner-product-wise and
 * outer-product-wise blocking).
 *
 * Conventions common to all entry points
 *   - One GPU, the current HIP device.  Every pointer documented as DEVICE must be device memory
 *     of that GPU; pointers documented as HOST are ordinary host memory.  The library never takes
 *     ownership of caller memory and never frees it.
 *   - Matrices are column-major (BLAS convention): element (i, j) of A is A[i + j*lda].
 *   - State (stream, workspace, profiling, last error) lives in a context.  Every host thread has a
 *     current context, initially the library's built-in default context; ozaki_context_use selects
 *     another one.  All calls below act on the calling thread's current context.  Two contexts with
 *     their own streams and workspaces are independent: their calls may be issued from two host
 *     threads, or interleaved from one, and run concurrently on the GPU.  One context is not
 *     thread-safe: one host thread drives it at a time, and two calls that share a workspace must
 *     be ordered on the same stream.
 *   - Work is enqueued on the context's stream (default: the null stream) and the calls return
 *     without waiting for the GPU unless stated otherwise.
 *   - Return value: 0 on success; a negative value -N means argument number N (1-based, in the
 *     order of the prototype) is invalid and nothing was launched; a positive value is one of the
 *     OZAKI_STATUS_* codes below.
 */
#ifndef OZAKI_DGEMM_H
#define OZAKI_DGEMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Type2 of the paper (Section 3): storage format of the slices = input format of the matrix unit. */
enum {
    OZAKI_SLICE_FP8_E4M3 = 0, /* OCP E4M3, 4 significand bits, FP32 accumulation (Section 4.1)        */
    OZAKI_SLICE_FP16 = 1,     /* IEEE binary16, 11 significand bits, FP32 accumulation (Section 4.1)  */
    OZAKI_SLICE_FP6_E2M3 = 2, /* OCP microscaling FP6 E2M3 (bias 1, no Inf/NaN): the 4 significand bits */
                              /* of E4M3, so the same slices and the same C as OZAKI_SLICE_FP8_E4M3,    */
                              /* on the twice as fast FP6 path of the matrix unit that Section 4.1      */
                              /* points to.  E2M3's smallest step is 1/8: a code holds twice the value  */
                              /* of Eq. 8, and the factor 1/4 per product is applied with the exponents */
    OZAKI_SLICE_FP6_E3M2 = 3, /* OCP microscaling FP6 E3M2 (bias 3), 3 significand bits: the FP6 column of    */
                              /* Table 2 (14 slices for a full FP64 significand); same FP6 matrix path        */
    OZAKI_SLICE_INT8 = 4      /* comparison path (the integer-matrix-unit variant of the scheme that Section 2 */
                              /* cites): slice entries are the integers q of Eq. 5-8 with |q| <= 2^6 stored as */
                              /* two's-complement bytes, products accumulate in INT32 (exact while             */
                              /* k_block * 4^b <= 2^31 - 1, which keeps b = 6 up to k_block = 524287)          */
};

/* How the slice-pair products are summed into FP64 (Section 3 after Eq. 11; Section 4.2). */
enum {
    OZAKI_ACCUM_FP64_HW = 0,      /* hardware FP64 additions                                            */
    OZAKI_ACCUM_FP64_INT_EMU = 1, /* FP64 additions emulated with 32/64-bit integer instructions only,  */
                                  /* round-to-nearest-even, bitwise equal to the hardware result        */
    OZAKI_ACCUM_EXACT_FIXED = 2   /* integer-only as well: the terms of a block are summed without any  */
                                  /* rounding in a 192-bit fixed-point integer per element (the sum of  */
                                  /* Eq. 10 free of rounding error, remark after Eq. 11) and rounded   */
                                  /* to FP64 once.  Unit: 2^-144 of the unit of the leading pair's      */
                                  /* product; a term whose scale lies further down is cut to that unit  */
                                  /* towards minus infinity.  Block sums are added to C with the        */
                                  /* emulated FP64 addition.  Not bitwise equal to the other two modes  */
                                  /* (fewer roundings).                                                 */
};

/* Which slice pairs (p, q) are multiplied. */
enum {
    OZAKI_PAIRS_TRIANGLE = 0, /* p + q <= s + 1: s(s+1)/2 products (terms below the last slice's weight are dropped)  */
    OZAKI_PAIRS_ALL = 1       /* all s * s products: the setting of the paper's Table 2 and Section 5.3              */
};

/* Where the FP64 roundings of the block sum happen (OZAKI_ACCUM_FP64_HW and _INT_EMU; Section 4 tunes the order of
 * the accumulation without giving it).  Either way the terms are visited anti-diagonal by anti-diagonal, p + q from
 * the largest (least significant) down to 2, p ascending inside one. */
enum {
    OZAKI_SUM_RUNS = 0,       /* consecutive terms of one anti-diagonal that carry the same power-of-two scale for an    */
                              /* element are summed exactly (matrix-unit accumulators, integer registers) and added      */
                              /* with ONE rounded FP64 addition: fewer roundings, less product traffic                   */
    OZAKI_SUM_PLAIN = 1       /* every term 2^(cA+cB) * product of Eq. 10 is added with its own rounded FP64 addition    */
};

enum {
    OZAKI_STATUS_OK = 0,
    OZAKI_STATUS_INFEASIBLE = 1,   /* no slice width b >= 0 keeps the accumulation of the matrix unit exact for this   */
                                   /* block length (condition after Eq. 8: k_block * 4^0 exceeds the exact window)      */
    OZAKI_STATUS_WORKSPACE = 3,    /* no workspace set, or it is smaller than ozaki_workspace_min_bytes    */
    OZAKI_STATUS_HIP_ERROR = 4,    /* a HIP runtime call failed; see ozaki_last_hip_error                  */
    OZAKI_STATUS_NONFINITE = 5,    /* reported by ozaki_last_device_status: A or B held an Inf or NaN      */
    OZAKI_STATUS_STATIC_LIMIT = 6, /* ozaki_dgemm_static: the problem needs more than OZAKI_STATIC_SCRATCH_BYTES */
    OZAKI_STATUS_SLICE_COUNT = 7,  /* num_slices is larger than OZAKI_MAX_SLICES                           */
    OZAKI_STATUS_TARGET = 8        /* reported by ozaki_last_device_status: a target of ozaki_linear_loss or    */
                                   /* ozaki_linear_loss_grad was neither a word of the vocabulary nor `ignore`  */
};

#define OZAKI_MAX_SLICES 32

/* ------------------------------------------------------------------------------------------------
 * Contexts
 * ---------------------------------------------------------------------------------------------- */
typedef struct ozaki_context_s* ozaki_context_t;

/* Creates a context (stream: null stream, no workspace, profiling off).  ctx_out: HOST. */
int ozaki_context_create(ozaki_context_t* ctx_out);
/* Destroys a context created by ozaki_context_create (releases its HIP events; never the caller's stream or
 * workspace).  If it is the calling thread's current context, the thread falls back to the default context.  It
 * must not be current in another thread, and its GPU work should have completed. */
int ozaki_context_destroy(ozaki_context_t ctx);
/* Makes ctx the calling host thread's current context; NULL selects the built-in default context. */
int ozaki_context_use(ozaki_context_t ctx);

/* Stream (a hipStream_t passed as void*; NULL = the null stream) used by all later calls of the current context. */
int ozaki_set_stream(void* hip_stream);

/*
 * ozaki_plan (host only, touches no GPU) -- the constants of Eq. 1-3 for one block length.
 *   k_block       length of the inner-product block the scheme is applied to (Section 4.3); >= 1
 *   slice_format  OZAKI_SLICE_*
 *   rho_out       HOST, may be NULL: rho = max(gamma, xi) of Eq. 3 with Type1 = FP64, Type3 = FP32 (INT32 for
 *                 OZAKI_SLICE_INT8)
 *   bits_out      HOST, may be NULL: b = 53 - rho, the magnitude bits of a slice entry: every entry is
 *                 q * 2^-b with integer |q| <= 2^b, and k_block * 4^b <= 2^24 keeps Eq. 11 exact
 * Returns 0, -1/-2 for invalid arguments, or OZAKI_STATUS_INFEASIBLE when rho > 53.
 */
int ozaki_plan(int64_t k_block, int slice_format, int* rho_out, int* bits_out);

/*
 * ozaki_dgemm -- C := A B by the Ozaki scheme (Section 3; blocking of Section 4.3).
 *   m, n, k       A is m x k, B is k x n, C is m x n; any non-negative sizes (internally zero-padded to
 *                 the tile sizes, which is exact).  m == 0 or n == 0: nothing is done.  k == 0: C := 0.
 *   A, lda        DEVICE, read-only, column-major, lda >= max(1, m)
 *   B, ldb        DEVICE, read-only, column-major, ldb >= max(1, k)
 *   C, ldc        DEVICE, written (every entry of the m x n matrix is overwritten), ldc >= max(1, m);
 *                 must not overlap A, B or the workspace
 *   slice_format  OZAKI_SLICE_*
 *   num_slices    s >= 1: number of slices taken from every row of A and every column of B (Eq. 4-8);
 *                 the slice pairs (p, q) with p + q <= s + 1 are multiplied (OZAKI_PAIRS_TRIANGLE) and summed
 *                 by the rule OZAKI_SUM_RUNS.  0 selects a data-independent default (ceil(61 / (b+1)) slices).
 *                 More than OZAKI_MAX_SLICES: OZAKI_STATUS_SLICE_COUNT.
 *   k_block       inner-product-wise block length (Section 4.3); 0 means k (no blocking).  A last,
 *                 shorter block is allowed.  Any length for which Eq. 1-3 leave b >= 0 is accepted; blocks of
 *                 more than 16384 elements are read two or three times for the slicing, and reserve 12 more bytes
 *                 of workspace per operand element (included in ozaki_workspace_bytes).
 *   accum_mode    OZAKI_ACCUM_*
 * The slices, exponents and slice-pair products live in the workspace (ozaki_set_workspace).
 * Inputs must be finite; an Inf/NaN raises a device flag readable with ozaki_last_device_status
 * and leaves C unspecified.  Results whose exponent leaves the normal FP64 range are unspecified in
 * the integer-only modes (the emulation omits overflow, underflow and subnormals, Section 4.2).
 */
int ozaki_dgemm(int64_t m, int64_t n, int64_t k,
                const double* A, int64_t lda, const double* B, int64_t ldb,
                double* C, int64_t ldc,
                int slice_format, int num_slices, int64_t k_block, int accum_mode);

/*
 * ozaki_dgemm_ex -- ozaki_dgemm with the pair set and the summation rule as arguments of their own.
 *   pair_set      OZAKI_PAIRS_*.  OZAKI_PAIRS_ALL with num_slices = the count of ozaki_count_slices is the paper's
 *                 error-free setting: the products then sum to the exact product (Eq. 9-10).
 *   sum_rule      OZAKI_SUM_* (ignored by OZAKI_ACCUM_EXACT_FIXED, whose sum has no intermediate rounding)
 *   mem_cap       0, or a cap in bytes on the part of the workspace the call may use: the call then works on
 *                 panels of rows of A and columns of B small enough for the cap (outer-product-wise blocking,
 *                 Section 4.3) and gives the same bits as the uncapped call, since rows of A and columns of B are
 *                 sliced independently of each other.  A cap below the need of one 256 x 256 panel:
 *                 OZAKI_STATUS_WORKSPACE.
 * ozaki_dgemm(...) is ozaki_dgemm_ex(..., OZAKI_PAIRS_TRIANGLE, OZAKI_SUM_RUNS, 0).
 */
int ozaki_dgemm_ex(int64_t m, int64_t n, int64_t k,
                   const double* A, int64_t lda, const double* B, int64_t ldb,
                   double* C, int64_t ldc,
                   int slice_format, int num_slices, int64_t k_block, int accum_mode,
                   int pair_set, int sum_rule, size_t mem_cap);

/*
 * ozaki_dgemm_static -- ozaki_dgemm for callers that cannot allocate device memory or hand over a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and
 * the same bits in C as ozaki_dgemm, but the slices, exponents and slice-pair products live in a fixed array of
 * OZAKI_STATIC_SCRATCH_BYTES bytes that is part of the library's device code (every GPU the library runs on holds
 * one copy from the first call until the process ends); the workspace of ozaki_set_workspace is neither needed nor
 * touched, and the call allocates and frees nothing.
 *   Limit: ozaki_workspace_min_bytes(m, n, k, slice_format, num_slices, k_block) must not exceed
 *   OZAKI_STATIC_SCRATCH_BYTES, else OZAKI_STATUS_STATIC_LIMIT is returned and nothing is launched (m = n = k = 256
 *   with 12 FP8 slices fits several times over, m = n = 600, k = 1000 with 11 slices just fits, m = n = k = 2048
 *   does not).
 *   Every call on a GPU uses that GPU's one array, which keeps what the previous call left: the kernels overwrite
 *   all they read, so nothing needs clearing between calls, but two calls that overlap in time on one GPU (two
 *   streams, two contexts, two host threads) race on it and give undefined results.  Enqueued on the current
 *   context's stream.  An Inf/NaN input is reported by ozaki_last_device_status as for ozaki_dgemm.
 */
#define OZAKI_STATIC_SCRATCH_BYTES (64u << 20)
int ozaki_dgemm_static(int64_t m, int64_t n, int64_t k,
                       const double* A, int64_t lda, const double* B, int64_t ldb,
                       double* C, int64_t ldc,
                       int slice_format, int num_slices, int64_t k_block, int accum_mode);

/*
 * ozaki_dgemm_scaled -- C := alpha (A B) + beta C, the GEMM of the BLAS that the paper emulates (Section 1), with
 * the FP64 multiplication of Section 4.2 beside the addition.
 *   alpha, beta   HOST values; zeros or normal numbers.
 *   The product P = A B is formed exactly as by ozaki_dgemm (same arguments, same bits), then every entry is
 *   combined as  C = fl(fl(alpha * P) + fl(beta * C))  -- one rounded multiplication per term and one rounded
 *   addition, no fused multiply-add; with beta == 0, C = fl(alpha * P) and the old C is not read (it may hold
 *   anything); with alpha == 1 and beta == 0 the call is ozaki_dgemm.  In the integer-only modes the
 *   multiplications and the addition are integer-only too (same bits; the old C must then hold zeros or
 *   normal numbers).  All other arguments as for ozaki_dgemm.
 *   The workspace must have ozaki_workspace_bytes_scaled bytes (ozaki_workspace_bytes plus the m x n product),
 *   or at least ozaki_workspace_min_bytes plus 8 m n rounded up to 256.
 * Returns as ozaki_dgemm; negative values count positions in THIS argument list.
 */
int ozaki_dgemm_scaled(int64_t m, int64_t n, int64_t k, double alpha,
                       const double* A, int64_t lda, const double* B, int64_t ldb,
                       double beta, double* C, int64_t ldc,
                       int slice_format, int num_slices, int64_t k_block, int accum_mode);
size_t ozaki_workspace_bytes_scaled(int64_t m, int64_t n, int64_t k, int slice_format, int num_slices, int64_t k_block);

/*
 * ozaki_suggest_k_block -- a block length for the inner dimension k (Section 4.3 leaves the choice to the user).
 * A heuristic from measurements on MI355X, not part of the method: FP8 / FP6 slices keep b = 4 up to k = 65536, so
 * they are blocked only above that (into blocks of 16384, the longest the fast slicing kernel takes); FP16 gains a
 * magnitude bit per factor 4 in the block length, and 4096 (b = 6) was the fastest block at k = 16384 (the paper
 * reports the same optimum on its GPU); INT8 keeps b = 6 up to 524287.  Returns the suggested k_block (0 = no
 * blocking), or a negative argument index.  HOST call.
 */
int64_t ozaki_suggest_k_block(int64_t k, int slice_format);

/*
 * Workspace (Section 5.1: work memory is allocated once, outside the timed region).
 *   ozaki_workspace_bytes      size that lets ozaki_dgemm keep all s(s+1)/2 pair products of one block
 *                              resident (capped at 160 GiB of products; more pairs are then processed in
 *                              several passes).  0 if the arguments are invalid or infeasible.
 *   ozaki_workspace_min_bytes  smallest size ozaki_dgemm accepts (the s products of the longest anti-diagonal
 *                              resident at a time).
 *   ozaki_workspace_bytes_ex   either of the two (minimum != 0: the smallest) for a pair set OZAKI_PAIRS_*.
 *   ozaki_set_workspace        dev_ptr: DEVICE memory, 256-byte aligned, owned by the caller, must stay
 *                              valid until replaced; bytes: its size.  (NULL, 0) clears it.
 */
size_t ozaki_workspace_bytes(int64_t m, int64_t n, int64_t k, int slice_format, int num_slices, int64_t k_block);
size_t ozaki_workspace_min_bytes(int64_t m, int64_t n, int64_t k, int slice_format, int num_slices, int64_t k_block);
size_t ozaki_workspace_bytes_ex(int64_t m, int64_t n, int64_t k, int slice_format, int num_slices, int64_t k_block,
                                int pair_set, int minimum);
int ozaki_set_workspace(void* dev_ptr, size_t bytes);

/* Waits for the stream, then returns OZAKI_STATUS_NONFINITE if a kernel since the last call of this
 * function met an Inf/NaN input, OZAKI_STATUS_TARGET if one met a target outside the vocabulary (the low-precision
 * operators below), OZAKI_STATUS_HIP_ERROR on a HIP failure, else 0.  A call reports one cause and clears that one: where both
 * were met, the next call returns OZAKI_STATUS_TARGET. */
int ozaki_last_device_status(void);
/* Numeric hipError_t of the most recent failed HIP call of the current context (0 if none). */
int ozaki_last_hip_error(void);
/* Static, NUL-terminated description of a return value of this library. */
const char* ozaki_status_string(int status);

/*
 * Per-phase GPU time.  ozaki_profile_enable(1) makes ozaki_dgemm bracket its kernels with HIP events
 * on the context's stream; ozaki_profile_read waits for the stream and returns, in HOST arrays of three
 * floats / three ints, the accumulated milliseconds and the number of kernel launches of the phases
 * [0] slicing (Eq. 4-8, includes the transposition of A), [1] slice-pair GEMMs (Eq. 10-11),
 * [2] accumulation and rescaling; then resets the counters.  Where a call forms products and sums in one pass, [1] is both
 * and [2] the launches that then find nothing to do.  ozaki_profile_enable(0) turns it off.
 * At most 4096 spans are kept between two reads (later ones are dropped), and nothing is recorded while the
 * stream is being captured into a HIP graph.
 */
int ozaki_profile_enable(int on);
int ozaki_profile_read(float* ms_out, int* launches_out);

/* ------------------------------------------------------------------------------------------------
 * Verification exports: the intermediate results the method defines, in plain layouts, for parity
 * checks against a reference implementation.  Not meant for timed use.  They use the workspace.
 * ---------------------------------------------------------------------------------------------- */

/*
 * ozaki_split -- Eq. 4-8 for one operand.
 *   is_B        0: X is A (rows x k, the vectors are the rows of A, ldx >= rows);
 *               1: X is B (k x rows, the vectors are the columns of B, ldx >= k)
 *   rows, k     number of vectors and their length
 *   X, ldx      DEVICE, column-major
 *   slices_out  DEVICE: T*s matrices in the order [block t][slice p], each `rows` vectors of
 *               kb_t = min(k_block, k - t*k_block) entries, vector-major (entry kk of vector r at
 *               r*kb_t + kk); 1 byte per entry (E4M3 code, E2M3 / E3M2 code in the low six bits, or the INT8
 *               integer) or 2 bytes (binary16 bits).  Blocks are packed back to back (block t starts after
 *               s*rows*kb_u entries of every earlier block u).
 *   exps_out    DEVICE: int32 [T][s][rows], the exponents c of Eq. 4 (32-bit for alignment's sake; every
 *               value fits 16 bits)
 */
int ozaki_split(int is_B, int64_t rows, int64_t k, const double* X, int64_t ldx,
                int slice_format, int num_slices, int64_t k_block,
                void* slices_out, int32_t* exps_out);

/*
 * ozaki_count_slices -- how many slices Eq. 4-8 extract from an operand until its remainder is zero (Section 3, the
 * paragraph before Eq. 4): the largest count over its vectors and k-blocks.  With that many slices (the larger
 * of the two operands' counts) and OZAKI_PAIRS_ALL the sum of the pair products is the exact product, which is
 * the error-free setting of the paper.
 *   is_B, rows, k, X, ldx, slice_format, k_block   as for ozaki_split
 *   count_out   HOST: the count; 0 for an all-zero operand; OZAKI_MAX_SLICES + 1 if OZAKI_MAX_SLICES slices do
 *               not exhaust it (ozaki_dgemm cannot run the error-free setting on it then)
 * Synchronises with the stream.  Workspace: 256 bytes, plus 8 * rows * k bytes (rounded up to 256) for A, plus 12
 * bytes per element of the (64-element padded) operand when the block is longer than 16384.
 */
int ozaki_count_slices(int is_B, int64_t rows, int64_t k, const double* X, int64_t ldx,
                       int slice_format, int64_t k_block, int* count_out);

/*
 * ozaki_pair_products -- the slice-pair products of Eq. 10-11, as the matrix unit produced them.
 *   pair_set    OZAKI_PAIRS_*
 *   chained     0: every pair is multiplied on its own (the kernel's run formation is switched off).
 *               1: run formation on: where all elements of a 32 x 32 tile share the scale of consecutive pairs of an
 *               anti-diagonal, the matrix unit keeps accumulating and ONE slot receives the exact sum of the run.
 *               Every anti-diagonal is cut into groups of floor(window / (k_block 4^b)) pairs (at least one), whose sum is
 *               inside the exact window (2^24; INT8: 2^31 - 1) whatever the data; a run ends with its group.
 *               2: the launch configuration of ozaki_dgemm with OZAKI_SUM_RUNS in this workspace, of its kernels that store
 *               products (where all exponents are regular ladders a call may form its sums without storing any).  Its groups are shorter
 *               where that is faster, and longer where the limit of 1 would cut the longest anti-diagonal into three
 *               groups or more (not for INT8): there the matrix unit sums on as long as the accumulators, together with
 *               a bound on every partial sum of the next pair, stay inside the window, so that the length of a run
 *               depends on the data.
 *   P_out       DEVICE: [T][pairs][n][m] 4-byte words: for block t and pair index z (pairs in accumulation order:
 *               anti-diagonals g = p+q from the largest down to 2, p ascending within one), an m x n column-major
 *               matrix (leading dimension m).  FP32 value sum_kk sliceA_p(i,kk) * sliceB_q(kk,j), the slices being
 *               the values of Eq. 8 (for FP6 the matrix unit's result times the exact factor 1/4); for
 *               OZAKI_SLICE_INT8 the INT32 integer sum_kk qA qB.  With chained != 0 the slot of a run's first pair
 *               holds the sum over the run and the other slots of the run hold 0.
 *   run_len_out DEVICE, may be NULL: uint8 [T][pairs][n][m]: how many consecutive pairs (starting with this one) the
 *               value in P_out sums; 0 where the pair is part of an earlier pair's run.  All 1 with chained == 0.
 */
int ozaki_pair_products(int64_t m, int64_t n, int64_t k,
                        const double* A, int64_t lda, const double* B, int64_t ldb,
                        int slice_format, int num_slices, int64_t k_block,
                        int pair_set, int chained, void* P_out, uint8_t* run_len_out);

/*
 * ozaki_fp64_add_emulated -- out[i] = a[i] + b[i] with the integer-only FP64 addition used by
 * OZAKI_ACCUM_FP64_INT_EMU (Section 4.2).  a, b, out: DEVICE arrays of n doubles (zeros and normal
 * numbers; out may alias a or b).
 */
int ozaki_fp64_add_emulated(const double* a, const double* b, double* out, int64_t n);

/* ------------------------------------------------------------------------------------------------
 * Low-precision operators for training and serving: FP8 with a scale for each block of 128, the product of
 * matrices in that form, and the cross entropy of a linear layer.
 *
 * A matrix of `rows` vectors is given by its first element, the distance ld between the starts of neighbouring vectors
 * (in elements) and its type; element e of vector i is X[i * ld + e].  (A row-major matrix's rows, or a column-major
 * one's columns.)  Vectors start at multiples of 16 bytes: pointers and ld * (bytes per element) are multiples of 16,
 * and the 16 bytes in which a vector ends may be read whole (what lies behind its end has no influence and is not written).
 * Results D, dH, dW may lie anywhere.  No size is above OZAKI_MAX_EXTENT, no vector longer than that many bytes or further from
 * its neighbour.  All pointers are DEVICE.
 * ---------------------------------------------------------------------------------------------- */
enum { OZAKI_TYPE_F32 = 0, OZAKI_TYPE_BF16 = 1, OZAKI_TYPE_F16 = 2 };

/* Which elements share a scale. */
enum {
    OZAKI_SCALE_VECTORS = 0, /* 128 neighbouring elements of a vector (activations, gradients)                   */
    OZAKI_SCALE_BLOCKS = 1   /* the same 128 elements of 128 neighbouring vectors (weights)                      */
};
#define OZAKI_SCALE_BLOCK 128
#define OZAKI_MAX_EXTENT (1 << 22)
#define OZAKI_MAX_QUANTISED (1LL << 34) /* rows * k of ozaki_quantise_fp8 (a launch has fewer than 2^32 threads)       */
#define OZAKI_MAX_LOGITS (1LL << 38)    /* tokens * vocab of ozaki_linear_loss and its gradient                       */

/* Quantises X (rows vectors of k elements of `type`) to OCP E4M3.  For each block, a being the largest finite magnitude in it
 * and at least 2^-100:
 *     scale = a / 448        code = E4M3(x * 448 / a), rounded once, to nearest, ties to even; NaN where x is not finite.
 *   Q, ldq    codes of X's vectors, one byte each; may be null (then so is S)
 *   S, lds    scales, S[(e / 128) * lds + i] for vector i, with OZAKI_SCALE_BLOCKS S[(e / 128) * lds + i / 128]; lds is at least
 *             the number of vectors or of blocks of vectors
 *   Qt, St    the same of the transpose of X, whose k vectors have `rows` elements; may be null
 * One of Q and Qt is there.  One read of X serves both. */
int ozaki_quantise_fp8(int64_t rows, int64_t k, const void* X, int64_t ldx, int type, int scaling, void* Q, int64_t ldq, float* S,
                       int64_t lds, void* Qt, int64_t ldqt, float* St, int64_t ldst);

/* D[i * ldd + j] = sum over b of Sa[b * ldsa + i] * Sb[..] * (sum over e of block b of A[i * lda + e] * B[j * ldb + e]), i < m, j < n:
 * A's vectors with OZAKI_SCALE_VECTORS, B's with `scaling_b`, as ozaki_quantise_fp8 leaves them.  Sums, and the products of two scales
 * (which have to lie in its range), in FP32; D of `type_d`, rounded once; with `accumulate` the sum is added to what D holds.  k == 0 gives zeros.
 * For a D of 32 bits every product A[i][e] * B[j][e] is exact.  For a D of 16 bits they are formed by the matrix unit's FP8 instructions, which
 * align the products of eight neighbouring elements to the largest of them and cut them 13 bits below its power of two: on normally distributed
 * codes 1.4e-5 of the result's norm, a hundredth of D's own rounding, but more than that where a sum nearly cancels.
 * Where few results leave compute units without work the inner dimension is cut and the shares meet in the context's
 * workspace: ozaki_gemm_fp8_workspace_bytes, 0 where none is needed.  The cut depends on m, n and k only. */
int ozaki_gemm_fp8(int64_t m, int64_t n, int64_t k, const void* A, int64_t lda, const float* Sa, int64_t ldsa, const void* B, int64_t ldb,
                   const float* Sb, int64_t ldsb, int scaling_b, void* D, int64_t ldd, int type_d, int accumulate);
size_t ozaki_gemm_fp8_workspace_bytes(int64_t m, int64_t n, int64_t k);

/* Softmax cross entropy of the outputs z = H W^T of a linear layer over a vocabulary, which are not kept:
 *     lse[t] = log(sum over v of exp(z[t][v]))          loss[t] = lse[t] - z[t][targets[t]], 0 where targets[t] == ignore
 * H: tokens vectors, W: vocab vectors of k elements, both of `type` (BF16 or F16); sums in FP32.  A target that is neither in
 * 0 .. vocab - 1 nor `ignore` gives a loss of NaN and raises OZAKI_STATUS_TARGET (ozaki_last_device_status).
 * Needs the context's workspace, ozaki_linear_loss_workspace_bytes(tokens, vocab, k, 0, 0). */
int ozaki_linear_loss(int64_t tokens, int64_t vocab, int64_t k, const void* H, int64_t ldh, const void* W, int64_t ldw, int type,
                      const int64_t* targets, int64_t ignore, float* loss, float* lse);

/* Its gradient, from the lse that the call above left and the gradient dloss[t] of whatever was made of the losses:
 *     g[t][v] = (exp(z[t][v] - lse[t]) - [v == targets[t]]) * dloss[t]      dH = g W      dW = g^T H
 * in the type of H and W; either result may be null.  Tokens with targets[t] == ignore (or an invalid target, which raises
 * OZAKI_STATUS_TARGET) have no share: their rows of dH are zeros, and what their rows of H hold does not matter.  g is formed a
 * piece of the vocabulary at a time, in 16 bits and without dloss; dW is formed with H times dloss[t] over the largest |dloss|, which is rounded to
 * 16 bits where the dloss of the tokens that count differ (dW's error is then about 1.4 times what it is with equal ones; in FP16, tokens of less
 * than 2^-19 of the largest lose more).  The piece follows from the workspace, of
 * ozaki_linear_loss_workspace_bytes(tokens, vocab, k, 1, minimum) bytes: minimum != 0 the least, 0 what is recommended.  With the
 * recommended size or more the result does not depend on the workspace. */
int ozaki_linear_loss_grad(int64_t tokens, int64_t vocab, int64_t k, const void* H, int64_t ldh, const void* W, int64_t ldw, int type,
                           const int64_t* targets, int64_t ignore, const float* lse, const float* dloss, void* dH, int64_t lddh, void* dW,
                           int64_t lddw);
size_t ozaki_linear_loss_workspace_bytes(int64_t tokens, int64_t vocab, int64_t k, int grad, int minimum);

/* ------------------------------------------------------------------------------------------------
 * A model's feed-forward block and its training step.  The same conventions as for the low-precision operators above: matrices of vectors,
 * inputs' vectors at multiples of 16 bytes (the 16 bytes in which one ends may be read whole), results anywhere, all pointers DEVICE unless
 * stated otherwise.  Inputs and results do not overlap unless it is said that they may.
 * ---------------------------------------------------------------------------------------------- */

/* act(z); GELU z * Phi(z) with the normal distribution's Phi, GELU_TANH z * (1 + tanh(sqrt(2/pi) * (z + 0.044715 z^3))) / 2, SILU z / (1 + exp(-z)) */
enum {
    OZAKI_ACTIVATION_NONE = 0, OZAKI_ACTIVATION_RELU = 1, OZAKI_ACTIVATION_GELU = 2, OZAKI_ACTIVATION_GELU_TANH = 3, OZAKI_ACTIVATION_SILU = 4
};
#define OZAKI_MAX_NORM 16384 /* elements of a row of ozaki_block_norm                                                 */

/* A linear layer with what follows it:     z = X W^T + bias          Y = act(z) + R
 * X: m vectors, W: n >= 1 vectors of k >= 1 elements of `type` (BF16 or F16), of which everything else is too; m * n, m * k and n * k are at most
 * OZAKI_MAX_LOGITS.
 *   bias      n elements; may be null
 *   R, ldr    m x n, may lie anywhere, may be Y with its ld; may be null
 *   Z, ldz    where z goes, for the gradient; may be null
 * Sums, activation and additions in FP32, from z that has not been rounded; one rounding of each result.  Where few results leave compute units without
 * work the inner dimension is cut and the shares meet in the context's workspace, ozaki_linear_workspace_bytes(m, n, k, 0); 0 where none is
 * needed.  The cut depends on m, n and k only. */
int ozaki_linear(int64_t m, int64_t n, int64_t k, const void* X, int64_t ldx, const void* W, int64_t ldw, int type, const void* bias, int activation,
                 const void* R, int64_t ldr, void* Y, int64_t ldy, void* Z, int64_t ldz);

/* Its gradient, from the gradient dY of Y (which is R's):
 *     dz = dY * act'(Z)          dX = dz W          dW = dz^T X          dbias[j] = sum over i of dz[i][j]
 *   Z, ldz    what ozaki_linear left, or anything else that dz is to be formed with; not read without an activation
 *   dX, dW    of `type`; dbias in 32 bits.  Each may be null, not all of them; X is read for dW, W for dX.
 * dz is formed once and rounded to `type` for the two products (without an activation it is dY; in FP16 magnitudes from 65520 on become infinite there); dbias is
 * summed in 32 bits from what has not been rounded.  Where few tiles leave compute units without work the sums over n or m are cut into shares; the cut depends on the sizes
 * and on which of dX and dW are asked for.  RELU's derivative at zero is zero.  m == 0 gives zeros in dW and dbias, and all results may be null then
 * (an empty dX is).  n is at most OZAKI_MAX_EXTENT / 2.  Needs the context's workspace, ozaki_linear_workspace_bytes(m, n, k, 1). */
int ozaki_linear_grad(int64_t m, int64_t n, int64_t k, const void* X, int64_t ldx, const void* W, int64_t ldw, int type, int activation, const void* Z,
                      int64_t ldz, const void* dY, int64_t lddy, void* dX, int64_t lddx, void* dW, int64_t lddw, float* dbias);
size_t ozaki_linear_workspace_bytes(int64_t m, int64_t n, int64_t k, int grad);

/* A pair of linear layers whose results are multiplied:     g = X Wg^T          u = X Wu^T          Y = act(g) * u
 * Wg and Wu: n vectors each, ldw apart (of one matrix that holds both: Wu = Wg + n * ldw elements).
 *   G, U      where g and u go, for the gradient; both may be null
 * Everything else as for ozaki_linear; workspace ozaki_gated_linear_workspace_bytes(m, n, k, 0). */
int ozaki_gated_linear(int64_t m, int64_t n, int64_t k, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw, int type, int activation,
                       void* Y, int64_t ldy, void* G, int64_t ldg, void* U, int64_t ldu);

/* Its gradient:
 *     dg = dY * U * act'(G)      du = dY * act(G)      dX = dg Wg + du Wu      dWg = dg^T X      dWu = du^T X
 * dg and du are formed once and rounded to `type`; dX is one sum of both terms.  Each result may be null, not all of them (dWg and dWu share lddw).  Everything else as for
 * ozaki_linear_grad; workspace ozaki_gated_linear_workspace_bytes(m, n, k, 1). */
int ozaki_gated_linear_grad(int64_t m, int64_t n, int64_t k, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw, int type,
                            int activation, const void* G, int64_t ldg, const void* U, int64_t ldu, const void* dY, int64_t lddy, void* dX,
                            int64_t lddx, void* dWg, void* dWu, int64_t lddw);
size_t ozaki_gated_linear_workspace_bytes(int64_t m, int64_t n, int64_t k, int grad);

/* What lies between two blocks of a model, for each of `rows` rows of k elements, 1 <= k <= OZAKI_MAX_NORM, with rho(v) = 1 / sqrt(mean(v^2) + eps):
 *     u = X * rho(X) * w_post   (w_post null: u = X)          the norm behind a block
 *     r = R + scale * gate * u                                its gate and scale, the sum that runs through the model
 *     H = r * rho(r) * w_pre                                  the norm in front of the next block
 *   X, H      of `type` (F32, BF16, F16); X null: nothing is added (r is R; R_out, w_post and gate are then null too, unless rows is 0: then
 *             nothing is done, and any address of rows may be null)
 *   w_post, w_pre      k elements in 32 bits
 *   gate, group        32 bits, rows i share row i / group of it: gate[(i / group) * k + e]; null: one
 *   R, R_out  of `type_r`, which is `type` or F32; R null: zeros.  R_out is r; may be null, may be R with its ld.
 *   H         may be null (then so may w_pre), not with R_out; may be X with its ld
 * Rounded once each: H is formed from the r that has not been rounded.  Sums in 32 bits; rows whose squares leave their range are normed all the same, as long as rho
 * itself is a number that 32 bits hold. */
int ozaki_block_norm(int64_t rows, int64_t k, const void* X, int64_t ldx, int type, const float* w_post, const float* gate, int64_t group, float scale,
                     float eps, const void* R, int64_t ldr, int type_r, void* R_out, int64_t ldro, const float* w_pre, void* H, int64_t ldh);

/* Its gradient, from those of H (dH, of `type`; null: none) and of R_out (dR_out, of `type_r`; null: none), with R_out here the r that the call above left:
 *     dR = dR_out + the gradient of r through H          dX = the gradient of X through scale * gate * u, from dR that has not been rounded
 *     dw_pre, dw_post (k elements), dgate (as gate), in 32 bits: sums over rows, in an order that depends on rows, k and group only
 * Each result may be null, not all of them; R_out and w_pre are read with dH (and only then); dw_pre asks for dH; dX, dw_post and dgate ask for X, dw_post for
 * w_post, dgate for gate.  dR may be dR_out, dX may be X or dH, each with its ld.  rows == 0 gives zeros in dw_pre and dw_post, and all
 * results may be null then.  For the sums over rows the call needs the context's workspace, ozaki_block_norm_workspace_bytes(rows, k, group) with group 0 without a gate. */
int ozaki_block_norm_grad(int64_t rows, int64_t k, const void* X, int64_t ldx, int type, const float* w_post, const float* gate, int64_t group,
                          float scale, float eps, const void* R_out, int64_t ldro, int type_r, const float* w_pre, const void* dH, int64_t lddh,
                          const void* dR_out, int64_t lddro, void* dX, int64_t lddx, void* dR, int64_t lddr, float* dw_post, float* dgate,
                          float* dw_pre);
size_t ozaki_block_norm_workspace_bytes(int64_t rows, int64_t k, int64_t group);

/* The norm of `count` tensors together:     *norm = |scale| * sqrt(sum over all elements of x^2)
 *   tensors, sizes, types      HOST: where each lies (DEVICE; aligned to its elements, no more), how many elements it has (at most 2^38, all of
 *                              them together at most 2^43), their type.  They are read before the call returns.  At most 2^27 tensors.
 *   scale                      what the elements are to be multiplied by (one over what the loss was multiplied by)
 *   norm                       DEVICE, one number in 32 bits; infinite or NaN where an element is
 * Squares of at most 33 elements are summed in 32 bits, those sums in twice as many; elements whose squares leave the range are no exception.  The order depends
 * on sizes, types and alignment only.  Needs the context's workspace,
 * ozaki_gradient_norm_workspace_bytes(count). */
int ozaki_gradient_norm(int count, const void* const* tensors, const int64_t* sizes, const int* types, float scale, float* norm);

/* The same, and the elements scaled so that the norm is at most max_norm:     out = x * scale * min(1, max_norm / *norm), rounded once
 *   out       HOST: where each tensor's results go (DEVICE, of its type); out[i] may be tensors[i]
 *   given     1: *norm is there already (that of all shares of a model, say) and read; 0: it is formed and written
 * A norm that is NaN makes every element NaN, one that is infinite makes finite ones zero: look at *norm before the results are used.
 * Workspace as above, none with `given`. */
int ozaki_clip_gradients(int count, const void* const* tensors, const int64_t* sizes, const int* types, float scale, float max_norm, void* const* out,
                         float* norm, int given);
size_t ozaki_gradient_norm_workspace_bytes(int64_t count);

#ifdef __cplusplus
}
#endif
#endif /* OZAKI_DGEMM_H */
