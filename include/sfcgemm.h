/*
 * sfcgemm.h -- C ABI of the MI355X (gfx950) space-filling-curve,
 * communication-avoiding bf16 GEMM.
 *
 * The operation is the GEMM of the paper's Section II.A, C = A * B with A of
 * M x K and B of K x N, executed as in Listing 1 (Section II.D): the M x N
 * output is cut into BM x BN blocks; the blocks are visited in generalized
 * Hilbert order (Section II.B); with ca_layers = c > 1 the contraction is
 * split into c contiguous K ranges, each computing a full copy of C, and the
 * copies are summed (Section II.C / II.D).  C is overwritten (Listing 1 zeroes
 * each block before the first contraction); there is no alpha or beta.
 *
 * Conventions for every entry point below
 *   - Matrices are row-major.  A[i][k] is at A[i*lda + k], B[k][j] at
 *     B[k*ldb + j], C[i][j] at C[i*ldc + j].  bf16 elements are 16-bit
 *     patterns (the upper half of an IEEE binary32).
 *   - A, B, C and workspace pointers are DEVICE pointers on the current HIP
 *     device; the caller owns them and keeps them alive until the work on
 *     `stream` has finished.  `stream` is a hipStream_t (NULL = null stream).
 *   - GEMM calls are asynchronous: they validate, enqueue kernels on `stream`
 *     and return.  Faults during execution surface at the next synchronisation.
 *   - On any error nothing is enqueued and C is not touched.
 *   - Elements of C outside the M x N region (ldc padding) are never written;
 *     elements of A and B outside their M x K and K x N regions are never used.
 *   - Accumulation is fp32 in every case.  For a fixed tile shape and layer
 *     count the result is bitwise reproducible and independent of the tile
 *     order and schedule.
 */
#ifndef SFCGEMM_H
#define SFCGEMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- return codes ------------------------------------------------------ */
#define SFC_OK               0
#define SFC_ERR_INVALID_ARG (-1) /* negative size, ld too small, null pointer, bad enum */
#define SFC_ERR_UNSUPPORTED (-2) /* misaligned element pointer, size beyond int32 tile indexing */
#define SFC_ERR_WORKSPACE   (-3) /* caller workspace smaller than sfc_gemm_ws_size() */
#define SFC_ERR_HIP         (-4) /* HIP runtime error; sfc_last_error() has the text */

/* ---- output element type (reading A8: fp32 accumulate, fp32 or bf16 out) */
#define SFC_OUT_F32  0           /* C holds float */
#define SFC_OUT_BF16 1           /* C holds bf16, rounded to nearest even */

/* ---- block (tile) shape BM x BN of the output grid --------------------- */
#define SFC_TILE_AUTO    0       /* chosen from M, N, K and ca_layers.  With one
                                    layer, 256-row blocks and a last round of
                                    blocks at most half full, the last block columns
                                    that make up that round are computed by a second
                                    launch (same stream) with 128-row blocks of the
                                    same width, which fill one round in about half
                                    the time; result bits are those of the single
                                    launch.  (fp8 operands: only where K is deep
                                    enough for that to pay.)  256x256 blocks with
                                    such a launch may also take the place of the
                                    128x256 blocks that sfc_gemm_model prefers.
                                    Small bf16 products and few rows with ca_layers
                                    SFC_CA_AUTO or 1 run on a kernel of 16-, 32- or
                                    64-row blocks, which are all in flight at once:
                                    order and sched are checked but mean nothing
                                    there (not with a caller's workspace and
                                    SFC_CA_AUTO: its layer copies are those of
                                    sfc_gemm_plan) */
#define SFC_TILE_128x128 1
#define SFC_TILE_256x128 2       /* BM = 256, BN = 128 */
#define SFC_TILE_128x256 3       /* BM = 128, BN = 256 */
#define SFC_TILE_256x256 4

/* ---- number of K layers (copies of C) ---------------------------------- */
#define SFC_CA_AUTO      0       /* ca_layers = 0: chosen with the block shape by the
                                    analytical model (Section III.B Eq. 1-4, used as in
                                    Section III.C's second option), among 1, 2, 4, 8, 16;
                                    small products and few rows on their own kernel take
                                    a count of their own, among the same */

/* ---- order of the output blocks ---------------------------------------- */
#define SFC_ORDER_HILBERT   0    /* generalized Hilbert curve (Section II.B) */
#define SFC_ORDER_ROW_MAJOR 1    /* plain row-major; for comparison only */

/* ---- how curve positions are dealt to the persistent workgroups --------- */
#define SFC_SCHED_INTERLEAVED 0  /* workgroup r takes positions r, r+P, ...: the blocks
                                    in flight form one contiguous curve segment, and each
                                    chiplet (XCD) owns a contiguous sub-segment of it */
#define SFC_SCHED_BLOCK       1  /* workgroup r takes the r-th contiguous range of
                                    positions (the block partition of Section III.A) */
#define SFC_SCHED_INTERLEAVED_PLAIN 2  /* as SFC_SCHED_INTERLEAVED with r = the
                                    hardware workgroup index, so consecutive positions
                                    go to different chiplets; for comparison only */

/*
 * sfc_tile_order -- the block order of a gm x gn grid (Section II.B; the map
 * built by create_sfc_map in Listing 1).
 *   gm, gn   grid sides (blocks along M and along N), both >= 1, gm*gn < 2^31.
 *   out_idx  HOST buffer of gm*gn int32, caller-owned.  On return out_idx[s]
 *            = im*gn + in for the block (im, in) visited at curve position s.
 * The table is produced on the current device by the same generator the GEMM
 * uses, then copied back; the call is synchronous.
 * Returns SFC_OK, SFC_ERR_INVALID_ARG (bad sides, NULL out_idx),
 * SFC_ERR_UNSUPPORTED (gm*gn too large) or SFC_ERR_HIP.
 */
int sfc_tile_order(int gm, int gn, int32_t *out_idx);

/* As sfc_tile_order, with an explicit SFC_ORDER_* mode. */
int sfc_tile_order_ex(int gm, int gn, int order, int32_t *out_idx);

/*
 * sfc_gemm -- C = A * B, fp32 output (Section II.A, Listing 1).
 *   M, N, K    >= 0.  M == 0 or N == 0: nothing to do, SFC_OK.  K == 0: C = 0.
 *   A, lda     bf16, M x K, lda >= K (A may be NULL when M*K == 0).
 *   B, ldb     bf16, K x N, ldb >= N (B may be NULL when K*N == 0).
 *   C, ldc     float, M x N, ldc >= N.
 *   ca_layers  c in [1, 64]: number of K ranges / copies of C.  The K blocks
 *              (64 deep) are split into min(c, ceil(K/64)) contiguous ranges,
 *              range l holding blocks [floor(l*nK/c), floor((l+1)*nK/c)).  For
 *              c > 1 the partial copies live in a workspace of
 *              sfc_gemm_ws_size() bytes that the library keeps per stream: it
 *              is allocated, and grown, in stream order (hipMallocAsync /
 *              hipFreeAsync on `stream`), and only work on that stream uses
 *              it, so calls on different streams may run concurrently.  It is
 *              kept, keyed by the stream handle, until the process ends.
 *              A call recorded into a graph uses the same layers, and so gives the
 *              same bits, as the call that runs at once; its copies and counters
 *              lie in memory that only recorded calls of that stream use and that
 *              is never freed, so replays may run on any stream and beside calls
 *              that run at once.  Replays of graphs that were recorded on one
 *              stream must not overlap each other.
 *              SFC_CA_AUTO (0): the library picks c (sfc_gemm_model's, or the
 *              small-block kernel's own: 13x1024x16384 takes 8 there, the model
 *              16).
 *   stream     hipStream_t or NULL.
 * No GEMM entry point synchronises the device or a stream.  The first call for
 * a block grid allocates its curve table (hipMalloc) and enqueues the
 * generator on `stream`; calls on other streams wait for it on the device.  A
 * call recorded into a graph before the table is complete has the generator in
 * the graph.
 */
int sfc_gemm(int64_t M, int64_t N, int64_t K,
             const void *A, int64_t lda,
             const void *B, int64_t ldb,
             void *C, int64_t ldc,
             int ca_layers, void *stream);

/* As sfc_gemm with a bf16 C (rounded to nearest even from the fp32 sums). */
int sfc_gemm_bf16out(int64_t M, int64_t N, int64_t K,
                     const void *A, int64_t lda,
                     const void *B, int64_t ldb,
                     void *C, int64_t ldc,
                     int ca_layers, void *stream);

/*
 * sfc_gemm_ws_size -- bytes of fp32 workspace that a ca_layers = c call needs
 * for the replicated C of Section II.C / II.D (Listing 1 keeps K_layers copies
 * of C, one per K range, and reduces them): c_eff dense M x N fp32 copies,
 * c_eff * M * N * 4 bytes with c_eff = min(c, ceil(K/64)) when c_eff > 1, else 0.
 * For c = SFC_CA_AUTO: the size for the largest count the model picks (16), a
 * bound that holds whatever it chooses.  Returns 0 for invalid arguments as well.
 */
size_t sfc_gemm_ws_size(int64_t M, int64_t N, int64_t K, int ca_layers);

/*
 * sfc_gemm_ex -- the general entry point behind sfc_gemm / sfc_gemm_bf16out.
 *   out_type   SFC_OUT_F32 or SFC_OUT_BF16.
 *   tile       SFC_TILE_*; order SFC_ORDER_*; sched SFC_SCHED_*.
 *   ws         device workspace of ws_bytes bytes, or NULL to use the library's
 *              internal one.  When c_eff > 1, layer l of the partial result is
 *              left in ws as a dense fp32 M x N matrix at ws + l*M*N floats.
 * Tile order and schedule never change the result bits; tile shape and layer
 * count change only the fp32 summation grouping.
 */
int sfc_gemm_ex(int64_t M, int64_t N, int64_t K,
                const void *A, int64_t lda,
                const void *B, int64_t ldb,
                void *C, int64_t ldc,
                int out_type, int ca_layers, int tile, int order, int sched,
                void *ws, size_t ws_bytes, void *stream);

/*
 * sfc_gemm_fused_ex -- sfc_gemm_ex with the reduction of the layer copies
 * fused into the GEMM launch (Listing 1's final add-reduce, Section II.D,
 * done by the GEMM's own workgroups): the workgroup that finishes a block's
 * layer copy publishes it (a release fence at device scope) and counts it on
 * the block's arrival counter (a device-scope atomic); the workgroup that
 * completes the count reads the c_eff copies of that block and sums them in
 * ascending layer order in fp32, so C is bit-identical to sfc_gemm_ex's.  No
 * workgroup waits for another.  One launch instead of two; the c_eff-way sum of
 * a block runs on one compute unit.  The counters are library memory kept per
 * stream (zero between launches; a call never leaves one raised), so `ws`, if
 * given, still needs only sfc_gemm_ws_size() bytes.  With c_eff = 1 this is
 * sfc_gemm_ex.  Arguments, errors and the contents left in ws as for
 * sfc_gemm_ex.
 */
int sfc_gemm_fused_ex(int64_t M, int64_t N, int64_t K,
                      const void *A, int64_t lda,
                      const void *B, int64_t ldb,
                      void *C, int64_t ldc,
                      int out_type, int ca_layers, int tile, int order, int sched,
                      void *ws, size_t ws_bytes, void *stream);

/*
 * sfc_gemm_noalloc_ex -- sfc_gemm_ex for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): the same kernels and results, bit for bit, with no
 * allocation and no synchronisation in the call.  Instead of the library's
 * per-stream workspace and cached curve tables it uses one static device
 * array per GPU, held until the process ends: SFC_NOALLOC_WS_BYTES of fp32
 * layer copies and two curve tables of SFC_NOALLOC_MAX_BLOCKS entries, which
 * every call that runs on the curve kernel rewrites on `stream` (a small kernel
 * before the GEMM); the small-block kernel's copies and counters lie there too.
 *   Arguments and errors as for sfc_gemm_ex without a workspace, plus:
 *   SFC_ERR_WORKSPACE   sfc_gemm_ws_size(M, N, K, ca_layers) exceeds
 *                       SFC_NOALLOC_WS_BYTES (checked before any HIP call);
 *   SFC_ERR_UNSUPPORTED the block grid has more than SFC_NOALLOC_MAX_BLOCKS
 *                       blocks.
 * Every call on a GPU uses that GPU's one array, whose contents are those the
 * last call left: calls that overlap on one GPU (on different streams, or
 * from different threads) race on it and must be ordered by the caller.  The
 * first call on a device looks up the array's address (hipGetSymbolAddress).
 */
#define SFC_NOALLOC_WS_BYTES   ((size_t)64 << 20)   /* 64 MiB of layer copies */
#define SFC_NOALLOC_MAX_BLOCKS (1 << 17)            /* blocks per curve table */
int sfc_gemm_noalloc_ex(int64_t M, int64_t N, int64_t K,
                        const void *A, int64_t lda,
                        const void *B, int64_t ldb,
                        void *C, int64_t ldc,
                        int out_type, int ca_layers, int tile, int order, int sched,
                        void *stream);

/*
 * sfc_gemm_f8_ex -- C = A * B with 8-bit float operands (the paper leaves the
 * data type a parameter of the method, Section III.A): A and B hold OCP FP8
 * E4M3 bytes (1 sign, 4 exponent bits with bias 7, 3 mantissa bits; no
 * infinities, 0x7F / 0xFF are NaN), row-major, lda and ldb in elements (=
 * bytes).  The products are exact in fp32 and the sums are fp32, as in
 * sfc_gemm_ex; C is fp32 or bf16 (out_type).  Same blocks-along-the-curve and
 * K-layer scheme, with K blocks 128 deep: ca_layers = c uses min(c,
 * ceil(K/128)) layers, whose workspace sfc_gemm_ws_size(M, N, K, c) bounds.
 * Restrictions (else SFC_ERR_UNSUPPORTED, nothing enqueued): A and B 16-byte
 * aligned, lda, ldb, K and N multiples of 16; tile SFC_TILE_AUTO,
 * SFC_TILE_256x256 or SFC_TILE_128x256.  SFC_TILE_AUTO and SFC_CA_AUTO pick the
 * free knobs with the model of sfc_gemm_model over those two block shapes,
 * evaluated on the bf16 problem with the same number of K blocks (K' =
 * 64*ceil(K/128)): a 128-deep fp8 block moves the bytes of a 64-deep bf16
 * block and takes the same MFMA time (ties go to 256x256); a half-height last
 * launch may then change 128x256 to 256x256 blocks (see SFC_TILE_AUTO).  K = 0
 * writes zeros for any N.  Other arguments and errors as for sfc_gemm_ex.
 */
int sfc_gemm_f8_ex(int64_t M, int64_t N, int64_t K,
                   const void *A, int64_t lda,
                   const void *B, int64_t ldb,
                   void *C, int64_t ldc,
                   int out_type, int ca_layers, int tile, int order, int sched,
                   void *ws, size_t ws_bytes, void *stream);

/* ---- 8-bit float formats --------------------------------------------------- */
#define SFC_FP8_E4M3 0   /* OCP E4M3: bias 7, 3 mantissa bits, no infinities, 0x7F/0xFF NaN */
#define SFC_FP8_E5M2 1   /* OCP E5M2: bias 15, 2 mantissa bits, 0x7C/0xFC = +-inf,
                            0x7D-0x7F/0xFD-0xFF NaN (the IEEE-style 8-bit format) */

/*
 * sfc_gemm_f8_fmt_ex -- sfc_gemm_f8_ex with the format of each operand chosen:
 * a_format and b_format are SFC_FP8_E4M3 or SFC_FP8_E5M2 (the two 8-bit float
 * formats of the same matrix instruction; mixed pairs allowed).  Every value of
 * either format is a bf16 value, so products are exact in fp32 as for E4M3.
 * Errors: SFC_ERR_INVALID_ARG for another format code, else as sfc_gemm_f8_ex.
 * sfc_gemm_f8_ex is this call with both formats SFC_FP8_E4M3.
 */
int sfc_gemm_f8_fmt_ex(int64_t M, int64_t N, int64_t K,
                       const void *A, int64_t lda,
                       const void *B, int64_t ldb,
                       void *C, int64_t ldc,
                       int out_type, int a_format, int b_format,
                       int ca_layers, int tile, int order, int sched,
                       void *ws, size_t ws_bytes, void *stream);

/*
 * sfc_gemm_plan -- what sfc_gemm_ex would launch, without launching
 * (fp32 output, 16-byte aligned operands).  ca_layers may be SFC_CA_AUTO and
 * tile SFC_TILE_AUTO; the plan then shows the choice of the curve kernel, for the
 * whole grid: the model's, or the 256x256 blocks that replace it together with a
 * half-height strip.  The strip itself is not shown, nor the small-block kernel
 * that SFC_TILE_AUTO uses for small products and few rows.
 *   plan[0] = BM, plan[1] = BN, plan[2] = gm, plan[3] = gn, plan[4] = c_eff,
 *   plan[5] = number of persistent workgroups, plan[6] = workgroups per CU.
 * Needs a device (it queries the CU count and kernel occupancy).
 */
int sfc_gemm_plan(int64_t M, int64_t N, int64_t K, int ca_layers, int tile, int64_t plan[7]);

/*
 * sfc_gemm_f8_plan -- what sfc_gemm_f8_ex (and sfc_gemm_f8_fmt_ex) would
 * launch, without launching (fp32 output); plan[] as for sfc_gemm_plan.  tile
 * is SFC_TILE_AUTO, SFC_TILE_128x256 or SFC_TILE_256x256, else
 * SFC_ERR_INVALID_ARG.  Needs a device.
 */
int sfc_gemm_f8_plan(int64_t M, int64_t N, int64_t K, int ca_layers, int tile, int64_t plan[7]);

/*
 * sfc_gemm_model -- the analytical model behind SFC_TILE_AUTO and SFC_CA_AUTO,
 * evaluated for given device parameters (host only: no device is touched).  Two
 * measured rules come after it: small products and few rows may run on the
 * small-block kernel, and 256x256 blocks with a half-height strip may replace
 * 128x256 blocks (see SFC_TILE_AUTO); both are outside this function.
 * The paper's fine-grained roofline (Section III.B, Eq. 1-4) on the GPU: a core
 * is a CU running `occupancy` persistent workgroups, one BRGEMM is one 64-deep
 * block of one task, at max(G*gamma, beta*(S_A + S_B)) with the panels of a
 * block shared by the tasks in flight on one XCD; the critical path is the
 * rounds of tasks times the blocks of the longest layer, plus the C traffic
 * (and, with layers, the copies written and read back) and the launches.
 * Every candidate (block shape x c in {1, 2, 4, 8, 16}, or only the fixed ones) is
 * evaluated and the fastest kept; near ties go to less padded work, then to
 * 256x256, 128x256, 256x128, 128x128 in that order, then to fewer layers.
 *   out_type   SFC_OUT_F32 or SFC_OUT_BF16 (bytes of C).
 *   ca_layers  SFC_CA_AUTO (0) or a fixed count in [1, 64].
 *   tile       SFC_TILE_AUTO or a fixed SFC_TILE_*.
 *   num_cus    compute units (>= 1).
 *   occupancy  host array: workgroups per CU of SFC_TILE_128x128, _256x128,
 *              _128x256, _256x256 (each >= 1).
 *   choice     host out: [0] SFC_TILE_* code, [1] effective layer count,
 *              [2] estimated shader clocks.
 * Returns SFC_OK or SFC_ERR_INVALID_ARG.
 */
int sfc_gemm_model(int64_t M, int64_t N, int64_t K, int out_type, int ca_layers, int tile, int num_cus,
                   const int32_t occupancy[4], int64_t choice[3]);

/*
 * sfc_probe_mfma -- measurement aid for the roofline (the counterpart of the
 * paper's compute micro-benchmark, Section III.B): register-only bf16 MFMA
 * 16x16x32 throughput (the GEMM kernel's instruction) of the current device,
 * 256 workgroups x 4 waves, each wave running `iterations` rounds of 64
 * independent MFMAs.
 *   random_operands  1: operands drawn at random (they change between MFMAs, as
 *                    in a GEMM); 0: constant operands.
 *   tflops, mhz      out: achieved TFLOP/s and the mean shader clock sampled
 *                    during the loop (MHz).  Host pointers.
 * Synchronous (null stream); allocates and frees a 257 KiB device buffer.
 * Returns SFC_OK, SFC_ERR_INVALID_ARG (iterations < 1, NULL outputs) or
 * SFC_ERR_HIP.
 */
int sfc_probe_mfma(int random_operands, int iterations, double *tflops, double *mhz);

/* ---- 4-bit operands ---------------------------------------------------------
 * A microscaled (OCP MX) 4-bit matrix of `rows` x `cols` values is two arrays:
 *   codes   E2M1 (1 sign, 2 exponent bits with bias 1, 1 mantissa bit: 0, 0.5, 1,
 *           1.5, 2, 3, 4, 6 and their negatives), two to a byte, the even column
 *           in the low bits; row i starts at byte i*ldq;
 *   scales  E8M0, one byte s for each 32 columns, the power 2^(s - 127), 255 = NaN
 *           (all 32 values are NaN); row i starts at byte i*lds.
 * Rows whose length is no multiple of 32 end in a block that is filled up with
 * zeros.  Rules for every call: codes 16-byte aligned, ldq a multiple of 16 and
 * >= 16*ceil(cols/32); scales 4-byte aligned, lds a multiple of 4 and >=
 * ceil(cols/32); both below 2^22.  The bytes of a row of scales up to the next
 * multiple of 4 may be read (the last row's too) but are never used or written.
 * Matrices that are not in 4 bits are row-major fp32 or bf16 (SFC_OUT_F32,
 * SFC_OUT_BF16) at element alignment, leading dimensions in elements.
 */

/*
 * sfc_mx4_quant -- a matrix to 4 bits, blocks along its rows (Q, S), along its
 * columns and transposed (Qt, St), or both; an output pair that is NULL is left out.
 *   X, ldx     rows x cols, in_type.
 *   order      NULL, or `rows` sorted slots as sfc_moe_sort writes them: row p is
 *              then X[order[p] / topk], X having x_rows rows, and a row of zeros
 *              where order[p] < 0 or that row does not exist.  (NULL: x_rows and topk
 *              are not used.)
 *   Q, S       rows x cols.    Qt, St   cols x rows.
 * Scale of a block: max(f - 2, 0), f the exponent field of the largest magnitude as
 * fp32, i.e. 2^(floor(log2 max) - 2), at least 2^-127; 255 if the block holds an
 * infinity or NaN.  Element: x over the scale rounded to the nearest E2M1 value,
 * ties to the even code, at most 6 in magnitude.  The codes of a block with scale
 * 255 are unspecified.
 */
int sfc_mx4_quant(int64_t rows, int64_t cols,
                  const void *X, int64_t ldx, int in_type,
                  const int32_t *order, int64_t x_rows, int topk,
                  void *Q, int64_t ldq, void *S, int64_t lds,
                  void *Qt, int64_t ldqt, void *St, int64_t ldst, void *stream);

/* sfc_mx4_dequant -- the values of a 4-bit matrix, rows x cols, as fp32 or bf16 (exact
 * but where a value exceeds the type: then infinity, rounded to nearest). */
int sfc_mx4_dequant(int64_t rows, int64_t cols,
                    const void *Q, int64_t ldq, const void *S, int64_t lds,
                    void *Y, int64_t ldy, int out_type, void *stream);

/*
 * sfc_gemm_mx4_ex -- C = A * B^T, A (M x K) and B (N x K) in 4 bits, both with their
 * blocks along K; C fp32 or bf16 (rounded to nearest even from the fp32 sums).
 *   K          a multiple of 32 (SFC_ERR_INVALID_ARG otherwise); K == 0: C = 0.
 * Products and block sums are exact, sums of blocks fp32.  Few rows run on kernels that
 * stream B once: up to 16 rows at any K (with A in registers while K <= 8192, or 16384 where N
 * is large), up to 32 while K <= 4096 and N < 2^28, up to 64 while K <= 4096 and
 * N <= 4096.  The others run on 256x256 or 128x128 blocks along the
 * curve, K in up to 16 layers where an estimate of the time favours it (copies in
 * library memory, as for sfc_gemm: replays of graphs recorded on one stream must then not
 * overlap each other, but with a workspace of their own).  The choice depends on M, N, K and
 * out_type alone, so equal calls give equal bits.
 * The gradients of C = A * B^T are two such calls: dA = dC * B with dC's blocks along N
 * and the transposed B (Qt of sfc_mx4_quant), dB = dC^T * A with both transposed.
 */
int sfc_gemm_mx4_ex(int64_t M, int64_t N, int64_t K,
                    const void *A, int64_t lda, const void *As, int64_t ldas,
                    const void *B, int64_t ldb, const void *Bs, int64_t ldbs,
                    void *C, int64_t ldc, int out_type, void *stream);

/*
 * sfc_gemm_mx4_ws_ex -- sfc_gemm_mx4_ex with its layer copies in the caller's workspace, so
 * that graphs with workspaces of their own may be replayed at once, wherever they were recorded.
 *   ws         NULL (library memory of the stream) or 16-byte aligned device memory of
 *              sfc_gemm_mx4_ws_size() bytes (SFC_ERR_WORKSPACE if ws_bytes is less); the call uses
 *              it until its work on `stream` has finished.
 * sfc_gemm_mx4_ws_size -- bytes that the call needs on the current device; 0 where it needs
 * none, the sizes are bad or there is no device.
 */
size_t sfc_gemm_mx4_ws_size(int64_t M, int64_t N, int64_t K, int out_type);
int sfc_gemm_mx4_ws_ex(int64_t M, int64_t N, int64_t K,
                       const void *A, int64_t lda, const void *As, int64_t ldas,
                       const void *B, int64_t ldb, const void *Bs, int64_t ldbs,
                       void *C, int64_t ldc, int out_type,
                       void *ws, size_t ws_bytes, void *stream);

/*
 * sfc_mx4_linear -- Y = X * W^T with X (M x K, fp32 or bf16) brought to 4 bits within the
 * call and W (N x K) kept in 4 bits.  K is the row length of X, W's rows hold
 * ceil(K/32) blocks; the result is that of sfc_mx4_quant and sfc_gemm_mx4_ex.  Up to 16
 * rows may be converted by the product's own launch; otherwise X's codes lie in library
 * memory, one per stream, as layer copies do: replays of graphs recorded on one stream must not
 * overlap each other, but with a workspace of their own.
 */
int sfc_mx4_linear(int64_t M, int64_t N, int64_t K,
                   const void *X, int64_t ldx, int in_type,
                   const void *W, int64_t ldw, const void *Ws, int64_t ldws,
                   void *Y, int64_t ldy, int out_type, void *stream);

/* sfc_mx4_linear_ws, sfc_mx4_linear_ws_size -- the same with X's codes, scales and the layer copies
 * in the caller's workspace, as for sfc_gemm_mx4_ws_ex. */
size_t sfc_mx4_linear_ws_size(int64_t M, int64_t N, int64_t K, int out_type);
int sfc_mx4_linear_ws(int64_t M, int64_t N, int64_t K,
                      const void *X, int64_t ldx, int in_type,
                      const void *W, int64_t ldw, const void *Ws, int64_t ldws,
                      void *Y, int64_t ldy, int out_type,
                      void *ws, size_t ws_bytes, void *stream);

/* ---- mixture of experts -------------------------------------------------------
 * A slot is one (token, choice) pair, slot = token*topk + choice.  Sorted rows belong to
 * slots: order[p] is the slot of row p (-1: none), pos[slot] its row (-1: dropped), and
 * rows offsets[e] .. offsets[e+1]-1 are expert e's.  All index arrays are int32 on
 * the device.  Indices that point outside their array count as none.
 */

/*
 * sfc_moe_sort -- slots sorted by expert, stable.
 *   ids        `slots` expert ids; an id outside 0 .. experts-1 drops the slot.
 *   align      every expert's rows start at a multiple of it (>= 1); the rows in between
 *              belong to no slot.
 *   rows       length of `order`, >= slots + experts*(align - 1).  offsets has
 *              experts + 1 entries, offsets[experts] being the rows in use (the rest of
 *              `order` is -1); pos has `slots`.
 *   ws         NULL (library memory of the stream, see sfc_mx4_linear for graphs) or
 *              sfc_moe_sort_ws_size() bytes.
 * At most 1024 experts.
 */
size_t sfc_moe_sort_ws_size(int64_t slots, int experts);
int sfc_moe_sort(int64_t slots, int experts, int align, const int32_t *ids,
                 int64_t rows, int32_t *offsets, int32_t *order, int32_t *pos,
                 void *ws, size_t ws_bytes, void *stream);

/*
 * sfc_moe_dispatch -- Xs[p] = w[order[p]] * X[order[p] / topk], a row of zeros where
 * order[p] < 0; X tokens x cols, Xs rows x cols, both of `type`; weights fp32 per slot,
 * or NULL: the rows as they are, bit for bit.
 */
int sfc_moe_dispatch(int64_t rows, int64_t cols, int64_t tokens, int topk,
                     const void *X, int64_t ldx, int type,
                     const int32_t *order, const float *weights,
                     void *Xs, int64_t ldxs, void *stream);

/*
 * sfc_moe_combine -- Y[t] = sum over j ascending of w[t, j] * Ys[pos[t, j]], in fp32,
 * dropped slots left out; Ys rows x cols, Y tokens x cols, both of `type`; weights
 * (tokens x topk, fp32) or NULL: 1.  Without weights this is the gradient of
 * sfc_moe_dispatch without weights.
 */
int sfc_moe_combine(int64_t tokens, int64_t cols, int64_t rows, int topk,
                    const void *Ys, int64_t ldys, int type,
                    const int32_t *pos, const float *weights,
                    void *Y, int64_t ldy, void *stream);

/*
 * sfc_moe_combine_grad -- the gradient of sfc_moe_combine: dYs[pos[t, j]] = w[t, j] * dY[t],
 * rows of no slot 0, and dW[t, j] = <dY[t], Ys[pos[t, j]]> (fp32, tokens x topk; 0 for a
 * dropped slot).  order and pos are those of one sfc_moe_sort.
 */
int sfc_moe_combine_grad(int64_t tokens, int64_t cols, int64_t rows, int topk,
                         const void *dY, int64_t lddy, const void *Ys, int64_t ldys, int type,
                         const int32_t *order, const int32_t *pos, const float *weights,
                         void *dYs, int64_t lddys, float *dW, void *stream);

/*
 * sfc_moe_gemm_mx4_ex -- C[p] = A[p] * B[e]^T for the rows p of every expert e; rows behind
 * the last segment are set to 0 (sfc_moe_sort's offsets start at 0; rows before a first
 * segment that starts later are not written).  A rows x K, B `experts` matrices of N x K that lie
 * stride_b (codes) and stride_bs (scales) bytes apart, multiples of 16 and 4; K a multiple
 * of 32.  The same call with the transposed weights gives the gradient of A.  The kernel
 * and its block shape are chosen from rows, N, K and experts; segment lengths are read
 * on the device.
 */
int sfc_moe_gemm_mx4_ex(int64_t rows, int64_t N, int64_t K, int experts,
                        const void *A, int64_t lda, const void *As, int64_t ldas,
                        const void *B, int64_t ldb, int64_t stride_b,
                        const void *Bs, int64_t ldbs, int64_t stride_bs,
                        const int32_t *offsets,
                        void *C, int64_t ldc, int out_type, void *stream);

/*
 * sfc_moe_wgrad_mx4_ex -- C[e] = A[:, seg] * B[:, seg]^T with seg = offsets[e] ..
 * offsets[e+1]-1, for every expert (zeros for one without rows): the weight gradient, A
 * being the transposed dY (M x rows) and B the transposed X (N x rows), both with their
 * blocks along the sorted rows.  Segments must start at multiples of 32
 * (sfc_moe_sort's align); a start that does not is taken down to one, and the end of the last
 * segment up to one, for 32 rows share a scale.  C[e] lies stride_c elements after C[e-1],
 * M x N, ldc; the experts' rows may lie in turn (stride_c < ldc) but not overlap.
 */
int sfc_moe_wgrad_mx4_ex(int64_t M, int64_t N, int64_t rows, int experts,
                         const void *A, int64_t lda, const void *As, int64_t ldas,
                         const void *B, int64_t ldb, const void *Bs, int64_t ldbs,
                         const int32_t *offsets,
                         void *C, int64_t ldc, int64_t stride_c, int out_type, void *stream);

/* ---- products of experts in bf16 ---------------------------------------------------
 * Operands are row-major bf16 at element alignment (16-byte aligned rows are fastest), sums fp32,
 * leading dimensions of operands in elements and below 2^22.  Weights W that act as C = A * W^T (N x K, as a
 * linear layer holds them) are SFC_B_NK; as C = A * W (K x N) SFC_B_KN.  What a product computes
 * with one of the two, its gradient computes with the other from the same memory.
 */
#define SFC_B_NK 0
#define SFC_B_KN 1

/*
 * sfc_moe_gemm_ex -- C[p] = A[p] * B[e]^T (SFC_B_NK) or A[p] * B[e] (SFC_B_KN) for the rows p of
 * every expert e; rows behind the last segment are set to 0 (rows before a first segment that starts
 * later are not written).
 *   A          rows x K; with `order` (rows slots, as sfc_moe_sort writes them) a_rows x K, and row p is
 *              A[order[p] / topk], or a row of zeros where order[p] < 0 or that row does not exist: the
 *              gather of sfc_moe_dispatch within the product.  It needs a_rows * lda < 2^31 - 2^11
 *              (SFC_ERR_UNSUPPORTED otherwise).  (order NULL: a_rows and topk are not used.)
 *   B          `experts` matrices, stride_b elements apart.
 *   offsets    experts + 1 segment bounds, on the device; bounds outside 0 .. rows count as the
 *              nearest of them.
 *   C          rows x N, out_type.
 * The gradient of A is the same call with the other layout.  The kernel and its block shape, and with them the order of
 * the sums, are chosen from rows, N, K, experts, b_layout, out_type, whether A, B, lda, ldb and stride_b make 16-byte
 * aligned rows, and the device's number of CUs: calls that are equal in these repeat their bits.
 */
int sfc_moe_gemm_ex(int64_t rows, int64_t N, int64_t K, int experts,
                    const void *A, int64_t lda, const int32_t *order, int64_t a_rows, int topk,
                    const void *B, int64_t ldb, int64_t stride_b, int b_layout,
                    const int32_t *offsets,
                    void *C, int64_t ldc, int out_type, void *stream);

/*
 * sfc_moe_wgrad_ex -- C[e] = A[seg]^T * B[seg] with seg = offsets[e] .. offsets[e+1]-1, for every
 * expert (zeros for one without rows): the weight gradient.  A rows x M and B rows x N, as they
 * lie: the gradient of SFC_B_NK weights with A = dC, B = A of sfc_moe_gemm_ex, that of
 * SFC_B_KN weights with the two exchanged.  C[e] lies stride_c elements after C[e-1],
 * M x N, ldc, out_type; the experts' rows may lie in turn (stride_c < ldc) but not overlap.
 */
int sfc_moe_wgrad_ex(int64_t M, int64_t N, int64_t rows, int experts,
                     const void *A, int64_t lda, const void *B, int64_t ldb,
                     const int32_t *offsets,
                     void *C, int64_t ldc, int64_t stride_c, int out_type, void *stream);

/* ---- low-rank adapters of many requests -------------------------------------------
 * Row t of a batch belongs to adapter a = ids[t] (int32, on the device; outside 0 .. adapters-1: to
 * none) and gets, beside what a shared projection of any type gave it,
 *     Y[t] = base[t] + V[t] * B[a]^T,   V[t] = scales[a] * X[t] * A[a]^T
 * with A[a] of rank x K and B[a] of N x rank, bf16, V fp32; ranks up to 256 (adapters of less are
 * filled up with zeros).  Rows in any order: runs of one adapter's rows (prompts) read its weights
 * least often.  A row sees its own adapter's weights only, so infinities and NaN stay with their adapter, and are
 * where the formulas have them, whatever the batch's size.
 * The gradients, with U[t] = scales[a] * dY[t] * B[a]: dBase = dY; dX = U[t] * A[a] (added to the shared
 * projection's); dA[a] = sum of U[t]^T X[t], dB[a] = sum of dY[t]^T V[t] over the adapter's rows t; all
 * of them calls below with the weights' other layout.  X, dY and weights at element alignment.
 */

/* sfc_lora_down -- V (rows x rank, fp32, ldv) as above from X (rows x K, bf16): A as rank x K (SFC_B_NK) or
 * K x rank (SFC_B_KN), stride_a elements from one adapter's to the next; scales NULL: 1; zeros in rows of no
 * adapter.  U is this call with X = dY and A = B, K x rank.  ldx and lda below 2^22.
 *   ws         NULL (library memory of the stream: replays of graphs recorded on one stream must then not
 *              overlap each other) or 16-byte aligned device memory of sfc_lora_down_ws_size() bytes
 *              (SFC_ERR_WORKSPACE if ws_bytes is less).
 * sfc_lora_down_ws_size -- bytes that the call needs on the current device; 0 where it needs none, the sizes
 * are bad or there is no device. */
size_t sfc_lora_down_ws_size(int64_t rows, int64_t K, int64_t rank, int adapters);
int sfc_lora_down(int64_t rows, int64_t K, int64_t rank, int adapters,
                  const void *X, int64_t ldx, const void *A, int64_t lda, int64_t stride_a, int layout,
                  const int32_t *ids, const float *scales,
                  float *V, int64_t ldv, void *ws, size_t ws_bytes, void *stream);

/* sfc_lora_up -- Y (rows x N, `type`) as above: B as N x rank (SFC_B_NK) or rank x N (SFC_B_KN); base rows x N
 * of Y's type, NULL: 0, or Y itself; rows of no adapter are base's.  V's products with B are fp32, rounded once
 * with base; bf16 Y: V may be taken to 16 bits (2^-16 of it), in any case to 2^-134. */
int sfc_lora_up(int64_t rows, int64_t N, int64_t rank, int adapters,
                const float *V, int64_t ldv, const void *B, int64_t ldb, int64_t stride_b, int layout,
                const int32_t *ids, const void *base, int64_t ld_base,
                void *Y, int64_t ldy, int type, void *stream);

/* sfc_lora_wgrad -- for every adapter G[a] = sum over t with ids[t] = a of Z[t]^T V[t], columns x rank
 * (SFC_B_NK), or of V[t]^T Z[t], rank x columns (SFC_B_KN): the gradient of sfc_lora_up's B in
 * its layout with Z = dY, that of sfc_lora_down's A in the other layout's name with V = U and Z = X (A of
 * rank x K: SFC_B_KN).  Zeros for an adapter without rows.  Z rows x columns, bf16; G out_type, stride_g
 * elements from one to the next, not overlapping.  Sums run over a fixed split of the rows: equal calls give
 * equal bits.
 *   ws         as for sfc_lora_down, of sfc_lora_wgrad_ws_size() bytes. */
size_t sfc_lora_wgrad_ws_size(int64_t rows, int64_t columns, int64_t rank, int adapters);
int sfc_lora_wgrad(int64_t rows, int64_t columns, int64_t rank, int adapters,
                   const void *Z, int64_t ldz, const float *V, int64_t ldv, const int32_t *ids,
                   void *G, int64_t ldg, int64_t stride_g, int layout, int out_type,
                   void *ws, size_t ws_bytes, void *stream);

/* Static text of a return code. */
const char *sfc_strerror(int code);

/* Text of the last error raised on the calling thread ("" if none). */
const char *sfc_last_error(void);

/* ABI version: 1. */
int sfc_version(void);

#ifdef __cplusplus
}
#endif

#endif /* SFCGEMM_H */
