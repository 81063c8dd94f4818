/* libspdp -- C ABI of the B200 (sm_100a) SPDP decode path.
 *
 * y = W_sp * (x masked by dynamic pruning): W_sp is an unstructured, statically pruned fp16
 * matrix held in the Tiled-CBC format (Sec. 4.1 of the paper), x is one token's fp16
 * activation vector, and columns whose activation fails the dynamic-pruning (DP) test are
 * never fetched from device memory (Sec. 4.2).
 *
 * Conventions that hold for every call
 *  - All tensor pointers named *_dev are CALLER-OWNED DEVICE memory on the device that was
 *    current when the handle was created; pointers named *_host are host memory.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *  - Every call returns an spdp_status; nothing throws; out-parameters are written only on
 *    SPDP_OK unless stated.  Host-detectable errors (null pointers, bad handle, unsupported
 *    shape) are returned before any work is enqueued.
 *  - A handle owns its packed arrays, its split-K workspace and a few staging buffers.  The
 *    workspace is per handle, so at most ONE spdp_spmspv per handle may be in flight; calls on
 *    one handle must be ordered (same stream, or events).  Different handles are independent.
 *    A call that was aborted, or that overlapped another call on the same handle, can leave a partial
 *    sum in the workspace; spdp_set_num_ctas (any value, also the current one) empties it again.
 *  - Format constants: column tile 256 x 1, GTile 256 x 16, four 64-bit bitmap words per column
 *    tile (Sec. 4.1); 16-byte padding of every column's values (Sec. 4.2.3).
 */
#ifndef SPDP_H_
#define SPDP_H_

#include <stdint.h>

#if defined(__GNUC__)
#define SPDP_API __attribute__((visibility("default")))
#else
#define SPDP_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef struct spdp_matrix* spdp_handle;   /* opaque; created by pack/import, released by spdp_free */

typedef enum {
    SPDP_OK = 0,
    SPDP_ERR_INVALID_ARG = -1,       /* null pointer, bad handle, bad enum, misaligned pointer */
    SPDP_ERR_UNSUPPORTED_SHAPE = -2, /* tile shape other than 256 x 16, M or K < 1, ldw < K      */
    SPDP_ERR_ALLOC = -3,             /* device or host allocation failed                        */
    SPDP_ERR_CUDA = -4,              /* a CUDA runtime call failed (see spdp_last_cuda_error)    */
    SPDP_ERR_OVERFLOW = -5,          /* Values would need 2^32 or more elements (TileOffset is 32-bit) */
    SPDP_ERR_TIMEOUT = -6            /* a bounded device-side wait expired (spdp_spmm; see spdp_last_device_status) */
} spdp_status;

/* Dynamic-pruning rule: which columns of W are fetched for this x (Sec. 2.2 "Dynamic Pruning",
 * W_dp(x) = W (.) M(x); Sec. 4.2 step (3): a magnitude metric of the activation against a
 * threshold calibrated offline, Sec. 5.1). */
typedef enum {
    SPDP_DP_NONE = 0,    /* every column is active                                              */
    SPDP_DP_ABS_GT = 1,  /* column j active iff NOT(|x_j| <= thr), compared in fp32 on the exactly
                            widened fp16 x_j: ties are skipped, thr = 0 skips exact zeros, thr < 0
                            keeps everything, NaN and +-Inf activations are active             */
    SPDP_DP_MASK = 2     /* explicit mask: bit (j % 32) of 32-bit word (j / 32) of mask_dev (Sec. 6:
                            DP variants that materialise a mask use the same column interface)  */
} spdp_dp_rule;

typedef enum { SPDP_Y_F16 = 0, SPDP_Y_F32 = 1 } spdp_ydtype;

/* Shape, sizes and device addresses of a packed matrix (all sizes in elements unless named bytes). */
typedef struct {
    int64_t M, K;              /* logical matrix shape                                          */
    int64_t R, C, NGT;         /* row tiles ceil(M/256), GTile columns ceil(K/16), R*C          */
    int64_t pad_elems;         /* every column's values are padded to a multiple of this (8 or 1) */
    int64_t nnz;               /* stored nonzeros                                               */
    int64_t values_len;        /* = TileOffset[NGT], padding included                           */
    int64_t packed_bytes;      /* bytes of TileOffset + ColInfo + Bitmap + Values               */
    int64_t workspace_bytes;   /* split-K scratch owned by the handle                           */
    /* The arrays lie inside cudaMalloc allocations, several in one: they may be read by a peer or exported to another process
     * (an exported handle stands for the whole allocation, whose start cuMemGetAddressRange tells), until the handle is freed. */
    const void* tileoffset_dev;  /* uint32[NGT+1]  start of each GTile in Values (elements)      */
    const void* colinfo_dev;     /* uint32[NGT*16] (column start inside its GTile) << 16 | nnz   */
    const void* bitmap_dev;      /* uint64[NGT*16*4] bit b of word w = row 64*w+b of the column tile */
    const void* values_dev;      /* fp16[values_len] nonzeros in tile-column order, zero padded  */
    int32_t num_ctas;          /* CTAs one spdp_spmspv launches                                 */
    int32_t device;            /* CUDA device ordinal the handle lives on                       */
} spdp_info;

/* Pack a dense, statically pruned matrix into Tiled-CBC (Sec. 4.1 "Storage Structure";
 * padding rule of Sec. 4.2.3).
 *   W_dev     fp16 [M][ldw] row-major, device; an element is "pruned" iff its value is +-0
 *             (bits & 0x7FFF == 0); every other bit pattern, NaN/Inf/subnormals included, is
 *             stored verbatim.
 *   M, K      >= 1; sides that are not multiples of 256 / 16 are zero-extended logically.  The matrix
 *             may hold at most 2^26 column tiles (ceil(M/256) * ceil(K/16) * 16), else
 *             SPDP_ERR_UNSUPPORTED_SHAPE.
 *   ldw       leading dimension in elements, >= K.
 *   tile_m, tile_k  must be 256 and 16 (the format's constants), else SPDP_ERR_UNSUPPORTED_SHAPE.
 *   out       receives the handle.  The call allocates device memory, runs on `stream` and
 *             synchronises it twice (packing is an offline step).  W_dev is not retained.
 * GTile (r, c) has linear index r*C + c; its 16 ColInfo words and 64 bitmap words are
 * contiguous; Values holds, per GTile and per column, the column's nonzeros in row order
 * followed by 0x0000 padding up to a multiple of 8 elements. */
SPDP_API spdp_status spdp_pack_tiled_cbc(const void* W_dev, int64_t M, int64_t K, int64_t ldw,
                                int tile_m, int tile_k, void* stream, spdp_handle* out);

/* Same as spdp_pack_tiled_cbc with the padding unit chosen: pad_elems = 8 (the format) or 1 (no
 * padding: the byte count then equals the storage formula of Sec. 4.1 exactly).  Handles packed
 * with pad_elems = 1 can be inspected, exported and unpacked; spdp_spmspv rejects them with
 * SPDP_ERR_UNSUPPORTED_SHAPE because its 16-byte loads need the padding. */
SPDP_API spdp_status spdp_pack_tiled_cbc_ex(const void* W_dev, int64_t M, int64_t K, int64_t ldw,
                                   int tile_m, int tile_k, int pad_elems, void* stream, spdp_handle* out);

/* Pack with a 4-bit Values payload (Sec. 5.1: 4-bit round-to-nearest weights, applied after static
 * pruning and before dynamic pruning; Sec. 6: Values are stored apart from the sparsity metadata, so
 * they can be low-bit).  The paper fixes no layout for it; this library's is: TileOffset, ColInfo and
 * Bitmap exactly as in Sec. 4.1, with offsets counted in CODES and every column padded to 32 codes
 * (16 bytes); Codes holds, per column tile, its n codes in row order, two per byte (even rank in the
 * low nibble), zero padded; Scales holds one fp16 per column tile (same index as ColInfo).
 *   scale = fp16(max|w| of the column tile / 7), computed in fp32;
 *   code  = clamp(rint(w / scale), -7, 7) + 8 in fp32, ties to even (8 where the scale is 0);
 *   the weight a code stands for is (code - 8) * scale.
 * Weights must be finite (codes of Inf/NaN are unspecified).  Arguments as spdp_pack_tiled_cbc.
 * The handle works with spdp_spmspv, spdp_spmspv_host, spdp_active_columns, spdp_get_info
 * (pad_elems = 32, values_len = number of codes), spdp_set_num_ctas and spdp_export_q4; the other
 * calls return SPDP_ERR_UNSUPPORTED_SHAPE for it.  spdp_spmspv on such a handle computes
 * y = sum over active columns of (code - 8) * scale * x_j with fp32 accumulation. */
SPDP_API spdp_status spdp_pack_tiled_cbc_q4(const void* W_dev, int64_t M, int64_t K, int64_t ldw, int tile_m,
                                   int tile_k, void* stream, spdp_handle* out);

/* Copy the arrays of a 4-bit handle to HOST buffers: tileoffset uint32[NGT+1], colinfo uint32[NGT*16],
 * bitmap uint64[NGT*64], codes uint8[values_len/2], scales fp16[NGT*16] (any pointer may be NULL).
 * Synchronous.  SPDP_ERR_INVALID_ARG for a handle that is not 4-bit. */
SPDP_API spdp_status spdp_export_q4(spdp_handle h, void* tileoffset_host, void* colinfo_host, void* bitmap_host,
                           void* codes_host, void* scales_host);

/* Build a handle from the four Tiled-CBC arrays in HOST memory (Sec. 4.1).  The arrays are
 * validated on the host (monotone TileOffset, ColInfo offsets equal to the prefix sums of the
 * padded counts, bitmap popcounts equal to the ColInfo counts); a mismatch returns
 * SPDP_ERR_INVALID_ARG.  The data is copied; the host arrays are not retained. */
SPDP_API spdp_status spdp_import_tiled_cbc(int64_t M, int64_t K, int pad_elems, const void* tileoffset_host,
                                  const void* colinfo_host, const void* bitmap_host,
                                  const void* values_host, int64_t values_len, spdp_handle* out);

/* y = W_sp * x over the active columns only (Sec. 4.2, Alg. 1; fp32 accumulation).
 *   x_dev     fp16 [K], device, 2-byte aligned.
 *   rule/thr  the DP rule; thr is used by SPDP_DP_ABS_GT only.
 *   mask_dev  uint32[ceil(K/32)], device; required for SPDP_DP_MASK, ignored otherwise.
 *   y_dev     [M] of ydt (fp16 rounded to nearest even from the fp32 sum, or fp32), device.
 *             Every one of the M entries is written, also when no column is active (zeros).
 * Asynchronous on `stream`; allocates nothing and never synchronises.  Launches one kernel.
 * The summation order is fixed for a given handle, so repeated calls give identical bits.
 * No CTA of the kernel ever waits for another one (the split-K combine is made of single atomic
 * exchanges), so there is nothing on the device that can time out; the handle's device status word,
 * readable with spdp_last_device_status, is reserved for device-side checks and stays 0. */
SPDP_API spdp_status spdp_spmspv(spdp_handle h, const void* x_dev, spdp_dp_rule rule, float thr,
                        const void* mask_dev, void* y_dev, spdp_ydtype ydt, void* stream);

/* Small-batch decode: Y[b] = W_sp * x_b for `batch` tokens (1..SPDP_MAX_BATCH) in one pass over
 * the packed matrix.  The paper treats one token per call and names batched DP decode as future
 * work (Sec. 6); this entry point applies its definition token by token: token b has its own
 * active set (the DP rule on x_b), a column tile is fetched once if ANY token keeps its column,
 * and a token that skips a column enters the product with 0 for it.  With finite weights that is
 * the omission of the column; a column tile that holds Inf or NaN and is fetched for another token
 * gives NaN instead (0 * Inf).  Likewise a NaN or Inf activation of a kept column reaches, through the
 * zeros of the fetched tiles, every row (0 * NaN), as in a dense product; the single-vector call
 * multiplies stored nonzeros only.
 *   x_dev        fp16 [batch][ldx], device, ldx >= K elements between tokens.
 *   mask_dev     uint32 [batch][mask_stride] words, mask_stride >= ceil(K/32); SPDP_DP_MASK only.
 *   y_dev        [batch][ldy] of ydt, ldy >= M elements between tokens; all batch*M entries are written.
 * Asynchronous on `stream`, allocates nothing; launches one kernel for 3 or more tokens and one
 * single-vector kernel per token below that (which is faster there).  The handle's workspaces allow
 * one such call in flight per handle.  Results are identical from call to call. */
#define SPDP_MAX_BATCH 8
SPDP_API spdp_status spdp_spmspv_batch(spdp_handle h, const void* x_dev, int64_t ldx, int batch, spdp_dp_rule rule,
                              float thr, const void* mask_dev, int64_t mask_stride, void* y_dev, int64_t ldy,
                              spdp_ydtype ydt, void* stream);

/* Prefill product on the same packed handle (Sec. 4.3, SPDP-SpMM): Y[n] = W_sp * X[n] for N tokens,
 * static pruning only (no dynamic pruning: every column is fetched once per block of tokens).
 * The column tiles are decoded from Tiled-CBC into dense fp16 operand tiles in shared memory (what
 * the paper's layout-alignment stage does for its tensor-core path), the contraction runs on the
 * 5th-generation tensor cores (tcgen05.mma, fp16 inputs, fp32 accumulation in tensor memory).
 *   X_dev   fp16 [N][ldx], device, one token per row, ldx >= K elements between tokens; X_dev must
 *           be 16-byte aligned and ldx a multiple of 8 (the tiles are read through a tensor map,
 *           encoded on the host at every call), else SPDP_ERR_INVALID_ARG.
 *   N       >= 1 tokens.
 *   Y_dev   [N][ldy] of ydt, device, ldy >= M elements between tokens; all N*M entries are written.
 * Asynchronous on `stream`; one to three kernels.  A tile of the result (256 rows x 32 to 512 tokens) is one CTA's
 * work, or a pair's.  Where whole tiles would leave SMs idle, which is the rule for short prompts and small
 * layers, the tiles that do not fill a round (often all of them) are cut along K: several CTAs leave fp32 partial
 * sums of a tile in scratch memory, and they (as a thread-block cluster) or a further kernel add them in a fixed order.  Which tiles are
 * cut follows from M, K, N, ydt and the device alone (its SMs and the clusters that it holds at once), so repeated calls give identical bits.
 * 32-bit results are added up in shorter pieces where the fastest cut would make them less exact.
 *   The scratch memory, up to 77 MB on 148 SMs, comes from a stream-ordered pool of the library's (cudaMallocFromPoolAsync /
 * cudaFreeAsync on `stream`; in a stream capture it becomes memory of the graph).  The pool keeps up to 96 MB until the
 * device's last handle is freed; spdp_free(NULL) gives back what is unused.  Where there is no memory for it the call
 * cuts nothing: slower, and the sums in another order.
 *   The handle's workspace is never touched, so calls on one handle may overlap.
 *   The waits inside the kernels (on shared-memory barriers that the copies and the tensor cores complete) are
 * bounded.  One that runs out records SPDP_ERR_TIMEOUT in the handle's status word, and the rows and tokens that the CTA
 * would have written, or left partial sums of, stay unwritten; TileOffset words that do not describe a K-block that fits
 * shared memory record SPDP_ERR_OVERFLOW the same way.  A status other than 0 therefore means that Y is incomplete.
 * SPDP_ERR_CUDA if the driver's tensor-map encoder cannot be found. */
SPDP_API spdp_status spdp_spmm(spdp_handle h, const void* X_dev, int64_t N, int64_t ldx, void* Y_dev, int64_t ldy,
                      spdp_ydtype ydt, void* stream);

/* Same product with HOST vectors (Sec. 4.2): brings x_host (fp16 [K], ideally pinned) to a
 * staging buffer of the handle, runs spdp_spmspv, leaves y in y_host ([M] of ydt) and
 * synchronises `stream`.  mask_host is uint32[ceil(K/32)] or NULL.  The buffers may start at any byte.  Where
 * all of them lie in page-locked memory (each in one allocation or registration) and on a multiple of their element's size,
 * the kernels read and write them directly; else they are copied before and after the kernel. */
SPDP_API spdp_status spdp_spmspv_host(spdp_handle h, const void* x_host, spdp_dp_rule rule, float thr,
                             const void* mask_host, void* y_host, spdp_ydtype ydt, void* stream);

/* The same product for callers that must not allocate (the paper has no counterpart: this entry
 * point exists for the library's users, not for the method).  Some hosts of this code cannot
 * call cudaMalloc at all: a serving process that hands all device memory to its own arena at
 * start-up, an embedding that forbids driver allocations after initialisation, a caller that
 * already holds the four Tiled-CBC arrays in memory it manages.  For them nothing here creates a
 * handle; the caller passes the packed arrays (device pointers, laid out as spdp_info describes,
 * 16-byte column padding), x, the DP rule and y, exactly as for spdp_spmspv.
 *
 * What spdp_spmspv keeps in a handle-owned allocation (the split-K partial sums that CTAs
 * exchange) lives in ONE fixed device array inside the library, about 0.5 MB, present on every
 * GPU that loads the library until the process exits.  It bounds the launch to 512 CTAs (the
 * library never asks for more); shapes beyond the library's general limit (2^26 column tiles)
 * return SPDP_ERR_UNSUPPORTED_SHAPE.  The call enqueues a small set-up kernel (which empties the
 * part of the array this call uses, whatever an earlier call left there) and the spMspV kernel
 * on `stream`; it calls no cudaMalloc, cudaFree or allocating library routine.
 *
 * The first call on each device looks up the array's device address (cudaGetSymbolAddress, with
 * that device current) and the SM count; make that first call outside any stream capture.
 * Every call on a device shares the one array: two calls that can overlap on the GPU (different
 * streams without ordering, or two host threads) race on it and give wrong sums; order them.
 * Results equal spdp_spmspv's for the same CTA count. */
SPDP_API spdp_status spdp_spmspv_noalloc(const void* tileoffset_dev, const void* colinfo_dev,
                                const void* bitmap_dev, const void* values_dev, int64_t M, int64_t K,
                                const void* x_dev, spdp_dp_rule rule, float thr, const void* mask_dev,
                                void* y_dev, spdp_ydtype ydt, void* stream);

/* Producer-fused dynamic pruning (Sec. 6: DP variants that materialise a mask map to the same column
 * interface; Sec. 4.2 step (3): a magnitude test against a threshold calibrated offline).  The input of
 * a gated MLP's down-projection is x = silu(gate) * up; this call computes it (fp32 arithmetic, one
 * rounding to fp16) and writes, in the same pass, the mask of the columns the following spdp_spmspv
 * should keep: bit (j % 32) of word (j / 32) is NOT(|x_j| <= thr) evaluated on the STORED fp16 x_j, i.e.
 * exactly the set SPDP_DP_ABS_GT would choose.  Pass the mask with SPDP_DP_MASK.  A caller with
 * another per-column score (say |x_j| times a column norm) gets its mask from spdp_active_columns on
 * the score vector and uses SPDP_DP_MASK in the same way.
 *   gate_dev, up_dev  fp16 [K], device.     x_dev_out  fp16 [K], device.
 *   mask_dev_out      uint32[ceil(K/32)], device (bits beyond K clear).
 *   count_dev_out     int32[1], device, or NULL: number of kept columns.
 * Asynchronous on `stream`; allocates nothing. */
SPDP_API spdp_status spdp_swiglu_dp(const void* gate_dev, const void* up_dev, int64_t K, float thr, void* x_dev_out,
                           void* mask_dev_out, void* count_dev_out, void* stream);

/* ---- around the projections of a decoder layer ------------------------------------------------------------
 * The calls of this part take no handle: they run on the current device, which must hold every *_dev pointer, are asynchronous
 * on `stream`, may be captured, and give the same bits for the same arguments.  Two of them take scratch memory, stream-ordered from
 * the pool that spdp_spmm describes (SPDP_ERR_ALLOC where there is none); each call has its own.  Calls with different outputs may
 * overlap.  An output may not overlap an input unless the call says so. */

/* Low-rank adapters of many requests beside a shared projection: Y[n] = base[n] + scale_a * B_a * (A_a * X[n]) with
 * a = adapter[n] (the paper has no adapters; merging B A into a statically pruned W would fill its zeros, so the adapters of a
 * packed layer stay beside it).  X is what spdp_spmspv, spdp_spmspv_batch or spdp_spmm got for the same tokens, base what it
 * wrote; dynamic pruning does not apply to the adapter's own product.
 *   X_dev        fp16 [N][ldx], ldx >= K, N <= 2^24.
 *   adapter_dev  int32 [N]; a value outside 0 .. count-1 means no adapter: Y[n] = base[n], bit for bit.
 *   A_dev, B_dev fp16 [count][rank][K] and [count][M][rank]: row strides lda >= K and ldb >= rank, adapters
 *                stride_a and stride_b apart (in elements): one after another, row between row, or (0) one A or B for all.
 *                1 <= rank <= SPDP_MAX_RANK.
 *   ranks_dev    int32 [count] or NULL: adapter a has only its first ranks[a] rows of A and columns of B; the others
 *                do not count, whatever they hold.  Values outside 0 .. rank are taken as the nearest of these.
 *   scales_dev   float [count] or NULL (1).
 *   base_dev     [N][ldbase] of ydt, ldbase >= M; may be Y_dev itself (with ldbase = ldy): the adapters are then added in place.
 *   Y_dev        [N][ldy] of ydt, ldy >= M.
 * Sums in 32 bits; the vector between the two products is rounded to 11 bits for 16-bit results and to 22 for 32-bit ones (below 2^-28
 * and 2^-17 of a token's largest to fewer, within 2^-39 of that), with the range of 32-bit numbers.  The tokens of an adapter need
 * not stand together.  The fast case: rows that start on 16-byte boundaries (addresses and strides), K, M and rank multiples of 8.
 * Launches one kernel for up to 16 tokens in the fast case and else two, with scratch memory: for each token 4 bytes and 2 (with 32-bit
 * results 4) times the rank rounded up to a multiple of 32; for each started 256 tokens 2432 bytes; 255 bytes at most between. */
#define SPDP_MAX_RANK 256
SPDP_API spdp_status spdp_lora(const void* X_dev, int64_t N, int64_t K, int64_t ldx, const void* adapter_dev, const void* A_dev, int64_t lda,
                      int64_t stride_a, const void* B_dev, int64_t ldb, int64_t stride_b, int64_t count, int rank, const void* ranks_dev,
                      const void* scales_dev, const void* base_dev, int64_t ldbase, void* Y_dev, int64_t M, int64_t ldy, spdp_ydtype ydt,
                      void* stream);

/* Norms of the query and key heads and their rotation by positions, in one pass over the output of the q/k projections.
 * Each head x of head_dim values becomes x / sqrt(mean(x^2) + eps) * weight, then its first 2 * pairs values turn: pair i by the
 * angle pos[axis of i][n] * inv_freq[i], (a, b) -> (a cos - b sin, b cos + a sin); values that do not turn stay.  Arithmetic in 32
 * bits, angles in 64, one rounding to fp16.  (A normed head's sum of squares, and their mean plus eps, have to be in the range of 32-bit
 * numbers: a concern for 32-bit rows beyond 10^18, and for heads of zeros or below 10^-18 with an eps of 0.)
 *   q_dev, k_dev      [N][ldq], [N][ldk] of dt (fp16 or fp32, a projection's output types), N <= 2^24: a token's q_heads
 *                     (kv_heads) heads one after another.  Either number may be 0 (its pointers are then ignored), not both.
 *   head_dim          even, 2 .. 256.
 *   q_weight_dev, k_weight_dev  fp16 [head_dim], or NULL: those heads are not normed.
 *   pos_dev           int32 [axes][pos_stride], pos_stride >= N: a token's position on each axis (1 axis for text; time, height
 *                     and width for video).  1 <= axes <= 4.
 *   sections          HOST int [axes]: the first sections[0] pairs turn by axis 0, the next sections[1] by axis 1, ...; their
 *                     sum is `pairs`.
 *   inv_freq_dev      float [pairs], radians per position (whatever scaling of the frequencies is in use is in them).
 *   pairs             0 .. head_dim / 2; 0: no rotation (pos, axes, sections and inv_freq are ignored).
 *   adjacent          0: pair i is (x[i], x[i + pairs]); 1: (x[2 i], x[2 i + 1]).
 *   q_out_dev, k_out_dev  fp16, as q_dev and k_dev; they may be those themselves (same pointer and stride) where dt is fp16.
 * Launches one kernel. */
SPDP_API spdp_status spdp_qk_norm_rope(const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk, spdp_ydtype dt, int64_t N, int q_heads, int kv_heads,
                              int head_dim, const void* q_weight_dev, const void* k_weight_dev, float eps, const void* pos_dev, int64_t pos_stride,
                              int axes, const int* sections, const void* inv_freq_dev, int pairs, int adjacent, void* q_out_dev,
                              int64_t ldq_out, void* k_out_dev, int64_t ldk_out, void* stream);

/* A paged key/value cache held in 4 bits.  A row (one token's key or value of one head, head_dim = 64, 128 or 256 values) is
 * head_dim codes and one fp16 scale to 32 dimensions, by the rule of the 4-bit Values (spdp_pack_tiled_cbc_q4):
 *   scale = fp16(max|x| / 7);  code = clamp(rint(x / scale), -7, 7) + 8 (8 where the scale is 0);  it stands for (code - 8) * scale.
 * Rows must be finite (what Inf or NaN leave is unspecified, within that row); values of 65492 and more may come to stand for Inf,
 * which 7 times their scale rounds to in fp16.
 * A page holds page_tokens = P tokens (a power of two, 16 .. 256); for each key head in turn: codes of the keys
 * [P][head_dim / 2] bytes, codes of the values [P][head_dim / 2], scales of the keys fp16 [P][head_dim / 32], scales of the values
 * [P][head_dim / 32].  In a row of codes, with G = head_dim / 32, dimension 32 g + 8 c + j (c < 4, j < 8) is bits 4 j .. 4 j + 3 of
 * 32-bit word c G + g.
 * A cache is `pages` such pages, 16-byte aligned, in any order; slot s is token s % P of page s / P.
 * spdp_kv4_page_bytes writes the bytes of a page (host arithmetic). */
SPDP_API spdp_status spdp_kv4_page_bytes(int kv_heads, int head_dim, int page_tokens, int64_t* bytes_out);

/* Stores N tokens' keys and values into the cache.
 *   k_dev        fp16 [N][ldk], heads one after another (what spdp_qk_norm_rope leaves), N <= 2^24.
 *   v_dev        [N][ldv] of vdt; 32-bit values are first rounded to fp16.
 *   slot_dev     int64 [N]; a slot below 0 or beyond the last page stores nothing.  A slot that occurs twice ends up with either
 *                token's row, or parts of both.
 *   k_values_dev_out, v_values_dev_out  fp16 [N][ld...], or NULL: the values that the codes stand for (rounded to fp16), also
 *                where nothing is stored: a prompt's own attention can then work on the keys and values that later tokens see.
 * Launches one kernel. */
SPDP_API spdp_status spdp_kv4_store(const void* k_dev, int64_t ldk, const void* v_dev, int64_t ldv, spdp_ydtype vdt, int64_t N, int kv_heads, int head_dim,
                           const void* slot_dev, void* cache_dev, int64_t pages, int page_tokens, void* k_values_dev_out, int64_t ldk_values,
                           void* v_values_dev_out, int64_t ldv_values, void* stream);

/* Attention of one new token for each of B requests over the 4-bit cache, fused with the pruning decision of the projection
 * behind it (as spdp_swiglu_dp is for a gated MLP): y = softmax(cap * tanh(scale * q k / cap)) v, query head i with key head
 * i / (q_heads / kv_heads).
 *   q_dev        fp16 [B][ldq], B <= 4096; q_heads a multiple of kv_heads.
 *   table_dev    int32 [B][table_stride], table_stride >= table_pages: the pages of each request in order, table_pages * page_tokens
 *                <= 2^31 - 8193.  The keys of a page outside 0 .. pages-1 are left out.
 *   length_dev   int32 [B]: keys of each request, the new token's own among them (store it first); values below 0 and above
 *                table_pages * page_tokens count as these.  A request without keys gets zeros.
 *   scale        between -10^16 and 10^16.
 *   cap          > 0 (10^38 at most): scores are capped; 0: they are not.
 *   window       > 0: only the last `window` keys count; 0: all do.
 *   y_dev        fp16 [B][ldy], ldy >= q_heads * head_dim.
 *   mask_dev_out uint32 [B][mask_stride], mask_stride >= q_heads * head_dim / 32, or NULL: the columns that the o-projection
 *                should keep, NOT(|y_j| <= thr) on the stored y, for SPDP_DP_MASK (thr is used for nothing else).
 * Refused as SPDP_ERR_UNSUPPORTED_SHAPE besides: B * kv_heads * (query heads of a key head / 8, rounded up) * (table_pages * page_tokens / 64 + 8) of
 * 2^31 and more.
 * What lies in the cache behind a request's last key is never used, whatever it is.  Sums in 32 bits; the softmax's weights, times
 * the scales of the values, are rounded to fp16 for their product with these.  Where the requests are few and table_pages (or the
 * window) says that they are short, the call launches one kernel; else two, with scratch memory (a few MB). */
SPDP_API spdp_status spdp_attn_kv4(const void* q_dev, int64_t ldq, int64_t B, int q_heads, int kv_heads, int head_dim, const void* cache_dev, int64_t pages,
                          int page_tokens, const void* table_dev, int64_t table_stride, int64_t table_pages, const void* length_dev, float scale,
                          float cap, int64_t window, float thr, void* y_dev, int64_t ldy, void* mask_dev_out, int64_t mask_stride, void* stream);

/* A paged key/value cache held in 8 bits, with a scale to every 16 tokens of a head.  A page holds page_tokens = P tokens (a power of
 * two, 16 .. 256): for each key head in turn P / 16 cells, one to 16 tokens.  A cell, with D = head_dim = 64, 128 or 256, is 32 D + 16
 * bytes: codes of the keys [D / 64][16 tokens][64 dimensions]; codes of the values, where token r and dimension d is byte
 * 512 (d / 32) + 64 (d % 8) + 16 (r % 8 / 2) + 4 (d % 32 / 8) + 2 (r / 8) + r % 2; the scale of the keys and that of the values (32-bit
 * floats); 8 bytes of zeros.  A code is an e4m3 number (1 sign, 4 exponent and 3 mantissa bits) and stands for itself times its
 * scale, which is a power of two: the smallest from 2^-15 up with max|x| <= 448 scale, over what the cell holds of its side.  So
 *   code = e4m3(x / scale), rounded once, ties to even, and what it stands for is an fp16 number.
 * Values are first brought between -61440 and 61440 (Inf too; NaN becomes one of the two).
 * A cache is `pages` such pages, 16-byte aligned, in any order.
 * spdp_kv8_page_bytes writes the bytes of a page, kv_heads * P * (2 D + 1) (host arithmetic). */
SPDP_API spdp_status spdp_kv8_page_bytes(int kv_heads, int head_dim, int page_tokens, int64_t* bytes_out);

/* Stores the keys and values of N tokens of B requests (B <= 4096) behind those that the requests have.
 *   k_dev        fp16 [N][ldk], heads one after another (what spdp_qk_norm_rope leaves), N <= 2^24.
 *   v_dev        [N][ldv] of vdt; 32-bit values are first rounded to fp16.
 *   first_dev    int32 [B + 1], ascending: the tokens first[b] .. first[b + 1] - 1 are request b's, in order (numbers below 0 and above N
 *                count as these; tokens of no request are passed over); NULL: N = B and token b is request b's.
 *   table_dev    int32 [B][table_stride], table_stride >= table_pages: the pages of each request in order, table_pages * page_tokens
 *                <= 2^31 - 8193.  Tokens of a page outside 0 .. pages-1 are not stored.  No page that is stored to may occur twice.
 *   length_dev   int32 [B]: tokens of each request with the new ones: its last new token becomes number length - 1 (values below 0 and
 *                above table_pages * page_tokens count as these; new tokens that then have numbers below 0 are passed over).
 *   k_values_dev_out, v_values_dev_out  fp16 [N][ld...], or NULL: the values that the codes of the new tokens stand for, also where
 *                they are not stored.  Rows of tokens that are passed over stay as they were.
 * A cell's first token makes the rest of it zeros.  One that joins a cell whose scale is too small for it makes the scale grow, and
 * the codes of the tokens before are rounded again (those that stand for less than 2^-6 of the new scale change, by half a step of
 * 2^-9 of it at most).  Where a request's length has gone back, its new tokens take the places of those that are no more: a cell that still holds older ones
 * keeps the scale it has, also where that was a lost token's.  Launches one kernel. */
SPDP_API spdp_status spdp_kv8_store(const void* k_dev, int64_t ldk, const void* v_dev, int64_t ldv, spdp_ydtype vdt, int64_t N, int kv_heads, int head_dim, int64_t B,
                           const void* first_dev, const void* table_dev, int64_t table_stride, int64_t table_pages, const void* length_dev, void* cache_dev,
                           int64_t pages, int page_tokens, void* k_values_dev_out, int64_t ldk_values, void* v_values_dev_out, int64_t ldv_values, void* stream);

/* Attention of N new tokens of B requests over the 8-bit cache (store them first), fused with the pruning decision of the projection behind
 * it: y = softmax(cap * tanh(scale * q k / cap)) v, query head i with key head i / (q_heads / kv_heads), for single tokens, a few
 * of each request, and prompts or pieces of them, also mixed in a call.
 *   q_dev        fp16 [N][ldq]; q_heads a multiple of kv_heads.
 *   first_dev, table_dev, length_dev  as for spdp_kv8_store: request b's last token first[b + 1] - 1 is its key number length[b] - 1, and
 *                a token sees the keys up to its own number.  The keys of a page outside 0 .. pages-1 are left out.
 *   scale        between -10^16 and 10^16.
 *   cap          > 0 (10^38 at most): scores are capped; 0: they are not.
 *   window       > 0: a token sees only the last `window` keys up to its own, and the request's first `sinks` keys (those of them that are not
 *                behind it); 0: all keys up to its own.  Pages that no token sees may be missing from the table.
 *   y_dev        fp16 [N][ldy], ldy >= q_heads * head_dim.  A token that sees no key gets zeros; tokens of no request stay as they were.
 *   mask_dev_out uint32 [N][mask_stride], mask_stride >= q_heads * head_dim / 32, or NULL: the columns that the o-projection
 *                should keep, NOT(|y_j| <= thr) on the stored y, for SPDP_DP_MASK (thr is used for nothing else).
 * Refused as SPDP_ERR_UNSUPPORTED_SHAPE besides: N * q_heads of 2^31 and more; with g = q_heads / kv_heads and T = table_pages * page_tokens, B * kv_heads *
 * (r / 8, rounded up) * (T / 64 + 8) of 2^31 and more, where r is g if first_dev is NULL and else 64 or N g, whichever is less; and, with first_dev,
 * kv_heads * (N g / 128 + B) * (T / 128 + 8) of 2^31 and more.
 * What lies in the cache behind a request's last key is never used, whatever it is.  Sums in 32 bits; the softmax's weights, times the
 * scales of the values, are rounded to fp16 for their product with these.  Requests of up to 64 rows (tokens times g) and longer ones are different kernels': the
 * call launches one to five, with scratch memory (up to 40 MB on 148 SMs, and 64 bytes to 128 rows) unless the requests are few and short.  The waits inside the
 * kernels are bounded; where one runs out, which none should, rows become NaN or stay unwritten. */
SPDP_API spdp_status spdp_attn_kv8(const void* q_dev, int64_t ldq, int64_t N, int q_heads, int kv_heads, int head_dim, int64_t B, const void* first_dev, const void* cache_dev,
                          int64_t pages, int page_tokens, const void* table_dev, int64_t table_stride, int64_t table_pages, const void* length_dev, float scale, float cap,
                          int64_t window, int64_t sinks, float thr, void* y_dev, int64_t ldy, void* mask_dev_out, int64_t mask_stride, void* stream);

/* The pages of a cache (4-bit, 8-bit, or any whose pages are a multiple of 16 bytes) between steps.  The state is the caller's, on the
 * device, and every call changes it in stream order, so all of this may be captured together with the steps that use the pages:
 *   ref_dev      int32 [pages] (1 <= pages <= 2^28): how many entries of the table name the page; 0 or less: the page is free.
 *   table_dev    int32 [rows][table_stride], table_stride >= table_pages, rows <= 2^24: a request's pages in order, -1 where there is none.
 *                rows * table_pages < 2^31.
 *   cache_dev    `layers` caches of `pages` pages each, layer_stride bytes apart (a multiple of 16, >= pages * page_bytes; ignored for one layer); all share
 *                the table.  16-byte aligned.
 * A call names n <= 4096 rows (or pairs) by int32 [n] arrays on the device; rows outside 0 .. rows-1 are passed over, entries are cut
 * to 0 .. table_pages.  n = 0 does nothing (an output of a number gets 0). */

/* Entries from[i] .. to[i] - 1 of row[i] each get a free page, whatever they held: the lowest free page to the first entry of row[0], and so on.
 * Those for which there is none get -1; short_dev_out (int32 [1], or NULL) gets their number.  No entry may be named twice.  One kernel. */
SPDP_API spdp_status spdp_kv_pages_take(void* ref_dev, int64_t pages, void* table_dev, int64_t rows, int64_t table_stride, int64_t table_pages, const void* row_dev,
                           const void* from_dev, const void* to_dev, int64_t n, void* short_dev_out, void* stream);

/* Entries from[i] .. to[i] - 1 of row[i] give their pages back and become -1 (those that name none too).  A finished request frees 0 ..
 * table_pages; one with a window frees what lies between its first tokens and the window.  One kernel. */
SPDP_API spdp_status spdp_kv_pages_free(void* ref_dev, int64_t pages, void* table_dev, int64_t rows, int64_t table_stride, int64_t table_pages, const void* row_dev,
                           const void* from_dev, const void* to_dev, int64_t n, void* stream);

/* Row child[i] becomes a request with the first length[i] tokens of row parent[i]: full pages (of page_tokens, a power of two, 1 .. 2^16) are shared, a last,
 * partly filled one is copied to a free page (the lowest to the first i) in all layers.  Entries behind these stay as they were.  Where the parent
 * has no page the child gets -1; so it does where there is no free page for a copy, and short_dev_out (int32 [1], or NULL) gets
 * the number of these.  Children are distinct rows that are no parents, whose first entries name no pages.  Two kernels. */
SPDP_API spdp_status spdp_kv_pages_fork(void* cache_dev, int layers, int64_t layer_stride, int64_t page_bytes, void* ref_dev, int64_t pages, void* table_dev, int64_t rows,
                           int64_t table_stride, int64_t table_pages, int page_tokens, const void* parent_dev, const void* child_dev, const void* length_dev, int64_t n,
                           void* short_dev_out, void* stream);

/* Page src[i] to page dst[i] in all layers.  Pairs of which one is outside 0 .. pages-1 are passed over.  What is a destination may be nothing
 * else in the call.  One kernel. */
SPDP_API spdp_status spdp_kv_pages_copy(void* cache_dev, int layers, int64_t layer_stride, int64_t page_bytes, int64_t pages, const void* src_dev, const void* dst_dev, int64_t n,
                           void* stream);

/* Brings the pages in use together: with `live` of them, the i-th free page below `live` gets the i-th page in use from `live` on, in all layers, counts and table
 * entries (of all rows) with it.  live_dev_out (int32 [1], or NULL) gets their number: the pages from there on are free.  Two
 * or three kernels, 8 bytes of scratch memory to a page. */
SPDP_API spdp_status spdp_kv_pages_compact(void* cache_dev, int layers, int64_t layer_stride, int64_t page_bytes, void* ref_dev, int64_t pages, void* table_dev, int64_t rows,
                           int64_t table_stride, int64_t table_pages, void* live_dev_out, void* stream);

/* Row-tile sharding over several GPUs (the paper names multi-GPU execution as future work, Sec. 6; the
 * natural split of y = W x keeps whole 256-row tiles together, so every rank packs its own rows as
 * an independent Tiled-CBC matrix, x is replicated, and the outputs are disjoint).  This is the split
 * every rank must agree on: the ceil(M/256) row tiles are dealt out in contiguous runs, the first
 * (tiles % world) ranks get one more.  Writes rank's first row and its number of rows (0 when there
 * are fewer row tiles than ranks).  Host arithmetic only. */
SPDP_API spdp_status spdp_row_shard(int64_t M, int world, int rank, int64_t* first_row_out, int64_t* rows_out);

/* Release the handle and everything it owns (waits for the work on its device).  Up to 512 MB per device of what freed handles
 * leave is kept for the next ones.  spdp_free(NULL), which is SPDP_OK, gives that back to the driver, and the unused scratch
 * memory of spdp_spmm (up to 96 MB, else kept until the device's last handle goes): call it when another allocator needs
 * the memory. */
SPDP_API spdp_status spdp_free(spdp_handle h);

/* ---- inspection surface (the format and the active set are checked bit for bit) ---- */

SPDP_API spdp_status spdp_get_info(spdp_handle h, spdp_info* out);

/* Copy the four arrays to HOST buffers sized as in spdp_info (any pointer may be NULL to skip
 * it).  Synchronous. */
SPDP_API spdp_status spdp_export(spdp_handle h, void* tileoffset_host, void* colinfo_host,
                        void* bitmap_host, void* values_host);

/* Decode the packed matrix back to dense fp16 [M][ldw] in device memory with the rule of
 * Sec. 4.2.1 (bit clear -> +0, else Values[base + number of set bits before the position]).
 * Asynchronous on `stream`. */
SPDP_API spdp_status spdp_unpack(spdp_handle h, void* W_dev_out, int64_t ldw, void* stream);

/* The active-column set spdp_spmspv would use for this x (Sec. 4.2 step (3)):
 * bitmask_dev_out uint32[ceil(K/32)] (bit j%32 of word j/32, bits beyond K clear) and, if not
 * NULL, count_dev_out int32[1], both device.  Asynchronous on `stream`. */
SPDP_API spdp_status spdp_active_columns(spdp_handle h, const void* x_dev, spdp_dp_rule rule, float thr,
                                const void* mask_dev, void* bitmask_dev_out, void* count_dev_out,
                                void* stream);

/* Context measurements for the benchmark (the paper has no counterpart; they compute nothing).
 * spdp_probe_stream_read reads the handle's Values array front to back with plain 16-byte loads;
 * spdp_probe_gather reads exactly what one spdp_spmspv call with these arguments must fetch -- the
 * ColInfo / TileOffset words of the active columns, their bitmaps and their padded values -- with
 * plain loads and no decoding (its first call, and any call with other arguments, first builds the
 * list of those tiles in a scratch buffer it allocates; repeated calls with the same pointers reuse
 * the list, so time the repeats).  Both are asynchronous on `stream` and write nothing the caller can
 * see; the caller times them.  They give the speed of a contiguous read and
 * the ceiling of the method's access pattern on this GPU, next to which the kernel is reported. */
SPDP_API spdp_status spdp_probe_stream_read(spdp_handle h, void* stream);
SPDP_API spdp_status spdp_probe_gather(spdp_handle h, const void* x_dev, spdp_dp_rule rule, float thr,
                              const void* mask_dev, void* stream);

/* Read (and clear) the handle's device status word: 0, or an spdp_status recorded by a kernel.
 * Synchronises the device. */
SPDP_API spdp_status spdp_last_device_status(spdp_handle h, int* out);

/* Tuning knob: number of CTAs spdp_spmspv launches (0 = default: one per SM, fewer on small
 * layers; at most 1024 and at most one per GTile are used).  Takes effect on
 * the next call; re-derives the handle's split-K workspace.  Waits for the device.  Where there is no memory for the new
 * workspace (SPDP_ERR_ALLOC) the handle stays as it was. */
SPDP_API spdp_status spdp_set_num_ctas(spdp_handle h, int num_ctas);

/* Text of the last CUDA runtime error seen by the library on this thread ("" if none). */
SPDP_API const char* spdp_last_cuda_error(void);

SPDP_API const char* spdp_status_string(spdp_status s);

#ifdef __cplusplus
}
#endif
#endif /* SPDP_H_ */
