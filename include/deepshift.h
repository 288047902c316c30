/*
 * deepshift.h -- C ABI of the DeepShift shift-operator library for GB300 (sm_103a).
 *
 * DeepShift (Elhoushi et al., "DeepShift: Towards Multiplication-Less Neural
 * Networks") replaces every multiply of a fully-connected or convolutional
 * layer by a bitwise shift and a sign flip (Sec. 3, Eq. 1-3).  With weight
 * codes s in {-1, 0, +1} (Eq. 2) and p in [-15, 0] (Sec. 4) and int32
 * activations / biases in 32-bit fixed point with 16 fraction bits (Sec. 4),
 * every operator of this library computes, per output,
 *
 *     y = ReLU?( sat32( b + sum_k s_k * (x_k >> -p_k) ) )
 *
 * with ">>" the two's-complement arithmetic right shift (floor division by
 * 2^-p, Eq. 1), the shift applied before the flip, the sum exact and the
 * result saturated to the int32 range.
 *
 * Conventions for every entry point:
 *   - Tensor pointers are DEVICE pointers owned by the caller.  The library
 *     allocates no memory in any call.
 *   - `stream` is a cudaStream_t passed as void* (NULL = legacy default
 *     stream).  Compute calls are asynchronous and stream-ordered; only
 *     ds_pack_shift_weights synchronises its stream.
 *   - Arguments are validated before anything is launched.  On an error the
 *     call returns a non-zero ds_status, launches nothing, writes no output,
 *     and ds_last_error() describes the problem.  A failed launch returns
 *     DS_ERR_CUDA.
 *   - Activation / output base pointers must be 16-byte aligned
 *     (DS_ERR_ALIGNMENT otherwise).  Any positive size is accepted; tails are
 *     handled inside the kernels.
 */
#ifndef DEEPSHIFT_H
#define DEEPSHIFT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DS_OK = 0,
  DS_ERR_INVALID_ARG = 1,      /* null pointer, bad flag, inconsistent descriptor */
  DS_ERR_SHAPE = 2,            /* non-positive or inconsistent dimension */
  DS_ERR_CODE_RANGE = 3,       /* s not in {-1,0,1} or p not in [-15,0] */
  DS_ERR_ALIGNMENT = 4,        /* pointer not 16-byte aligned */
  DS_ERR_BUFFER_TOO_SMALL = 5, /* caller buffer smaller than required */
  DS_ERR_UNSUPPORTED = 6,      /* valid but not supported (e.g. too large) */
  DS_ERR_CUDA = 7              /* a CUDA runtime call or launch failed */
} ds_status;

/* Devices.  Kernel attributes (the opt-in shared-memory size, non-portable
 * cluster sizes) are set once per process, on the device that is current at a
 * kernel's first launch: drive one GPU per process (one process per GPU, as
 * the multi-GPU replicas do).  A launch on a second device from the same
 * process is not supported: kernels that need such an attribute fail with
 * DS_ERR_CUDA, and every launch goes to the device that is current, so that
 * device has to be the memory's (the tensor helpers of the 8-bit operators
 * check it).  The device's SM count, which sizes grids, split reductions and
 * cluster choices, is likewise read once per process. */

/* Size limits.  Every size the library forms from caller dimensions is
 * bounded before it can overflow 64 bits.  A code matrix holds at most 2^48
 * codes, with n_out <= 2^31 and k_red <= 2^40 (2^36 for the expanded and
 * bf16 layouts); a tensor holds at most 2^62 bytes; a zero-padded image
 * extent (H + 2 pad) is at most 2^31 - 1; one convolution image has at most
 * 2^31 input values (C x H x W) and 2^30 output positions (OH x OW).  Larger
 * dimensions give DS_ERR_UNSUPPORTED, and 0 from the size queries. */

/* Description of the last error on the calling thread ("" if none). */
const char* ds_last_error(void);

/* Library version: major * 10000 + minor * 100 + patch (a library utility: no counterpart in the paper). */
int ds_version(void);

/* sizeof of the ABI structs as compiled into the library (0: ds_weights, 1: ds_layer, 2: ds_f8_matrix,
 * 3: ds_expert_slots, 4: ds_adamw_tensor, 5: ds_adamw_options), so that bindings can check their layout; 0 for any
 * other argument (a library utility: no counterpart in the paper). */
size_t ds_abi_struct_size(int which);

/* ---------------------------------------------------------------------------
 * Flags of the compute calls
 * ------------------------------------------------------------------------- */
#define DS_RELU 1u      /* y = max(y, 0) after saturation (and after the residual add) */
#define DS_AMAX_IN 2u   /* amax_io[0] already holds max|x| of the input: skip the pre-pass */
#define DS_AMAX_OUT 4u  /* write max|y| over this call's outputs into amax_io[1] */
#define DS_RESIDUAL 8u  /* conv only: y = sat32(sat32(conv) + residual) before the ReLU */
#define DS_FORCE_INT64 16u /* always use the 64-bit accumulator path (testing / worst case) */
#define DS_CONV_IM2COL 32u /* conv only: use the implicit-GEMM (im2col gather) kernel instead of the
                              direct halo-tile kernel (testing / comparison) */

/* ---------------------------------------------------------------------------
 * Packed weights.
 *
 * A layer's codes are given as two int8 matrices s[n_out][k_red] and
 * p[n_out][k_red], row-major (a conv layer's OIHW codes flattened, so
 * k_red = C*R*S in (c, r, s) order).  They are packed once into a blob of
 * ds_packed_weight_bytes(n_out, k_red) bytes in caller-owned device memory.
 *
 * Blob layout (format DS_FORMAT_PLANES6, all offsets in bytes, little endian):
 *   [0, 256)          header written by the pack kernel:
 *                       u32 magic (0x31575344 "DSW1"), u32 format,
 *                       i64 n_out, i64 k_red, i64 n_chunks,
 *                       u32 invalid_count, u32 nnz_max, u64 a_max
 *   nib  @ 256        n_chunks x n_out records of 4 u32: for chunk g, column n,
 *                     word w holds in bits 4i..4i+3 the value -p (0..15) of
 *                     reduction index k = 32g + 8w + i
 *   bits @ nib + n_chunks*n_out*16
 *                     n_chunks x n_out records of 2 u32 {sign, nz}: bit j of
 *                     `sign` is set iff s = -1 and bit j of `nz` iff s != 0,
 *                     for k = 32g + j
 *   colA @ bits + n_chunks*n_out*8
 *                     n_out u64: A[n] = sum_k |s| * 2^(15 + p)  (sum of |w| in
 *                     units of 2^-15; used to prove int32 accumulation exact)
 *   nnz  @ colA + n_out*8
 *                     n_out u32: number of non-zero codes of column n
 * Entries with k >= k_red are zero codes.  n_chunks = ceil(k_red / 32).
 * Storage is 6 bits per weight: 4 shift bits + sign + non-zero.  The paper's
 * 5-bit count (Sec. 4) has 32 states, one short of the 33 states of a ternary
 * sign times 16 shifts, so the non-zero plane is the sixth bit (layers whose
 * shifts stay in [-14, 0] can be stored in 5 bits: DS_FORMAT_CODES5 below).
 * ------------------------------------------------------------------------- */
#define DS_FORMAT_PLANES6 1u
#define DS_WEIGHTS_MAGIC 0x31575344u

typedef struct ds_weights {
  uint32_t magic;       /* DS_WEIGHTS_MAGIC once filled by ds_pack_shift_weights */
  uint32_t format;      /* DS_FORMAT_PLANES6 */
  int64_t n_out;        /* output columns (FC: N, conv: K) */
  int64_t k_red;        /* reduction length (FC: K, conv: C*R*S) */
  int64_t n_chunks;     /* ceil(k_red / 32) */
  const void* packed;   /* device pointer to the blob (caller-owned, must outlive use) */
  size_t packed_bytes;  /* size of the blob */
  uint64_t a_max;       /* max over columns of A[n] */
  uint32_t nnz_max;     /* max over columns of the non-zero count */
  uint32_t reserved;
  const void* expanded; /* NULL, or the execution layout set by ds_expand_shift_weights */
  size_t expanded_bytes;
  const void* weights_bf16; /* NULL, or the bf16 weights set by ds_expand_shift_weights_bf16 */
  size_t weights_bf16_bytes;
} ds_weights;

/* Bytes needed for the packed blob of an n_out x k_red code matrix (0 if invalid). */
size_t ds_packed_weight_bytes(int64_t n_out, int64_t k_red);

/*
 * Pack codes (Eq. 3's shift matrix P and sign matrix S, Sec. 4 range).
 *   s, p       device int8 [n_out][k_red], row-major.
 *   packed     device buffer of at least ds_packed_weight_bytes(n_out, k_red)
 *              bytes, 256-byte aligned (cudaMalloc / torch allocations are).
 *   desc       host struct filled on success.
 * Synchronises `stream` (an offline call) so that it can report
 * DS_ERR_CODE_RANGE when any s is outside {-1,0,1} or p outside [-15,0]
 * (the blob is then unusable and desc is not filled).
 */
ds_status ds_pack_shift_weights(const int8_t* s, const int8_t* p, int64_t n_out, int64_t k_red,
                                void* packed, size_t packed_bytes, ds_weights* desc, void* stream);

/* ---------------------------------------------------------------------------
 * Strict 5-bit code storage (Sec. 4: 4 shift bits and a sign bit per weight).
 *
 * With every shift of a nonzero weight in [-14, 0], a ternary sign times 15
 * shifts plus the zero weight is 31 states, which fit 5 bits: code 0 is the
 * zero weight, 1 + (-p) a weight with s = +1, 16 + (-p) one with s = -1 (31
 * is never written).  This is a storage format for such layers: compute calls
 * take the 6-bit blob above, made from the codes that ds_unpack_shift_weights5
 * returns.  The p of a zero weight is not stored and reads back as 0 (no term
 * depends on it).
 *
 * Blob layout (format DS_FORMAT_CODES5, little endian):
 *   [0, 256)     header: u32 magic (0x31575344), u32 format (2), i64 n_out,
 *                i64 k_red, i64 n_chunks = ceil(k_red / 32), u32 invalid_count
 *   @ 256        n_out x n_chunks records of 5 u32, record (n, g) at
 *                256 + 20 (n n_chunks + g): bit j of word b is bit b of the
 *                code of k = 32 g + j (zero beyond k_red)
 * 5 bits per weight, the total rounded up to 256 bytes.
 * ------------------------------------------------------------------------- */
#define DS_FORMAT_CODES5 2u

/* Bytes of the 5-bit blob of an n_out x k_red code matrix (0 if invalid). */
size_t ds_packed5_weight_bytes(int64_t n_out, int64_t k_red);

/*
 * Store codes (s, p: device int8 [n_out][k_red], row-major) in the 5-bit blob
 * `packed5` (device, 256-byte aligned, at least ds_packed5_weight_bytes bytes,
 * caller-owned).  Synchronises `stream` (an offline call) so that it can
 * report DS_ERR_CODE_RANGE when a code has no 5-bit state (s outside
 * {-1, 0, 1}, or p outside [-14, 0] for s != 0, or outside [-15, 0] for s = 0);
 * the blob is then unusable.
 */
ds_status ds_pack_shift_weights5(const int8_t* s, const int8_t* p, int64_t n_out, int64_t k_red, void* packed5,
                                 size_t packed5_bytes, void* stream);

/*
 * Read a 5-bit blob back into s, p (device int8 [n_out][k_red], caller-owned;
 * p = 0 where s = 0).  Synchronises `stream`: the header is checked on the
 * host first (DS_ERR_INVALID_ARG: not a 5-bit blob; DS_ERR_SHAPE: other
 * dims), and DS_ERR_CODE_RANGE reports codes 31 (written as zero weights).
 */
ds_status ds_unpack_shift_weights5(const void* packed5, size_t packed5_bytes, int64_t n_out, int64_t k_red,
                                   int8_t* s, int8_t* p, void* stream);

/* ---------------------------------------------------------------------------
 * Expanded execution layout (optional).  The packed blob is the storage
 * format; decoding it inside every CTA of every launch costs a measurable
 * share of the integer issue slots of these ALU-bound kernels.  A layer may
 * therefore be expanded once into 32-bit shift / sign words laid out as the
 * kernels stage them:
 *   int32 [ceil(n_out / 32)][k_red][64]: for column block cb and reduction
 *   index k, words 0..31 hold -p and words 32..63 hold s of columns
 *   32*cb .. 32*cb + 31 (zero beyond n_out).
 * 8 bytes per weight (plus padding of the last column block).  Kernels use
 * it when desc->expanded is set and decode the blob otherwise; results are
 * identical either way.
 * ------------------------------------------------------------------------- */

/* Bytes of the expanded layout of an n_out x k_red code matrix (0 if invalid). */
size_t ds_expanded_weight_bytes(int64_t n_out, int64_t k_red);

/*
 * Expand packed weights (the codes of Eq. 3's flip(2^P, S)) into `expanded` (device, 16-byte aligned, at least
 * ds_expanded_weight_bytes bytes, caller-owned and outliving every use) and
 * record it in *w (w->expanded, w->expanded_bytes).  Stream-ordered and
 * asynchronous; the blob must stay valid.  Errors: DS_ERR_INVALID_ARG for an
 * unfilled descriptor, DS_ERR_BUFFER_TOO_SMALL, DS_ERR_ALIGNMENT.
 */
ds_status ds_expand_shift_weights(ds_weights* w, void* expanded, size_t expanded_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Float variant (bf16 activations, fp32 accumulation on the tensor cores).
 *
 * With x in bf16 the product x * s * 2^p is exact (s * 2^p is a power of two
 * with p in [-15, 0]), so LinearShift is an ordinary dense contraction
 *     y[m][n] = ReLU?( bias[n] + sum_k x[m][k] * W[n][k] ),  W = flip(2^P, S)  (Eq. 3)
 * with fp32 accumulation.  Its result is not bit-exact: the sum is rounded
 * in an implementation-defined order; |y - exact| <= 1e-5 * (sum_k |x W| + |bias|)
 * is the tolerance the tests hold it to.
 * ------------------------------------------------------------------------- */

/* Bytes of the bf16 weight layout: bf16 [n_out][kpad], kpad = ceil(k_red / 8) * 8. */
size_t ds_bf16_weight_bytes(int64_t n_out, int64_t k_red);

/*
 * Decode packed weights into bf16 W[n][k] = s * 2^p = flip(2^P, S) of Eq. 3 (sign bit, exponent 127 + p,
 * zero mantissa; +0 for s = 0) in `buf` (device, 16-byte aligned, caller-owned)
 * and record it in w->weights_bf16.  Stream-ordered, asynchronous.
 */
ds_status ds_expand_shift_weights_bf16(ds_weights* w, void* buf, size_t bytes, void* stream);

/*
 * Float LinearShift (Eq. 3, fully-connected form, in the float form the paper trains with, Sec. 4) on tcgen05
 * tensor cores (TMA-fed, TMEM accumulator).
 *   x     device bf16 bit patterns (uint16) [M][K], row-major, K % 8 == 0
 *   w     weights with w->weights_bf16 set, n_out == N, k_red == K
 *   bias  device fp32 [N] or NULL
 *   y     device fp32 [M][N]
 *   flags DS_RELU or 0
 * Errors: DS_ERR_UNSUPPORTED when K % 8 != 0 or the bf16 weights are missing.
 */
ds_status ds_linear_shift_bf16(const uint16_t* x, const ds_weights* w, const float* bias, float* y, int64_t M,
                               int64_t K, int64_t N, uint32_t flags, void* stream);

/* 1 if a bounded wait of the float kernel gave up in any ds_linear_shift_bf16 launch since the previous call of
 * this function (or since the library loaded), 0 if none did, -1 if the flag could not be read.  Reading clears
 * the flag.  The flag is device-wide and not per call: synchronise the streams of the calls it should cover
 * first (the read itself is a synchronous copy).  A launch whose wait gave up stops early, so its y is
 * incomplete.  A library utility: no counterpart in the paper. */
int ds_bf16_fault_flag(void);

/* Diagnostic: the limit, in SM clock cycles, of each bounded wait of the float kernel's later launches; cycles <= 0
 * restores the default (4e9 cycles, about 2 s).  A launch whose wait runs out stops issuing work, lets the copies and
 * tensor-core operations it already issued finish, frees its tensor memory and sets the fault flag above, so a test
 * can make the waits run out on purpose and the context stays usable.  Process-wide (not per stream or thread).
 * A library utility: no counterpart in the paper. */
void ds_bf16_set_wait_limit(long long cycles);

/* ---------------------------------------------------------------------------
 * Accumulator width.  Each compute call proves, on the device and with no
 * host round trip, whether 32-bit accumulation is exact:
 *     ceil(amax * A[n] / 2^15) + nnz[n] + |b[n]| <= 2^31 - 1   for every n
 * where amax = max|x| of the input.  If so the 32-bit path runs (no
 * wrap-around and no saturation can occur); otherwise a 64-bit path runs and
 * the exact sum is saturated.  amax comes from amax_io[0] when DS_AMAX_IN is
 * set, else from a pre-pass over x that writes it to amax_io[0].  amax_io
 * (device, 2 x u32) may be NULL: then no bound is available and the 64-bit
 * path is always taken (DS_AMAX_IN and DS_AMAX_OUT need amax_io).
 * ------------------------------------------------------------------------- */

/*
 * LinearShift forward (Eq. 3, Y = flip(2^P, S) X + b; Sec. 4 fixed point):
 *   y[m][n] = sat32( bias[n] + sum_k s[n][k] * (x[m][k] >> -p[n][k]) ), ReLU if DS_RELU.
 *   x     device int32 [M][K] row-major (Q16.16)
 *   w     packed weights with n_out == N and k_red == K
 *   bias  device int32 [N] or NULL (zero bias)
 *   y     device int32 [M][N] row-major; must not overlap x
 *   amax_io device u32[2] or NULL (see above); DS_AMAX_OUT writes max|y| to amax_io[1]
 */
ds_status ds_linear_shift(const int32_t* x, const ds_weights* w, const int32_t* bias, int32_t* y,
                          int64_t M, int64_t K, int64_t N, uint32_t flags, uint32_t* amax_io,
                          void* stream);

/*
 * ConvShift forward (Eq. 3, Y = flip(2^P, S) (*) X + b; cross-correlation with
 * zero padding, as the paper's PyTorch operator):
 *   y[n][k][oh][ow] = sat32( bias[k] + sum_{c,r,q} s[k][c][r][q] *
 *                            (xpad[n][c][oh*sh + r][ow*sw + q] >> -p[k][c][r][q]) )
 *   then, with DS_RESIDUAL, y = sat32(y + residual[n][k][oh][ow]); then ReLU if DS_RELU.
 *   x        device int32 NCHW [N][C][H][W]
 *   w        packed weights with n_out == K and k_red == C*R*S
 *   bias     device int32 [K] or NULL
 *   residual device int32 NCHW [N][K][OH][OW], required iff DS_RESIDUAL
 *   y        device int32 NCHW [N][K][OH][OW], OH = (H + 2*pad_h - R)/stride_h + 1
 *   amax_io  as for ds_linear_shift
 */
ds_status ds_conv2d_shift(const int32_t* x, const ds_weights* w, const int32_t* bias,
                          const int32_t* residual, int32_t* y, int N, int C, int H, int W, int K,
                          int R, int S, int stride_h, int stride_w, int pad_h, int pad_w,
                          uint32_t flags, uint32_t* amax_io, void* stream);

/*
 * LinearShift for callers that cannot allocate device memory.  The paper has
 * no counterpart: this is a deployment convenience of this library.
 *
 * Same operation, arguments and errors as ds_linear_shift, except that the
 * two scratch words of amax_io come from a static device array of 64 u32
 * (256 bytes) that every GPU loading this library holds until the process
 * exits.  It suits callers that must not call cudaMalloc or any allocating
 * routine: a plugin given only its input and output buffers, a host callback,
 * a real-time path that must stay out of the allocator.  Each call uses two of
 * the 64 words whatever the problem size; a build whose per-call need exceeded
 * the array would be rejected with DS_ERR_UNSUPPORTED.  DS_AMAX_IN and
 * DS_AMAX_OUT are rejected (DS_ERR_INVALID_ARG): they need caller scratch.
 *   - The first call on each device looks up the array's device address
 *     (cudaGetSymbolAddress with that device current) and caches it; make that
 *     first call before any stream capture.
 *   - All calls share the array, which keeps the last call's contents; the
 *     max|x| pre-pass clears its word before writing it.  Calls that overlap on
 *     the GPU (different streams without ordering, or several threads) race on
 *     the array and may compute wrong results: order them on one stream.
 *   - It allocates nothing: no cudaMalloc, cudaFree or allocating library call.
 */
ds_status ds_linear_shift_static_scratch(const int32_t* x, const ds_weights* w, const int32_t* bias,
                                         int32_t* y, int64_t M, int64_t K, int64_t N, uint32_t flags,
                                         void* stream);

/* ---------------------------------------------------------------------------
 * Chained forward (ResNet / VGG shaped networks of shift layers).
 *
 * A network is an array of ds_layer run in program order.  Tensors
 * live in numbered slots: slot 0 is the network input x, slot 1 the network
 * output y, slots >= 2 are carved from the caller's workspace.  Activations
 * are NCHW int32 Q16.16; an FC layer reads its input slot as [batch][C*H*W].
 * The ops are the paper's operators (Eq. 3: DS_OP_CONV, DS_OP_FC with the
 * fused bias / saturation / residual / ReLU epilogue) plus the integer pools
 * that ResNet and VGG need (DS_OP_MAXPOOL: max over the window, padded taps
 * ignored; DS_OP_AVGPOOL: floor(sum / (R*S)), no padding).  Each shift layer
 * proves its accumulator width on the device from the max|x| that its
 * producer wrote (the network input gets one pre-pass), so the whole forward
 * runs without a host round trip and can be captured in a CUDA graph.  Make one
 * eager call with the same program and batch first: the first launch of each
 * kernel shape sets kernel attributes and queries cluster occupancy, host calls
 * that a capture in the default (global) mode may refuse.
 * ------------------------------------------------------------------------- */
#define DS_OP_CONV 1
#define DS_OP_FC 2
#define DS_OP_MAXPOOL 3
#define DS_OP_AVGPOOL 4

typedef struct ds_layer {
  int32_t op;          /* DS_OP_* */
  int32_t in;          /* input slot */
  int32_t aux;         /* residual slot (DS_RESIDUAL), else -1 */
  int32_t out;         /* output slot (not 0; distinct from in and aux) */
  int32_t C, H, W;     /* input channels and spatial size, per image */
  int32_t K;           /* conv / FC: output channels or features (pools: ignored) */
  int32_t R, S;        /* conv / pool window */
  int32_t stride, pad; /* conv / pool */
  uint32_t flags;      /* DS_RELU, DS_RESIDUAL (conv only) */
  const ds_weights* w; /* conv / FC weights (n_out = K, k_red = C*R*S or C*H*W) */
  const int32_t* bias; /* conv / FC bias (device int32 [K]) or NULL */
} ds_layer;

/*
 * Workspace bytes for running n layers at the given batch (0 if invalid):
 * every slot >= 2 sized for the largest tensor written to it, plus the
 * max|x| words.  Validates the program like ds_shift_forward.
 */
size_t ds_shift_forward_workspace_bytes(const ds_layer* layers, int n, int batch);

/*
 * Runs the program (shift layers of Eq. 3 with the Sec. 4 fixed point, pools as described above):
 * x = slot 0 (device, [batch][C0][H0][W0] of layer 0),
 * y = slot 1 (device, the tensor of the last layer that writes slot 1),
 * ws = workspace (device, 256-byte aligned, >= the bytes above).
 * Validation errors (DS_ERR_SHAPE, DS_ERR_INVALID_ARG, ...) are reported
 * before anything is launched.  Asynchronous, stream-ordered, no device
 * allocation; the planner's small host arrays are allocated before the first
 * launch, and a failed host allocation returns DS_ERR_UNSUPPORTED ("host
 * memory allocation failed") with nothing launched.  No C++ exception leaves
 * any entry point.
 * A layer that depends on neither its predecessor's output nor a slot that
 * its predecessor reads or writes (a ResNet block's shortcut beside the main
 * branch) runs on a side stream of the calling thread, ordered by events on
 * the slots it reads and writes; the caller's stream waits for the side
 * stream before the call returns, so `stream` orders everything as before.
 * The side stream and its events are created on a thread's first call (one
 * set per host thread, kept until the thread ends); if they cannot be
 * created, every layer runs on `stream`.
 */
ds_status ds_shift_forward(const ds_layer* layers, int n, const int32_t* x, int32_t* y, void* ws,
                           size_t ws_bytes, int batch, void* stream);

/* ---------------------------------------------------------------------------
 * Input gradient (Eq. 7 and its footnote: dC/dX = dC/dY W_q^T for LinearShift,
 * W_q^rot180 (*) dC/dY for ConvShift).  The gradient dY is int32 Q16.16 and
 * each term is the forward's shift-then-flip, s * (dy >> -p); the exact sum
 * is saturated to int32 (no bias, no ReLU).
 *
 * ds_pack_shift_weights_backward packs the code matrices of that pass from
 * the forward codes s, p (device int8, [K][C][R][S]; an FC layer's [N][K_in]
 * is K = N, C = K_in, R = S = 1, strides 1).  A layer of strides (sh, sw) has
 * sh * sw tap phases (a, b): input position i = sh i' + rho receives only the
 * taps r = a + sh t with a = (rho + pad) mod sh, so each phase is a stride-1
 * correlation of dY with a sub-kernel of Th(a) = ceil((R - a) / sh) x Tw(b)
 * taps.  Phase (a, b) is packed as a matrix of C columns and reduction length
 * K * Th * Tw (index (k, t, u) holds the code of (k, c, a + sh (Th-1-t),
 * b + sw (Tw-1-u)); for stride 1 this is W^rot180 with the channels swapped)
 * into desc[a * sw + b]; a phase with no taps gets a descriptor with
 * k_red = 0 and no blob.  desc points to sh * sw caller-owned descriptors,
 * packed to ds_packed_weight_bytes_backward(K, C, R, S, sh, sw) bytes
 * (256-byte aligned; phases at 256-byte aligned offsets).  Synchronises its
 * stream once per phase; DS_ERR_CODE_RANGE on bad codes; strides in [1, 16].
 *
 * ds_linear_shift_backward_x: dx [M][K] from dy [M][N] (row-major, 16-byte
 * aligned) with w_bwd packed by ds_pack_shift_weights_backward(s, p, N, K,
 * 1, 1, 1, 1, ...).  Flags: DS_AMAX_IN / DS_AMAX_OUT (amax_io as in
 * ds_linear_shift) and DS_FORCE_INT64 only.
 *
 * ds_conv2d_shift_backward_x: dx [N][C][H][W] from dy [N][K][OH][OW] of the
 * forward geometry (H, W, R, S, strides, pads as given to ds_conv2d_shift;
 * OH = (H + 2 pad_h - R) / stride_h + 1, likewise OW), w_bwd the
 * stride_h * stride_w descriptors of ds_pack_shift_weights_backward(s, p, K,
 * C, R, S, stride_h, stride_w, ...).  Stride 1 runs the forward ConvShift of
 * dy with padding R-1-pad (direct / pointwise kernels); larger strides run one
 * implicit GEMM per output phase (no term of a skipped window position is
 * computed) and zero-fill the positions no tap reaches.  Flags: DS_AMAX_IN,
 * DS_AMAX_OUT, DS_FORCE_INT64, and DS_CONV_IM2COL (the per-phase implicit
 * GEMM also at stride 1).  Errors as ds_conv2d_shift.
 * ------------------------------------------------------------------------- */
size_t ds_packed_weight_bytes_backward(int K, int C, int R, int S, int stride_h, int stride_w);
ds_status ds_pack_shift_weights_backward(const int8_t* s, const int8_t* p, int K, int C, int R, int S, int stride_h,
                                         int stride_w, void* packed, size_t packed_bytes, ds_weights* desc,
                                         void* stream);
ds_status ds_linear_shift_backward_x(const int32_t* dy, const ds_weights* w_bwd, int32_t* dx, int64_t M, int64_t K,
                                     int64_t N, uint32_t flags, uint32_t* amax_io, void* stream);
ds_status ds_conv2d_shift_backward_x(const int32_t* dy, const ds_weights* w_bwd, int32_t* dx, int N, int C, int H,
                                     int W, int K, int R, int S, int stride_h, int stride_w, int pad_h, int pad_w,
                                     uint32_t flags, uint32_t* amax_io, void* stream);

/* ---------------------------------------------------------------------------
 * Conversion of float models (the step before packing).
 *
 * ds_quantize_shift_weights: the DeepShift-Q quantizer (Sec. 3.1, Eq. 4-6,
 * with the shift clipping of Sec. 4) of n float32 weights w (device, 4-byte
 * aligned, any layout; conv weights flattened as [K][C][R][S]) into the
 * int8 codes s (device, n bytes) and p (device, n bytes) that
 * ds_pack_shift_weights takes:
 *   s = sign(w) in {-1, 0, +1},  p = clip(round(log2|w|), p_min, 0).
 * round(log2|w|) is the integer n with 2^(n-1/2) <= |w| < 2^(n+1/2), decided
 * exactly (no float log; no float weight is a tie).  p_min is -15 (the
 * 6-bit code format) or -14 (codes that also fit the strict 5-bit format of
 * Sec. 4); other values in [-15, 0] are accepted.  w = 0 and NaN give s = 0,
 * p = p_min; +-inf gives s = +-1, p = 0.  Stream-ordered, no synchronisation.
 * Errors: DS_ERR_INVALID_ARG (NULL pointer, p_min outside [-15, 0]),
 * DS_ERR_SHAPE (n <= 0), DS_ERR_ALIGNMENT (w not 4-byte aligned).
 *
 * ds_quantize_q16: Sec. 4's rounding of float inputs (and biases) to 32-bit
 * fixed point with 16 fraction bits: q = round-half-to-even(x * 2^16),
 * saturated to [INT32_MIN, INT32_MAX]; NaN gives 0.  x (n float32) and q
 * (n int32) are device pointers, 4-byte aligned (16-byte alignment takes
 * the vectorised path).  Errors: DS_ERR_INVALID_ARG, DS_ERR_SHAPE,
 * DS_ERR_ALIGNMENT as above.
 * ------------------------------------------------------------------------- */
ds_status ds_quantize_shift_weights(const float* w, int64_t n, int p_min, int8_t* s, int8_t* p, void* stream);
ds_status ds_quantize_q16(const float* x, int64_t n, int32_t* q, void* stream);

/*
 * max |x| over n int32 values, written to *amax (device u32; |INT32_MIN| = 2^31): the input of the
 * accumulator-width proof above (the paper is silent on overflow; Sec. 4 fixes only the 32-bit format).
 */
ds_status ds_absmax(const int32_t* x, int64_t n, uint32_t* amax, void* stream);

/* ---------------------------------------------------------------------------
 * Weight-specialised ConvShift (Eq. 3, as ds_conv2d_shift; specialising the kernels to the weights at run time is
 * the future work of Sec. 6.1).  For a small layer the library writes a kernel in which every weight's shift and
 * sign are immediates and the zero weights are left out, so a term is one shift by an immediate and one add or
 * subtract (no shift for p = 0), with no code loads; it compiles the kernel at run time with NVRTC (libnvrtc,
 * opened on first use) for the current device and keeps it in the returned handle.  Meant for the few-thousand-
 * weight layers at the input of a network (VGG16's first conv: 1728 weights), where the whole layer fits the
 * instruction stream.
 *
 * ds_specialize_conv2d_shift: s, p HOST int8 codes [K][C][R][S] (s in {-1, 0, +1}, p in [-15, 0]); square
 * stride (1 or 2) and padding (below R and S); K*C*R*S <= DS_SPECIALIZE_MAX_WEIGHTS, R, S <= 11.  Compiles and
 * loads (seconds for the largest layers; not stream-ordered, not for a capture).  On success *out owns the kernel
 * until ds_specialized_destroy.  Errors: DS_ERR_INVALID_ARG (NULL), DS_ERR_SHAPE, DS_ERR_CODE_RANGE,
 * DS_ERR_UNSUPPORTED (too many weights or channels for the shared-memory tile, NVRTC missing or failing),
 * DS_ERR_CUDA.
 *
 * ds_conv2d_shift_specialized: the layer on x [N][C][H][W] -> y [N][K][OH][OW] (NCHW int32, 16-byte aligned,
 * not overlapping), bias, residual, flags (DS_RELU, DS_RESIDUAL, DS_AMAX_IN, DS_AMAX_OUT, DS_FORCE_INT64) and
 * amax_io exactly as ds_conv2d_shift; the same accumulator-width proof picks 32- or 64-bit sums per CTA.  Use it
 * on the device it was specialised on.  Stream-ordered, allocates nothing.
 * ------------------------------------------------------------------------- */
#define DS_SPECIALIZE_MAX_WEIGHTS 4096
typedef struct ds_specialized ds_specialized;
ds_status ds_specialize_conv2d_shift(const int8_t* s, const int8_t* p, int K, int C, int R, int S, int stride,
                                     int pad, ds_specialized** out);
ds_status ds_conv2d_shift_specialized(const ds_specialized* h, const int32_t* x, const int32_t* bias,
                                      const int32_t* residual, int32_t* y, int N, int H, int W, uint32_t flags,
                                      uint32_t* amax_io, void* stream);
void ds_specialized_destroy(ds_specialized* h);

/* ---------------------------------------------------------------------------
 * 8-bit floating point: matrices with a scale per block of 128, their product,
 * and the operators around it in a feed-forward block.
 *
 * The paper keeps activations in fixed point and names 8 bits as the next step
 * (Sec. 5.2.1); on this GPU the 8-bit path with twice the bf16 rate is floating
 * point.  A shift weight s * 2^p, p in [-15, 0], is exact in e4m3 with the
 * scale 2^-8, so a shift layer runs on it with its own weights; float layers
 * run on it with weights rounded to blocks.
 *
 * A ds_f8_matrix describes device memory (the library keeps no pointer to it
 * after a call): 8-bit values q, row r at q + r * ld, and float32 scales; the
 * value of an element is q[r][c] * scale.  `blocks` says which scale:
 *   DS_F8_ROWS   scale[r * ld_scale + c / 128]: one per row and 128 columns
 *   DS_F8_TILES  scale[(r / 128) * ld_scale + c / 128]: one per 128 x 128
 * q is 16-byte aligned and ld a multiple of 16 (cols need not be; bytes beyond
 * cols are neither read into results nor written).  The last block of a row or
 * column may be short.
 *
 * Writing a block: with amax the largest finite magnitude in it and MAX the
 * largest value of the format (448, 57344),
 *   scale = max(amax / MAX, 2^-126),  q = value * min(MAX / amax, 2^126)
 * (each a float32 operation) rounded to nearest, ties to even; with DS_F8_POW2
 * the scale is rounded up to a power of two and q = value / scale.
 * Infinities and NaN become the 8-bit NaN.  With DS_F8_POW2 q * scale needs no
 * rounding in float32, and changing the blocks of such a matrix later changes
 * only values that fall below the format's range.
 *
 * Rows: 0 is accepted everywhere (an expert or a step without tokens): nothing
 * is launched for the outputs that then have no elements, and sums over rows
 * are written as zeros.  Types of the other tensors are DS_TYPE_*; their base
 * pointers need only their type's alignment (16 bytes take the vector path),
 * except `weight`, 16 bytes.  Arithmetic is float32; a value is rounded once,
 * where it is stored.  Limits: rows and cols below 2^31 - 256, rows * ld at
 * most 2^48.  Outputs must not overlap inputs except where a call says so, and
 * the 8-bit outputs of one call have one format.
 * ------------------------------------------------------------------------- */
#define DS_TYPE_F32 0
#define DS_TYPE_BF16 1
#define DS_TYPE_F16 2

#define DS_F8_E4M3 0
#define DS_F8_E5M2 1

#define DS_F8_ROWS 0
#define DS_F8_TILES 1

#define DS_F8_POW2 1u /* scales are powers of two */

typedef struct ds_f8_matrix {
  void* q;          /* device, 8-bit values */
  float* scale;     /* device, 4-byte aligned */
  int64_t rows, cols;
  int64_t ld;       /* bytes between rows */
  int64_t ld_scale; /* floats between rows of scales */
  int32_t format;   /* DS_F8_E4M3, DS_F8_E5M2 */
  int32_t blocks;   /* DS_F8_ROWS, DS_F8_TILES */
} ds_f8_matrix;

/*
 * Rounds x (device, [rows][cols] of `type`, row stride ldx elements) to 8 bits:
 *   out    [rows][cols], DS_F8_ROWS or DS_F8_TILES, or NULL
 *   out_t  the transposed matrix [cols][rows] (its DS_F8_ROWS blocks run down
 *          the columns of x: the operand of a product that sums over rows), or
 *          NULL; with DS_F8_TILES it is the exact transpose of a DS_F8_TILES out
 * At least one is given; both cost one pass over x.  flags: DS_F8_POW2 or 0.
 */
ds_status ds_quantize_f8(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const ds_f8_matrix* out,
                         const ds_f8_matrix* out_t, uint32_t flags, void* stream);

/* The same from the values of another 8-bit matrix: other blocks, another format, or the transpose. */
ds_status ds_requantize_f8(const ds_f8_matrix* x, const ds_f8_matrix* out, const ds_f8_matrix* out_t, uint32_t flags,
                           void* stream);

/* The weights s * 2^p of packed codes (Eq. 3) as an e4m3 matrix in tiles: q = s * 2^(p + 8), every scale 2^-8; exact.
 * out is [n_out][k_red], DS_F8_E4M3, DS_F8_TILES.  Stream-ordered. */
ds_status ds_expand_shift_weights_f8(const ds_weights* w, const ds_f8_matrix* out, void* stream);

/*
 * y[m][n] = bias[n] + add[m][n] + sum_k x[m][k] * w[n][k] over 8-bit matrices
 * x [M][K] and w [N][K], on the tensor cores (tcgen05).  Each operand has its
 * own format and blocks.  Products within a block of 128 k are summed by the
 * tensor core; a block's sum is multiplied by its two scales and added in
 * float32 (a sum times either scale has to stay within the normal numbers; the
 * scales' own product need not).  So y = x w^T for a layer's forward pass,
 * dy (w_t)^T for its input gradient, and dy_t (x_t)^T for its weight gradient.
 *   bias  device float32 [N] or NULL
 *   add   device float32 [M][N], row stride ld_add, or NULL; may be y itself
 *         (DS_TYPE_F32, ldy == ld_add): gradients accumulate in place
 *   y     device, `type`, row stride ldy elements
 * K = 0 gives bias + add.  Results do not depend on timing; their rounding
 * depends on M (the reduction of small calls is split).
 */
ds_status ds_linear_f8(const ds_f8_matrix* x, const ds_f8_matrix* w, const float* bias, const float* add,
                       int64_t ld_add, void* y, int type, int64_t ldy, void* stream);

/* Diagnostic: the tile that ds_linear_f8 takes for these arguments on the current device: 256 or 128 rows of w (the
 * kernel of large products), or 64, 32 or 16 rows of x (the other one); 0 where it launches nothing or refuses them. */
int ds_linear_f8_tile(const ds_f8_matrix* x, const ds_f8_matrix* w, const float* add, int64_t ld_add, void* y, int type,
                      int64_t ldy);

/* As ds_bf16_fault_flag and ds_bf16_set_wait_limit, for ds_linear_f8, ds_gated_f8_backward and the experts' products. */
int ds_f8_fault_flag(void);
void ds_f8_set_wait_limit(long long cycles);

/*
 * Root-mean-square norm of a residual stream with an 8-bit output:
 *   h = x + residual;  rstd = (mean_c h^2 + eps)^(-1/2);  out = h * rstd * weight, in 8 bits (DS_F8_ROWS)
 *   x, residual  device [rows][cols] of `type`; residual may be NULL (h = x)
 *   weight       device float32 [cols]
 *   h            device, `type`, row stride ldh, or NULL; may be x or residual
 *                itself (same row stride).  The norm is that of the unrounded h.
 *   rstd         device float32 [rows] or NULL
 * flags: DS_F8_POW2 or 0.
 *
 * Backward (the rounding to 8 bits passes gradients unchanged, as the paper's
 * straight-through estimate does for its own, Eq. 8): with dy the gradient of
 * out, h and rstd from the forward call and dh the gradient of h from the
 * stream that continues (or NULL),
 *   dx = dh + rstd * (dy weight - h rstd mean_c(dy weight h rstd))   (of x and of residual alike)
 *   dw[c] = sum_r dy[r][c] h[r][c] rstd[r]                           (float32 [cols], overwritten)
 * dx may be dy, h or dh itself (same row stride).  ws: device, 16-byte aligned,
 * of ds_rmsnorm_f8_backward_workspace_bytes(rows, cols) bytes.  The sum over
 * rows has a fixed order.
 */
ds_status ds_rmsnorm_f8(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight, int type,
                        int64_t rows, int64_t cols, float eps, const ds_f8_matrix* out, void* h, int64_t ldh,
                        float* rstd, uint32_t flags, void* stream);
size_t ds_rmsnorm_f8_backward_workspace_bytes(int64_t rows, int64_t cols);
ds_status ds_rmsnorm_f8_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, const float* rstd,
                                 const float* weight, const void* dh, int64_t lddh, int type, int64_t rows,
                                 int64_t cols, void* dx, int64_t lddx, float* dw, void* ws, size_t ws_bytes,
                                 void* stream);

/*
 * SiLU-gated activation a = silu(g) * u with an 8-bit output, and a checkpoint
 * of g and u in 8 bits for its backward pass.
 *   gu    device [rows][up + features] of `type`, row stride ld: g in columns
 *         [0, features), u in [up, up + features), up = features rounded up to
 *         a multiple of 128 (no block holds both; columns between are ignored)
 *   out   a, [rows][features], DS_F8_ROWS
 *   ckpt  g and u as [rows][up + features], DS_F8_ROWS (zeros between), or NULL
 *
 * Backward: with g and u the values of ckpt and da [rows][features] of `type`
 * (row stride ld) the gradient of a,
 *   du = da silu(g),  dg = da u sig(g) (1 + g (1 - sig(g)))
 *   dgu    [rows][up + features], DS_F8_ROWS (zeros between), or NULL
 *   dgu_t  its transpose [up + features][rows], DS_F8_ROWS, or NULL
 *   a_t    a again, from ckpt, transposed: [features][rows], DS_F8_ROWS, or NULL
 * At least one is given; each is rounded from float32, not from another.
 * flags: DS_F8_POW2 or 0.
 */
ds_status ds_gated_f8(const void* gu, int type, int64_t ld, int64_t rows, int64_t features, const ds_f8_matrix* out,
                      const ds_f8_matrix* ckpt, uint32_t flags, void* stream);
ds_status ds_gated_f8_backward(const ds_f8_matrix* ckpt, const void* da, int type, int64_t ld, int64_t features,
                               const ds_f8_matrix* dgu, const ds_f8_matrix* dgu_t, const ds_f8_matrix* a_t,
                               uint32_t flags, void* stream);

/* ---------------------------------------------------------------------------
 * Experts: a feed-forward block of which each token takes `top_k` of `experts`
 * parts.  Its slots s = t * top_k + j (choice j of token t) are put in order of
 * their expert, tokens in their order within one; the operators of an expert's
 * part then work on its segment of rows:
 *   counts[e]    slots of expert e
 *   offsets[e]   its first row; offsets[e + 1] = offsets[e] + counts[e] rounded
 *                up to a multiple of `align` (offsets[experts]: the rows in use)
 *   position[s]  the row of a slot, -1 where its expert is not in
 *                [0, experts): such a slot (padding of a batch) goes nowhere
 *   slot[r]      the slot of a row, -1 for rows that hold none (the gaps behind
 *                segments, and the rows from offsets[experts] on)
 * All of it is made and read on the device; `rows` is what the host knows of
 * it, enough for any choice of experts: ds_expert_rows().  With align = 128 the
 * segments start at blocks of the 8-bit matrices, so that these hold no two
 * experts' rows also where they are transposed; with 1 there are no gaps.
 *
 * A ds_expert_slots describes this device memory (int32, 4-byte aligned; the
 * library keeps no pointer to it).  What the calls below read of it has to be
 * what ds_expert_order wrote; rows and slots out of range are passed over.
 * Rows that hold no slot are written as zeros by the calls that write rows (the
 * products take the gaps for rows of their expert: zeros, or the bias).
 * Limits: rows below 2^31 - 256, 1 <= experts <= DS_EXPERTS_MAX, 1 <= align
 * <= 2^20.  tokens = 0 is accepted.  Types, strides and alignment are as for
 * the 8-bit operators; arithmetic is float32, in the order of j, and a value
 * is rounded once, where it is stored.  No result depends on timing.
 * ------------------------------------------------------------------------- */
#define DS_EXPERTS_MAX 1024

#define DS_INDEX_I32 0
#define DS_INDEX_I64 1

typedef struct ds_expert_slots {
  int32_t* offsets;  /* device [experts + 1] */
  int32_t* counts;   /* device [experts] */
  int32_t* position; /* device [tokens * top_k] */
  int32_t* slot;     /* device [rows] */
  int64_t tokens, rows;
  int32_t top_k, experts, align, reserved;
} ds_expert_slots;

/* Rows that hold the segments of any choice of experts: the largest multiple of align not above
 * tokens * top_k + min(experts, tokens * top_k) * (align - 1); -1 for arguments out of range. */
int64_t ds_expert_rows(int64_t tokens, int32_t top_k, int32_t experts, int32_t align);

/* Writes all of `s` (its rows at least ds_expert_rows) from ids, device [tokens][top_k] of DS_INDEX_*, contiguous. */
ds_status ds_expert_order(const void* ids, int id_type, const ds_expert_slots* s, void* stream);

/* out[r] = x[slot[r] / top_k]: x [tokens][cols] and out [rows][cols] of `type`, or 8-bit matrices of one format with
 * DS_F8_ROWS blocks, whose values and scales are copied as they are. */
ds_status ds_expert_gather(const void* x, int type, int64_t ldx, int64_t cols, const ds_expert_slots* s, void* out,
                           int64_t ldo, void* stream);
ds_status ds_expert_gather_f8(const ds_f8_matrix* x, const ds_expert_slots* s, const ds_f8_matrix* out, void* stream);

/*
 * out[t] = add[t] + sum_j weights[t][j] * y[position[t][j]], over the slots that have a row
 *   y        device [rows][cols] of `type`
 *   weights  device float32 [tokens][top_k], contiguous, or NULL: all 1.  With these, the sum is the gradient of
 *            ds_expert_gather's x, y being that of its rows.
 *   add      device [tokens][cols] of `type`, or NULL; may be out itself (same stride)
 *   out      device [tokens][cols] of `type`
 * Backward, dout being the gradient of out (and of add):
 *   dy[position[t][j]] = weights[t][j] * dout[t]     (zeros in the other rows)
 *   dweights[t][j] = sum_c dout[t][c] * y[position[t][j]][c]     (0 for a slot without a row)
 * dweights may be NULL, and y then too.  dy may be y itself (same stride).
 */
ds_status ds_expert_combine(const void* y, int type, int64_t ldy, int64_t cols, const ds_expert_slots* s,
                            const float* weights, const void* add, int64_t ld_add, void* out, int64_t ldo,
                            void* stream);
ds_status ds_expert_combine_backward(const void* dout, int64_t ldd, const void* y, int64_t ldy, int type, int64_t cols,
                                     const ds_expert_slots* s, const float* weights, void* dy, int64_t lddy,
                                     float* dweights, void* stream);

/*
 * The products of the experts' parts, over 8-bit matrices as ds_linear_f8 takes them:
 *   y[r] = bias[e] + x[r] w_e^T     for the rows r of each segment e (gaps too: x holds zeros there)
 *   x     [rows][K], DS_F8_ROWS (or DS_F8_TILES where align is a multiple of 128)
 *   w     [experts * N][K], w_e its rows [e N, (e + 1) N); in tiles only where N is a multiple of 128
 *   bias  device float32 [experts][N], contiguous, or NULL
 *   y     device [rows][N] of `type`; zeros from row offsets[experts] on
 * and their weight gradients
 *   dw_e[n][k] = add_e[n][k] + sum over the rows r of segment e of dy_t[n][r] x_t[k][r]
 *   dy_t  [N][rows], x_t [K][rows]: transposed, so that blocks run along the rows; align a multiple of 128
 *   dw    device float32 [experts * N][K], row stride lddw; add the same, ld_add, or NULL; may be dw itself
 * A bounded wait that gives up is reported by ds_f8_fault_flag.
 */
ds_status ds_expert_linear_f8(const ds_f8_matrix* x, const ds_f8_matrix* w, const ds_expert_slots* s, const float* bias,
                              void* y, int type, int64_t ldy, void* stream);
ds_status ds_expert_weight_grad_f8(const ds_f8_matrix* dy_t, const ds_f8_matrix* x_t, const ds_expert_slots* s,
                                   const float* add, int64_t ld_add, float* dw, int64_t lddw, void* stream);

/* ---------------------------------------------------------------------------
 * Optimizer: one step of Adam with decoupled weight decay over many tensors.
 * For each value, with t the step's number (from 1) and each operation rounded
 * to float32 (the factors are computed in float64 and rounded once; those of a
 * t or lr on the device in float32, within 2^-21 of it):
 *   g' = g * grad_scale
 *   m  = beta1 * m + (1 - beta1) * g'
 *   v  = beta2 * v + (1 - beta2) * (g' * g')
 *   p  = p * (1 - lr * weight_decay)
 *        - m * (lr / (1 - beta1^t)) / (sqrt(v) * (1 - beta2^t)^(-1/2) + eps)
 * p is rounded once to its type, to the nearest; `copy` is p, as it was before
 * that, rounded to another.  A 16-bit p keeps no update below half its step:
 * for these, p is float32 and `copy` the 16-bit values.
 *
 * The states m and v are float32, or 8 bits: e4m3 values of m and of sqrt(v),
 * with a float32 scale for each 128 consecutive values of a tensor,
 *   scale = max(amax / 448, 2^-126),  u = value * min(448 / amax, 2^126),
 * amax the block's largest finite magnitude.  u becomes one of its two e4m3
 * neighbours, the one of larger magnitude with the probability of u's distance
 * from the other one, so that its expected value is u.  (To the nearest a state
 * would stand still: a step changes v by 1 - beta2 of itself, a rounding to 3
 * bits loses up to 12%.)  For m that makes the expected value what the
 * recurrence says; v is the square of the root that is held, and each
 * rounding's variance is added to it: its mean is above the recurrence's, by at
 * most 2/15 while a block's scale stays and its roots are at least 2^-6 of it
 * (with beta2 = 0.999 5.5% for normal gradients, 7% where one in 20 is not
 * zero; the mean of 1 / sqrt(v) is then 1.2 and 2% above).  A positive sqrt(v)
 * is held as at least the smallest value, 2^-9, and its square is not 0 where
 * the block's largest root is at least 2^-57 and beta2 above 1/2, so that a
 * later step divides by a root and not by eps alone.  Infinities and NaN become
 * NaN.  The
 * step itself takes m and v before they are rounded.  With i the index of a
 * value in its tensor and n the tensor's number in the call, the random bits
 * of m and sqrt(v) are the low and the high half of a hash of
 *   x = i * 0x9E3779B1 + t * 0xBB67AE85 + n * 0x6A09E667 + seed    (mod 2^32):
 *   x ^= x >> 16;  x *= 0x243F6A89;  x ^= x >> 15;  x *= 0xB7E15163;
 *   x ^= x >> 16
 * and the value is the upper neighbour where its distance plus (half + 1/2) /
 * 2^16 reaches 1.
 * ------------------------------------------------------------------------- */
typedef struct ds_adamw_tensor {
  void* p;            /* device [n] of p_type */
  const void* g;      /* device [n] of g_type */
  void *m, *v;        /* device [n]: float32, or e4m3 where the scales are given */
  float *m_scale, *v_scale; /* device [ceil(n / 128)], or both NULL */
  void* copy;         /* device [n] of copy_type, or NULL */
  int64_t n;
  float weight_decay;
  int32_t p_type, g_type, copy_type; /* DS_TYPE_* */
} ds_adamw_tensor;

typedef struct ds_adamw_options {
  double lr, beta1, beta2, eps;
  int64_t step;            /* t, from 1; not read where step_dev is given */
  const int64_t* step_dev; /* device: t, or NULL.  A captured call is replayed with the value that is there then */
  const float* lr_dev;     /* device: lr, or NULL */
  const float* grad_scale; /* device: a factor of all gradients (a clipped norm, a loss scale), or NULL */
  uint32_t seed, reserved;
} ds_adamw_options;

/*
 * Updates `count` tensors (a host array, read during the call): p, m, v, their
 * scales and copy in place.  The tensors' memories are contiguous, aligned to
 * their type (eight values take the vector path), and apart from each other;
 * all states are of one kind.  n = 0 is accepted.  One launch for up to 400
 * tensors.  Errors: DS_ERR_INVALID_ARG (NULL, a type, betas outside [0, 1),
 * step below 1, overlap), DS_ERR_SHAPE, DS_ERR_ALIGNMENT, DS_ERR_UNSUPPORTED
 * (n above 2^40).
 */
ds_status ds_adamw(const ds_adamw_tensor* tensors, int count, const ds_adamw_options* options, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DEEPSHIFT_H */
