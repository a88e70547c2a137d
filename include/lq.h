/*
 * lq.h - C ABI of the B200 (sm_100a) implementation of the LoRaQ fully quantized linear layer
 *
 *     Y = deq( Q4(X) * Q4(W - L1 L2) )  +  deq( Qb( Qb(X) * Qb(L1) ) * Qb(L2) )
 *
 * Notation follows the paper (Section 3.1): X in R^{m x d} activations, W in R^{d x n} weights,
 * Y = X W.  Here M = m rows (tokens x batch), K = d input features, N = n output features,
 * r = the rank of the low-rank branch, G = ceil(K / group) blocks of the 4-bit main format.
 *
 * Two main formats (Appendix A.3, Table 2), chosen by lq_config.group:
 *   group = 64  SINT4: signed 4-bit codes in [-7, 7], one fp16 scale per block of 64 along K;
 *               the per-block scale products are applied by the GEMM's epilogue warps.
 *   group = 32  MXINT4: the same codes, one power-of-two scale 2^e per block of 32 along K,
 *               e the smallest integer with 7 * 2^e >= max|v| of the block (the paper does not
 *               spell the rule out; this one never clips); the scales are applied by the tensor
 *               core itself (block-scaled MMA).  Every branch format; with the fp16 reference branch the
 *               tensor core also adds the branch product onto the same accumulator.
 *
 * Every function returns an lq_status; nothing throws, aborts or prints.  "host" / "device"
 * in a parameter comment says which address space the pointer lives in.  Device pointers and
 * the stream belong to the caller (e.g. a torch tensor's data_ptr() and a torch stream's
 * cuda_stream); everything behind lq_layer* / lq_act* is allocated and owned by the library
 * and released by the matching _free call.  Calls that take a stream are asynchronous on it.
 * There is no CPU fallback: without a CUDA device the device-side calls return LQ_ERR_CUDA.
 */
#ifndef LQ_H_
#define LQ_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LQ_OK = 0,
  LQ_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, handle/shape mismatch          */
  LQ_ERR_UNSUPPORTED = 2, /* a size or format outside what the kernels are built for         */
  LQ_ERR_ALLOC = 3,       /* host or device allocation failed                                 */
  LQ_ERR_CUDA = 4,        /* a CUDA runtime/driver call failed (or no device)                 */
  LQ_ERR_TIMEOUT = 5,     /* a bounded device-side wait expired (see lq_get_device_status)    */
  LQ_ERR_NUMERIC = 6      /* non-finite value met where the method needs finite ones          */
} lq_status;

/* Precision of the low-rank branch: bits of the two factors (W) and of the activations that
 * enter it, incl. the rank-r intermediate (A).  Section 3.3 quantizes the branch with an
 * operator Q2; the integer per-token / per-channel variants are this build's configurations. */
typedef enum {
  LQ_BRANCH_NONE = 0,   /* rank 0: plain W4A4                                  */
  LQ_BRANCH_W16A16 = 1, /* fp16 factors, fp16 activations (reference variant)  */
  LQ_BRANCH_W8A8 = 2,
  LQ_BRANCH_W6A6 = 3,
  LQ_BRANCH_W4A8 = 4,
  /* MX branches of the mixed-precision study (Section 4.3, Tables 3-4; Appendix A.3 "MX Formats"): factors in
   * blocks of 32 with a power-of-two scale and e4m3 / e2m3 / e2m1 elements; the activations of BOTH branches and
   * the rank-r intermediate are MXFP8e4.  Only with main_fmt = LQ_MAIN_MXFP4. */
  LQ_BRANCH_MXFP8 = 5,
  LQ_BRANCH_MXFP6 = 6,
  LQ_BRANCH_MXFP4 = 7,
  /* Integer MX branches of the same study (Table 3's integer rows): factors in blocks of 32 with a power-of-two
   * scale and signed 8-bit / 4-bit integer codes; the activations of BOTH branches and the rank-r intermediate
   * are MXINT8.  Only with main_fmt = LQ_MAIN_MXINT4_A8; rank <= 64 with MXINT8 factors, <= 128 with MXINT4 factors. */
  LQ_BRANCH_MXINT8 = 8,
  LQ_BRANCH_MXINT4 = 9
} lq_branch_fmt;

/* 4-bit format of the residual (main) branch, Appendix A.3. */
typedef enum {
  LQ_MAIN_AUTO = 0,    /* from `group`: 64 -> SINT4 (integer codes, fp16 scale per 64), 32 -> MXINT4           */
  LQ_MAIN_MXFP4 = 2,   /* MXFP4e2 weights (e2m1 elements, power-of-two scale per 32; group must be 32) times
                          MXFP8e4 activations, all scales applied by the tensor core (Tables 3-4)              */
  LQ_MAIN_MXINT4_A8 = 3 /* MXINT4 weights (group must be 32) times MXINT8 activations (Table 3's integer rows): an
                          8-bit code travels as two 4-bit digits, code = 16 hi + lo, each an exact E4M3 operand
                          with block scales 2^(e+4) and 2^e, so the tensor core applies every scale here too    */
} lq_main_fmt;

/* Element format of the activations (X for both branches, and the rank-r intermediate) of an MXFP layer.  The rank
 * study of Section 4.3 (Table 4) gives activations and factors ONE sub-16-bit format: MXFP8e4, or MXFP6e2. */
typedef enum {
  LQ_ACT_DEFAULT = 0,  /* SINT4 / MXINT4 main formats: their own 4-bit activations; MXFP4: MXFP8e4; MXINT4_A8: MXINT8 */
  LQ_ACT_MXFP6 = 6     /* MXFP6e2 activations; only with main_fmt = LQ_MAIN_MXFP4 (the weights' kernels do not change:
                          every e2m3 value is an e4m3 value)                                                     */
} lq_act_fmt;

typedef enum { LQ_OUT_F16 = 0, LQ_OUT_F32 = 1 } lq_out_dtype;

/* One layer's shape and calibration settings. */
typedef struct {
  int32_t K, N, rank; /* d, n and rho of Sections 3.1-3.2; rank in [0, 128]; K and N multiples of 8,
                         K <= 8192 (anything else: LQ_ERR_UNSUPPORTED)                              */
  int32_t group;      /* 64 = SINT4 (default), 32 = MXINT4: block length of the 4-bit main format  */
  int32_t branch;     /* an lq_branch_fmt                                                         */
  int32_t steps;      /* Adam steps on (L, R); 1000 in Appendix A "Optimization"                  */
  float lr;           /* 1e-4 for integer formats (Appendix A)                                    */
  float beta1, beta2, eps; /* Adam moments / epsilon; the paper is silent: 0.9, 0.999, 1e-8       */
  int32_t rot_steps;  /* steps of the rotation-aware optimisation of Section 3.3; 0 (default) = none,  */
  float rot_lr;       /* 500 steps at 0.5 (0.1 for the mixed-precision study) in Appendix A           */
  uint64_t seed;      /* start vectors of the host SVD iteration                                  */
  int32_t main_fmt;   /* an lq_main_fmt; 0 (default) = SINT4 / MXINT4 as `group` says                */
  int32_t act_fmt;    /* an lq_act_fmt; 0 (default) = the main format's own activations                 */
} lq_config;

typedef struct lq_layer lq_layer; /* opaque: Q1(P) codes+scales, Q2(L1), Q2(L2), bias (Figure 1)  */
typedef struct lq_act lq_act;     /* opaque: device buffers holding one batch of quantized
                                     activations for one layer shape (qx, sx, qb, sXb, tq, sT)   */

/* Fill *cfg with the defaults above for the given shape. */
lq_status lq_config_default(lq_config* cfg, int32_t K, int32_t N, int32_t rank, int32_t branch);

/* Data-free calibration of one weight, entirely on the host (Sections 3.2-3.3, Appendix A,
 * Appendix B.2): SVD initialisation L = -L0, R = R0; Adam on
 * mean((Q1(W + L R) - W - L R)^2) with the quantizer's derivative taken as zero; the best
 * iterate is kept; with cfg->rot_steps > 0 an orthogonal rotation Om of the factors (L1 Om,
 * Om^T L2: the same product) is then optimised to lower Q2's error (Cayley retraction steps,
 * best iterate kept); the factors are quantized with Q2; P = W - Q2(L1) Q2(L2) is quantized
 * with Q1 (SINT4 or MXINT4 blocks along K per output column, as cfg->group says; MXINT4 weight
 * exponents are kept within [-24, 15] so that 2^e is a finite fp16 number).  With main_fmt = LQ_MAIN_MXFP4,
 * Q1 is MXFP4e2 and Q2 the branch's MXFP format (blocks of 32 along each factor's contraction axis; exponent
 * floor(log2 max) - emax as in the OCP Microscaling conversion the paper cites; no rotation step: rot_steps must be 0).
 * With main_fmt = LQ_MAIN_MXINT4_A8, Q1 is MXINT4 and Q2 the branch's MX integer format (blocks of 32 along each
 * factor's contraction axis, the smallest power-of-two scale that does not clip; rot_steps must be 0).
 *   W_f16_host     [K][N] row-major IEEE half bits (the paper's d x n orientation), host
 *   bias_f16_host  [N] half bits or NULL, host
 *   out            receives a new layer (host copy only; see lq_layer_to_device)
 *   objective_trace[steps + 1] doubles or NULL, host: objective at every iterate, [0] = init
 * Errors: INVALID_ARG (null / bad shape), UNSUPPORTED (group not 64 or 32, ...),
 * NUMERIC (non-finite W), ALLOC. */
lq_status lq_calibrate(const lq_config* cfg, const uint16_t* W_f16_host,
                       const uint16_t* bias_f16_host, lq_layer** out, double* objective_trace);

/* Build a layer from already quantized parts (all host pointers, copied):
 *   Wq_packed [K][N/2] bytes: codes in [-7,7] as two's-complement nibbles, column 2j in the
 *             low nibble, column 2j+1 in the high nibble
 *   sw        [G][N] half bits: scale of block g of output column n (MXINT4: an exact power of
 *             two 2^e with e in [-24, 15], anything else is INVALID_ARG)
 *   L1, L2    integer branches: int8 codes [K][rank] and [rank][N]; W16A16: half bits, same shapes
 *   sL1, sL2  fp32 per-column scales [rank] and [N]; NULL for W16A16
 *   bias      [N] half bits or NULL
 * With rank == 0 or LQ_BRANCH_NONE the branch pointers are ignored.
 * MXFP layers (main_fmt = LQ_MAIN_MXFP4):
 *   Wq_packed [K][N/2] bytes: e2m1 bit patterns (sign, two exponent bits, one mantissa bit) as nibbles, same order
 *   sw        [ceil(K/32)][N] half bits: the block's power-of-two scale 2^e, e in [-24, 15]
 *   L1, L2    [K][rank] and [rank][N] bytes: e4m3 bit patterns of the elements (every e2m3 and e2m1 value is an
 *             e4m3 value, so the three MXFP branch formats arrive in one encoding)
 *   sL1, sL2  fp32 powers of two: [ceil(K/32)][rank] (blocks of L1 along K) and [ceil(rank/32)][N] (of L2 along rank)
 * Integer MX layers with 8-bit activations (main_fmt = LQ_MAIN_MXINT4_A8): Wq_packed and sw as for MXINT4;
 *   L1, L2    int8 codes [K][rank] and [rank][N], within [-127, 127] (LQ_BRANCH_MXINT8) or [-7, 7] (LQ_BRANCH_MXINT4)
 *   sL1, sL2  fp32 powers of two 2^e, e in [-120, 120]: [ceil(K/32)][rank] and [ceil(rank/32)][N] */
lq_status lq_layer_import(const lq_config* cfg, const uint8_t* Wq_packed, const uint16_t* sw,
                          const void* L1, const float* sL1, const void* L2, const float* sL2,
                          const uint16_t* bias, lq_layer** out);

/* Copy a layer's parts out into caller-sized host buffers (same layouts as lq_layer_import;
 * any pointer may be NULL to skip that part). */
lq_status lq_layer_export(const lq_layer* layer, uint8_t* Wq_packed, uint16_t* sw, void* L1,
                          float* sL1, void* L2, float* sL2, uint16_t* bias);

/* Shape of a layer handle. */
lq_status lq_layer_info(const lq_layer* layer, lq_config* cfg_out);

/* Upload the layer to `device` in the kernels' operand layout (allocates device memory;
 * synchronous).  Must precede lq_act_create / lq_quantize_act / lq_linear_forward. */
lq_status lq_layer_to_device(lq_layer* layer, int device);

lq_status lq_layer_free(lq_layer* layer);

/* Allocate the activation record for up to M_max rows of `layer`'s shape on `device`. */
lq_status lq_act_create(const lq_layer* layer, int32_t M_max, int device, lq_act** out);
lq_status lq_act_free(lq_act* act);

/* Dynamic activation quantization fused with the branch's down-projection (Figure 1;
 * Appendix A.2 "Quantization": both the residual and the low-rank branch consume quantized X).
 * One read of X produces
 *   qx, sx   4-bit codes / scales per token and block along K (Appendix A.3): fp16 scales per
 *            block of 64 (SINT4) or one exponent byte per block of 32 (MXINT4)
 *   qb, sXb  per-token branch codes / fp32 scale
 *   tq, sT   per-token codes / scale of the rank-r intermediate T = deq(qb) deq(L1)
 *   X_f16_dev  [M][K] row-major half, device, 16-byte aligned
 *   M          1 <= M <= M_max of `out`
 * X must be finite: the kernel does not look for infinities or NaNs (a row that holds one gets an
 * undefined scale and codes; nothing is flagged).  LQ_ERR_NUMERIC is raised only by the host-side
 * calls, for non-finite weights or scales.
 * Asynchronous on `cuda_stream` (a cudaStream_t). */
lq_status lq_quantize_act(const lq_layer* layer, const void* X_f16_dev, int32_t M, lq_act* out,
                          void* cuda_stream);

/* Y = sum_g sx sw (qx_g Wq_g) + sT sL2 (tq L2q) + bias: the 4-bit main product per group on
 * the tensor cores, per-group scales and the branch's up-projection applied in one epilogue
 * (Figure 1; Section 3.3).  For an MXINT4 layer the tensor core applies sx sw itself and the
 * epilogue only adds the branch and the bias.
 *   act    result of lq_quantize_act for this layer
 *   Y_dev  [M][N] row-major, half or float per `dtype`, device, 16-byte aligned
 * A row's codes and scales depend on that row alone.  So does its Y for the MX formats; for SINT4 the fp32 sum over
 * the groups may be cut in two to eight parts where M is small, so Y of the same row may differ by rounding (some 1e-7
 * of the sum of the terms' magnitudes) between calls of different M - not between the row chunks of one host call.
 * Asynchronous on `cuda_stream`. */
lq_status lq_linear_forward(const lq_layer* layer, const lq_act* act, void* Y_dev,
                            lq_out_dtype dtype, void* cuda_stream);

/* Whole path from host memory: copies X to the device, runs lq_quantize_act and
 * lq_linear_forward, copies Y back and waits for it.  X_f16_host [M][K], Y_host [M][N].
 * Rows are independent, so for M >= 512 the call is pipelined over two to eight row chunks: one chunk
 * is computed on `cuda_stream` while the next travels host -> device and the previous one
 * device -> host on two internal copy streams (this needs pinned host memory to overlap;
 * pageable memory works but serialises).  Staging buffers, streams and events inside `act`
 * are created on the first call.  Afterwards `act` holds the codes of all M rows. */
lq_status lq_linear_forward_host(const lq_layer* layer, lq_act* act, const void* X_f16_host,
                                 int32_t M, void* Y_host, lq_out_dtype dtype, void* cuda_stream);

/* The same without the final wait: returns once everything is queued; Y_host is complete when
 * `cuda_stream` has been synchronised (the stream is made to wait for the last copy).  X_f16_host
 * and Y_host must be pinned and must stay valid until then.  Calls for different layers on
 * different streams (each with its own `act`) overlap their copies in both directions, which a
 * sequence of waiting calls cannot: one layer's output travels device -> host while the next
 * layer's input travels host -> device.  Figure 1's data flow; the paper has no counterpart for
 * the transport itself. */
lq_status lq_linear_forward_host_async(const lq_layer* layer, lq_act* act, const void* X_f16_host,
                                       int32_t M, void* Y_host, lq_out_dtype dtype, void* cuda_stream);

/* (The paper has no counterpart for this entry point; it exists for deployment.)
 * Same result as lq_quantize_act followed by lq_linear_forward, for callers that may not
 * allocate device memory when they call: servers whose own pool owns all device memory once
 * start-up is over, loops with a fixed memory budget, plugins inside a framework that owns the
 * allocator - a raw allocation there can fail, fragment the pool, and stalls every stream while
 * it synchronises the device.  This call performs no allocation (no cudaMalloc / cudaFree,
 * no allocating library routine): the activation record lives in one fixed device array of
 * LQ_STATIC_SCRATCH_BYTES that is part of the library image, so every GPU that loads the
 * library holds that much memory until the process exits.  The caller passes only inputs and
 * outputs:
 *   layer      uploaded with lq_layer_to_device (that earlier call is where the layer's
 *              own device memory was allocated)
 *   X_f16_dev  [M][K] row-major half, device, 16-byte aligned
 *   Y_dev      [M][N] row-major half or float per `dtype`, device, 16-byte aligned
 * Limit: with Mp = M rounded up to 128, Kp = K rounded up to 128 and G2 = Kp / 64, the record
 * needs about 2*Mp*Kp + 4*G2*Mp + 136*Mp bytes (each part rounded up to 256); if that exceeds
 * LQ_STATIC_SCRATCH_BYTES - or if the layer's main format is MXINT4, which this entry point
 * does not cover - the call returns LQ_ERR_UNSUPPORTED and launches nothing
 * (8 MiB holds e.g. M = 256 at any supported K, or M = 1024 at K = 2240).
 * The first call on each device looks up the array's device address (one-time set-up, done
 * with that device current); make that first call before starting any stream capture.
 * All calls share the one array, which keeps the previous call's contents: a call writes all of
 * the record that it reads, so nothing is cleared in between.  Two calls that overlap on the
 * GPU - other streams, other threads - race on the array; serialise them.  Asynchronous on
 * `cuda_stream`. */
#define LQ_STATIC_SCRATCH_BYTES (8u << 20)
lq_status lq_linear_forward_static(const lq_layer* layer, const void* X_f16_dev, int32_t M, void* Y_dev,
                                   lq_out_dtype dtype, void* cuda_stream);

/* ---- low-rank adapters of many requests beside a shared projection ----------------------------------------------
 * (The paper has one low-rank branch per layer, fixed at calibration.  A server that answers many requests with one
 * quantized layer adds each request's own fp16 branch to the shared output.)
 *
 *     Y[m] = Y0[m] + scale_a ( X[m] A_a ) B_a,     a = the adapter of row m, or none: Y[m] = Y0[m]
 *
 * lq_adapters holds up to `slots` adapters (A_a [K][r_a], B_a [r_a][N], scale_a) of projections of one shape on one
 * device; lq_rowmap says which adapter each row of a batch uses.  One map serves every projection of a step.        */
typedef struct lq_adapters lq_adapters;
typedef struct lq_rowmap lq_rowmap;

/* A set of `slots` empty adapters of rank up to max_rank for projections of K inputs and N outputs (allocates
 * 2 * slots * r * (K + N) bytes of device memory, r = max_rank rounded up to 16 or a multiple of 32; synchronous).
 * 1 <= slots <= 1023, 1 <= max_rank <= 128, K <= 8192, N <= 2^20, K and N multiples of 8; anything else is UNSUPPORTED. */
lq_status lq_adapters_create(int32_t K, int32_t N, int32_t max_rank, int32_t slots, int device, lq_adapters** out);
lq_status lq_adapters_free(lq_adapters* set);

/* Puts an adapter into a slot, or another one in its place; rank 0 empties the slot (A and B are then ignored).
 *   A_f16_dev  [K][rank] row-major half bits, device        B_f16_dev  [rank][N] row-major half bits, device
 *   scale      finite, below 2^96 in magnitude (UNSUPPORTED); applied to the product in fp32.  Where the scale times the largest entry of a
 *              row's X A is below 2^-111, what is added loses bits
 * The set keeps its own copy.  Asynchronous on `cuda_stream`: forwards queued there earlier use what was there before,
 * later ones the new adapter; forwards on other streams must be ordered by the caller.  May be captured. */
lq_status lq_adapters_set(lq_adapters* set, int32_t slot, int32_t rank, const void* A_f16_dev, const void* B_f16_dev, float scale,
                          void* cuda_stream);

/* A map of up to M_max rows to the slots 0 .. slots - 1 (1 <= slots <= 1023, M_max <= 2^24), with the workspace of the forwards
 * that use it (synchronous): 520 bytes a row. */
lq_status lq_rowmap_create(int32_t M_max, int32_t slots, int device, lq_rowmap** out);
lq_status lq_rowmap_free(lq_rowmap* map);

/* Sorts the rows by adapter (stable; on the device, so a captured graph sorts anew on each replay what the array then holds).
 *   row_adapter_dev  [M] int32, device: the slot of each row; anything outside 0 .. slots - 1 means none
 *   M                1 <= M <= M_max; the rows of every forward until the next call.  A replayed graph that sorts leaves its own rows in the
 *                    map: a forward of another M behind it needs a call before it (without one it writes nothing, and lq_get_device_status
 *                    says INVALID_ARG)
 * Asynchronous on `cuda_stream`. */
lq_status lq_rowmap_set(lq_rowmap* map, const int32_t* row_adapter_dev, int32_t M, void* cuda_stream);

/* Y = Y0 + the rows' adapters.  Products and sums in fp32; the rank-r intermediate travels as two halves under a power-of-two
 * scale of its row (22 bits of the row's largest entry); rounded once to `dtype`.  Beside an fp32 Y0 the result can be some four times
 * farther from the exact one than fp32 products and sums throughout (relative errors of 1e-7 to 4e-7), or nearer.
 *   X_f16_dev  [M][K] row-major half, device, 16-byte aligned, finite
 *   Y0_dev     [M][N] row-major half or float per `dtype`, device, 16-byte aligned: the projection's output
 *   Y_dev      the same shape and type: Y0_dev itself (rows without an adapter are then left alone) or memory apart from it
 *              (INVALID_ARG where they overlap otherwise), and apart from X
 * The map's slots must not be more than the set's, and map and set must be on one device.  No sum depends on the order of execution, so
 * equal calls give equal bits; a row may differ by rounding between calls of other M or other maps.
 * Calls that use one map, lq_rowmap_set among them, share its workspace: they must not overlap on the GPU (one stream, or events;
 * graphs that were captured with one map must not run side by side).  Asynchronous on `cuda_stream`. */
lq_status lq_adapters_forward(const lq_adapters* set, const lq_rowmap* map, const void* X_f16_dev, const void* Y0_dev, void* Y_dev,
                              lq_out_dtype dtype, void* cuda_stream);

/* ---- queries and keys behind a projection: norm of each head and rotation by position, in one pass ---------------
 * (Outside the paper's layer: what an attention block does with the output of its qkv projection.)                  */
typedef enum {
  LQ_NORM_NONE = 0,
  LQ_NORM_RMS = 1,        /* x / sqrt(mean x^2 + eps) * weight                       */
  LQ_NORM_LAYER = 2       /* (x - mean) / sqrt(var + eps) * weight + bias            */
} lq_norm;

#define LQ_ROPE_MAX_AXES 4
typedef struct {
  int32_t axes;                    /* 0 (no rotation) .. LQ_ROPE_MAX_AXES: e.g. 1 = text, 2 = rows and columns, 3 = time, height, width */
  int32_t dims[LQ_ROPE_MAX_AXES];  /* entries of a head that turn with each axis: even, >= 0; their sum, rot_dim, is what is rotated;
                                      the head's other entries, behind them, only see the norm                        */
  int32_t halves;                  /* 0: pair i is entries (2 i, 2 i + 1); 1: (i, i + rot_dim / 2), rot_dim a multiple of 8 */
  int32_t shared;                  /* 0: each axis has its own frequencies theta^(-2 j / dims[axis]), j from 0;
                                      1: pair i has theta^(-2 i / rot_dim), and the axes take dims[axis] / 2 pairs each in turn */
  double theta;                    /* > 0                                                                             */
} lq_rope_config;

typedef struct lq_rope lq_rope;    /* opaque: axis and frequency of each pair, on one device                          */

/* Fill *cfg: `axes` axes of dims[0 .. axes - 1] entries (host), neighbouring pairs, frequencies of each axis its own, theta 10000. */
lq_status lq_rope_config_default(lq_rope_config* cfg, int32_t axes, const int32_t* dims);

/* A table of rotations (synchronous).
 *   freq_host  NULL (frequencies as the configuration says) or rot_dim / 2 finite doubles, radians a position, pair by pair: scaled or
 *              interpolated frequencies.  Below 2^64 in magnitude, as must be the configuration's (UNSUPPORTED)
 *   axis_host  NULL or rot_dim / 2 axes, pair by pair (the configuration's dims then only give rot_dim)
 * Frequencies are kept as 64-bit fractions of a turn and multiplied by the position in integers: modulo a turn an angle is within 1.5e-9
 * radians of frequency times position at any position (theta below 1: times the frequency).  What is left of it beside the nearest quarter
 * turn becomes a float, within 1.4e-7 radians; cosine and sine are within 4 * 2^-24. */
lq_status lq_rope_create(const lq_rope_config* cfg, const double* freq_host, const int32_t* axis_host, int device, lq_rope** out);
lq_status lq_rope_free(lq_rope* rope);

/* The queries or the keys of a call.  Entry d of head h of row s of sequence b lies at b * seq + s * row + h * head + d elements. */
typedef struct {
  const void* in;                          /* device, 16-byte aligned; half or float per in_dtype                     */
  void* out;                               /* device, 16-byte aligned; half or float per out_dtype; `in` itself, with its strides and
                                              type (INVALID_ARG otherwise), or memory apart from all inputs           */
  int64_t in_seq, in_row, in_head;         /* strides in elements, multiples of 8, below 2^31, a head's below 2^26 (the memory they span
                                              may be larger)                                                          */
  int64_t out_seq, out_row, out_head;      /* no two outputs of the call on one place, none on an input (INVALID_ARG;
                                              UNSUPPORTED where dimensions run through one another too often to tell);
                                              may be negative, like those of `in`                                     */
  const float* weight;                     /* [head_dim] device, 16-byte aligned, or NULL (ones); NULL without a norm */
  const float* bias;                       /* [head_dim] device, 16-byte aligned, or NULL (zeros); LQ_NORM_LAYER only */
  int32_t heads;                           /* 1 .. 4096                                                               */
} lq_heads;

/* Norm of each head, then the rotation of its leading rot_dim entries: entries (u, v) of a pair become
 * (u cos - v sin, v cos + u sin) of the row's angle.  In fp32, rounded once to out_dtype.
 *   q, k       either may be NULL (no such heads)
 *   head_dim   a multiple of 8 up to 256, >= rot_dim
 *   sequences, seq_len   >= 1; rows = sequences * seq_len < 2^31
 *   pos_dev    [sequences][seq_len][axes] int32, any value, device; ignored (may be NULL) if the table has no axes
 * Writes nothing but the heads' entries: what lies between them (values of the same rows, say) stays.
 * Runs on the table's device.  Asynchronous on `cuda_stream`. */
lq_status lq_qk_norm_rope(const lq_heads* q, const lq_heads* k, int32_t head_dim, int32_t sequences, int32_t seq_len, lq_norm norm, float eps,
                          const lq_rope* rope, const int32_t* pos_dev, lq_out_dtype in_dtype, lq_out_dtype out_dtype, void* cuda_stream);

/* The queries, keys and values of an attention block in one call, three to five kernels on the stream: lq_quantize_act and
 * lq_linear_forward of a layer whose N output columns are q_heads heads of queries, kv_heads of keys and kv_heads of values; the rows'
 * adapters, if any, added to all of them; norm and rotation of the queries and keys, in place.  Equal to the bit to those calls one by one. */
typedef struct {
  int32_t head_dim, q_heads, kv_heads;     /* (q_heads + 2 kv_heads) head_dim = N                              */
  int32_t sequences;                       /* M = sequences * rows of each                                     */
  int32_t norm;                            /* an lq_norm                                                       */
  float eps;
  const float *q_weight, *k_weight;        /* as lq_heads.weight and .bias                                     */
  const float *q_bias, *k_bias;
  const lq_rope* rope;                     /* a table of no axes: no rotation                                  */
  const int32_t* pos_dev;                  /* [M][axes]                                                        */
} lq_qkv;

/*   act, X_f16_dev, M   as for lq_quantize_act
 *   set, map            the rows' adapters of this projection (set's K and N the layer's, map's rows M), or both NULL
 *   Y_dev               [M][N] row-major half or float per `dtype`, device, 16-byte aligned, apart from weights, biases and positions
 *                       and, with adapters, from X (INVALID_ARG)
 * Nothing is launched if an argument is refused.  Asynchronous on `cuda_stream`. */
lq_status lq_qkv_forward(const lq_layer* layer, lq_act* act, const void* X_f16_dev, int32_t M, const lq_adapters* set, const lq_rowmap* map,
                         const lq_qkv* qkv, void* Y_dev, lq_out_dtype dtype, void* cuda_stream);

/* ---- a cache of keys and values in 8 bits, and attention over it --------------------------------------------------
 * (Outside the paper's layer: what an attention block does with the rows that lq_qkv_forward has written.)
 *
 * Tokens are kept in pages of page_tokens, pages in any order; every 32 tokens of a head share one step 2^e for their keys and one
 * for their values, e the smallest integer in [-20, 9] with 127 * 2^e >= the largest magnitude written, and are stored as
 * rint(x / 2^e) in [-127, 127].  (What is beyond 127 * 2^9 = 65024 becomes that.)  Tokens that come to 32 which hold some already may
 * need a larger e': the codes c that are there become rint(c / 2^(e' - e)).  Every value c 2^e is a half.                          */
#define LQ_KV_BLOCK 32
#define LQ_KV_MAX_SEQUENCES 65535
typedef struct lq_kvcache lq_kvcache;

/* A cache of `layers` layers of `pages` pages each on one device (allocates layers * pages * page_tokens / 32 * kv_heads * (64 Dp + 32) bytes,
 * Dp = head_dim rounded up to 64, 80, 96, 112, 128, 192 or 256, and the attention's workspace; synchronous).  page_tokens a multiple of 32
 * up to 65536, kv_heads <= 4096, head_dim a multiple of 8 up to 256; anything else is UNSUPPORTED.  Holds zeros at first. */
lq_status lq_kvcache_create(int32_t layers, int32_t pages, int32_t page_tokens, int32_t kv_heads, int32_t head_dim, int device, lq_kvcache** out);
lq_status lq_kvcache_free(lq_kvcache* cache);

/* The sequences of a step, the same for every layer.  The arrays are device memory and are read when the kernels run, so a captured graph
 * goes by what they then hold.  A sequence that does not fit them (a length below 0, above its pages' or, where that matters, below its rows;
 * a page outside the cache) makes the kernels leave its tokens, or those of that page, out; lq_get_device_status then says INVALID_ARG. */
typedef struct {
  int32_t sequences;                       /* 1 .. LQ_KV_MAX_SEQUENCES                                                */
  int32_t rows;                            /* rows of the call's tensors, >= 0                                        */
  const int32_t* row_start;                /* [sequences + 1], not falling: sequence s has rows row_start[s] .. row_start[s + 1] - 1, its
                                              newest tokens in order (none is fine); rows behind row_start[sequences] are no sequence's
                                              and are left alone.  NULL: rows / sequences rows each                   */
  const int32_t* length;                   /* [sequences] tokens of each sequence, those of this step among them      */
  const int32_t* pages;                    /* [sequences][page_stride] pages of each sequence, from its first token on */
  int32_t page_stride;                     /* >= 1                                                                    */
} lq_kvbatch;

/* Keys and values as rows, or as an output.  Entry d of head h of row i lies at i * row + h * head + d elements (an output's of token i
 * of sequence s: s * seq more).  Pointers 16-byte aligned; strides multiples of 8, of less than 2^40 in magnitude. */
typedef struct {
  void *k, *v;                             /* device; half or float                                                   */
  int64_t k_seq, k_row, k_head;            /* (seq: of outputs alone)                                                 */
  int64_t v_seq, v_row, v_head;
} lq_kvrows;

/* Writes the batch's rows, finite keys and values, as each sequence's last tokens: tokens length - n .. length - 1 of one with n rows
 * (length >= n).  A token that is the first of its 32 begins them anew.  Pages that are written belong to one sequence of the batch.
 * kv_heads * ceil(rows / 32) < 2^31, else UNSUPPORTED.  Asynchronous on `cuda_stream`. */
lq_status lq_kvcache_append(lq_kvcache* cache, int32_t layer, const lq_kvbatch* batch, const lq_kvrows* rows, lq_out_dtype dtype, void* cuda_stream);

/* Reads tokens begin .. length - 1 of each sequence, at most max_tokens of them, into rows 0, 1, .. of its part of the output; what lies
 * behind stays.  Values are exact in either type.  Uses the batch's sequences, lengths and pages alone; rows and row_start have to be such as the
 * other calls take, and what row_start points to is not read (rows = 0 and NULL will do).
 *   begin_dev  [sequences] int32, device, >= 0; NULL: from the first token on
 *   rows       k or v may be NULL (not wanted); no two entries on one place and none on lengths, pages or begin_dev (INVALID_ARG;
 *              UNSUPPORTED where dimensions run through one another too often to tell)
 * kv_heads * sequences * (max_tokens / 32 + 2) < 2^31 (max_tokens, or page_stride * page_tokens where that is less), else UNSUPPORTED.
 * Asynchronous on `cuda_stream`. */
lq_status lq_kvcache_read(const lq_kvcache* cache, int32_t layer, const lq_kvbatch* batch, const int32_t* begin_dev, int32_t max_tokens,
                          const lq_kvrows* rows, lq_out_dtype dtype, void* cuda_stream);

typedef struct {
  const void* q;                           /* device, half, 16-byte aligned, finite: entry d of head h of row i at i * q_row + h * q_head + d */
  void* out;                               /* the same, of what the row's head attends to; apart from q and the batch's arrays, no two
                                              entries on one place (INVALID_ARG; UNSUPPORTED where it cannot be told) */
  int64_t q_row, q_head;                   /* strides in elements, multiples of 8, below 2^40 in magnitude            */
  int64_t out_row, out_head;
  int32_t q_heads;                         /* a multiple of the cache's heads, up to 4096: heads h * q_heads / kv_heads and on share head h   */
  int32_t causal;                          /* 1: row i of a sequence's n is token p = length - n + i (length >= n) and sees tokens 0 .. p;
                                              0: every row sees the whole sequence, of any length (0: the output is zeros) */
  int32_t window;                          /* with causal: > 0: of those the last `window` ones, p among them, and    */
  int32_t sinks;                           /* the sequence's first `sinks` (only with a window)                       */
  float scale;                             /* of the products, e.g. 1 / sqrt(head_dim); below 2^64 in magnitude       */
} lq_attn;

/* Attention of the batch's rows over what the cache holds: out = sum_j w_j v_j / sum_j w_j, w_j = exp(scale q . k_j), j over the tokens that
 * the row sees.  Products on the tensor cores from halves, sums in fp32; beside the values weights are rounded to halves, to 2^-11 of
 * each down to 2^-21 of the largest and by at most 2^-32 of that below.  One token a sequence, a few, whole prompts, or all of these in one batch.  No sum depends on the order of execution: equal calls give equal bits; a
 * row may differ by rounding between calls of other batches.
 * rows * q_heads / kv_heads <= 2^30, rows * q_heads <= 2^34.  Attention calls of one cache, of any of its layers, share its workspace: they
 * must not overlap on the GPU (one stream, or events; graphs that were captured with one cache must not run side by side).
 * Asynchronous on `cuda_stream`. */
lq_status lq_cache_attention(const lq_kvcache* cache, int32_t layer, const lq_kvbatch* batch, const lq_attn* attn, void* cuda_stream);

/* ---- the residual stream between two blocks: gate, sum and norms in one pass ---------------------------------------
 * (Outside the paper's layer: what lies between a block's last projection and the next one's lq_quantize_act.)
 *
 *     x' = x + factor * gate * N1(y),     h = (N2(x') * weight + bias) * (1 + scale) + shift                              */
typedef struct {
  const void* x;                           /* [rows][features], device: the stream                                    */
  const void* y;                           /* the block's output, or NULL: x' = x                                     */
  void* x_out;                             /* x', or NULL (not wanted); may be x itself, with its stride              */
  void* h;                                 /* the normed rows, or NULL; may be y itself, with its stride and type     */
  int64_t x_row, y_row, x_out_row, h_row;  /* strides of rows in elements, multiples of 8                             */
  const float* after_weight;               /* [features] of N1, or NULL (ones); NULL without that norm                */
  const float* weight;                     /* [features] of N2, or NULL (ones); NULL without that norm                */
  const float* bias;                       /* [features] or NULL; LQ_NORM_LAYER only                                  */
  const void *gate, *scale, *shift;        /* [features] for each sequence, mod_seq elements apart (a multiple of 8; 0: one for all), of
                                              mod_dtype; NULL: gate 1, scale 0, shift 0                               */
  int64_t mod_seq;
  int32_t rows, features, sequences;       /* rows = sequences * rows of each; features a multiple of 8 up to 8192    */
  int32_t after, norm;                     /* lq_norm of N1 and N2                                                    */
  int32_t x_dtype, y_dtype, h_dtype, mod_dtype;    /* lq_out_dtype; x_out's is x_dtype                                */
  float factor, eps;
  int32_t device;
} lq_residual;

/* All pointers 16-byte aligned; outputs on no input but in place as said (INVALID_ARG).  In fp32; h is made of x' before it is rounded.
 * Runs on r->device.  Asynchronous on `cuda_stream`. */
lq_status lq_residual_norm(const lq_residual* r, void* cuda_stream);

/* Decode the activation record of the last lq_quantize_act into plain host arrays (for
 * parity checks); NULL skips a part.  qx int8 [M][K], sx half bits [M][G] (MXINT4: the block
 * exponents e as int16 [M][G], since 2^e may lie below the fp16 range), qb int8 [M][K],
 * sXb float [M], tq int8 [M][rank] (W16A16: half bits [M][rank]), sT float [M].
 * MXFP: qx and tq are the e4m3 bytes, sT the block exponents of the intermediate as floats [M][ceil(rank/32)].
 * Integer MX with 8-bit activations: qx and tq are the int8 codes (16 hi + lo of the two stored digits), sx the
 * block exponents as for MXINT4, sT the block exponents of the intermediate as floats [M][ceil(rank/32)].
 * Synchronises `cuda_stream`. */
lq_status lq_act_export(const lq_act* act, int8_t* qx, uint16_t* sx, int8_t* qb, float* sXb,
                        void* tq, float* sT, void* cuda_stream);

/* Status word the kernels write when a bounded wait expires (or a map holds other rows than its forward's): code is an lq_status
 * (LQ_OK if none), stage identifies the waiting role.  Reading clears it.  Synchronises
 * the device. */
lq_status lq_get_device_status(int device, int32_t* code, int32_t* stage);

/* Self-test of the kernels' failure detection (the paper has no counterpart).  Every wait inside the
 * kernels is bounded: a role that waits longer than its limit records LQ_ERR_TIMEOUT and its
 * stage in the status word, and the kernel returns instead of hanging.  This call launches a
 * one-warp kernel that waits, with a limit of about 0.1 s, on a barrier that nothing ever arrives
 * on; afterwards lq_get_device_status must report {LQ_ERR_TIMEOUT, 4} and the device stays usable.
 * Asynchronous on `cuda_stream`. */
lq_status lq_selftest_wait_timeout(int device, void* cuda_stream);

/* Process-wide switches, read when a call is made; they are plain globals, so set them while no other
 * thread is inside the library (distinct handles may otherwise be used from distinct threads).
 *   "store_qb"     1: lq_quantize_act also writes the branch activation codes to HBM so that lq_act_export can
 *                  return them (parity tests); 0 (default): they stay on chip
 *   "gemm_ctas"    CTAs of the GEMM kernels; 0 (default) = one per SM
 *   "gemm_width"   columns of the MX GEMM's tiles: 64, 128, 160, 192 or 224 (with an integer branch at most 160, without one
 *                  not 160; a forward that cannot have the width returns INVALID_ARG); 0 (default) = chosen by the library
 *   "gemm_split"   1, 2, 4, 8: so many CTAs share a tile of the SINT4 GEMM where they fit; 0 (default): chosen by the launcher
 *   "gemm_pair"    1 (default): from 256 rows on, pairs of CTAs share an MX GEMM's tile; 0: never
 *   "quant_warps", "quant_ctas"   how the quantizer kernel is cut: row groups of 8 per tile (at most 8 count) and 128-value
 *                  stages of K per chunk; 0 = chosen by the library.  What a launch cannot have (more than 15 groups times stages,
 *                  more stages than K has) becomes the largest that it can, stages first
 *   "overlap"      1 (default): kernels are launched with programmatic stream serialization - a kernel's CTAs may take
 *                  their SMs and set up while the previous kernel on the stream drains, and wait (in the kernel) for
 *                  that kernel's completion before touching global memory; 0: plain launches
 *   "main_kind"    byte format that carries the 4-bit codes into the tensor cores; only 1 (E4M3) exists
 * Returns INVALID_ARG for an unknown name or value. */
lq_status lq_set_option(const char* name, int32_t value);

const char* lq_status_string(lq_status s);
/* Text of the last CUDA runtime error this host thread met inside the library ("no error" if none);
 * what LQ_ERR_CUDA stood for. */
const char* lq_last_cuda_error(void);
int lq_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LQ_H_ */
