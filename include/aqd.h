/*
 * aqd.h -- C ABI of libaqd: integer-only quantized convolution for GB300 (sm_103a).
 *
 * Implements the inference path of AQD (Chen et al., "AQD: Towards Accurate Quantized
 * Object Detection", arXiv 2007.06919, Sec. 3.2): convolution on low-bit integer codes
 * (Eq. 4) followed by a fused integer epilogue -- the folded batch-norm bias (Eq. 6,
 * optionally one parameter set per FPN level for multi-level BN, Sec. 3.2.2 / Fig. 3),
 * the dyadically rescaled skip add (Eq. 7 with F of Eq. 8), and the fixed-point rescale,
 * round and clip that produce the next layer's k-bit codes (Eq. 2). No floating point
 * value crosses a layer boundary.
 *
 * Conventions for every entry point
 *   - Pointers inside aqd_tensor / parameter structs are DEVICE pointers owned by the
 *     caller; the structs themselves live in host memory and are read before return.
 *   - `stream` is a cudaStream_t (NULL = legacy default stream). Work is enqueued on it;
 *     no entry point synchronizes except aqd_device_status.
 *   - The library allocates no device memory. Errors come back as aqd_status; argument
 *     errors are detected before any launch and launch nothing. C++ exceptions never
 *     cross this boundary. aqd_last_error() gives a message for the calling thread.
 *   - Device-side failures (a bounded wait that timed out, a failed device check) are
 *     latched in a device status word that aqd_device_status() reads and clears.
 *
 * Tensor layout (NHWC, one "row" = the C channels of one pixel)
 *   bits 2, 4, 8 (unsigned codes, Eq. 2 range [0, 2^k - 1]):
 *     a row is a run of 32-bit little-endian words; word w holds channels [w*q, (w+1)*q)
 *     with q = 32/bits, and channel i of its word sits at bit 8*(i%4) + bits*(i/4).
 *     bits 8 is plain bytes. bits 2 and 4 need C % 32 == 0.
 *   bits 3: each group of 32 channels takes 12 bytes = 3 words; words 0 and 1 hold the
 *     low 2 bits of channels 0..15 and 16..31 in the 2-bit layout, word 2 holds bit 2 of
 *     channel i at bit 8*(i%4) + i/4. Needs C % 32 == 0.
 *   bits 32: one int32 per channel (accumulator-domain values, e.g. detection-head
 *     outputs whose scale is passed on to the next stage, Sec. 3.2.1).
 *   Rows are contiguous: pixel (n, h, w) starts at byte ((n*H + h)*W + w) * row_bytes.
 *   Code tensors must be 16-byte aligned.
 *
 * Arithmetic of one output element (all integer; rhu(v, R) = floor((v + 2^(R-1)) / 2^R),
 * rhu(v, 0) = v; sat32 saturates to int32):
 *   acc = sum_{r,s,c} x[n, ho*S - P + r, wo*S - P + s, c] * w[co, r, s, c]   (Eq. 4;
 *         taps outside the image read code 0, the zero point of Eq. 2)
 *   t   = acc + bias[l][co]                                                   (Eq. 6)
 *   with a skip tensor s (Eq. 7, F(m, n) = c / 2^d of Eq. 8):
 *     scale_main = 0 (skip coarser): t = t + rhu(s * c[l][co], d[l][co])
 *     scale_main = 1 (main coarser): t = rhu(sat32(t) * c[l][co], d[l][co]) + s
 *   u   = sat32(t)
 *   out = u                                            for 32-bit outputs
 *   out = min(max(rhu(u * M0[l][co], 31 + shift[l][co]), 0), 2^k - 1)   for k-bit codes
 *         (Eq. 2 applied to the BN output; the clip at 0 is the ReLU)
 * Weights: signed integers w, either k-bit two's complement (AQD_W_TWOS) or Eq. 3's
 * unsigned eta_w standing for 2*eta_w - (2^k - 1) (AQD_W_ODD, the odd grid of Eq. 4).
 */
#ifndef AQD_H
#define AQD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef void* aqd_stream_t; /* a cudaStream_t */

typedef enum {
  AQD_OK = 0,
  AQD_ERR_INVALID = 1,      /* bad argument; nothing launched */
  AQD_ERR_UNSUPPORTED = 2,  /* valid but outside what the kernels implement */
  AQD_ERR_CUDA = 3,         /* a CUDA runtime call failed */
  AQD_ERR_TIMEOUT = 4,      /* a bounded device-side wait expired (device status) */
  AQD_ERR_DEVICE_CHECK = 5  /* a device-side consistency check failed (device status) */
} aqd_status;

enum { AQD_W_TWOS = 0, AQD_W_ODD = 1 };

typedef struct {
  int32_t n, h, w, c; /* logical NHWC shape */
  int32_t bits;       /* 2, 3, 4, 8: packed unsigned codes; 32: int32 values */
  void* data;         /* device pointer, layout above */
} aqd_tensor;

/* Per-(level, output channel) requant tables, each [levels][cout] row-major (Eq. 6, the
 * multi-level BN of Sec. 3.2.2 keeps one row per FPN level over shared weights).
 * m0/shift may be NULL when the output is 32-bit; bias may be NULL (all zero).
 * shift must lie in [-31, 31] (total right shift 31 + shift in [0, 62]). */
typedef struct {
  const int32_t* m0;
  const int8_t* shift;
  const int32_t* bias;
  int32_t levels;
} aqd_requant_params;

/* Skip-add rescale of Eq. 7/8, tables [levels][cout]: c any int32, d in [0, 62].
 * upsample = 2 reads the skip at (h/2, w/2): the nearest 2x interpolation of the FPN
 * top-down path (Sec. 3.2.3 occasion 3 with Sec. 3.2.4). */
typedef struct {
  const int32_t* c;
  const int8_t* d;
  int32_t upsample;   /* 1 or 2 */
  int32_t scale_main; /* 0: the skip is rescaled; 1: the main branch is rescaled */
} aqd_skip_params;

/* Prepared weights: written once by aqd_conv_prepare_weights, read by every conv call. */
typedef struct {
  const void* data; /* device buffer of aqd_conv_weights_bytes() bytes, 256-byte aligned */
  int32_t cout, kh, kw, cin;
  int32_t w_bits;   /* 2, 3, 4 or 8 */
  int32_t w_format; /* AQD_W_TWOS or AQD_W_ODD */
} aqd_conv_weights;

/* One image group of a grouped convolution (e.g. one FPN level). */
typedef struct {
  aqd_tensor x;    /* input codes */
  aqd_tensor y;    /* output: codes or int32 */
  aqd_tensor skip; /* skip operand; skip.data == NULL means no skip for this job */
  int32_t level;   /* row of the requant / skip tables */
} aqd_conv_job;

/* ---- host helpers ---------------------------------------------------------------- */

/* Bytes of one packed row of c channels at `bits`, or -1 if the layout does not exist. */
int64_t aqd_row_bytes(int32_t c, int32_t bits);

/* Eq. 8: the dyadic approximation m0 * 2^-(31 + shift) of `real` with |m0| < 2^31 and
 * 31 + shift in [0, 62] that minimizes the absolute error (largest shift whose
 * round-half-up m0 still fits). real = 0 gives (0, 0). Host only; no device work. */
aqd_status aqd_quantize_multiplier(double real, int32_t* m0, int8_t* shift);

const char* aqd_status_string(aqd_status s);
const char* aqd_last_error(void);

/* Reads and clears the device status word of the current device (synchronizes the
 * stream). *code receives AQD_OK or the first latched AQD_ERR_TIMEOUT /
 * AQD_ERR_DEVICE_CHECK. */
aqd_status aqd_device_status(aqd_stream_t stream, int32_t* code);

/* Diagnostics: force the convolution kernel (0 = automatic choice, 1 = tensor-core
 * kernel when the shape allows it, 2 = CUDA-core kernel, 3 = as 1 but never on CTA
 * pairs, 4 = as 1 but never on the FP4 pipe, 5 = as 1 but on neither); returns the previous
 * setting, or -1 for an unknown value. aqd_last_conv_path() reports the kernel the calling thread's last
 * successful conv call used (1 tensor core unpacking in-kernel, 2 CUDA core, 3 tensor core
 * fed from the expanded workspace, 4 the same on CTA pairs sharing each weight tile, 5 the
 * F16 tensor-core kernel of a network's first conv on a 3-channel 8-bit image with a 7x7
 * kernel, 6 the FP4 tensor-core pipe for 2-bit codes, 0 none yet). Forcing 2 also turns
 * paths 5 and 6 off.
 *
 * The FP4 pipe (path 6, kind::mxf4nvf4 with unit block scales) takes 2-bit activation codes
 * with weights |w| <= 4 (2-bit two's complement or Eq. 3's odd grid, 3-bit two's complement),
 * cin % 256 == 0 and at most 240 output channels per tile, on the workspace path, in
 * aqd_conv_int / aqd_conv_int_grouped (which expand their own input) and for the last layer
 * of aqd_conv_int_grouped_tower; each code and weight is the E2M1 value n / 2, w / 2, so
 * every product is exact and the FP32 sum is 1/4 of the integer sum, as exact as the E4M3
 * embedding. The split calls (expand / expanded / chain) always use byte images. */
int32_t aqd_set_conv_path(int32_t path);
int32_t aqd_last_conv_path(void);

/* Diagnostics (the paper has no counterpart): exercises the device-side failure path that
 * every tensor-core kernel uses, without faulting anything. One thread waits, with the
 * kernels' bounded mbarrier wait shortened to 2 ms, on a barrier that nobody arrives at; the
 * wait expires and latches AQD_ERR_TIMEOUT in the device status word; a second thread,
 * waiting the kernels' full 1 s limit on another such barrier, leaves through the kernel's
 * shared abort flag. out: 5 int64 in device memory, written by the kernel:
 * [0] 1 if the short wait expired, [1] its duration in ns, [2] 1 if the second wait
 * returned without its phase, [3] its duration in ns, [4] 1 if a control barrier whose
 * phase completed was seen as complete, and two sets of warps that take a loop's tiles in
 * turn, one of which loses a wait, met at every barrier of that loop. The next aqd_device_status() returns
 * AQD_ERR_TIMEOUT once and clears it. */
aqd_status aqd_selftest_wait_timeout(int64_t* out, aqd_stream_t stream);

/* ---- codes <-> int32 ----------------------------------------------------------- */

/* Packs rows x c int32 codes (device) into the k-bit layout (low k bits of each value;
 * signed weights therefore pack as two's complement). bits 2/3/4/8. */
aqd_status aqd_pack_codes(const int32_t* codes, int64_t rows, int32_t c, int32_t bits,
                          void* out, aqd_stream_t stream);
/* Inverse of aqd_pack_codes; is_signed sign-extends two's-complement fields. */
aqd_status aqd_unpack_codes(const void* packed, int64_t rows, int32_t c, int32_t bits,
                            int32_t is_signed, int32_t* out, aqd_stream_t stream);

/* ---- convolution (Eq. 4 + fused epilogue) ----------------------------------------- */

/* Size of the prepared-weights buffer for a [cout][kh][kw][cin] kernel. */
size_t aqd_conv_weights_bytes(int32_t cout, int32_t kh, int32_t kw, int32_t cin);

/* Converts packed signed weights [cout][kh][kw][cin] (rows packed along cin in the
 * w_bits layout) into the prepared layout at w->data (the struct's shape fields must be
 * filled in). Done once per model load; conv calls then read the prepared form. */
aqd_status aqd_conv_prepare_weights(const void* w_packed, const aqd_conv_weights* w,
                                    void* w_prepared, size_t bytes, aqd_stream_t stream);

/* One convolution y = epilogue(conv(x, w)) at the given level of the tables.
 * skip may be NULL (no skip; sp ignored). y->bits selects the output: 2/3/4/8 codes or
 * 32 (int32, rq->m0/shift unused). rq may be NULL only for 32-bit outputs (no bias).
 * workspace (device, 256-byte aligned, owned by the caller, contents not preserved) may be
 * NULL; see aqd_conv_workspace_bytes. Results are identical with and without it. */
aqd_status aqd_conv_int(const aqd_tensor* x, const aqd_conv_weights* w, int32_t stride,
                        int32_t pad, int32_t level, const aqd_requant_params* rq,
                        const aqd_tensor* skip, const aqd_skip_params* sp, aqd_tensor* y,
                        void* workspace, size_t ws_bytes, aqd_stream_t stream);

/* The same convolution over up to 8 jobs with shared weights in ONE launch: the shared
 * detector head applied to every FPN level, each with its own level's BN row. All jobs
 * share x->c, y->bits, skip presence and the weights; spatial sizes and batch differ. */
aqd_status aqd_conv_int_grouped(const aqd_conv_job* jobs, int32_t njobs,
                                const aqd_conv_weights* w, int32_t stride, int32_t pad,
                                const aqd_requant_params* rq, const aqd_skip_params* sp,
                                void* workspace, size_t ws_bytes, aqd_stream_t stream);

/* Workspace that lets a convolution expand its packed input codes once into a zero-padded
 * byte image (one byte per code, two per 8-bit code: sum over jobs of
 * n*(h+2*pad)*(w+2*pad)*cin bytes, twice that at 8 bits) and feed the tensor cores from it with TMA tile loads, instead of unpacking every code once per
 * kernel tap inside the convolution. Returns 0 when this path does not apply (stride != 1,
 * cin % 64 != 0, codes or weights wider than 4 bits with cin % 128 != 0, K * 3825 >= 2^24
 * with 8-bit codes or weights); a NULL or smaller workspace passed
 * to the conv calls then selects the in-kernel unpacking path. */
size_t aqd_conv_workspace_bytes(const aqd_conv_job* jobs, int32_t njobs,
                                const aqd_conv_weights* w, int32_t stride, int32_t pad);

/* The two steps of the workspace path as separate calls, for callers that expand an input
 * once and convolve it more than once (e.g. two heads over one feature map) or time the
 * steps apart. aqd_conv_expand_input writes the byte image of the jobs' inputs (only x of
 * each job is read; y, skip and level are ignored). aqd_conv_int_grouped_expanded is
 * aqd_conv_int_grouped reading that image: `workspace` must hold the expansion of exactly
 * these jobs' inputs, for the same weights' geometry, stride and pad, written by an
 * earlier aqd_conv_expand_input on this stream. That image does not depend on the weights' bits or
 * format: weights of any width may read it. Both need the workspace path to apply
 * (aqd_conv_workspace_bytes > 0) and a large enough workspace: otherwise AQD_ERR_INVALID,
 * or AQD_ERR_UNSUPPORTED when the tensor-core kernel does not take the convolution. */
aqd_status aqd_conv_expand_input(const aqd_conv_job* jobs, int32_t njobs, const aqd_conv_weights* w,
                                 int32_t stride, int32_t pad, void* workspace, size_t ws_bytes,
                                 aqd_stream_t stream);
aqd_status aqd_conv_int_grouped_expanded(const aqd_conv_job* jobs, int32_t njobs,
                                         const aqd_conv_weights* w, int32_t stride, int32_t pad,
                                         const aqd_requant_params* rq, const aqd_skip_params* sp,
                                         void* workspace, size_t ws_bytes, aqd_stream_t stream);

/* Layer chaining on the workspace path: aqd_conv_int_grouped_expanded that, besides the
 * packed k-bit outputs y (k = 2, 3 or 4), writes the same codes one byte each into
 * `next_workspace` as the zero-padded byte image that a following stride-1 convolution
 * with padding `next_pad` over these outputs reads (the layout aqd_conv_expand_input
 * writes for inputs of the outputs' shape, jobs in the same order), so that convolution
 * can be called with aqd_conv_int_grouped_expanded (or this function) without an
 * expansion pass. Only the interior of the image is written: its border must already hold
 * zeros (fill next_workspace with zeros once, or expand an input of the same shape into it
 * once; no call writes the border afterwards). Needs cout % 64 == 0, a next_workspace of
 * at least sum(n * (ho + 2 next_pad) * (wo + 2 next_pad)) * cout bytes, 256-byte aligned
 * and not overlapping `workspace`; otherwise AQD_ERR_INVALID. The paper's layers pass
 * k-bit codes from one layer to the next (Eq. 2, Fig. 1); this is the same codes stored one
 * per byte for the tensor cores. */
aqd_status aqd_conv_int_grouped_chain(const aqd_conv_job* jobs, int32_t njobs,
                                      const aqd_conv_weights* w, int32_t stride, int32_t pad,
                                      const aqd_requant_params* rq, const aqd_skip_params* sp,
                                      void* workspace, size_t ws_bytes, int32_t next_pad,
                                      void* next_workspace, size_t next_ws_bytes, aqd_stream_t stream);

/* ---- a chained tower, layers overlapped tile by tile -------------------------------- */

/* Bytes of per-tile counters that aqd_conv_int_grouped_tower needs to overlap its layers:
 * 4 x (layers - 1) x the tiles of one layer (256 output positions of the padded-width grid
 * per tile). 0 for invalid arguments or a single layer. */
size_t aqd_conv_tower_sync_bytes(const aqd_conv_job* jobs, int32_t njobs, int32_t layers, int32_t pad);

/* Runs `layers` grouped stride-1 convolutions in a chain, as the shared detector head applies
 * its tower to every FPN level (Sec. 3.2.2, Fig. 3: one weight set per layer, one parameter
 * row per level): layer i is Eq. 4 -> Eq. 6 -> Eq. 2 (no skip) of w[i] and rq[i] on layer
 * i-1's output codes.
 *   jobs: layers x njobs, row-major: jobs[i * njobs + j] is job j of layer i; its x must be
 *     jobs[(i-1) * njobs + j].y (same data pointer and shape) for i > 0; skip must be empty.
 *     Every layer keeps the spatial size: w[i].kh = w[i].kw = 2 pad + 1.
 *   Layers 0 .. layers-2 write 2/3/4-bit codes (their packed y, and, in the same epilogue,
 *     the next layer's zero-padded byte image); the last layer any output (int32 heads).
 *   ws_a, ws_b: two expanded-activation workspaces of ws_bytes each (256-byte aligned, each
 *     at least aqd_conv_workspace_bytes of every layer); layer i reads ws_a for even i, ws_b
 *     for odd i. input_expanded == 0: the call expands layer 0's input into ws_a first
 *     (aqd_conv_expand_input); nonzero: ws_a already holds it (written by that call, or by a
 *     chained previous layer). The call never writes ws_b's zero border: zero ws_b once
 *     before its first use.
 *   sync: device counters of aqd_conv_tower_sync_bytes() bytes (4-byte aligned), cleared on
 *     `stream` by the call's first kernel. With sync given, the longest leading run of
 *     layers of one shape (same weight geometry and code widths, at most 4, each running on
 *     CTA pairs with one output-channel tile, cout <= 256) runs as ONE persistent launch in
 *     layer-major tile order: each tile waits (a bounded wait, AQD_ERR_TIMEOUT on expiry)
 *     only for the tiles of the previous layer whose rows it reads. The remaining layers,
 *     and every layer when sync is NULL, run one launch each, each waiting for the whole
 *     previous launch. Calls that share sync or the workspaces must not overlap in time.
 * Every layer is validated before anything is launched; an error names the layer. */
aqd_status aqd_conv_int_grouped_tower(const aqd_conv_job* jobs, int32_t njobs, int32_t layers,
                                      const aqd_conv_weights* w, const aqd_requant_params* rq, int32_t pad,
                                      void* ws_a, void* ws_b, size_t ws_bytes, void* sync, size_t sync_bytes,
                                      int32_t input_expanded, aqd_stream_t stream);

/* ---- convolution without a caller workspace ---------------------------------------- */

/* Size of the library's own expanded-activation workspace (16 MiB per device context). */
#define AQD_STATIC_WORKSPACE_BYTES (16u << 20)

/* aqd_conv_int on the expanded-activation workspace path, with the workspace taken from a
 * fixed array inside the library instead of from the caller; it allocates nothing. The
 * paper has no counterpart: this exists for callers that cannot allocate device memory
 * (a serving loop whose device memory was all reserved at start-up, a host plugin without
 * an allocator of its own). Results are the same bytes as aqd_conv_int with a workspace.
 * The first call on a device looks the array up (cudaGetSymbolAddress); make it before any
 * stream capture. Every call on a device shares the one array: calls that overlap in time
 * (other streams, other host threads) race on it and must be ordered by the caller;
 * nothing in it needs to start at zero (each call writes every byte it reads).
 * The array's address is looked up once per (device, context): a context created later on
 * the same device (after cudaDeviceReset) gets its own lookup on its first call.
 * Argument errors return AQD_ERR_INVALID as aqd_conv_int does. Returns AQD_ERR_UNSUPPORTED,
 * launching nothing, whenever the call would not run on the workspace path: the path does
 * not apply (aqd_conv_workspace_bytes would be 0), the kernel choice would take a kernel
 * that reads no workspace (8-bit codes with a skip, or a forced CUDA-core path), or the
 * problem needs more than AQD_STATIC_WORKSPACE_BYTES. */
aqd_status aqd_conv_int_static_workspace(const aqd_tensor* x, const aqd_conv_weights* w, int32_t stride,
                                         int32_t pad, int32_t level, const aqd_requant_params* rq,
                                         const aqd_tensor* skip, const aqd_skip_params* sp, aqd_tensor* y,
                                         aqd_stream_t stream);

/* ---- training side (Sec. 3.1.2, Sec. 3.2.2) --------------------------------------- */

/* The quantizers with learnable intervals. weight = 0: Eq. 2 on activations,
 *   eta = round(clip(x / nu, 0, 1) (2^b - 1)), y = eta nu / (2^b - 1);
 * weight = 1: Eq. 3 on weights,
 *   eta = round((clip(w / nu, -1, 1) + 1) / 2 (2^b - 1)), y = (2 eta / (2^b - 1) - 1) nu.
 * "round" is half-up. Every code is decided in float32 in that order (one correctly rounded
 * division x / nu, the clip, the products, floor(v + 0.5); no fused multiply-add), so a float32
 * restatement of the equations gives the same codes and values. x, y: n float32 (device,
 * 4-byte aligned; 16-byte alignment takes vector loads); codes: n uint8 codes eta or NULL;
 * y may be NULL when codes is given. bits 1..8, nu > 0. */
aqd_status aqd_fake_quant(const float* x, int64_t n, float nu, int32_t bits, int32_t weight, float* y,
                          uint8_t* codes, aqd_stream_t stream);

/* The Straight-Through Estimator backward of aqd_fake_quant (the rounding's derivative taken
 * as 1). gx = gy where the value lies inside the clip range (0 < x / nu < 1 for Eq. 2,
 * -1 < w / nu < 1 for Eq. 3), else 0 (gx may be NULL). *gnu (one device float64) =
 * sum of gy * d y / d nu with d y / d nu = eta / Q - x / nu inside, 1 above, 0 below (Eq. 2) and
 * 2 eta / Q - 1 - w / nu inside, 1 above, -1 below (Eq. 3), Q = 2^b - 1: float32 within runs of
 * a thread, float64 across threads, a fixed order across blocks (deterministic).
 * workspace: aqd_fake_quant_backward_workspace_bytes() bytes, 8-byte aligned. */
size_t aqd_fake_quant_backward_workspace_bytes(void);
aqd_status aqd_fake_quant_backward(const float* x, const float* gy, int64_t n, float nu, int32_t bits, int32_t weight,
                                   float* gx, double* gnu, void* workspace, size_t ws_bytes, aqd_stream_t stream);

/* Batch statistics of the multi-level BN (Sec. 3.2.2, Fig. 3: one BN per FPN level over a
 * shared head) during training: for level l, the per-channel mean and biased variance of the
 * float32 tensor z[l] ([pixels[l]][c], channels last, device) over all its pixels, written as
 * float64 mean[l][c], var[l][c] (device). z and pixels are host arrays of `levels` (1..8)
 * entries. Sums are shifted by the level's first pixel, float32 over runs of 32 pixels and
 * float64 beyond. workspace: aqd_bn_level_stats_workspace_bytes(levels, c) bytes (0 for
 * invalid arguments), 8-byte aligned. */
size_t aqd_bn_level_stats_workspace_bytes(int32_t levels, int32_t c);
aqd_status aqd_bn_level_stats(const float* const* z, const int64_t* pixels, int32_t levels, int32_t c, double* mean,
                              double* var, void* workspace, size_t ws_bytes, aqd_stream_t stream);

/* ---- 8-bit language-model operators -------------------------------------------------- */

/* The quantized path of a decoder's feed-forward and output layers beside the convolutions: every
 * token's activations become int8 codes with one float32 scale per token (value = code * scale, Eq. 1's
 * uniform quantizer with the interval taken from the row), layers multiply codes exactly as integers
 * (Eq. 4), and the two scales return once per output. The paper's own layers are convolutions; these are the
 * same quantizer and product on matrices of tokens.
 *
 * Matrices are row-major with a row stride in elements (ld); elements of a row are adjacent. Types: */
enum { AQD_F32 = 0, AQD_F16 = 1, AQD_BF16 = 2, AQD_I32 = 3 };

/* Where the quantizers write rows of 8-bit codes. codes or values may be NULL, not both. */
typedef struct {
  int8_t* codes;        /* [rows][ld_codes], in [-127, 127] */
  int64_t ld_codes;
  float* scales;        /* [rows] */
  void* values;         /* the values that the codes stand for, code * scale rounded to values_dtype */
  int64_t ld_values;
  int32_t values_dtype; /* AQD_F32, AQD_F16 or AQD_BF16 */
} aqd_row_codes;

/* How a row u of float32 values becomes codes: a = max |u_k|, scale = a / 127, code = u / scale
 * rounded to nearest, ties to even (computed as u * (127 / a)). A row with a < 2^-120 (under the norm: with every
 * |h_k weight_k| below that) has scale 0 and codes 0. A row
 * that holds a NaN or an infinity (or, under the norm, whose sum of squares passes float32's range)
 * has scale NaN, codes 0 and values NaN, so the products that read it give NaN.
 * All pointers are device pointers aligned to their element; rows that start at 16-byte boundaries
 * take vector accesses. cols >= 1; rows may be 0. Every row stride of an output must be >= cols; an
 * input's may be any value >= 0. Outputs do not overlap inputs, except where said. */

/* u = x. */
aqd_status aqd_quant_rows(int64_t rows, int32_t cols, const void* x, int64_t ldx, int32_t dtype,
                          const aqd_row_codes* out, aqd_stream_t stream);

/* The norm before a layer, with the residual's addition: h = x + residual (residual NULL: h = x),
 *   u_k = h_k / sqrt(mean(h^2) + eps) * weight_k,
 * in float32 throughout; `sum` (NULL: not wanted) receives h rounded to `dtype`, the type of x, residual
 * and sum; the norm reads the unrounded h. sum may be x or residual itself (same pointer and ld): the residual
 * stream updated in place. weight: cols values of weight_dtype. eps >= 0; with eps = 0 rows whose squares lie below
 * float32's range are normalized like others. */
typedef struct {
  int64_t rows;
  int32_t cols, dtype;
  const void* x;
  int64_t ldx;
  const void* residual;
  int64_t ld_residual;
  void* sum;
  int64_t ld_sum;
  const void* weight;
  int32_t weight_dtype;
  float eps;
} aqd_rms_norm_args;
aqd_status aqd_rms_norm_quant(const aqd_rms_norm_args* args, const aqd_row_codes* out, aqd_stream_t stream);

/* Between a gated feed-forward's products: u = act(gate) * up in float32. act: AQD_ACT_SILU,
 * g / (1 + e^-g), or AQD_ACT_GELU_TANH, g/2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))). gate and up are matrices of
 * one type (two halves of one product's output, say: same ld, up = gate + cols). */
enum { AQD_ACT_SILU = 0, AQD_ACT_GELU_TANH = 1 };
typedef struct {
  int64_t rows;
  int32_t cols, dtype;
  const void* gate;
  int64_t ld_gate;
  const void* up;
  int64_t ld_up;
  int32_t act;
} aqd_gated_act_args;
aqd_status aqd_gated_act_quant(const aqd_gated_act_args* args, const aqd_row_codes* out, aqd_stream_t stream);

/* Prepared weights of an 8-bit layer: n output channels of k int8 codes and a scale per channel. */
typedef struct {
  const void* data;    /* device buffer of aqd_linear_weights_bytes(n, k) bytes, 256-byte aligned */
  const float* scales; /* [n] (device; read by every call, not copied) */
  int32_t n, k;
} aqd_linear_weights;

/* Size of the prepared-weights buffer; 0 for sizes that are not supported (n or k < 1, k > 131,071, beyond which
 * a sum of k products of two int8 codes could pass int32, or over 2^40 bytes). */
size_t aqd_linear_weights_bytes(int32_t n, int32_t k);
/* Lays codes[n][ld] (any int8 values) out at w->data, once per model load. */
aqd_status aqd_linear_prepare_weights(const int8_t* codes, int64_t ld, const aqd_linear_weights* w, void* prepared,
                                      size_t bytes, aqd_stream_t stream);

/* y[m][n] = (sum_k x[m][k] w[n][k]) * x_scale[m] * w_scale[n] + bias[n]: the sum is the exact int32,
 * converted to float32 once, then the products in this order and the addition in float32, rounded once to y_dtype. bias (float32) may be
 * NULL. With y_dtype AQD_I32, y receives the integer sums and x_scale, the weights' scales and bias are not read.
 * x: int8 codes, any ldx >= 0. workspace: aqd_linear_workspace_bytes(m, w) bytes or more, 256-byte aligned,
 * or NULL; its contents do not matter, and calls that share it must not overlap in time. Results are identical with
 * and without it: with more than 16 tokens, or rows of codes that are not 16-byte aligned, it may hold the codes as the kernels read
 * them, and a call without it runs on slower ones. */
typedef struct {
  int64_t m;
  const int8_t* x;
  int64_t ldx;
  const float* x_scale;
  const float* bias;
  void* y;
  int64_t ldy;
  int32_t y_dtype;
} aqd_linear_args;
size_t aqd_linear_workspace_bytes(int64_t m, const aqd_linear_weights* w);
aqd_status aqd_linear_int8(const aqd_linear_args* args, const aqd_linear_weights* w, void* workspace, size_t ws_bytes,
                           aqd_stream_t stream);

/* ---- attention of an 8-bit decoder ------------------------------------------------------ */

/* What lies between a decoder's 8-bit query-key-value product and its 8-bit output product: norms of queries and keys with
 * the position rotation, a cache of keys and values in 4 bits (Eq. 1's uniform quantizer, its interval taken from each row as above),
 * attention over that cache, and attention over whole prompts.
 *
 * Tensors of heads are [tokens][heads][head_dim] with strides in elements: ld from a token to the next, ldh from a head to the
 * next, both >= 0 and any for an input; the values of a head are adjacent. kv_heads divides heads: query head h reads key and value
 * head h / (heads / kv_heads). Outputs do not overlap inputs or each other, except where said. */

/* A cache of `pages` pages; a page holds page_size places (a power of two, 16..1024) of every key-value head. Place p of page g is
 * slot g * page_size + p. A place holds, of each head, a key row and a value row: head_dim (64, 128, 192 or 256) codes of 4 bits,
 * the row's lowest value and its step, both bfloat16:
 *   low = the largest bfloat16 <= min_k x_k,  step = the least bfloat16 >= (max_k x_k - low) / 15 (at least 2^-126, but 0 where max = low),
 *   code_k = (x_k - low) / step to the nearest, ties to even (0 where step = 0; what is within 2^-18 of a tie without being one may go to
 *   either side);  value = low + step * code.
 * So a value is off by half a step at most, and by 2^-18 of one more beside a tie. Rows that hold a NaN or an infinity, or whose values span more than float32's range, read back
 * as NaN. The layout within a page is the library's own. */
typedef struct {
  void* data; /* aqd_kv_cache_bytes(...) bytes (device), 256-byte aligned; its first contents do not matter */
  int64_t pages;
  int32_t page_size, kv_heads, head_dim;
} aqd_kv_cache;
/* 0 for sizes that are not supported (pages < 1, kv_heads outside 1..65535, over 2^40 bytes, and as above). */
size_t aqd_kv_cache_bytes(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim);

/* Queries and keys before attention, per token and head, in float32, rounded once to `dtype` (AQD_F32, AQD_F16, AQD_BF16, of all tensors here but
 * the weights and tables):
 *   u_k = x_k / sqrt(mean(x^2) + eps) * weight_k  (weight NULL: u = x, for queries and keys each; head_dim values of weight_dtype),
 *   then pair f of the first rot_dim places turns by the angle a = positions[token] * inv_freq[f], f < rot_dim / 2:
 *   (u_i, u_j) -> (u_i cos a - u_j sin a, u_j cos a + u_i sin a), with i = f, j = f + rot_dim / 2, or, if interleaved, i = 2 f, j = 2 f + 1.
 * eps >= 0. Rows of any finite values are normalized alike, those whose squares leave float32's range too (a row of zeros with eps = 0: NaN).
 * The angle is exact to 2^-24 of a turn while |position| (1 + |inv_freq|) < 2^38 (it is reduced in fixed point). rot_dim: even, 0..head_dim.
 * head_dim: even, 2..512 (with a cache: its own). q_out may be q, and k_out k (same pointer and strides).
 * heads may be 0 (keys alone). cache NULL: v and slots are not read. With a cache, each token's keys (rotated and rounded to `dtype`) and
 * values v are written to place slots[token] too, the bytes that aqd_cache_write would write; k_out may then be NULL. A slot outside the cache is
 * skipped. The slots inside it are distinct; of one listed twice a row may mix both tokens'. */
typedef struct {
  int64_t tokens;
  int32_t heads, kv_heads, head_dim, dtype;
  const void* q;
  int64_t ldq, ldqh;
  const void* k;
  int64_t ldk, ldkh;
  const void* v;
  int64_t ldv, ldvh;
  void* q_out;
  int64_t ldq_out, ldqh_out;
  void* k_out;
  int64_t ldk_out, ldkh_out;
  const void* q_weight;
  const void* k_weight;
  int32_t weight_dtype;
  float eps;
  const int64_t* positions;
  const float* inv_freq;
  int32_t rot_dim, interleaved;
  const int64_t* slots;
} aqd_qk_rope_args;
aqd_status aqd_qk_norm_rope(const aqd_qk_rope_args* args, const aqd_kv_cache* cache, aqd_stream_t stream);

/* Rows of keys and values (k, v: [tokens][kv_heads][head_dim] of dtype) to places slots[token], and the values that the places hold back from there
 * (a slot outside the cache: skipped by the write, zeros from the read). Reading, k or v may be NULL. Slots as above; a read may list one twice. */
typedef struct {
  int64_t tokens;
  int32_t dtype;
  void* k;
  int64_t ldk, ldkh;
  void* v;
  int64_t ldv, ldvh;
  const int64_t* slots;
} aqd_cache_rows;
aqd_status aqd_cache_write(const aqd_cache_rows* rows, const aqd_kv_cache* cache, aqd_stream_t stream);
aqd_status aqd_cache_read(const aqd_cache_rows* rows, const aqd_kv_cache* cache, aqd_stream_t stream);

/* Attention of each sequence's last tokens over the cache. Sequence s has lengths[s] places, place t in page pages[s][t / page_size] (a row of
 * `columns` entries of the table; longer lengths are cut to columns * page_size, negative ones are 0), and the queries of tokens starts[s] .. starts[s+1] - 1
 * (starts NULL: token s alone; tokens = seqs then). Query j of its n sees the places t < lengths[s] - n + j + 1: its own token's and those before.
 *   o = sum_t p_t v_t,  p = softmax over the places seen of scale * q . k_t,  lse = ln sum_t exp(scale * q . k_t).
 * k_t and v_t are the cache's values. A query that sees no place gets o = 0 and lse = -infinity. Places in a page outside [0, pages) are not there.
 * Rows of out behind the last sequence are left as they were. dtype (q and out): AQD_F16 or AQD_BF16. starts[0] >= 0, not falling, at most tokens.
 * scale > 0, finite. q takes part as float16 after a power-of-two factor per row (values below 2^-29 of the row's largest lose bits); scores,
 * statistics and sums are float32, p times the value's step is float16 with the largest step's power in front.
 * Work is split over places by the lengths at hand; parts join in a fixed order. workspace: aqd_cache_attention_workspace_bytes(...) bytes,
 * 256-byte aligned; its contents do not matter, and calls that share it must not overlap in time. */
typedef struct {
  int64_t tokens;
  int32_t seqs, heads, dtype;
  float scale;
  const void* q;
  int64_t ldq, ldqh;
  void* out;
  int64_t ldo, ldoh;
  float* lse;               /* [tokens][heads] or NULL */
  const int32_t* starts;    /* [seqs + 1] or NULL */
  const int32_t* lengths;   /* [seqs] */
  const int32_t* page_table; /* [seqs][ld_table], `columns` of them used; ld_table 0: one row for all */
  int64_t ld_table;
  int32_t columns;
} aqd_cache_attention_args;
size_t aqd_cache_attention_workspace_bytes(int64_t tokens, int32_t seqs, int32_t heads, const aqd_kv_cache* cache);
aqd_status aqd_cache_attention(const aqd_cache_attention_args* args, const aqd_kv_cache* cache, void* workspace, size_t ws_bytes, aqd_stream_t stream);

/* Attention over whole sequences, packed one after another: sequence s has the queries starts[s] .. starts[s+1] - 1 and the keys and values
 * kv_starts[s] .. kv_starts[s+1] - 1 (kv_starts NULL: the same). causal: query j of n sees the first m - n + j + 1 of its sequence's m keys; else all.
 * o and lse as above; a query that sees nothing gets 0 and -infinity; rows behind the last sequence are left as they were. dtype (q, k, v, out): AQD_F16 or
 * AQD_BF16; head_dim 64, 128, 192 or 256; every pointer of them 16-byte aligned, every stride a multiple of 8 elements. Scores, statistics and sums
 * are float32; p is rounded to dtype before it meets v. A key or value that a query does not see reaches no output of it, be it NaN or infinite. tokens and kv_tokens: rows of q and of k. */
typedef struct {
  int64_t tokens, kv_tokens;
  int32_t seqs, heads, kv_heads, head_dim, dtype, causal;
  float scale;
  const void* q;
  int64_t ldq, ldqh;
  const void* k;
  int64_t ldk, ldkh;
  const void* v;
  int64_t ldv, ldvh;
  void* out;
  int64_t ldo, ldoh;
  float* lse;               /* [tokens][heads] or NULL */
  const int32_t* starts;    /* [seqs + 1] */
  const int32_t* kv_starts; /* [seqs + 1] or NULL */
} aqd_prompt_attention_args;
aqd_status aqd_prompt_attention(const aqd_prompt_attention_args* args, aqd_stream_t stream);

/* ---- distillation from a teacher's top logits ----------------------------------------- */

/* The loss that trains a low-bit student from a float teacher of which only the `top` largest logits of each
 * token are kept (teacher[t][j] float32, at vocabulary places index[t][j]):
 *   p = softmax(teacher / tau) over the kept places, q = softmax(logits / tau) over the whole vocabulary,
 *   loss[t] = row_weight[t] * sum_j p_j (ln p_j - ln q_index[j]),
 *   grad[t][v] = d loss[t] / d logits[t][v] = row_weight[t] / tau * (q_v sum_j p_j - sum_{j: index[j] = v} p_j).
 * A place whose index lies outside [0, vocab) is empty (a token may have fewer kept logits), as is one whose teacher
 * logit is -infinity; a token with none has loss 0 and gradient 0. A place listed twice counts twice.
 * A token of weight 0 has loss 0 and gradient 0 whatever its logits hold. A logit of -infinity has q = 0; where a
 * kept place of p > 0 has it, the loss is +infinity. A NaN or +infinity among a token's logits or kept
 * teacher logits makes its loss and gradient NaN, as do logits that are all -infinity. logit / tau has to lie
 * within float32's range; differences from a row's maximum count alone, so rows of the lowest value are even ones. Statistics are
 * float32; each thread sums a fixed share of a row and shares combine in a fixed order (deterministic).
 *   loss, lse: [tokens] float32 or NULL; lse = ln sum_v exp(logits[v] / tau), which the backward reads.
 *   grad: NULL (loss alone) or rows of the logits' type; it may be the logits themselves (same pointer and ld).
 *   row_weight: [tokens] float32, or NULL for all 1. tau > 0. top: 1..1024. index: int64. */
typedef struct {
  int64_t tokens;
  int32_t vocab, dtype;
  const void* logits;
  int64_t ld_logits;
  const int64_t* index;  /* [tokens][top], rows adjacent */
  const float* teacher;  /* [tokens][top], rows adjacent */
  int32_t top;
  float tau;
  const float* row_weight;
  void* grad;
  int64_t ld_grad;
} aqd_distill_args;
aqd_status aqd_distill_topk(const aqd_distill_args* args, float* loss, float* lse, aqd_stream_t stream);
/* The gradient alone, from the lse that aqd_distill_topk wrote; row_weight is the factor of each token's gradient
 * (the weight times the gradient that arrives at its loss). q carries the rounding of lse, |lse| 2^-24 of its value;
 * aqd_distill_topk's own gradient does not. */
aqd_status aqd_distill_topk_backward(const aqd_distill_args* args, const float* lse, aqd_stream_t stream);

/* ---- elementwise ------------------------------------------------------------------ */

/* y = requant(sat32(acc + bias)) per channel at `level`: Eq. 6 + Eq. 2 on an int32
 * accumulator tensor. y->bits 2/3/4/8 (or 32: sat32(acc + bias)). */
aqd_status aqd_requant(const aqd_tensor* acc, const aqd_requant_params* rq, int32_t level,
                       aqd_tensor* y, aqd_stream_t stream);

/* Eq. 7 on two tensors: a plays the accumulator (codes or int32), b the skip (codes or
 * int32, half size when sp->upsample == 2). rq NULL: 32-bit output sat32(result) with no
 * bias; otherwise bias is added to a first and y->bits selects the output as above. */
aqd_status aqd_residual_add_int(const aqd_tensor* a, const aqd_tensor* b,
                                const aqd_skip_params* sp, const aqd_requant_params* rq,
                                int32_t level, aqd_tensor* y, aqd_stream_t stream);

/* Sec. 3.2.4: k x k max-pooling (stride, zero-or-more padding < k) directly on codes;
 * padded taps are ignored. y has x's bits. */
aqd_status aqd_maxpool_codes(const aqd_tensor* x, int32_t k, int32_t stride, int32_t pad,
                             aqd_tensor* y, aqd_stream_t stream);

/* Sec. 3.2.4's max-pool fused with the first step of the workspace path of the convolution
 * that reads its output (the stem's 3x3 stride-2 pool feeding the first residual stage):
 * y = aqd_maxpool_codes(x, k, stride, pad) is written as packed codes (for any other reader,
 * e.g. a skip), and in the same pass `workspace` receives the zero-padded byte image that
 * aqd_conv_expand_input would write for the single job {x = y} of weights w with conv_stride
 * and conv_pad. A following aqd_conv_int_grouped_expanded of that job then reads it, so the
 * pooled map is never read back for its expansion and no separate pooling launch runs.
 * The pool must be 3x3 with stride 2 on 2- or 4-bit codes (else AQD_ERR_UNSUPPORTED);
 * x and y: same n, c and bits, y the pooled shape, distinct storage. The workspace path must apply to that convolution and the workspace
 * hold aqd_conv_workspace_bytes of it: otherwise AQD_ERR_UNSUPPORTED (AQD_ERR_INVALID for a
 * NULL workspace or bad shapes). Results are the bytes the two separate calls produce. */
aqd_status aqd_maxpool_expand(const aqd_tensor* x, int32_t k, int32_t stride, int32_t pad, aqd_tensor* y,
                              const aqd_conv_weights* w, int32_t conv_stride, int32_t conv_pad,
                              void* workspace, size_t ws_bytes, aqd_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* AQD_H */
