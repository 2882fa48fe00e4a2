/*
 * laud.h -- C ABI of the MI355X (gfx950) dynamic-bottleneck library.
 *
 * The library implements the inference hot path of the LAUDNet block (Sec. 3.1-3.2,
 * Fig. 2): a spatial masker scores coarse S x S patches, the active patches are turned
 * into an index list, and the residual bottleneck (1x1 -> 3x3 -> 1x1) is evaluated on
 * those patches only and added back into the feature map in place of the skip value.
 * Channel skipping and layer skipping (Sec. 3.1) use the same compaction machinery.
 *
 * Conventions that hold for every entry point
 *   - All tensor pointers are DEVICE pointers owned by the caller; the library never
 *     allocates, frees or keeps them.  Scratch memory is a caller-owned device workspace
 *     sized with laud_workspace_size(); its contents are undefined between calls.
 *   - Feature maps are dense NHWC: element (n,y,x,c) at ((n*H + y)*W + x)*C + c.  One
 *     pixel's channel vector is contiguous.  dtype is LAUD_F32 or LAUD_BF16; C, c_in,
 *     c_mid and c_out must be multiples of 8 and every tensor base 16-byte aligned.
 *     One feature map or scratch activation (N*H*W*max(c_in, c_mid) elements) has to stay
 *     below 2 GiB (the kernels address an operand with 32-bit byte offsets); larger
 *     shapes return LAUD_ERR_UNSUPPORTED.  The output of a first block may have any size
 *     where c_out is more than both (results are addressed with 64 bits).  One weight matrix
 *     of more than 2 GiB is unsupported too, except w2 and w3 of laud_channel_skip_conv,
 *     which may have any size.
 *   - Weights have the feature map's dtype: w1 [c_mid][c_in], w2 [c_mid][3][3][c_mid]
 *     (out, ky, kx, in; stride 1, zero padding 1, cross-correlation), w3 [c_out][c_mid].
 *     The per-channel affine (folded BN, Sec. 3.4) is float32: s1,t1,s2,t2 [c_mid],
 *     s3,t3 [c_out].  Accumulation, affine and the residual add are float32; h1, h2 and
 *     the output are rounded (nearest-even) to dtype.
 *   - Patch p of an H x W map with granularity S (S divides H and W; Hp = H/S, Wp = W/S)
 *     has flat index (n*Hp + py)*Wp + px and covers pixels [py*S, py*S+S) x [px*S, px*S+S).
 *   - Every call is asynchronous on `stream` (a hipStream_t passed as void*; NULL = the
 *     default stream) and never synchronises.  Data-dependent counts stay on the device.
 *   - Return value: LAUD_OK or a negative laud_status.  Arguments are validated on the
 *     host before anything is launched; on error nothing has been launched.
 *   - Threads: entry points may be called from several host threads at once as long as the calls
 *     use different workspaces (and, for in-place calls, different feature maps).  The library
 *     keeps no state between calls except (a) idempotent per-kernel launch attributes, requested on a
 *     kernel's first launch per device or all at once by laud_init(); (b) the optional stage-timing
 *     collector (laud_stage_timing_*), which is NOT re-entrant; (c) the fixed scratch array of
 *     laud_dyn_bottleneck_noalloc, shared by all calls on one GPU.  No environment variable is read.
 */
#ifndef LAUD_H
#define LAUD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LAUD_OK = 0,
  LAUD_ERR_INVALID_ARG = -1, /* null pointer, non-positive dim, S not dividing H/W, D not dividing c_mid */
  LAUD_ERR_UNSUPPORTED = -2, /* dtype/shape outside what the kernels cover (e.g. channels % 8 != 0) */
  LAUD_ERR_WORKSPACE = -3,   /* workspace missing or smaller than laud_workspace_size() */
  LAUD_ERR_HIP = -4,         /* a HIP launch failed */
  LAUD_ERR_SCRATCH_LIMIT = -5 /* laud_dyn_bottleneck_noalloc: the shapes need more scratch memory than the
                                 library's fixed LAUD_NOALLOC_SCRATCH_BYTES; use laud_dyn_bottleneck */
} laud_status;

/* LAUD_E4M3 (OCP 8-bit floating point, 1-4-3 bits, largest value 448) is a type of the token operators' operands only; feature
 * maps and the blocks above them are float32 or bf16. */
typedef enum { LAUD_F32 = 0, LAUD_BF16 = 1, LAUD_E4M3 = 2 } laud_dtype;

typedef enum {
  LAUD_OP_MASK_GEN = 0,
  LAUD_OP_COMPACT = 1,
  LAUD_OP_GATHER = 2,
  LAUD_OP_DYN_BOTTLENECK = 3,
  LAUD_OP_CHANNEL_SKIP = 4
} laud_op;

/* Shape of a dense NHWC feature map. */
typedef struct {
  int32_t N, H, W, C;
  int32_t dtype; /* laud_dtype */
} laud_fmap;

/* Folded parameters of one residual bottleneck (Fig. 2(a); Sec. 3.4). Device pointers. */
typedef struct {
  int32_t c_in, c_mid, c_out; /* c_out must equal c_in (identity shortcut) */
  const void* w1;
  const void* w2;
  const void* w3;
  const float* s1;
  const float* t1;
  const float* s2;
  const float* t2;
  const float* s3;
  const float* t3;
  int32_t relu_out; /* non-zero: ReLU after the residual add, on computed pixels only */
  const void* packed; /* NULL, or the block's weights re-ordered once by laud_pack_weights() (device memory of
                         laud_packed_weights_size() bytes).  With it no call spends time re-ordering weights; without
                         it the entry points do the same re-ordering themselves on every call, into their workspace.
                         It must be re-made whenever w1 / w2 / w3 change. */
} laud_bottleneck;

/* Human-readable name of a status code (static storage). */
const char* laud_status_string(int status);

/* Library ABI version (increments when a signature changes). */
int laud_abi_version(void);

/*
 * Optional one-time set-up for the CURRENT device: requests the launch attributes of every kernel (large
 * dynamic LDS) and resolves the device address of the allocation-free entry point's scratch array, so that
 * no first call has to do it -- e.g. inside a stream capture.  Allocates nothing, launches nothing; may be
 * called again (per device, from any thread).  Entry points work without it.
 */
int laud_init(void);

/*
 * Weights in the order the MFMA kernels stream them (a data layout, no arithmetic: every 16-byte piece of w1, w2, w3
 * is copied to the place where the lane that multiplies it will read it, so that a wave loads 1 KB in a row straight
 * into registers).  Made once per block -- e.g. when a model is loaded -- and handed over in laud_bottleneck.packed.
 * laud_packed_weights_size returns 0 for shapes / dtypes whose kernels read the plain layout (then packed stays
 * NULL).  p->packed itself is ignored by both calls.
 */
size_t laud_packed_weights_size(const laud_bottleneck* p, int dtype);
int laud_pack_weights(const laud_bottleneck* p, int dtype, void* packed, void* stream);

/*
 * Workspace bytes an entry point needs for the given shapes.  `op` is a laud_op; `p` may be
 * NULL for ops that take no bottleneck; `S_or_D` is the spatial granularity S (mask-gen,
 * gather, dyn-bottleneck), the element count n (compact) or the number of channel groups D
 * (channel-skip).  Returns 0 for invalid arguments.
 */
size_t laud_workspace_size(int op, laud_fmap fx, const laud_bottleneck* p, int S_or_D);

/*
 * Spatial masker + index generation (Sec. 3.2 "Masker design"; App. B, operator fusion
 * items 1-2).  For every patch:  logit = bias + sum_c w[c] * mean over the S x S patch of
 * x[...,c]  (the one-channel form W_0 - W_1 of the two-logit masker), mask = logit > 0
 * (strict; 0 and NaN are inactive), optionally AND-ed with a per-sample layer gate.  Then
 * the ascending list of active flat patch indices and its length are produced.
 *   x        [N,H,W,C] dtype                      in
 *   w        [C] float32                          in
 *   keep     [N] bytes or NULL: sample n's patches are all inactive when keep[n] == 0
 *   mask     [N*Hp*Wp] bytes (0/1)                out
 *   idx      [N*Hp*Wp] int32, first *count valid  out
 *   count    [1] int32                            out
 *   sample_offsets [N+1] int32 or NULL: number of active patches before sample n  out
 *   logits   [N*Hp*Wp] float32 or NULL            out
 */
int laud_mask_gen(const void* x, laud_fmap fx, int S, const float* w, float bias,
                  const uint8_t* keep, uint8_t* mask, int32_t* idx, int32_t* count,
                  int32_t* sample_offsets, float* logits,
                  void* ws, size_t ws_bytes, void* stream);

/*
 * Stable compaction of a byte mask (Sec. 3.1 layer gates; App. B item 2 for patch masks
 * supplied from outside): idx = ascending positions i in [0,n) with keep[i] != 0,
 * *count = their number.  idx has capacity n.  n == 0 writes *count = 0.
 */
int laud_layer_skip_compact(const uint8_t* keep, int n, int32_t* idx, int32_t* count,
                            void* ws, size_t ws_bytes, void* stream);

/*
 * Stand-alone gather (Sec. 3.1, step 1 of the three-step schedule): for p < *count,
 * out[p][dy][dx][:] = x[n][py*S - halo + dy][px*S - halo + dx][:] if that pixel is inside
 * the image, else 0, with (n,py,px) decoded from idx[p]; halo is 0 or 1 (1 = the
 * neighbours a 3x3 kernel needs).  out is [cap][S+2*halo][S+2*halo][C] dtype with
 * cap >= *count (N*Hp*Wp always suffices); entries p >= *count are not written.
 */
int laud_gather_patches(const void* x, laud_fmap fx, int S, int halo,
                        const int32_t* idx, const int32_t* count, void* out, void* stream);

/*
 * Spatially adaptive bottleneck (Fig. 2(b); Sec. 3.4; App. B items 2-3).  For every pixel of
 * an active patch:  out = act(x + s3*conv1x1(h2;w3) + t3),  h2 = relu(s2*conv3x3(h1;w2) + t2),
 * h1 = relu(s1*conv1x1(x;w1) + t1) evaluated from the true x on the patch and its one-pixel
 * halo, with h1 := 0 outside the image (the padding is the 3x3's).  Pixels of inactive
 * patches: out == x bit for bit.  act = ReLU iff p->relu_out.
 *   idx/count  ascending active patch indices and their number (device), as produced by
 *              laud_mask_gen or laud_layer_skip_compact; with S == H == W the indices are
 *              sample ids and the call is layer skipping.
 *   out        [N,H,W,C]; may be the same pointer as x (in place, the scatter-add of
 *              App. B item 3); partial overlap is not allowed.
 */
int laud_dyn_bottleneck(const void* x, laud_fmap fx, const laud_bottleneck* p, int S,
                        const int32_t* idx, const int32_t* count, void* out,
                        void* ws, size_t ws_bytes, void* stream);

/*
 * laud_dyn_bottleneck for callers that cannot allocate or hand over a workspace: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and bit-identical
 * results; the scratch activations (dilated pixel list, h1, h2) live in a fixed array of
 * LAUD_NOALLOC_SCRATCH_BYTES in the library's device image (one copy per GPU, held until the process ends)
 * instead of a caller workspace.  The call allocates nothing (no hipMalloc / hipFree, no allocating library
 * routine).  Shapes whose laud_workspace_size(LAUD_OP_DYN_BOTTLENECK, ...) exceeds LAUD_NOALLOC_SCRATCH_BYTES
 * return LAUD_ERR_SCRATCH_LIMIT (e.g. one 56 x 56 x 256 float32 image with c_mid 64 needs 1.6 MB; batch 8 of the
 * bf16 stage-3 map 14 x 14 x 1024 with c_mid 256 needs 1.6 MB).  All calls on one GPU share the array, which keeps
 * the last call's contents: calls that overlap in time on one GPU (different streams or threads) race and must
 * be serialised by the caller; nothing in it needs clearing between calls.
 */
#define LAUD_NOALLOC_SCRATCH_BYTES (16u << 20)
int laud_dyn_bottleneck_noalloc(const void* x, laud_fmap fx, const laud_bottleneck* p, int S,
                                const int32_t* idx, const int32_t* count, void* out, void* stream);

/* What a group-convolution / squeeze-and-excitation bottleneck adds to laud_bottleneck (the RegNetY
 * backbones of Sec. 4; Sec. 3.2 states that the dynamic block carries over to group convolutions). */
typedef struct {
  int32_t group_width; /* g: channels per group of the 3x3 (as many in as out); divides c_mid; 8, 16, 32 or 64.
                          The block's w2 is then [c_mid][3][3][g]: output channel o reads the input channels
                          (o/g)*g .. (o/g)*g + g-1. */
  int32_t se_width;    /* hidden width of the SE module, <= 1024; 0 = no SE module (pointers below unused) */
  const float* w_se1;  /* [se_width][c_mid] float32, device */
  const float* b_se1;  /* [se_width] */
  const float* w_se2;  /* [c_mid][se_width] */
  const float* b_se2;  /* [c_mid] */
} laud_group_se;

/*
 * Spatially adaptive bottleneck whose 3x3 is a group convolution, with an optional squeeze-and-excitation
 * module between the 3x3 (after its affine and ReLU) and the last 1x1 (Sec. 4, RegNetY; Fig. 2(b) otherwise).
 * Everything is as in laud_dyn_bottleneck except
 *   h2 = relu(s2*groupconv3x3(h1;w2) + t2),
 *   gate[n][c] = sigmoid(w_se2 * relu(w_se1 * z[n] + b_se1) + b_se2),  z[n] = mean of h2 over the ACTIVE
 *   pixels of sample n (the paper does not say what the squeeze averages over when only some locations are
 *   computed; with every patch active, and for layer skipping with S == H == W, this is the ordinary
 *   global average),
 *   out = act(x + s3*conv1x1(h2 * gate[n]; w3) + t3) on active pixels.
 * h2 * gate is rounded to dtype before the last 1x1 (c_mid <= 4096 and N <= 65535 when se_width > 0).  Workspace:
 * laud_workspace_size(LAUD_OP_DYN_BOTTLENECK, ...).  Errors as laud_dyn_bottleneck; a group width other
 * than 8/16/32/64 returns LAUD_ERR_UNSUPPORTED, a null `e` or one that does not divide c_mid
 * LAUD_ERR_INVALID_ARG.
 */
int laud_dyn_group_se_bottleneck(const void* x, laud_fmap fx, const laud_bottleneck* p,
                                 const laud_group_se* e, int S, const int32_t* idx, const int32_t* count,
                                 void* out, void* ws, size_t ws_bytes, void* stream);

/*
 * The same block with the masker fused into the first 1x1 (Sec. 3.4 "Operator fusion for spatial
 * maskers"; App. B item 1): conv1 is evaluated on EVERY pixel (spatially static) and the masker's
 * per-pixel projection sum_c w[c]*x[n,y,x,c] is accumulated from the same reads of x; the
 * projection is pooled over S x S patches, thresholded and turned into the index list, and conv2 /
 * conv3 + scatter-add run on the active patches as in laud_dyn_bottleneck.  One call replaces
 * laud_mask_gen followed by laud_dyn_bottleneck and produces the same mask / idx / count /
 * sample_offsets / logits outputs (same meaning, same optional NULLs) and the same `out`; logits
 * differ from laud_mask_gen's only in float32 summation order.  It pays off when the dilated
 * activation ratio is close to 1 (small S); c_in <= 4096.  Workspace: as LAUD_OP_DYN_BOTTLENECK.
 * With a layer gate (`keep`) and logits == NULL the first 1x1 and the projection are evaluated on the kept samples
 * only (the gates are compacted first); with logits wanted they cover every sample, gated ones included.
 */
int laud_masker_dyn_bottleneck(const void* x, laud_fmap fx, const laud_bottleneck* p, int S,
                               const float* w, float bias, const uint8_t* keep,
                               uint8_t* mask, int32_t* idx, int32_t* count,
                               int32_t* sample_offsets, float* logits, void* out,
                               void* ws, size_t ws_bytes, void* stream);

/*
 * The UNFUSED three-step schedule of Sec. 3.1 (gather, compute, scatter), kept as the baseline of
 * the operator-fusion ablation (Tab. 1): a stand-alone gather of the active patches with their halo
 * into a dense buffer, the three convolutions on that buffer (conv1 on all (S+2)^2 gathered
 * positions, with h1 := 0 at positions outside the image; the 3x3 inside the gathered tile; the last
 * 1x1 into a dense float32 buffer), and a stand-alone scatter that adds the residual.
 * Same arguments and same result as laud_dyn_bottleneck.  Workspace:
 * laud_dyn_bottleneck_unfused_workspace(fx, p, S) bytes.
 */
size_t laud_dyn_bottleneck_unfused_workspace(laud_fmap fx, const laud_bottleneck* p, int S);
int laud_dyn_bottleneck_unfused(const void* x, laud_fmap fx, const laud_bottleneck* p, int S,
                                const int32_t* idx, const int32_t* count, void* out,
                                void* ws, size_t ws_bytes, void* stream);

/*
 * Channel-skipping bottleneck (Fig. 2(c); Sec. 3.1-3.2).  cmask is [N][D] bytes; group g of
 * sample n covers mid channels [g*G, (g+1)*G), G = c_mid / D.  The mask multiplies the input
 * and the output of the 3x3 conv.  Two schedules, same result: in general the kept-channel weight
 * gather is fused into the three convs and dropped channels are never computed (one set of tiles per
 * sample); for bf16 blocks with c_mid = 256, c_out = 1024, groups of whole 64-channel slices (D <= 4),
 * square maps and N <= 4096 the samples are ordered by mask pattern, the first 1x1 stores zeros in the
 * dropped groups of h1, and the fused 3x3 -> last 1x1 kernel skips every 64-channel input slice that no
 * row of a tile keeps and stores zeros in the dropped groups of h2 (p->packed is used when given).
 * out = act(x + s3*conv1x1(h2 masked; w3) + t3) on every pixel; with all groups dropped
 * out = act(x + t3).  out may be the same pointer as x.  Workspace: LAUD_OP_CHANNEL_SKIP.
 */
int laud_channel_skip_conv(const void* x, laud_fmap fx, const laud_bottleneck* p,
                           const uint8_t* cmask, int D, void* out,
                           void* ws, size_t ws_bytes, void* stream);

/*
 * Static parts of the ResNet body (always executed, no mask).  The paper's
 * formulation assumes stride 1 inside dynamic blocks (Sec. 3.1); the first block of every stage
 * (projection shortcut, stride 2 in stages 2-4, placed on the 3x3 as in the torchvision models the
 * paper starts from) and the stem run as ordinary dense layers.
 *
 * laud_static_bottleneck: out = relu(s3*conv1x1(h2;w3)+t3 + s_sc*conv1x1_stride(x;w_sc)+t_sc), with
 * h1 = relu(affine1(conv1x1(x;w1))), h2 = relu(affine2(conv3x3 stride, pad 1 (h1;w2))).  x is
 * [N,H,W,c_in]; out is [N,Ho,Wo,c_out] with Ho = (H-1)/stride + 1 (stride 1 or 2) and must not alias x;
 * w_sc is [c_out][c_in] in x's dtype, s_sc/t_sc float32 [c_out]; p->c_out may differ from p->c_in.
 *
 * laud_stem: x [N,Hin,Win,3] dtype; 7x7 stride-2 pad-3 conv with w7 [c_out][7][7][3] (dtype),
 * affine s,t (float32), ReLU, then 3x3 stride-2 pad-1 max pooling; out [N,Hp,Wp,c_out] with
 * Hc = (Hin-1)/2 + 1, Hp = (Hc-1)/2 + 1; c_out a multiple of 8.
 *
 * laud_stem3x3 (the stem of the RegNet backbones, Sec. 4): x [N,Hin,Win,3] dtype; 3x3 stride-2 pad-1 conv with
 * w3 [c_out][3][3][3] (dtype), affine s,t (float32), ReLU, no pooling; out [N,Ho,Wo,c_out], Ho = (Hin-1)/2 + 1;
 * c_out a multiple of 8, at most 256.  No workspace.
 */
size_t laud_static_bottleneck_workspace(laud_fmap fx, const laud_bottleneck* p, int stride);
int laud_static_bottleneck(const void* x, laud_fmap fx, const laud_bottleneck* p, const void* w_sc,
                           const float* s_sc, const float* t_sc, int stride, void* out,
                           void* ws, size_t ws_bytes, void* stream);
size_t laud_stem_workspace(int N, int Hin, int Win, int c_out, int dtype);
int laud_stem3x3(const void* x, int N, int Hin, int Win, int dtype, const void* w3, const float* s,
                 const float* t, int c_out, void* out, void* stream);
int laud_stem(const void* x, int N, int Hin, int Win, int dtype, const void* w7, const float* s,
              const float* t, int c_out, void* out, void* ws, size_t ws_bytes, void* stream);

/*
 * Dynamic first block of a stage (Sec. 3.1: the mask decides at which OUTPUT locations the
 * convolutions run; locations that are not selected take the value of the skip connection, which in
 * this block is the strided 1x1 projection):
 *   out = act(s_sc*conv1x1_stride(x;w_sc)+t_sc + M * (s3*conv1x1(h2;w3)+t3)),
 * h1, h2 as in laud_static_bottleneck.  The mask lives on the output grid [N,Ho,Wo], Ho = (H-1)/stride+1,
 * in patches of S x S output pixels (S divides Ho and Wo); idx/count are the ascending list of active
 * patch indices (n*Hp + py)*Wp + px on that grid and its length, both device memory, e.g. from
 * laud_mask_gen called on x with granularity stride*S (adaptive pooling of x to the output patch grid,
 * Sec. 3.2) or from laud_layer_skip_compact.  conv1 runs only on the input pixels under the 3x3 windows
 * of active output pixels, conv2/conv3 only on active output pixels; the shortcut runs everywhere.
 * x [N,H,W,c_in], out [N,Ho,Wo,c_out] (must not alias x), stride 1 or 2, act = ReLU iff p->relu_out.
 * Errors as laud_static_bottleneck; LAUD_ERR_INVALID_ARG if S does not divide the output size.
 */
size_t laud_dyn_projection_workspace(laud_fmap fx, const laud_bottleneck* p, int stride);
int laud_dyn_projection_bottleneck(const void* x, laud_fmap fx, const laud_bottleneck* p,
                                   const void* w_sc, const float* s_sc, const float* t_sc, int stride,
                                   int S, const int32_t* idx, const int32_t* count, void* out,
                                   void* ws, size_t ws_bytes, void* stream);

/*
 * The same first block for the group-convolution / SE backbones (Sec. 4, RegNetY): the stride sits on the group
 * 3x3 (w2 [c_mid][3][3][g]), and the SE gate (see laud_dyn_group_se_bottleneck) is taken over the sample's active
 * OUTPUT pixels.  With every patch of the output grid in the index list this is the static first block of a
 * stage.  Arguments, workspace (laud_dyn_projection_workspace) and errors as laud_dyn_projection_bottleneck and
 * laud_dyn_group_se_bottleneck.
 */
int laud_dyn_group_se_projection_bottleneck(const void* x, laud_fmap fx, const laud_bottleneck* p,
                                            const laud_group_se* e, const void* w_sc, const float* s_sc,
                                            const float* t_sc, int stride, int S, const int32_t* idx,
                                            const int32_t* count, void* out, void* ws, size_t ws_bytes,
                                            void* stream);


/*
 * Channel masker (Sec. 3.2 "Masker design"; Fig. 3(b)): g = mean of x over H x W per sample and
 * channel; h = relu(wa*g + ba) (the paper does not name the non-linearity; ReLU is assumed);
 * l = wb*h + bb, 2D logits viewed row-major as [D][2]; group d is kept iff l[d][0] > l[d][1]
 * (strict; NaN drops the group).  The paper sets hidden = max(floor(D/16), 16); any positive
 * width is accepted.  All weights float32 device arrays: wa [hidden][C], ba [hidden],
 * wb [2*D][hidden], bb [2*D].  Outputs: cmask [N][D] bytes (the input of laud_channel_skip_conv),
 * logits2 [N][2*D] float32 or NULL.  Workspace: laud_channel_masker_workspace(fx) bytes.
 */
size_t laud_channel_masker_workspace(laud_fmap fx);
int laud_channel_masker(const void* x, laud_fmap fx, const float* wa, const float* ba, int hidden,
                        const float* wb, const float* bb, int D, uint8_t* cmask, float* logits2,
                        void* ws, size_t ws_bytes, void* stream);

/*
 * ---- Token operators ------------------------------------------------------------------------------------------------------
 * What surrounds a dynamic block when the map is a list of tokens (Sec. 3.1: the block carries over to transformers, which skip
 * tokens and layers): norms with gate and residual, products of 8-bit operands, and a feed-forward layer that is itself
 * conditional (a router picks a few experts per token).  A token list is a feature map of N = rows, H = W = 1: laud_mask_gen
 * with S = 1 scores it, and its mask is the `keep` argument below.
 *   - Rows may be further apart than they are long: an `ld` argument is the distance of two rows in elements, at least the
 *     row length and, like it, a multiple of 8 (of 16 for LAUD_E4M3 operands of a product).  Bases are 16-byte aligned.
 *   - No row (rows, M or T = 0): LAUD_OK, nothing is launched.
 *   - What is written shares no byte with anything else of the call, except where an argument says what it may be
 *     (LAUD_ERR_INVALID_ARG).
 *   - Rows are addressed with 64 bits: tensors are limited by memory, and by what one launch takes where an entry point
 *     says so (LAUD_ERR_UNSUPPORTED beyond).
 *   - Sums, statistics and accumulators are float32; each result is rounded once, to nearest even.
 */

/* 8-bit blocks: an E4M3 tensor [rows][cols] comes with one float32 scale for each block of block_rows x 128 elements, row-major
 * [ceil(rows/block_rows)][ceil(cols/128)]; the last blocks of a row or column may be shorter.  Element = code * scale. */

/*
 * Quantises x [rows][cols] (dtype, cols a multiple of 8): scale = max(max|x| / 448, 2^-126) over the block, q = e4m3(x / scale), the
 * quotient in float32, ties to even.  A NaN or an infinity makes its block's codes NaN.  block_rows: 1 (activations) or 128
 * (weights; then cols at most 2^31 - 128).
 */
int laud_quantize_e4m3(const void* x, int64_t ldx, int rows, int cols, int dtype, int block_rows, void* q, int64_t ldq,
                       float* scale, void* stream);

typedef enum { LAUD_NORM_RMS = 0, LAUD_NORM_LAYER = 1 } laud_norm_kind;

/* The norm after a block and the norm before the next one.  Weights and biases are float32 [C], device. */
typedef struct {
  int32_t C;            /* channels: a multiple of 8, at most 32768 */
  int32_t dtype;        /* LAUD_F32 or LAUD_BF16: x, y and out */
  int32_t kind;         /* laud_norm_kind of both norms */
  float eps;
  const float* post_w;  /* NULL: y as it is */
  const float* post_b;  /* NULL: none */
  const float* pre_w;   /* may be NULL where z is NULL */
  const float* pre_b;   /* NULL: none */
  float alpha, beta;    /* scales of the residual and of the branch */
} laud_norm_block;

/*
 * The seam between two residual blocks, in one pass over the rows:
 *   p = y, or norm(y; post_w, post_b);   r = x + branch on the rows a block ran on:  r = alpha * x + beta * gate * p  if keep, else x;
 *   out = r;   z = norm(r; pre_w, pre_b), taken from r before its rounding.
 * norm(v) = v / sqrt(mean(v^2) + eps) * w + b (RMS) or (v - mean(v)) / sqrt(var(v) + eps) * w + b (LAYER).  Squares are float32:
 * where their sum passes 2^128 it is infinite, and what it divides is 0.
 *   x     [rows][C]   residual stream
 *   y     [rows][C]   the block's result, or NULL: r = x (only the norm before a block; keep, gate must be NULL)
 *   keep  [rows] bytes or NULL (all kept): a row with 0 passes x on bit for bit; its y is not read
 *   gate  [ceil(rows/rows_per_gate)][C] float32 or NULL: row t uses gate row t / rows_per_gate (1: a gate per token, rows
 *         of a sample: a gate per sample, rows: one per channel)
 *   out   [rows][C] or NULL; may be x or y
 *   z     [rows][C] of z_dtype, or NULL (not both NULL): p->dtype, or LAUD_E4M3 with z_scale [rows][ceil(C/128)] as
 *         laud_quantize_e4m3 defines them (the operand of laud_matmul_e4m3); may be x or y where it has their type and ld
 */
int laud_norm_residual(const laud_norm_block* p, int rows, const void* x, int64_t ldx, const void* y, int64_t ldy,
                       const uint8_t* keep, const float* gate, int rows_per_gate, void* out, int64_t ldo, void* z, int64_t ldz,
                       int z_dtype, float* z_scale, void* stream);

/*
 * out[m][n] = sum_k a[m][k] * sa[m][k/128] * b[n][k] * sb[n/128][k/128]: products of 8-bit operands are added over a block of
 * 128, the block's sum takes its two scales (their product, in float32), blocks are added in float32.  a [M][K], b [N][K] E4M3, K a
 * multiple of 16, N of 8, rows at most 2^22 elements apart; sa [M][ceil(K/128)], sb [ceil(N/128)][ceil(K/128)]
 * (laud_quantize_e4m3 with block_rows 1 and 128); out [M][N] of out_dtype (LAUD_F32 or LAUD_BF16), no alias of an input.  Codes
 * are widened to bf16, which holds them exactly; products and sums are float32 for every shape and both types of result, so that
 * the number of rows changes a row's result by the order of its sums only.  At most 2^27 - 16 columns for up to 16 rows; for more
 * rows 2^23 - 8 tiles of 64 x 64 (larger ones where the results are many).
 * Workspace: laud_matmul_e4m3_workspace(M, N, K) bytes; no shape needs any at present (then ws may be NULL).
 */
size_t laud_matmul_e4m3_workspace(int M, int N, int K);
int laud_matmul_e4m3(const void* a, int64_t lda, const float* sa, const void* b, int64_t ldb, const float* sb, int M, int N,
                     int K, void* out, int64_t ldo, int out_dtype, void* ws, size_t ws_bytes, void* stream);

/* One mixture-of-experts layer.  Device pointers; matrices are dense. */
typedef struct {
  int32_t C, F;         /* token width and hidden width of an expert: multiples of 8 (of 16 with E4M3 weights) */
  int32_t E, top_k;     /* experts (at most 1024), experts a token goes to (1 .. min(E, 32)) */
  int32_t dtype;        /* LAUD_F32 or LAUD_BF16: x, router and out */
  int32_t w_dtype;      /* experts' weights: dtype, or LAUD_E4M3 where dtype is LAUD_BF16 */
  const void* router;   /* [E][C] */
  const void* up;       /* [E][2][F][C]: gate projection, up projection */
  const void* down;     /* [E][C][F] */
  const float* s_up;    /* E4M3: [E][2][ceil(F/128)][ceil(C/128)], else unused */
  const float* s_down;  /* E4M3: [E][ceil(C/128)][ceil(F/128)] */
  int32_t renormalise;  /* non-zero: a token's weights are divided by their sum */
  float scale;          /* factor on all weights */
} laud_moe_layer;

/*
 * A whole mixture-of-experts layer for a few tokens: l = router * x; the top_k experts by l (of equal ones the lower index; a NaN
 * comes last); weight = softmax(l over all experts) of the chosen ones, renormalised if asked for, times scale;
 *   out = sum over the chosen e of weight_e * down_e * (silu(gate_e * x) * (up_e * x)).
 * The hidden values stay float32.  A token with keep 0 is not routed: out row 0, experts -1, weights 0.
 *   x [T][C], out [T][C] dtype (out may be x); keep [T] bytes or NULL
 *   experts [T][top_k] int32 (ascending) and weights [T][top_k] float32: outputs, each may be NULL
 * T is at most LAUD_MOE_MAX_TOKENS (LAUD_ERR_UNSUPPORTED beyond).  An expert's weights are fetched once for every sixteen of its tokens;
 * where T * top_k <= E the down projection's once for each.  A result depends, in its last bits, on which of the two T makes it.
 * Workspace: laud_moe_workspace(p, T) bytes.
 */
#define LAUD_MOE_MAX_TOKENS 1024
size_t laud_moe_workspace(const laud_moe_layer* p, int T);
int laud_moe(const laud_moe_layer* p, int T, const void* x, int64_t ldx, const uint8_t* keep, void* out, int64_t ldo,
             int32_t* experts, float* weights, void* ws, size_t ws_bytes, void* stream);

/*
 * ---- Attention of a token block -------------------------------------------------------------------------------------------
 * The mixing step between a block's projections: over the tokens of this call (laud_attention), or of new tokens over a cache of
 * earlier tokens' keys and values (laud_cache_attention).  The conventions of the token operators hold.  Rows of q and out are
 * [token][heads][D], rows of k and v [token][kv_heads][D]: columns of one wider array (a projection's result) will do.
 * Query head h belongs to key head h / (heads / kv_heads).
 *   - Sequences lie one behind the other: offsets [B + 1] int32 (device) names the rows offsets[b] .. offsets[b + 1] - 1 of sequence b,
 *     ascending, within 0 .. T; a sequence may have no row.  Rows outside all sequences count for nothing, and are left as they were.
 *   - Weights are softmax(scale * q k) over the tokens that a query sees, and nothing else of the call has any part in its result
 *     (a NaN or an infinity in a token that it does not see stays there).  A score of -infinity has no weight; a query that sees
 *     nothing, or has no weight, gets zeros.  A value that is not finite makes its element of every query that sees it an infinity or NaN,
 *     whatever its weight, unless the query has none at all.  scale * log2(e) * score beyond float32's range is an infinite score, and sums
 *     are divided by the weights' at the end: values of more than 2^119 / (tokens that a query sees) may end in an infinity.
 *   - Scores, statistics and sums are float32.  Weights of float32 rows are not rounded.  With bf16 rows (bf16 operands of the instructions) a weight
 *     is rounded where it meets its value, by 2^-15 of itself; by 2^-8 where tiles of 128 query rows keep the matrix cores busy: in
 *     laud_attention with T * heads above 8192 and T above 14 B, over a bf16 cache with T * heads / kv_heads at least 512 B.  Codes of a cache in 8 bits
 *     are widened, a key's scale multiplies its scores and a value's scale its weights, before they are rounded.
 *   - The same call gives the same bits.  Which kernel and how many parts it takes follows from its sizes, so that a token's result
 *     may differ in its last bits between calls of other sizes.
 */
typedef struct {
  int32_t heads, kv_heads; /* heads: a multiple of kv_heads */
  int32_t D;               /* width of a head: a multiple of 8, at most 128 (LAUD_ERR_UNSUPPORTED beyond) */
  int32_t dtype;           /* LAUD_F32 or LAUD_BF16: q, k, v and out */
  int32_t causal;          /* non-zero: a query sees its own token and those before it; else all of its sequence */
  float scale;             /* of the products, positive and finite (1 / sqrt(D)) */
} laud_heads;

/*
 * out = attention of every token over its sequence.
 *   q, out [T] rows, k, v [T] rows; out may be q.  T at most 2^30, (B + T / 128) * heads at most 2^24 - 8, rows at most 2^22 elements apart
 *   (LAUD_ERR_UNSUPPORTED beyond).
 *   keep [T] bytes or NULL: a token with 0 (the masker's) is no key, and its row of out is zeros
 */
int laud_attention(const laud_heads* p, int B, const int32_t* offsets, int T, const void* q, int64_t ldq, const void* k, int64_t ldk,
                   const void* v, int64_t ldv, const uint8_t* keep, void* out, int64_t ldo, void* stream);

/* A cache of keys and values in pages.  Device pointers, dense; 16-byte aligned. */
typedef struct {
  int32_t pages, page;  /* number of pages; tokens a page holds: 16, 32, 64, 128 or 256; pages * page below 2^31 */
  int32_t kv_heads, D;  /* as in laud_heads; D a multiple of 16 for LAUD_E4M3 */
  int32_t dtype;        /* LAUD_F32, LAUD_BF16 or LAUD_E4M3 */
  void* k;              /* [pages][kv_heads][page][D] */
  void* v;
  float* k_scale;       /* LAUD_E4M3: [pages][kv_heads][page], a scale for each token's row of D, as laud_quantize_e4m3 defines it; else */
  float* v_scale;       /* unused */
} laud_cache;

/*
 * Which rows of a call belong to which sequence, and where its tokens are in the cache: the rows of sequence b are the last
 * ones of its lens[b] tokens (row i of n is at position lens[b] - n + i), position j is row j % page of page table[b][j / page].
 * Device pointers.  A position before the first or past the table, and one whose page is not 0 .. pages - 1, is no place: nothing
 * is written there, zeros are read, no query sees it.
 */
typedef struct {
  int32_t B;
  int32_t table_ld;       /* pages of a row of table, at least 1; table_ld * page at most 2^30 */
  const int32_t* offsets; /* [B + 1] */
  const int32_t* lens;    /* [B] */
  const int32_t* table;   /* [B][table_ld] */
  const int32_t* prefix;  /* [ceil(prefix_len / page)] pages of the tokens that come before the first of every sequence, or NULL */
  int32_t prefix_len;     /* their number (0: none; at most 2^30); laud_cache_attention only */
} laud_batch;

/*
 * laud_cache_write puts the rows k, v [T] of dtype (LAUD_F32 or LAUD_BF16: the cache's type, or any of them into LAUD_E4M3) where the
 * batch says, quantised by the way; laud_cache_read brings the rows from there, code * scale rounded once.  Two rows of a
 * call that are written to one place leave it undefined.  T * kv_heads is below 2^31 (LAUD_ERR_UNSUPPORTED beyond).
 */
int laud_cache_write(const laud_cache* c, const laud_batch* b, int T, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype,
                     void* stream);
int laud_cache_read(const laud_cache* c, const laud_batch* b, int T, void* k, int64_t ldk, void* v, int64_t ldv, int dtype,
                    void* stream);

/*
 * out = attention of new tokens (one, or some) over the cached tokens of their sequence, themselves among them, and over
 * the prefix: a query sees the whole prefix, and the positions up to its own (all of them where p->causal is 0).  The prefix is read
 * once for all sequences.  p->dtype is the cache's type, or LAUD_BF16 where that is LAUD_E4M3.
 *   q, out [T] rows; out may be q
 * Long sequences are shared out over workgroups, by the table's size and the number of rows; their parts are joined in order.
 * T * heads is below 2^31, and below 2^24 where parts are joined (the workspace is not 0; LAUD_ERR_UNSUPPORTED beyond).
 * Workspace: laud_cache_attention_workspace(p, c, b, T) bytes (0 for shapes that need none, and for arguments that the call refuses).
 */
size_t laud_cache_attention_workspace(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T);
int laud_cache_attention(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T, const void* q, int64_t ldq, void* out,
                         int64_t ldo, void* ws, size_t ws_bytes, void* stream);

/*
 * Instrumentation (host side; not part of the paper's method): per-stage GPU time of the
 * kernels the entry points launch.  While enabled, every stage is bracketed by a pair of HIP
 * events recorded on the call's stream (at most 65536 stage launches are kept per collection;
 * later ones are dropped).  laud_stage_timing_enable(1) clears what was collected and starts,
 * (0) stops.  laud_stage_timing_read() waits for the recorded events, adds up the elapsed
 * milliseconds and launch counts per stage into two HOST arrays of LAUD_STAGE_COUNT entries,
 * and clears the collection.  Not thread-safe against concurrent entry-point calls.  The token operators are not
 * collected: they are one launch each (laud_moe three or four).
 */
typedef enum {
  LAUD_STAGE_MASK_LOGITS = 0, /* pooled masker + threshold */
  LAUD_STAGE_COMPACT = 1,     /* ordered index generation */
  LAUD_STAGE_GATHER = 2,      /* stand-alone gather */
  LAUD_STAGE_COPY_INACTIVE = 3, /* unfused schedule only; elsewhere the copy of inactive patches is part of the block's last
                                   launch and of its time (CONV3, or CONV2 where the 3x3 and the last 1x1 are one kernel) */
  LAUD_STAGE_NEED = 4,        /* dilated active pixel list for conv1 */
  LAUD_STAGE_CONV1 = 5,
  LAUD_STAGE_CONV2 = 6,
  LAUD_STAGE_CONV3 = 7,
  LAUD_STAGE_CS1 = 8,
  LAUD_STAGE_CS2 = 9,
  LAUD_STAGE_CS3 = 10,
  LAUD_STAGE_SCATTER = 11,    /* stand-alone scatter + residual add (unfused schedule) */
  LAUD_STAGE_SE = 12,         /* squeeze-and-excitation gate + rescale (group-conv / SE blocks) */
  LAUD_STAGE_COUNT = 13
} laud_stage;
int laud_stage_timing_enable(int on);
int laud_stage_timing_read(double* total_ms, int64_t* launches);
const char* laud_stage_name(int stage);

/*
 * Achievable-peak probes (measurement aids, not part of the paper's method): the denominators a roofline fraction
 * can be read against besides the published peaks.  laud_probe_mfma launches `blocks` workgroups of 8 waves that
 * each issue 4*iters MFMAs (32x32x16 bf16, or the same FLOPs as 32x32x2 float32 steps) on register operands and
 * stores the FLOPs of the launch in *flops (host, may be NULL); sink is a device word nobody reads.
 * laud_probe_copy copies `bytes` (a multiple of 16, both pointers 16-byte aligned) with a plain grid-stride kernel;
 * laud_probe_read only reads them (sink: at least 16 device words nobody reads).
 * All only enqueue on `stream`; the caller times them with events.
 */
int laud_probe_mfma(int dtype, int iters, int blocks, double* flops, float* sink, void* stream);
int laud_probe_copy(const void* src, void* dst, size_t bytes, void* stream);
int laud_probe_read(const void* src, size_t bytes, float* sink, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LAUD_H */
