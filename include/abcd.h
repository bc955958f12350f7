/*
 * abcd.h -- C ABI of the ABCD active-block step on MI355X (gfx950).
 *
 * ABCD (Alpha-Composited Block Coordinate Descent) trains a radiance field one
 * spatial partition at a time: a step draws the active partition alone; its
 * image is composited between a foreground F and a background B that hold the
 * pre-accumulated renders of the frozen partitions in front of and behind it,
 * and gradients flow into the active parameters only (paper, Method section).
 * Because "over" is associative, the cached per-partition renders collapse
 * into F and B (Abstract; Method section). The renderer is 3D Gaussian
 * Splatting (Introduction), whose constants the paper does not state; they
 * are runtime parameters here (abcd_raster_params).
 *
 * One step on one camera is
 *   abcd_stage_cached     pinned host cache -> device chunk (per camera, in chunks)
 *   abcd_composite_cache  cached partition renders -> F, B (once per camera)
 *   abcd_project          parameters -> screen-space Gaussians
 *   abcd_bin_sort         -> per 16x16 tile, Gaussians sorted by (depth, index)
 *   abcd_render_fwd       -> out = F over A over B
 *   (loss gradient, e.g. abcd_loss_l1_grad)
 *   abcd_render_bwd       -> gradients of the active parameters only
 *
 * Conventions for every entry point:
 *  - Returns an abcd_status (int32). Arguments are validated on the host before
 *    any HIP call; an invalid call returns ABCD_E_INVALID and touches nothing.
 *  - Array arguments are DEVICE pointers owned by the caller unless marked
 *    "host". The library never allocates device memory: scratch space is a
 *    caller-provided workspace whose size the *_workspace_size helpers give.
 *  - All work is enqueued on `stream` and is asynchronous, except where a call
 *    is documented to synchronise.
 *  - Floating-point data is fp32 unless stated; fp16 is IEEE binary16 passed as
 *    uint16_t. Images are row-major [height][width][4] premultiplied RGBA.
 *  - Parameter arrays are contiguous structure-of-arrays:
 *      means [n][3], log_scales [n][3], quats [n][4] (w, x, y, z; any norm),
 *      opacity_logits [n], sh [n][(sh_degree+1)^2][3].
 *  - Alignment: quats, d_quats, conic_opacity and RGBA images 16 bytes,
 *    means2d 8 bytes, workspaces 256 bytes (an unaligned call is rejected).
 *  - Functions are stateless and reentrant; concurrent calls on one stream
 *    must not share a workspace.
 *  - Device arrays must be ordinary (coarse-grained) device memory, as
 *    hipMalloc and PyTorch's CUDA allocator return it. The library is built
 *    with hardware fp32 atomic adds (-munsafe-fp-atomics) for gradients,
 *    screen-space gradient sums and counters; on fine-grained, host-mapped or
 *    managed memory those atomics are not guaranteed to take effect, so the
 *    workspaces and every gradient output must not live there.
 */
#ifndef ABCD_H
#define ABCD_H

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ABCD_API __attribute__((visibility("default")))

#define ABCD_TILE 16           /* tile side in pixels */
#define ABCD_MAX_TILES 32768   /* ceil(W/16) * ceil(H/16) limit */
#define ABCD_MAX_GAUSSIANS (1LL << 30)

typedef enum {
  ABCD_OK = 0,
  ABCD_E_INVALID = 1,   /* bad argument; nothing was enqueued */
  ABCD_E_CAPACITY = 2,  /* intersection count exceeds the capacity given */
  ABCD_E_OVERFLOW = 3,  /* intersection count does not fit 32 bits */
  ABCD_E_HIP = 4        /* a HIP call failed; see abcd_last_error() */
} abcd_status;

/* Pinhole camera. x_cam = R x_world + t with OpenCV axes (x right, y down,
 * z forward); pixel (i, j) covers [i, i+1) x [j, j+1) and is sampled at its
 * centre (i + 0.5, j + 0.5). campos is the camera centre in world space (for
 * the view direction of the SH colour). Gaussians with view depth <= near_plane
 * are culled. near_plane must be positive (depth keys are the fp32 bit
 * patterns of positive depths, which sort as unsigned integers); a call with
 * near_plane <= 0 returns ABCD_E_INVALID. */
typedef struct {
  int32_t width, height;
  float fx, fy, cx, cy;
  float R[9]; /* row major */
  float t[3];
  float campos[3];
  float near_plane;
} abcd_camera;

/* Rasteriser constants of the 3D Gaussian Splatting renderer. */
typedef struct {
  float alpha_min;     /* blends with alpha below this are skipped (1/255) */
  float alpha_max;     /* alpha is clamped to this (0.99) */
  float t_min;         /* a blend that would take transmittance below this ends the pixel (1e-4) */
  float eps2d;         /* dilation added to every 2D covariance, px^2 (0.3) */
  float radius_sigmas; /* support radius in sigmas of the major axis (3) */
  float guard;         /* guard-band factor on the field of view inside the Jacobian (1.3) */
  int32_t sh_degree;   /* 0..3 */
  uint32_t flags;      /* ABCD_FLAG_* bits; others must be 0 */
} abcd_raster_params;

/* Compositing-aware stop (Limitations section: what a near-opaque foreground
 * hides need not be rendered). In abcd_render_fwd a pixel stops when the
 * weight the next blend would leave for later ones in the composited image,
 * (1 - F_alpha) T (1 - alpha), is below t_min, instead of T (1 - alpha); a
 * pixel whose F leaves it less than t_min blends nothing, and a tile whose
 * pixels all do so is skipped. Without F the rule is the plain one. The image
 * then differs from the plain rule's by at most t_min / (1 - alpha_max) per
 * channel times the largest colour plus one. abcd_render_bwd follows the
 * forward's final_T and last, so it needs no flag. */
#define ABCD_FLAG_FB_STOP 1u

/* ------------------------------------------------------------------------ */
/* Projection (3DGS EWA splatting: Introduction; Method section -- "only the
 * active partition is rendered").
 *
 * Per Gaussian i writes
 *   means2d[i][2]        pixel-space mean (u, v)
 *   conic_opacity[i][4]  (l11, l21, l22, o): the inverse 2D covariance (the
 *                        conic) [[a, b], [b, c]] as its Cholesky factor,
 *                        a = l11^2, b = l11 l21, c = l21^2 + l22^2 (computed
 *                        in fp64; the blend kernels evaluate the quadratic
 *                        form as a sum of two squares, which a badly
 *                        conditioned conic does not amplify), and opacity
 *                        o = sigmoid(logit)
 *   depth[i]             view-space z
 *   extent[i][2]         (ex, ey): half extents in pixels of the box that bins
 *                        the Gaussian: the support square (radius_sigmas times
 *                        the square root of the largest eigenvalue of the 2D
 *                        covariance) cut per axis to the extent of the ellipse
 *                        where alpha can reach alpha_min (|dx| <= sqrt(L A),
 *                        |dy| <= sqrt(L C), A and C the covariance's diagonal,
 *                        L = 1.001 tau + 0.001 and tau = 2 ((1 - e) ln 2 +
 *                        min(logit, 0)) >= 2 ln(o / alpha_min) for alpha_min =
 *                        m 2^e, m in [0.5, 1)); no pixel of a cut-off tile
 *                        could blend the Gaussian, so images are unchanged
 *   tiles_touched[i]     number of 16x16 tiles of that box
 *   rgb[i][3]            colour max(0, SH(view direction) + 0.5)
 * A culled Gaussian (behind near_plane, degenerate, non-finite, with no tile
 * on screen, or with alpha_min out of reach) gets zeros in every output. The
 * values deciding culling, the tile box and the depth key follow one fixed
 * fp32 operation order (the numerical contract of this library); extent must
 * be 8-byte aligned. n may be 0. */
ABCD_API int32_t abcd_project(const abcd_camera* cam /* host */, const abcd_raster_params* prm /* host */,
                     int64_t n, const float* means, const float* log_scales, const float* quats,
                     const float* opacity_logits, const float* sh, float* means2d,
                     float* conic_opacity, float* depth, float* extent, uint32_t* tiles_touched,
                     float* rgb, hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Binning: every (tile, Gaussian) pair of the support rectangles, sorted by
 * key = tile << 32 | fp32 bits of depth, ties by Gaussian index (the unique
 * front-to-back order of each tile's list).
 *
 * Outputs: values_sorted[M] Gaussian indices; keys_sorted[M] the keys (may be
 * NULL, then not written); tile_ranges[tiles][2] = [start, end) per tile
 * (start = number of pairs of lower tiles); tile_order[tiles] (may be NULL,
 * then not written): a schedule for abcd_render_fwd, the tile indices
 * ordered by decreasing list length kept to its leading three bits (the
 * octave and its quarter), ties in tile order.
 *
 * capacity: number of elements values_sorted (and keys_sorted) can hold. If
 * the intersection count M exceeds it (or does not fit 32 bits), nothing is
 * written to values_sorted or keys_sorted, every tile range is written empty
 * (so the blend calls that follow render nothing of the active block and read
 * no list entry) and tile_order is the identity.
 * n_isect (host, may be NULL): if given, the call synchronises `stream` once,
 * stores M there and returns ABCD_E_CAPACITY when M > capacity. If NULL, the
 * call does not synchronise; M (uint64) is left at the start of the workspace,
 * where the caller can read it later (M > capacity: that call overflowed).
 * capacity must be below 2^32.
 * workspace: at least abcd_bin_sort_workspace_size(n, capacity, width, height)
 * bytes, 256-byte aligned; it grows with the capacity (8 bytes per element for
 * an intermediate list of (Gaussian, 8x8-tile block) pairs, which never holds
 * more than M elements). */
ABCD_API int32_t abcd_bin_sort_workspace_size(int64_t n, int64_t capacity, int32_t width,
                                              int32_t height, size_t* bytes);
ABCD_API int32_t abcd_bin_sort(int32_t width, int32_t height, int64_t n, const float* means2d,
                      const float* extent, const float* depth, const uint32_t* tiles_touched,
                      int64_t capacity, void* workspace, size_t ws_bytes, uint64_t* keys_sorted,
                      uint32_t* values_sorted, uint32_t* tile_ranges, uint32_t* tile_order,
                      int64_t* n_isect /* host */, hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Split of long tiles between the forward and the backward (a scheduling
 * choice of this library; the paper's renderer is unchanged). The backward of
 * a tile walks its list back to front; a tile with a list of many thousand
 * entries would keep one workgroup busy after the rest of the GPU is idle.
 * With a split, whenever a tile's walk in the forward crosses a chunk
 * boundary (every `chunk` list positions, up to 63 boundaries: the 64th
 * chunk runs to the end of the list) it takes a 4 KB slot and stores each
 * pixel's transmittance and colour there, plus one slot for the end of the
 * walk; the backward then processes each (tile, chunk) as its own work item,
 * starting from those states, heaviest items first by the number of entries
 * the forward staged per chunk. Slots are taken in the forward's tile order
 * (heaviest first); a tile that finds none left is not split. The same
 * split must be given to a forward and its backward; results agree with the
 * unsplit backward up to rounding.
 * workspace: device memory of abcd_split_workspace_size(n_slots) bytes (or
 * more: the slots that fit are used), 256-byte aligned; chunk: a positive
 * multiple of 256, at most 2^24. Slots a frame needs: about (sum over tiles
 * of the longest walk in the tile) / chunk + (number of tiles split). */
typedef struct {
  void* workspace;
  size_t bytes;
  int32_t chunk;
  int32_t reserved;
} abcd_split;
ABCD_API int32_t abcd_split_workspace_size(int64_t n_slots, size_t* bytes);

/* ------------------------------------------------------------------------ */
/* Forward render and composite (Method section: F over active over B).
 *
 * Per pixel, front to back over its tile's list, starting from T = 1, C = 0:
 *   power = -(a dx^2 + c dy^2)/2 - b dx dy, (dx, dy) = pixel centre - mean;
 *   skip if power > 0; alpha = min(alpha_max, o exp(power)); skip if
 *   alpha < alpha_min; stop (without blending) if T (1 - alpha) < t_min;
 *   else C += rgb alpha T, T *= 1 - alpha.
 * The active render A = (C, 1 - T) is composited as out = F over A over B:
 *   out_rgb = F_rgb + (1 - F_a)(C + T B_rgb),
 *   out_a   = F_a + (1 - F_a)(1 - T (1 - B_a)).
 * F or B may be NULL (transparent); tile_ranges, values_sorted, means2d,
 * conic_opacity, rgb and the three outputs may not (ABCD_E_INVALID; a
 * placeholder buffer serves when the lists are empty). Also writes final_T[H][W] and last[H][W]
 * (entries of the tile's list walked up to and including the last blended
 * one), both needed by abcd_render_bwd. n_blends (may be NULL): the number of
 * blended (pixel, Gaussian) pairs of this call is ADDED to *n_blends.
 * tile_order (may be NULL): the order in which workgroups take tiles, a
 * permutation of the tiles such as abcd_bin_sort's tile_order (heaviest
 * first balances the GPU); it changes no output. NULL takes tiles in raster
 * order. split (host, may be NULL): see abcd_split. */
ABCD_API int32_t abcd_render_fwd(const abcd_camera* cam /* host */, const abcd_raster_params* prm /* host */,
                        const uint32_t* tile_ranges, const uint32_t* tile_order,
                        const uint32_t* values_sorted,
                        const float* means2d, const float* conic_opacity, const float* rgb,
                        const float* F, const float* B, float* out_rgba, float* final_T,
                        uint32_t* last, unsigned long long* n_blends, const abcd_split* split,
                        hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Cached render of a partition (Method section: the frozen partitions' renders
 * are cached per camera and refreshed after the block they belong to has been
 * trained): the forward above with F = B = transparent, written as
 * premultiplied fp16 RGBA, image_f16[H][W][4] = binary16 (round to nearest
 * even) of (C, 1 - T). Its input is that partition's projection and binning on
 * the camera; its output feeds abcd_composite_cache. tile_order as in
 * abcd_render_fwd (may be NULL). image_f16 8-byte aligned.
 * rect (device, may be NULL): int32[4] = (x0, y0, x1, y1), the bounding box
 * of the 16x16 tiles holding a pixel that blended anything, clipped to the
 * image; the image is zero outside it (x1 <= x0 when nothing blended). It is
 * the coverage box abcd_composite_cache takes. tile_ranges, values_sorted,
 * means2d, conic_opacity, rgb and image_f16 may not be NULL. */
ABCD_API int32_t abcd_render_cache(const abcd_camera* cam /* host */,
                          const abcd_raster_params* prm /* host */, const uint32_t* tile_ranges,
                          const uint32_t* tile_order, const uint32_t* values_sorted,
                          const float* means2d, const float* conic_opacity, const float* rgb,
                          uint16_t* image_f16, int32_t* rect, hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Backward (Method section: gradients are back-propagated only through the
 * active parameters; F and B are constants).
 *
 * Given dL_dout[H][W][4], writes the gradient of L with respect to every
 * active parameter: d_means [n][3], d_log_scales [n][3], d_quats [n][4],
 * d_opacity_logits [n], d_sh [n][(sh_degree+1)^2][3]; d_means2d [n][2] (may be
 * NULL) receives dL/d(u, v). With accumulate != 0 the gradients are added to
 * the arrays, otherwise they overwrite them. The derivative is exact for the
 * forward above, including zero derivative of a clamped alpha and of a
 * clamped colour. Inputs are those of the forward call on the same camera.
 * workspace: at least abcd_render_bwd_workspace_size(n) bytes, 256-byte
 * aligned (screen-space gradients, 36 bytes per Gaussian with n rounded up
 * to a multiple of 1024, and the work
 * schedule of the backward, heaviest walk first, 16 bytes per tile at the
 * maximum tile count). split (host, may be NULL): the one the forward used. */
ABCD_API int32_t abcd_render_bwd_workspace_size(int64_t n, size_t* bytes);
ABCD_API int32_t abcd_render_bwd(const abcd_camera* cam /* host */, const abcd_raster_params* prm /* host */,
                        int64_t n, const float* means, const float* log_scales, const float* quats,
                        const float* opacity_logits, const float* sh, const float* means2d,
                        const float* conic_opacity, const float* rgb, const float* extent,
                        const uint32_t* tile_ranges, const uint32_t* values_sorted,
                        const float* F, const float* B, const float* final_T, const uint32_t* last,
                        const float* dL_dout, void* workspace, size_t ws_bytes, float* d_means,
                        float* d_log_scales, float* d_quats, float* d_opacity_logits, float* d_sh,
                        float* d_means2d, int32_t accumulate, const abcd_split* split,
                        hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Allocation-free backward, for callers that cannot allocate device memory
 * (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): abcd_render_bwd without the workspace arguments, same outputs.
 * Its scratch (screen-space gradients and the backward's work schedule) is a
 * static device array of ABCD_NOALLOC_SCRATCH_BYTES inside the library; each
 * GPU the library runs on holds its own copy until the process ends. n may be
 * at most ABCD_NOALLOC_MAX_GAUSSIANS; a larger n returns ABCD_E_INVALID with
 * nothing enqueued. The call allocates nothing: no hipMalloc, no hipFree, no
 * allocating library routine (its first call on a device looks up that
 * device's copy of the array, with hipGetSymbolAddress, and keeps the
 * address). The calling thread's current device must be the one of `stream`.
 * Every call on a GPU shares that GPU's array, which keeps the last call's
 * contents; each call clears what must start at zero itself (with a fill
 * kernel, no memset node). Calls that overlap on one GPU (on other streams or
 * threads) race on the array and give wrong gradients: serialise them. */
#define ABCD_NOALLOC_MAX_GAUSSIANS (1LL << 20)
#define ABCD_NOALLOC_SCRATCH_BYTES 38275072ULL /* workspace of 2^20 Gaussians */
ABCD_API int32_t abcd_render_bwd_noalloc(const abcd_camera* cam /* host */,
                                         const abcd_raster_params* prm /* host */, int64_t n,
                                         const float* means, const float* log_scales,
                                         const float* quats, const float* opacity_logits,
                                         const float* sh, const float* means2d,
                                         const float* conic_opacity, const float* rgb,
                                         const float* extent, const uint32_t* tile_ranges,
                                         const uint32_t* values_sorted, const float* F,
                                         const float* B, const float* final_T,
                                         const uint32_t* last, const float* dL_dout,
                                         float* d_means, float* d_log_scales, float* d_quats,
                                         float* d_opacity_logits, float* d_sh, float* d_means2d,
                                         int32_t accumulate, const abcd_split* split,
                                         hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Collapse of cached partition renders into F and B (Abstract; Method section:
 * the stored renders of the frozen partitions are merged, front to back in
 * their depth order, into the two layers).
 *
 * images: k premultiplied RGBA fp16 renders [k][H][W][4]. order (host): a
 * permutation of 0..k-1, front to back. F = images[order[0]] over ... over
 * images[order[n_front-1]], B = images[order[n_front]] over ... over
 * images[order[k-1]], both fp32 [H][W][4]. flags: ABCD_COMPOSITE_ACCUMULATE
 * (1) continues the fold behind the incoming F and B (F <- F over fold, B <- B
 * over fold), so chunks of cached images can stream in front to back;
 * without it they are overwritten. k = 0 writes transparent F and B (or
 * leaves them unchanged when accumulating). ABCD_COMPOSITE_BESIDE (2) runs the
 * collapse on at most two workgroups per CU, each taking many pixels, so that
 * work enqueued on other streams meanwhile (the binning of the same step)
 * finds room on the CUs; alone on the GPU it is slower. Other bits:
 * ABCD_E_INVALID.
 * rects (device, may be NULL, 16-byte aligned): int32 [k][4] = (x0, y0, x1,
 * y1) per image, the pixel box [x0, x1) x [y0, y1) outside which that image
 * is fully transparent (all four channels zero), as abcd_render_cache
 * reports it; the image is not read outside its box. A box that cuts off
 * non-zero pixels gives wrong results. NULL: every image covers the frame.
 * stop_t (0 <= stop_t < 1; Limitations section: occluded renders can be
 * ignored): 0 folds every layer; above 0 a front layer is skipped once
 * 1 - F_alpha < stop_t and a back layer once (1 - F_alpha)(1 - B_alpha) <
 * stop_t (alphas accumulated so far), which changes F over B by at most
 * 2 stop_t per channel. */
ABCD_API int32_t abcd_composite_cache(int32_t width, int32_t height, int32_t k, const uint16_t* images,
                             const int32_t* order /* host */, int32_t n_front,
                             const int32_t* rects, float stop_t, float* F, float* B,
                             int32_t flags, hipStream_t stream);
#define ABCD_COMPOSITE_ACCUMULATE 1
#define ABCD_COMPOSITE_BESIDE 2

/* ------------------------------------------------------------------------ */
/* Upload of cached renders from pinned host memory (Method section: the cache
 * of camera-partition renders is kept in system memory or on disk, and the
 * renders a camera needs go to the GPU when a block becomes active). For each
 * j < k, copies the coverage box rects[j] (as in abcd_composite_cache; NULL:
 * the whole image) of host_images[j] (fp16 RGBA [H][W][4] in pinned host
 * memory) to the same pixels of dst[j] (device, [k][H][W][4]), as one 2D
 * copy per image, asynchronously on `stream`. Pixels of dst outside the box
 * keep their old contents, which abcd_composite_cache with the same rects
 * never reads; an empty box copies nothing. host_images (k pointers) and rects
 * ([k][4] int32) are host arrays; the host images must stay unchanged until
 * the copies complete. A box outside the image is an error. */
ABCD_API int32_t abcd_stage_cached(int32_t width, int32_t height, int32_t k,
                          const uint16_t* const* host_images /* host */,
                          const int32_t* rects /* host */, uint16_t* dst, hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* L1 reconstruction loss gradient (the paper evaluates a reconstruction loss
 * without naming it, Method section). img = out_rgb + (1 - out_a) bg;
 * dL/dimg = sign(img - target) / (3 H W) (sign(0) = 0); writes dL_dout[H][W][4]
 * (alpha channel -sum_c bg_c dL/dimg_c). bg (host) may be NULL (black). loss
 * (may be NULL): sum |img - target| / (3 H W) is ADDED to *loss. */
ABCD_API int32_t abcd_loss_l1_grad(int32_t width, int32_t height, const float* out_rgba,
                          const float* target_rgb, const float* bg /* host, 3 floats */,
                          float* dL_dout, float* loss, hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Adam update of the active parameters after the backward (the step on the
 * optimizer side; the paper trains with gradient steps but does not name the
 * optimizer, the 3DGS line it builds on uses Adam with one learning rate per
 * parameter group). For every element of every group, in place, fp32:
 *   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2;
 *   param -= lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * (Kingma and Ba 2015, Algorithm 1). groups (host array of n_groups <=
 * ABCD_ADAM_MAX_GROUPS): device arrays of `count` floats each; param,
 * exp_avg (m) and exp_avg_sq (v) are read and written, grad is read; a group
 * with count 0 is skipped. step >= 1 counts the updates made so far, this one
 * included; 0 <= beta1, beta2 < 1; eps >= 0. One launch. */
#define ABCD_ADAM_MAX_GROUPS 8
typedef struct abcd_adam_group {
  float* param;
  const float* grad;
  float* exp_avg;
  float* exp_avg_sq;
  int64_t count;
  float lr;
} abcd_adam_group;
ABCD_API int32_t abcd_adam_step(const abcd_adam_group* groups /* host */, int32_t n_groups,
                                float beta1, float beta2, float eps, int64_t step,
                                hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Operators of a decoder that turns learned features, one row per Gaussian,
 * into attributes, and of its training. A block of it is
 *   x + dropout(ffn(layer_norm(x))).
 * Matrices are row-major with unit stride along a row; ld* is the distance
 * between rows in elements (>= the width) and may be odd, and an array needs its
 * element's alignment only. All arrays of a call hold elements of `dtype`
 * unless stated; statistics, products and sums are kept in fp32 (in the order
 * that the launch fixes: the same call gives the same result) and every output
 * is rounded once, to nearest, from fp32. n >= 0 rows, up to
 * ABCD_MAX_GAUSSIANS; widths 1..ABCD_MAX_WIDTH. */
typedef enum { ABCD_F32 = 0, ABCD_F16 = 1, ABCD_BF16 = 2 } abcd_dtype;
#define ABCD_MAX_WIDTH 65536

/* Layer norm over rows of width d: mean and rstd = 1 / sqrt(var + eps) with
 * var = mean((x - mean)^2); y = (x - mean) rstd weight + bias. weight and bias
 * (d elements of type wdtype: dtype or ABCD_F32) may be NULL, then 1 and 0.
 * mean and rstd (fp32, n each) may be NULL, then not written; the backward needs
 * them. eps >= 0 (with eps = 0 a constant row gives NaN). y may be x itself. */
ABCD_API int32_t abcd_layer_norm(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx,
                                 int32_t wdtype, const void* weight, const void* bias, float eps,
                                 void* y, int64_t ldy, float* mean, float* rstd,
                                 hipStream_t stream);

/* Its gradients, with z = (x - mean) rstd and v = dy weight:
 *   dx = add + rstd (v - mean(v) - z mean(v z));  dweight = sum dy z;  dbias = sum dy
 * (sums over the rows, written, not added to; type wdtype). add (may be NULL) is
 * a gradient that reaches x by another path, the residual one. dx, dweight and
 * dbias may be NULL, then not computed; dx may be dy or add itself. workspace:
 * at least abcd_layer_norm_bwd_workspace_size bytes, 256-byte aligned. */
ABCD_API int32_t abcd_layer_norm_bwd_workspace_size(int32_t dtype, int64_t n, int64_t d,
                                                    size_t* bytes);
ABCD_API int32_t abcd_layer_norm_bwd(int32_t dtype, int64_t n, int64_t d, const void* dy,
                                     int64_t lddy, const void* x, int64_t ldx, const float* mean,
                                     const float* rstd, int32_t wdtype, const void* weight,
                                     const void* add, int64_t ldadd, void* dx, int64_t lddx,
                                     void* dweight, void* dbias, void* workspace, size_t ws_bytes,
                                     hipStream_t stream);

/* Dropout: y = residual + keep x / (1 - p), 0 <= p <= 1 (p = 1: nothing is
 * kept; what is dropped becomes 0, infinities and NaN too). residual may be NULL
 * (then 0) and y may be x or residual itself. keep is never stored: element
 * (row, col) takes word col % 4 of the Philox 4x32 block with 7 rounds (Salmon
 * et al. 2011) of the counter (col / 4, row, offset low, offset high) under the
 * key (seed low, seed high), and is kept if the word is >= floor(p 2^32). The
 * gradient is the same call on dy without a residual. Calls whose masks are to
 * be independent differ in offset. */
ABCD_API int32_t abcd_dropout(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx,
                              const void* residual, int64_t ldr, void* y, int64_t ldy, double p,
                              uint64_t seed, uint64_t offset, hipStream_t stream);

/* Gated feed-forward block over rows x[n][d]:
 *   h = act(x w_gate' + b_gate) * (x w_up' + b_up);  y = residual + dropout(h w_down' + b_down)
 * with h of width `h` and y of width `o`. Weights are contiguous, one row per
 * output: w_gate and w_up [h][d], w_down [o][h]; biases [h], [h], [o], each may be
 * NULL (0). Dropout as in abcd_dropout over y's n rows (p = 0: none). act:
 * ABCD_ACT_SILU g sigmoid(g), ABCD_ACT_GELU g Phi(g) (Phi the normal distribution,
 * by the error function; in 16-bit types within 5e-6 of its size), ABCD_ACT_RELU
 * max(g, 0); of a NaN each gives NaN, as value and as derivative. Products and act are
 * computed in fp32. (ABCD_ACT_SIGMOID and ABCD_ACT_NONE are a linear layer's.) h, its derivatives by the pre-activations and the gradients that
 * reach these are rounded to dtype where they go from one product to the next, in
 * memory or in registers, and the weights' and biases' gradients are sums of what was
 * rounded. In float16 this bounds their range too: beyond 65,504 they are infinities,
 * below 2^-25 zeros, whatever y and the weights' gradients come to, so that a loss is
 * scaled as float16 training does. In float32 a product may give NaN where an infinity
 * among what it multiplies (x, dy, a weight, h) would make it infinite, and numbers below
 * 2^-110 have fewer digits in it. */
enum { ABCD_ACT_SILU = 0, ABCD_ACT_GELU = 1, ABCD_ACT_RELU = 2, ABCD_ACT_SIGMOID = 3, ABCD_ACT_NONE = 4 };
typedef struct abcd_ffn {
  int32_t dtype, act;
  int64_t d, h, o;
  const void *w_gate, *w_up, *w_down;
  const void *b_gate, *b_up, *b_down;
  double p;
  uint64_t seed, offset;
} abcd_ffn;

/* *keeps = 1 if a training step does best to let the forward keep by_gate, by_up and
 * hidden for the backward, 0 if the backward makes them again faster than it would
 * read them (narrow blocks). Either way both are correct. */
ABCD_API int32_t abcd_gated_ffn_keeps(const abcd_ffn* ffn /* host */, int64_t n, int32_t* keeps);

/* Forward. residual (may be NULL) and y: [n][o], y may be residual itself. by_gate,
 * by_up, hidden: all NULL, or arrays [n][(h + 7) / 8 * 8] of dtype, 16-byte
 * aligned, that receive for the backward h's derivatives by the two
 * pre-activations and h itself (columns past h: zeros). workspace: at least
 * abcd_gated_ffn_workspace_size(ffn, n, saved) bytes (saved: 1 if by_gate, by_up
 * and hidden are given, else 0), 256-byte aligned. With and without these the sums may
 * be taken in another order. */
ABCD_API int32_t abcd_gated_ffn_workspace_size(const abcd_ffn* ffn /* host */, int64_t n,
                                               int32_t saved, size_t* bytes);
ABCD_API int32_t abcd_gated_ffn(const abcd_ffn* ffn /* host */, int64_t n, const void* x,
                                int64_t ldx, const void* residual, int64_t ldr, void* y,
                                int64_t ldy, void* by_gate, void* by_up, void* hidden, void* workspace,
                                size_t ws_bytes, hipStream_t stream);

/* Backward: gradients of x (not counting the residual path, whose gradient is dy
 * itself) and of every weight and bias, written, of dtype, laid out as what they
 * belong to; each may be NULL, then not computed. by_gate, by_up, hidden: the
 * forward's, or all NULL: then they are computed again from x (one product more, and no
 * memory held between the passes). p, seed and offset are the forward's. No output may
 * overlap an input. */
ABCD_API int32_t abcd_gated_ffn_bwd_workspace_size(const abcd_ffn* ffn /* host */, int64_t n,
                                                   int32_t saved, size_t* bytes);
ABCD_API int32_t abcd_gated_ffn_bwd(const abcd_ffn* ffn /* host */, int64_t n, const void* dy,
                                    int64_t lddy, const void* x, int64_t ldx, const void* by_gate,
                                    const void* by_up, const void* hidden, void* dx, int64_t lddx,
                                    void* dw_gate, void* dw_up, void* dw_down, void* db_gate,
                                    void* db_up, void* db_down, void* workspace, size_t ws_bytes,
                                    hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Operators around the decoder's blocks, for the same rows and element types. */

/* Features that rows share: y[i] = scale table[index[i]] for n indexes (index_bits:
 * 32 or 64, signed) into a table of m rows (1 <= m <= ABCD_MAX_GAUSSIANS, type tdtype:
 * dtype or ABCD_F32; scale finite). An index outside [0, m), as of a place of a batch that holds
 * nothing, gives a row of zeros. y may not overlap the table. */
ABCD_API int32_t abcd_embed(int32_t dtype, int64_t n, int64_t m, int64_t d, int32_t tdtype,
                            const void* table, int64_t ldt, int32_t index_bits, const void* index,
                            float scale, void* y, int64_t ldy, hipStream_t stream);

/* The n positions by index: order[n] (positions; of equal indexes in order, those
 * outside the table last), rows[n] (their indexes, m for those outside the table) and
 * ranges[m][2] (where row r's positions begin and end in order; 0, 0 for a row with none). A
 * set of indexes that does not change is sorted once for all its gradients. workspace: at
 * least abcd_embed_sort_workspace_size bytes, 256-byte aligned. */
ABCD_API int32_t abcd_embed_sort_workspace_size(int64_t n, int64_t m, size_t* bytes);
ABCD_API int32_t abcd_embed_sort(int64_t n, int64_t m, int32_t index_bits, const void* index,
                                 int32_t* order, int32_t* rows, int32_t* ranges, void* workspace,
                                 size_t ws_bytes, hipStream_t stream);

/* The table's gradient: dtable[r] = scale times the sum of dy[i] over the i with index
 * r, zeros for a row with none (written, not added to; type wdtype: dtype or ABCD_F32; ldt
 * elements between its rows). order, rows and ranges: abcd_embed_sort's, of the same n and
 * m, unchanged (what they hold is not checked on the host; with others the result is wrong). workspace: at least abcd_embed_bwd_workspace_size
 * bytes, 256-byte aligned. */
ABCD_API int32_t abcd_embed_bwd_workspace_size(int64_t n, int64_t d, size_t* bytes);
ABCD_API int32_t abcd_embed_bwd(int32_t dtype, int64_t n, int64_t m, int64_t d, const void* dy,
                                int64_t lddy, const int32_t* order, const int32_t* rows,
                                const int32_t* ranges, float scale, int32_t wdtype, void* dtable,
                                int64_t ldt, void* workspace, size_t ws_bytes, hipStream_t stream);

/* The same gradient from the indexes themselves, for up to ABCD_EMBED_FEW positions: one
 * launch, without a sort or a workspace. */
#define ABCD_EMBED_FEW 64
ABCD_API int32_t abcd_embed_bwd_few(int32_t dtype, int64_t n, int64_t m, int64_t d, const void* dy,
                                    int64_t lddy, int32_t index_bits, const void* index, float scale,
                                    int32_t wdtype, void* dtable, int64_t ldt, hipStream_t stream);

/* The joint between two blocks: a block's result f, normed, gated and scaled, goes
 * onto the residual path x, and the next block takes that normed:
 *   t = post(f);  y = x + scale gate t;  z = pre(y)
 * post and pre are each ABCD_NORM_NONE (t = f; no z), ABCD_NORM_LAYER, (v - mean) rstd
 * weight + bias with mean and rstd as in abcd_layer_norm, or ABCD_NORM_RMS, v rstd weight
 * with rstd = 1 / sqrt(mean(v^2) + eps). Weights, biases and scale (d elements of type
 * wdtype: dtype or ABCD_F32) may be NULL, then 1 and 0; they go with the norm that has them
 * (no bias with ABCD_NORM_RMS). gate: ABCD_GATE_NONE (1), ABCD_GATE_ROW, one number a row
 * (row r's at gate + r ldg), or ABCD_GATE_ELEMENT, [n][d]; of dtype, taken as it is. */
enum { ABCD_NORM_NONE = 0, ABCD_NORM_LAYER = 1, ABCD_NORM_RMS = 2 };
enum { ABCD_GATE_NONE = 0, ABCD_GATE_ROW = 1, ABCD_GATE_ELEMENT = 2 };
typedef struct abcd_joint {
  int32_t dtype, wdtype;
  int32_t post, pre, gate;
  float eps;
  int64_t d;
  const void *post_weight, *post_bias, *pre_weight, *pre_bias, *scale;
} abcd_joint;

/* Forward. z is the norm of y before y is rounded; z is NULL if and only if pre is
 * ABCD_NORM_NONE. The statistics (fp32, n each; means of layer norms only) may be NULL, then not
 * written; the backward needs them. No output may overlap an input. */
ABCD_API int32_t abcd_residual_norm(const abcd_joint* joint /* host */, int64_t n, const void* f,
                                    int64_t ldf, const void* x, int64_t ldx, const void* gate,
                                    int64_t ldg, void* y, int64_t ldy, void* z, int64_t ldz,
                                    float* post_mean, float* post_rstd, float* pre_mean,
                                    float* pre_rstd, hipStream_t stream);

/* Backward, from the gradients dz of z (NULL if and only if there is no z) and dy that
 * reaches y by other paths (NULL: none, with a z only); y and the statistics are the forward's:
 * gradients of x, f, gate (laid out as the gate is) and of the parameters (sums over the
 * rows, type wdtype), written, not added to; each may be NULL, then not computed, and is
 * NULL where there is no such gate or norm (dscale may be given without a scale). workspace: at
 * least abcd_residual_norm_bwd_workspace_size bytes, 256-byte aligned. No output may overlap an input. */
ABCD_API int32_t abcd_residual_norm_bwd_workspace_size(const abcd_joint* joint /* host */,
                                                       int64_t n, size_t* bytes);
ABCD_API int32_t abcd_residual_norm_bwd(
    const abcd_joint* joint /* host */, int64_t n, const void* dz, int64_t lddz, const void* dy,
    int64_t lddy, const void* f, int64_t ldf, const void* y, int64_t ldy, const void* gate,
    int64_t ldg, const float* post_mean, const float* post_rstd, const float* pre_mean,
    const float* pre_rstd, void* dx, int64_t lddx, void* df, int64_t lddf, void* dgate, int64_t lddg,
    void* dpost_weight, void* dpost_bias, void* dpre_weight, void* dpre_bias, void* dscale,
    void* workspace, size_t ws_bytes, hipStream_t stream);

/* Checkpoints of activations in 8 bits. Of every ABCD_PACK8_BLOCK consecutive elements
 * of a row (the last block may have fewer), with 2^e the largest power of two that does
 * not exceed the largest finite magnitude (e at least -120):
 *   q = rint(x 2^(6 - e)) between -127 and 127, which stands for q 2^(e - 6);
 * an infinity or a NaN is q = -128 and comes back as NaN. q: [n][blocks][32] (elements past
 * the row's end 0), 16-byte aligned; e: [n][blocks], the byte e + 127; blocks = (d + 31) / 32.
 * What was packed and unpacked packs to the same again. abcd_unpack8 writes dtype, which
 * is the packed one's: its numbers hold q 2^(e - 6) exactly. */
#define ABCD_PACK8_BLOCK 32
ABCD_API int32_t abcd_pack8(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx,
                            int8_t* q, uint8_t* e, hipStream_t stream);
ABCD_API int32_t abcd_unpack8(int32_t dtype, int64_t n, int64_t d, const int8_t* q,
                              const uint8_t* e, void* y, int64_t ldy, hipStream_t stream);

/* Linear layer of rows x[n][i]: y = residual + act(x w' + b), [n][o]. w: [o][i],
 * contiguous, one row per output; b [o] may be NULL (0). act: those of the gated block, as
 * it computes them, ABCD_ACT_SIGMOID 1 / (1 + e^-z) or ABCD_ACT_NONE. Products, act and sums in
 * fp32, with the gated block's limits in float32. */
typedef struct abcd_layer {
  int32_t dtype, act;
  int64_t i, o;
  const void *w, *b;
} abcd_layer;

/* Forward. residual (may be NULL), and y, which may be residual itself but may not overlap x. slope: NULL, or
 * [n][(o + 7) / 8 * 8], 16-byte aligned, that receives for the backward act's derivative (floats
 * with ABCD_F32, else a code of 16 bits, 30,800 times the slope's root; columns past o: zeros; with
 * ABCD_ACT_NONE nothing is written). workspace: at least
 * abcd_linear_workspace_size bytes, 256-byte aligned; NULL where that is 0. */
ABCD_API int32_t abcd_linear_workspace_size(const abcd_layer* layer /* host */, int64_t n, size_t* bytes);
ABCD_API int32_t abcd_linear(const abcd_layer* layer /* host */, int64_t n, const void* x, int64_t ldx,
                             const void* residual, int64_t ldr, void* y, int64_t ldy, void* slope,
                             void* workspace, size_t ws_bytes, hipStream_t stream);

/* Backward, with dz = dy act'(x w' + b): dx = dz w, dw = dz' x, db = the sum of dz's rows
 * (the residual's gradient is dy itself); written, of dtype, laid out as what they belong to;
 * each may be NULL, then not computed. Both products take dz rounded to dtype; db sums it as
 * it was before that, or rounded where the slopes of many rows of a wide layer are made again. x: the forward's
 * rows, or NULL and q and e, an 8-bit checkpoint of them (abcd_pack8), whose numbers are then x,
 * in the slopes too where these are made again. slope: the forward's, or NULL: made again
 * from x, w and b. workspace: at least abcd_linear_bwd_workspace_size bytes, 256-byte
 * aligned. No output may overlap an input. */
ABCD_API int32_t abcd_linear_bwd_workspace_size(const abcd_layer* layer /* host */, int64_t n, size_t* bytes);
ABCD_API int32_t abcd_linear_bwd(const abcd_layer* layer /* host */, int64_t n, const void* dy, int64_t lddy,
                                 const void* x, int64_t ldx, const int8_t* q, const uint8_t* e,
                                 const void* slope, void* dx, int64_t lddx, void* dw, void* db,
                                 void* workspace, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------ */
/* Helpers. abcd_last_error: message of the last failure on this thread.
 * abcd_timing_*: optional per-kernel HIP-event timing of every launch made by
 * this thread (off by default; enabling it adds two event records per launch
 * on the caller's stream). abcd_timing_read synchronises, and returns the
 * accumulated milliseconds and launch count of the kernel named `kernel`
 * (names: composite, project, bin_zero, depth_keys, radix_pass, l1_place,
 * l2_count, l2_scatter, bin_small_sort, bin_small_collect, bin_empty, bin_count,
 * render_fwd, loss_l1, zero_fill, bwd_order, render_bwd, project_bwd, adam,
 * render_cache, cache_rect_init, layer_norm, layer_norm_bwd, layer_norm_cols,
 * sum_parts, dropout, pack_rows, column_sums, ffn_in, ffn_out, ffn_dhidden, ffn_dx,
 * ffn_join, ffn_dweight, ffn_dweight_sum, ffn_narrow, ffn_narrow_bwd, ffn_few_in, ffn_few_out,
 * embed, embed_count, embed_scan, embed_scatter, embed_ranges, embed_rank, embed_bwd, embed_bwd_few,
 * embed_join, pack8, unpack8, residual_norm, residual_norm_bwd, residual_norm_sums,
 * linear_out, linear_few, linear_dz, linear_dx, linear_slope, linear_narrow,
 * linear_narrow_bwd). */
ABCD_API const char* abcd_last_error(void);
ABCD_API const char* abcd_version(void);
ABCD_API const char* abcd_status_string(int32_t status);
ABCD_API int32_t abcd_timing_enable(int32_t enable);
ABCD_API int32_t abcd_timing_reset(void);
ABCD_API int32_t abcd_timing_read(const char* kernel, double* total_ms, int64_t* launches);

#ifdef __cplusplus
}
#endif
#endif /* ABCD_H */
