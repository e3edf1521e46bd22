/*
 * dab.h - C ABI of the MI355X (gfx950) hot path of distribution-aware
 * binarization, after "Distribution-Aware Binarization of Neural Networks for
 * Sketch Recognition" (arXiv 1804.02941).
 *
 * The path: a layer's real-valued filters W_f (n = c*w*h weights each) are
 * replaced by W~_f = alpha_f*e_f + beta_f*(1 - e_f) with a 0/1 mask e_f
 * (Section 4.1, Theorem 2); the mask comes from a split of the sorted weights
 * found with prefix sums (Section 4.3.1, Algorithm 1); inputs of the layer are
 * binary, +1 / -1 (Section 4); the layer output is the ordinary convolution of
 * the binary input with W~ (Section 4.3.2).  Since W~ takes two values,
 *     y = alpha*s1 + beta*s2,  s1 = sum a_i e_i,  s2 = sum a_i (1 - e_i),
 * over the taps inside the image, with s1 + s2 = sA = sum a_i.  One bit per
 * weight and per activation is what crosses this interface; s1 is an exact
 * integer contraction of the two bit tensors and the two scalars recombine it
 * with the per-pixel sum sA.
 *
 * General rules
 *   - All data pointers are DEVICE pointers unless a comment says "host".
 *     The caller owns every buffer; the library allocates nothing and never
 *     frees or retains a pointer.  Its only state is a one-time set-up per
 *     device (dab_init), which every entry point that needs it performs on
 *     its first call on that device.
 *   - "stream" is a hipStream_t passed as void* (NULL = the null stream).
 *     Work is enqueued on it and the call returns without synchronising.
 *   - Every call returns a dab_status.  Arguments are validated on the host
 *     before anything is enqueued: on DAB_ERR_NULL, _SHAPE, _ALIGN, _WORKSPACE
 *     and _UNSUPPORTED nothing was launched.  A failing launch gives
 *     DAB_ERR_HIP (the status of that launch call, kept for
 *     dab_last_hip_error()); kernels of the same call enqueued before it
 *     stay enqueued and only write the call's own outputs and workspace.
 *     Faults inside a kernel surface at the caller's next synchronisation,
 *     as with any HIP work.
 *   - Float buffers are fp32, 4-byte aligned; packed buffers and Y are
 *     16-byte aligned (DAB_ERR_ALIGN otherwise).
 *   - Inputs must be finite.  A NaN activation binarizes to -1 (x >= tau is
 *     false); NaN weights give unspecified masks.
 *
 * Packed layouts (bit k of a word = (word >> k) & 1, least significant first)
 *   Activations  uint32 [B][H][W][Cw], Cw = ceil(C/32).  Bit (c mod 32) of
 *                word (c div 32) of pixel (b,h,w) is 1 iff a[b,c,h,w] = +1.
 *                Bits past C are 0.  A fully-connected input is H = W = 1.
 *   Weights      uint32 [R][Fp], R = kh*kw*Cw, Fp = 64*ceil(F/64).  Row
 *                r = (ky*kw + kx)*Cw + (c div 32), column f, bit (c mod 32) is
 *                e[f,c,ky,kx].  Bits past C and columns past F are 0.
 *                (Word-major: the word of one reduction position is contiguous
 *                over the filters, which is how both packing and expansion walk it.)
 *   Tap counts   uint32 [F][kh*kw]: ecnt[f][ky*kw+kx] = sum_c e[f,c,ky,kx]; their sum
 *                over the taps is K_f.  They describe the mask (and check it); the
 *                layer kernels do not need them.
 */
#ifndef DAB_H
#define DAB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum dab_status {
    DAB_OK = 0,
    DAB_ERR_NULL = 1,        /* a required pointer is NULL                          */
    DAB_ERR_SHAPE = 2,       /* a size is non-positive, n < 2, or the output empty  */
    DAB_ERR_ALIGN = 3,       /* a buffer is not aligned as stated above             */
    DAB_ERR_WORKSPACE = 4,   /* ws is NULL or smaller than the *_workspace_bytes    */
    DAB_ERR_UNSUPPORTED = 5, /* valid problem outside what the kernels cover        */
    DAB_ERR_HIP = 6          /* a HIP call failed; see dab_last_hip_error()         */
} dab_status;

typedef enum dab_layout {
    DAB_LAYOUT_NHWC = 0,     /* X[b][h][w][c], the native layout                    */
    DAB_LAYOUT_NCHW = 1      /* X[b][c][h][w], packed through a transposing kernel  */
} dab_layout;

/* One binarized convolution.  Output size Ho = (H + 2*pad_h - kh)/stride_h + 1,
 * Wo likewise; both must be >= 1. */
typedef struct dab_conv_desc {
    int32_t B, C, H, W;                 /* input: batch, channels, height, width */
    int32_t F, kh, kw;                  /* filters and their spatial extent      */
    int32_t pad_h, pad_w;               /* zero padding on each side             */
    int32_t stride_h, stride_w;
} dab_conv_desc;

/* Text for a status code (static storage, never NULL). */
const char* dab_strerror(int status);

/* hipError_t of the last failed HIP call made by this thread (0 if none). */
int dab_last_hip_error(void);

/*
 * dab_init - one-time set-up of the current device: raises the dynamic-LDS limit of the kernels
 * that stage more than the default 48 KB and looks up the address of the library's own device
 * memory.  Optional: entry points that depend on it do the same on their first call on a device.
 * Callers that capture a stream into a graph call it before the capture begins, so that no
 * attribute call falls inside it.  Thread-safe; later calls return at once.
 */
int dab_init(void);

/*
 * dab_estimate_alpha_beta - optimal alpha, beta, K and split of every filter.
 * Section 4.1 (Theorem 2) and Section 4.3.1 / Algorithm 1: sort the n weights
 * of a filter, form prefix sums P_i, score every split i = 1..n-1 with
 * D_i = P_i^2/i + (T - P_i)^2/(n - i), take the largest i of maximal D.  The
 * lower group is the i smallest weights (ties by original index), the upper
 * group the rest; alpha is the mean of the group whose mean has the greater
 * magnitude (the upper group if equal), beta the other mean, K the size of
 * the alpha group.  Sums and scores are accumulated in fp64; alpha and beta
 * are rounded to fp32 at the end.
 *
 *   W              [F][n] fp32, row f = filter f flattened in (c,ky,kx) order
 *   alpha, beta    [F] fp32 out
 *   K              [F] int32 out, 1 <= K <= n-1
 *   thr_val        [F] fp32 out: value of the largest element of the lower group
 *   thr_idx        [F] int32 out: its index in the row; element i is in the lower
 *                  group iff w_i < thr_val or (w_i == thr_val and i <= thr_idx)
 *   alpha_is_upper [F] uint8 out: 1 if the alpha group is the upper group
 *   ws, ws_bytes   scratch of at least dab_estimate_workspace_bytes(F, n) bytes (one flag per
 *                  filter for rows of 4096 weights and more, nothing for shorter rows).
 *                  Most rows are estimated without a full sort: value
 *                  buckets with exact integer sums give D at every bucket end and an
 *                  upper bound inside every bucket, and only the few elements of the
 *                  buckets that can hold the arg-max are ranked exactly; rows where that
 *                  does not apply (many equal values) are sorted, the long ones through
 *                  their flag in ws by a second kernel.  The result is the same split.
 *                  ws may be NULL (or too small): then every long row is sorted.
 * Errors: NULL pointers, F < 1 or n < 2 (a filter needs both groups non-empty)
 * -> DAB_ERR_SHAPE; n above the largest supported row (dab_estimate_max_n())
 * -> DAB_ERR_UNSUPPORTED.
 */
int dab_estimate_alpha_beta(const float* W, int32_t F, int32_t n,
                            float* alpha, float* beta, int32_t* K,
                            float* thr_val, int32_t* thr_idx, uint8_t* alpha_is_upper,
                            void* ws, size_t ws_bytes, void* stream);
size_t dab_estimate_workspace_bytes(int32_t F, int32_t n);
int32_t dab_estimate_max_n(void);

/*
 * dab_estimate_alpha_beta_noalloc - dab_estimate_alpha_beta for callers that cannot allocate
 * device memory or bring a workspace: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  The per-row hand-over flags live in a device array that is part of the
 * library (dab_estimate_noalloc_max_filters() bytes, held by every GPU the library runs on until
 * the process ends), so the call takes no workspace and makes no allocating call (its address is
 * looked up once per device, by dab_init or by the first call).  Same kernels, same outputs, bit
 * for bit, as dab_estimate_alpha_beta with a workspace.
 *
 *   arguments as for dab_estimate_alpha_beta, without ws / ws_bytes
 * Errors: as dab_estimate_alpha_beta; F above dab_estimate_noalloc_max_filters()
 * -> DAB_ERR_UNSUPPORTED.  All calls on one GPU share the one array (every flag a call reads it
 * has written itself, so nothing needs clearing between calls): two such calls whose work may
 * overlap on the same GPU (different streams) race; calls on one stream are safe.
 */
int dab_estimate_alpha_beta_noalloc(const float* W, int32_t F, int32_t n,
                                    float* alpha, float* beta, int32_t* K,
                                    float* thr_val, int32_t* thr_idx, uint8_t* alpha_is_upper, void* stream);
int32_t dab_estimate_noalloc_max_filters(void);

/*
 * dab_estimate_alpha_beta_bounded - the same estimate with the split kept near the previous
 * iteration's.  Section 5 remarks that on natural images the algorithm needs K restricted to
 * change by slight amounts only and gives no rule; here the partition may move by at most
 * max_change elements: with i_prev the previous size of the lower group (K_prev if the alpha group
 * was the lower one, n - K_prev otherwise, pulled into 1 .. n-1), the best split is searched over
 * max(1, i_prev - max_change) .. min(n-1, i_prev + max_change) only.  Ties, labelling and outputs
 * are as above; max_change >= n gives dab_estimate_alpha_beta's result, max_change = 0 keeps the
 * previous partition sizes and refreshes alpha, beta and the descriptor for the new weights.
 *
 *   K_prev              [F] int32, alpha_is_upper_prev [F] uint8: the previous call's outputs; they
 *                       may be the very buffers passed as K and alpha_is_upper
 * Errors as above; max_change < 0 -> DAB_ERR_SHAPE.
 */
int dab_estimate_alpha_beta_bounded(const float* W, int32_t F, int32_t n, const int32_t* K_prev,
                                    const uint8_t* alpha_is_upper_prev, int32_t max_change, float* alpha,
                                    float* beta, int32_t* K, float* thr_val, int32_t* thr_idx,
                                    uint8_t* alpha_is_upper, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_estimate_sign_split - the baseline the paper compares with, in the estimator's output form.
 * Section 4.1 notes that XNOR-Net / binary-weight networks are the special case that ignores the
 * weight distribution: e = [w >= 0], alpha = mean |w| over the filter, beta = -alpha.  The outputs
 * can be passed to dab_pack_weights and to the layer calls unchanged, which gives the comparison
 * axis of the paper's tables on the same kernels.
 *
 *   W, alpha, beta, thr_val, thr_idx, alpha_is_upper   as for dab_estimate_alpha_beta
 *   K              [F] int32 out: number of non-negative weights, 0 <= K <= n
 * The lower group is the negative weights: thr_val is the largest negative weight and thr_idx the
 * last index holding it (thr_val = -inf and thr_idx = 0 for a filter without negative weights);
 * alpha_is_upper is 1.  n >= 1; any row length is supported.
 */
int dab_estimate_sign_split(const float* W, int32_t F, int32_t n,
                            float* alpha, float* beta, int32_t* K,
                            float* thr_val, int32_t* thr_idx, uint8_t* alpha_is_upper, void* stream);

/*
 * dab_pack_weights - the mask e of Corollary 1 as bits, plus per-tap counts.
 * e[f,i] = 1 iff weight i of filter f belongs to the alpha group, decided from
 * the split descriptor of dab_estimate_alpha_beta (so the mask is defined by
 * stable rank, not by the sign of the kept values).
 *
 *   W          [F][C][kh][kw] fp32 (kh = kw = 1, C = n for a fully-connected layer)
 *   thr_val, thr_idx, alpha_is_upper   [F], as returned by the estimator
 *   E_packed   uint32 [kh*kw*Cw][Fp] out, every word written (layout above)
 *   ecnt       uint32 [F][kh*kw] out
 * Kernels of up to 384 taps (kh*kw; more -> DAB_ERR_UNSUPPORTED).
 */
int dab_pack_weights(const float* W, int32_t F, int32_t C, int32_t kh, int32_t kw,
                     const float* thr_val, const int32_t* thr_idx, const uint8_t* alpha_is_upper,
                     uint32_t* E_packed, uint32_t* ecnt, void* stream);

/*
 * dab_binarize_weights_multi - the whole weight side of several layers in a few launches (one per
 * class of row length present: up to 2304 weights, up to 4608, up to 9216, longer; plus one behind them
 * for the rows handed to the sort):
 * for every job, dab_estimate_alpha_beta (or, with K_prev, dab_estimate_alpha_beta_bounded) of its
 * filters followed by dab_pack_weights of the resulting masks.  Section 4.3.1 handles all filters of
 * a layer together; filters of different layers are just as independent, so they share the
 * launches (a workgroup looks up its job), and a filter's mask (Corollary 1) is packed by the
 * workgroup that has just found its split, while the row is still in cache.  Results are, bit
 * for bit, those of the separate calls, with one exception: for a row in which several splits have
 * scores that are equal to the last bit or differ only by the rounding of the float64 sums (a
 * constant row is the extreme case), the two may return different ones of those splits, because
 * their sort kernels cut such a row into different per-thread pieces.
 *
 *   jobs      host array of n_jobs descriptors (read during the call only); every pointer inside is a
 *             device pointer with the meaning it has in dab_estimate_alpha_beta / dab_pack_weights.
 *             E_packed and ecnt may both be NULL (estimation only); K_prev and alpha_is_upper_prev
 *             may both be NULL (unrestricted search), else max_change >= 0 bounds the split's move.
 *   ws        scratch of dab_binarize_weights_multi_workspace_bytes(jobs, n_jobs) bytes, 8-byte aligned
 *             (one flag per filter of the jobs whose unfinished rows go to the sort kernel; 0 for a
 *             few layers with rows of at most 4608 weights, which are finished in their own launch)
 * Errors: per job as in the separate calls (rows above dab_estimate_max_n(), more than 128 taps with
 * packing -> DAB_ERR_UNSUPPORTED: such a layer takes the separate calls); more than 16 jobs -> DAB_ERR_UNSUPPORTED; ws missing or too
 * small -> DAB_ERR_WORKSPACE; ws not 8-byte aligned -> DAB_ERR_ALIGN.
 */
typedef struct dab_weight_job {
    const float* W;                       /* [F][C][kh][kw] fp32 */
    int32_t F, C, kh, kw;
    float* alpha; float* beta; int32_t* K; float* thr_val; int32_t* thr_idx; uint8_t* alpha_is_upper;   /* [F] out */
    uint32_t* E_packed; uint32_t* ecnt;   /* out, or both NULL */
    const int32_t* K_prev; const uint8_t* alpha_is_upper_prev; int32_t max_change;   /* previous split, or both NULL */
} dab_weight_job;
size_t dab_binarize_weights_multi_workspace_bytes(const dab_weight_job* jobs /* host */, int32_t n_jobs);
int dab_binarize_weights_multi(const dab_weight_job* jobs /* host */, int32_t n_jobs, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_pack_activations - sign binarization of a layer input (Section 4: inputs
 * are +1 / -1) into bits along the channel dimension: bit = [x >= tau_c],
 * tau = 0 when tau is NULL (sign(0) = +1).
 *
 *   X          fp32, NHWC [B][H][W][C] or NCHW [B][C][H][W] according to layout
 *   tau        [C] fp32 per-channel thresholds, or NULL
 *   A_packed   uint32 [B][H][W][Cw] out, every word written
 */
int dab_pack_activations(const float* X, int32_t layout, int32_t B, int32_t C, int32_t H, int32_t W,
                         const float* tau, uint32_t* A_packed, void* stream);

/*
 * dab_pack_activations_multi - dab_pack_activations for several tensors in one launch: the inputs
 * of all binarized layers of a network that are resident together (Section 4: every binarized
 * layer's input is +1 / -1).  Each job is one NHWC tensor with its own thresholds and output; the
 * results are those of n_jobs separate calls.
 *
 *   jobs      host array of n_jobs descriptors (read during the call only); pointers inside are device pointers
 * Errors: as dab_pack_activations per job; more than 16 jobs -> DAB_ERR_UNSUPPORTED.
 */
typedef struct dab_pack_job {
    const float* X;              /* fp32 NHWC [B][H][W][C] */
    const float* tau;            /* [C] or NULL */
    uint32_t* A_packed;          /* uint32 [B][H][W][ceil(C/32)] out */
    int32_t B, C, H, W;
} dab_pack_job;
int dab_pack_activations_multi(const dab_pack_job* jobs /* host */, int32_t n_jobs, void* stream);

/*
 * dab_prepare_layers - everything that precedes the binary products of a set of resident layers:
 * dab_binarize_weights_multi(wjobs) and dab_pack_activations_multi(pjobs) in the launches of the
 * former.  The weight side (Section 4.3.1, Corollary 1) and the binarization of the inputs (Section 4)
 * do not depend on each other and load different parts of the chip (vector instructions and LDS
 * against memory), so some workgroups of the weight-side launches pack the activations beside
 * the others, which take the filters, and the two overlap inside one launch.  Results are, bit for bit, those of the two
 * separate calls; arguments, workspace and errors are theirs.  In addition: fewer filters in all
 * wjobs together than tensors in pjobs -> DAB_ERR_UNSUPPORTED (call the two separately).
 */
int dab_prepare_layers(const dab_weight_job* wjobs /* host */, int32_t n_wjobs, const dab_pack_job* pjobs /* host */,
                       int32_t n_pjobs, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_binconv2d - binarized convolution, Section 4.3.2's I (*) W~ on packed
 * operands: cross-correlation, zero padding (a padded tap contributes 0),
 * no bias.  For every output pixel p and filter f, over the taps inside the image,
 *     s1 = sum a_i e_i   (exact integer; a = +1/-1 from the activation bits, e from the weight bits),
 *     sA = sum a_i = 2*popc(A) - C * (number of those taps),
 *     Y[p][f] = alpha_f*s1 + beta_f*(sA - s1), evaluated in fp32 as
 *               (alpha_f - beta_f)*s1 + beta_f*sA  (|beta| <= |alpha|, so the rounding
 *               error stays within a few ulp of |alpha||s1| + |beta||s2|).
 *
 *   A_packed   uint32 [B][H][W][Cw]
 *   E_packed   uint32 [kh*kw*Cw][Fp]
 *   alpha,beta [F] fp32
 *   Y          fp32 NHWC [B][Ho][Wo][F] out
 *   dbg_s1     optional int32 [B][Ho][Wo][F] out: the integer s1 of every output
 *              (NULL to skip); this is what bit-exact tests compare
 *   ws         scratch of at least dab_binconv2d_workspace_bytes(d) bytes, 256-byte
 *              aligned (0 bytes for most layers: the kernels then read the packed bits
 *              directly.  Long reductions over many rows ask for room to expand their
 *              operands into, also where the kernel then taken does not write to it);
 *              dead when the call's work has completed (DAB_ERR_WORKSPACE if NULL,
 *              too small or misaligned)
 * Padding may reach or exceed the kernel extent (windows entirely in the border give 0).
 * Errors: |s1| can reach C*kh*kw, which must stay below 2^24 -> DAB_ERR_UNSUPPORTED
 * beyond (also for tensors past 2^31 bytes expanded).
 */
int dab_binconv2d(const dab_conv_desc* d /* host */, const uint32_t* A_packed, const uint32_t* E_packed,
                  const float* alpha, const float* beta,
                  float* Y, int32_t* dbg_s1, void* ws, size_t ws_bytes, void* stream);
size_t dab_binconv2d_workspace_bytes(const dab_conv_desc* d /* host */);

/*
 * dab_binfc - binarized fully-connected layer: the same product with a 1x1
 * spatial extent.  Y[b][f] = alpha_f*s1 + beta_f*s2 over the Kin inputs.
 *
 *   A_packed   uint32 [B][ceil(Kin/32)],  E_packed uint32 [ceil(Kin/32)][Fp]
 *   Y          fp32 [B][F] out;  dbg_s1 optional int32 [B][F]
 *   ws         as for dab_binconv2d, sized by dab_binfc_workspace_bytes
 */
int dab_binfc(int32_t B, int32_t Kin, int32_t F, const uint32_t* A_packed, const uint32_t* E_packed,
              const float* alpha, const float* beta,
              float* Y, int32_t* dbg_s1, void* ws, size_t ws_bytes, void* stream);
size_t dab_binfc_workspace_bytes(int32_t B, int32_t Kin, int32_t F);

/*
 * dab_binconv2d_bits / dab_binfc_bits - the same products with a re-binarizing epilogue: when
 * the next layer is binarized as well (Section 4: its inputs are +1 / -1; the appendix's block
 * puts the sign right after the previous binarized layer), the fp32 output is never needed, only
 *     A_next bit f of pixel p = [ Y[p][f] >= tau_out[f] ],
 * with Y[p][f] evaluated in fp32 exactly as dab_binconv2d evaluates it, so the result is identical,
 * bit for bit, to dab_pack_activations applied to dab_binconv2d's output.  1/32 of the output
 * bytes are written.
 *
 *   tau_out    [F] fp32 thresholds of the next layer's sign, or NULL for 0
 *   A_next     uint32 [B][Ho][Wo][ceil(F/32)] out (dab_binfc_bits: [B][ceil(F/32)]), every word
 *              written, bits past F are 0; this is the packed activation layout above with C = F
 *   other arguments, workspace and errors as for dab_binconv2d / dab_binfc
 */
int dab_binconv2d_bits(const dab_conv_desc* d /* host */, const uint32_t* A_packed, const uint32_t* E_packed,
                       const float* alpha, const float* beta, const float* tau_out, uint32_t* A_next,
                       void* ws, size_t ws_bytes, void* stream);
int dab_binfc_bits(int32_t B, int32_t Kin, int32_t F, const uint32_t* A_packed, const uint32_t* E_packed,
                   const float* alpha, const float* beta, const float* tau_out, uint32_t* A_next,
                   void* ws, size_t ws_bytes, void* stream);

/*
 * dab_pool_bits - max-pooling between two binarized layers, on the packed signs.  The sign of a
 * window's maximum is +1 iff any element's sign is +1 (one threshold per channel), so
 * sign(maxpool(y) - tau) is the bitwise OR of the window's packed words.  Windows lie inside the
 * image (no padding): Ho = (H - kh)/stride_h + 1, Wo likewise.  The Sketch-A-Net architecture that
 * Section 5.1 trains (the network of the work it cites) pools 3x3 with stride 2 between binarized
 * layers.
 *
 *   A_packed   uint32 [B][H][W][ceil(C/32)];  A_pooled uint32 [B][Ho][Wo][ceil(C/32)] out
 * Errors: a window larger than the image -> DAB_ERR_SHAPE.
 */
int dab_pool_bits(const uint32_t* A_packed, int32_t B, int32_t C, int32_t H, int32_t W, int32_t kh, int32_t kw,
                  int32_t stride_h, int32_t stride_w, uint32_t* A_pooled, void* stream);

/*
 * dab_wbin_conv2d / dab_wbin_fc - the weights-only binarized layer (Section 5.1's WBin: the
 * convolutional weights binarized, the inputs left real): y = x (*) W~ with
 * W~ = alpha e + beta (1 - e) (Sections 4.1, 4.3.2), evaluated as
 *     y[p][f] = beta[f] * sum_i x_i + (alpha[f] - beta[f]) * sum_i x_i e_i
 * over the taps inside the image (zero padding, cross-correlation, no bias).  The second sum is a
 * dense contraction and runs on the matrix cores: each fp32 input is split exactly into three bf16
 * pieces, the mask is bf16 0 / 1, so every product is exact and only the fp32 accumulation rounds.
 *
 *   X          fp32 NHWC [B][H][W][C] (dab_wbin_fc: [B][Kin]), finite, 16-byte aligned
 *   E_packed, alpha, beta   as for dab_binconv2d (the outputs of dab_pack_weights / the estimator)
 *   Y          fp32 NHWC [B][Ho][Wo][F] out (dab_wbin_fc: [B][F])
 *   ws         workspace of dab_wbin_conv2d_workspace_bytes(d) bytes (dab_wbin_fc_workspace_bytes),
 *              256-byte aligned.  (The operands are expanded on the way into the matrix cores, so nothing is
 *              written there; the size is still asked for, and a call that brings less refused.)
 * Accuracy: fp32 accumulation of exact terms; the error is bounded by about (3*n/16 + T) * 2^-24
 * times sum_i |x_i| |w~_i| (n = C*kh*kw, T = kh*kw) and is typically a few 1e-7 of that scale.
 * Errors as for dab_binconv2d.
 */
size_t dab_wbin_conv2d_workspace_bytes(const dab_conv_desc* d /* host */);
size_t dab_wbin_fc_workspace_bytes(int32_t B, int32_t Kin, int32_t F);
int dab_wbin_conv2d(const dab_conv_desc* d /* host */, const float* X, const uint32_t* E_packed, const float* alpha,
                    const float* beta, float* Y, void* ws, size_t ws_bytes, void* stream);
int dab_wbin_fc(int32_t B, int32_t Kin, int32_t F, const float* X, const uint32_t* E_packed, const float* alpha,
                const float* beta, float* Y, void* ws, size_t ws_bytes, void* stream);

/*
 * Weight-side steps of one training iteration (Algorithm 2).  The real weights are mean-centred
 * and clamped, every filter is binarized (dab_estimate_alpha_beta on the result), W~ is formed for
 * the forward and backward pass, and the gradient with respect to W~ is turned into the gradient
 * applied to the real weights (Theorem 4).  All buffers are device memory; W is [F][C][kh][kw]
 * fp32, seen as F rows of n = C*kh*kw.
 */
typedef enum {
    DAB_CENTER_FILTER = 0,   /* subtract the mean of the filter's n weights                    */
    DAB_CENTER_CHANNEL = 1   /* subtract, per filter and tap, the mean over the C channels     */
} dab_center_axis;

/*
 * dab_mean_center_clamp - MeanCenter, then Clamp(lo, hi) (Algorithm 2 lists them in this order
 * and does not name the axis of the mean; both conventions above are provided).  The mean is
 * accumulated in double, the centred value is rounded once to fp32.
 *
 *   W      [F][C][T] fp32 in (T = kh*kw);  W_out the same shape, may be W itself (in place)
 * Errors: lo > hi or a non-positive size -> DAB_ERR_SHAPE; another axis -> DAB_ERR_UNSUPPORTED.
 */
int dab_mean_center_clamp(const float* W, int32_t F, int32_t C, int32_t T, int32_t axis, float lo, float hi,
                          float* W_out, void* stream);

/*
 * dab_binarized_weights - W~ = alpha e + beta (1 - e) as fp32 (the last line of Algorithm 2's
 * binarization loop), with e taken from the split descriptor exactly as dab_pack_weights takes it.
 *
 *   W, alpha, beta, thr_val, thr_idx, alpha_is_upper   as for dab_estimate_alpha_beta
 *   W_tilde  [F][n] fp32 out, every element alpha[f] or beta[f]; must not overlap W
 */
int dab_binarized_weights(const float* W, int32_t F, int32_t n, const float* alpha, const float* beta,
                          const float* thr_val, const int32_t* thr_idx, const uint8_t* alpha_is_upper,
                          float* W_tilde, void* stream);

/*
 * dab_weight_gradient - Theorem 4 (derived in the appendix): G~ = G~1 + G~2, element-wise.  With e
 * the mask of the split descriptor, K its number of ones, T_k = W o e and R = W - T_k,
 *     G~_i = e_i/K + (||T_k||_1 / K) T_k^i [|W_i| <= 1] + (1-e_i)/(n-K) + (||R||_1 / (n-K)) R^i [|W_i| <= 1]
 * (the theorem's sgn(T_k) and sgn(W - T_k) are the masks e and 1 - e, as its derivation
 * substitutes them; STE passes the value where |W_i| <= 1).  With an upstream gradient dC/dW~ the
 * output is its element-wise product with G~, the gradient applied to the real weights.
 *
 *   W         [F][n] fp32, the mean-centred, clamped weights that were binarized (n >= 2)
 *   upstream  [F][n] fp32 or NULL
 *   G_out     [F][n] fp32 out; must not overlap W
 * K and the two l1 norms are recomputed from W and the descriptor (double accumulation).  A
 * descriptor whose mask is empty or full is outside the theorem; that group's terms are 0.
 */
int dab_weight_gradient(const float* W, int32_t F, int32_t n, const float* thr_val, const int32_t* thr_idx,
                        const uint8_t* alpha_is_upper, const float* upstream, float* G_out, void* stream);

/*
 * The real-valued ends of a binarized network: what a training step keeps for its backward pass, the
 * loss, and the layers that are not binarized when they serve.  Section 5.1 leaves a network's first
 * and last layers real; with a large vocabulary behind the last one these are a language model's
 * largest matrices.
 *
 * Element types of these calls, and the strides of their inputs: a matrix [rows][cols] is given with
 * the distance ld of its rows in elements (ld >= cols), so that a slice of columns whose first element is 16-byte
 * aligned needs no copy: base pointers are 16-byte aligned (DAB_ERR_ALIGN), the rows behind the first one at any
 * element.  fp32 vectors, scale bytes and targets are aligned as their type wants.  Outputs are contiguous, and overlap nothing else of
 * the call but what its description names.  Offsets are 64-bit.
 * Larger sizes than each call names are DAB_ERR_UNSUPPORTED.
 */
typedef enum dab_dtype {
    DAB_F32 = 0,
    DAB_BF16 = 1,
    DAB_F16 = 2
} dab_dtype;

/*
 * dab_ckpt8_save / dab_ckpt8_restore - a layer's real input held in 8 bits until its backward pass.
 * A group is 32 neighbouring channels of a row (the last one may be short).  With a the largest
 * magnitude of a group and f = floor(log2 a), its exponent is e = f - 6, or f - 5 where a 2^-e would
 * lie at or above 127.5; a value is q = x 2^-e rounded to the nearest integer, ties to even, so |q| <= 127 and
 * |x - q 2^e| <= 2^(e-1) < a/127, for groups with a from 2^-104 to 127.5 2^121.  f - 6 is kept within -110 .. 120 and |q| at
 * 127: below, steps are 2^-110 and a group loses its digits; above, at the end of fp32's range, e is 121 and
 * magnitudes are cut to 127 steps, by less than one of them.  The scale is a
 * power of two because undoing it is then exact in every type that has 8 significant bits: a
 * restored value is a bf16 number.
 *
 *   X    [rows][cols] of dtype, rows ldx apart
 *   Q    int8 [rows][32*ceil(cols/32)] out, zeros behind the last channel
 *   S    uint8 [rows][ceil(cols/32)] out: e + 127 (17 .. 248); a group of zeros has 17; a group with an
 *        infinity or a NaN has 255, and is restored as NaN throughout
 * restore writes [rows][cols] of dtype, rows ldx apart (f16: rounded to nearest, infinite where too large).
 */
int dab_ckpt8_save(const void* X, int32_t dtype, int32_t rows, int32_t cols, int64_t ldx, int8_t* Q, uint8_t* S, void* stream);
int dab_ckpt8_restore(const int8_t* Q, const uint8_t* S, int32_t rows, int32_t cols, void* X, int32_t dtype, int64_t ldx,
                      void* stream);

/*
 * dab_ckpt8_weight_gradient - the upstream gradient of a fully-connected layer's weights from its saved
 * input: dW[f][c] = sum over rows of dY[row][f] * (q 2^e)[row][c], which is what dab_weight_gradient takes as
 * `upstream` for a binarized layer.  On the matrix cores in bf16: the saved values are bf16 numbers, a
 * bf16 gradient is used as it is, an f16 one as the sum of two bf16 numbers and an fp32 one as the sum of
 * three, so that every product is exact (pieces have steps of 2^-133) and only the fp32 accumulation rounds.  Infinities and NaN in dY come
 * out as in the sum itself.
 *
 *   dY   [rows][F] of dtype, rows lddy apart;   dW  fp32 [F][cols] out.  F, cols and lddy are below 2^22, rows below 2^31 - 63
 *   ws   dab_ckpt8_weight_gradient_workspace_bytes(...) bytes, 256-byte aligned
 */
size_t dab_ckpt8_weight_gradient_workspace_bytes(int32_t rows, int32_t cols, int32_t F, int32_t dtype, int64_t lddy);
int dab_ckpt8_weight_gradient(const void* dY, int32_t dtype, int64_t lddy, const int8_t* Q, const uint8_t* S, int32_t rows,
                              int32_t cols, int32_t F, float* dW, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_head_loss - softmax cross entropy of L = H W^T over a vocabulary, without the logits: for every token t
 *     lse_t = log sum_v exp(L_tv),   loss_t = lse_t - L_t,target(t).
 * The products run on the matrix cores a block of the vocabulary at a time; of a block only its rows'
 * maxima and sums and the targets' logits leave the compute unit.  Sums and logits are fp32.  fp32
 * inputs are multiplied as they are where tokens are few, else as sums of three bf16 numbers (six
 * products of pieces, what is left out is below 2^-24 of a term): the workspace then holds 6 bytes for every
 * element of H and W, in the loss and in the gradient.
 *
 *   H        [T][D] of dtype (DAB_BF16 or DAB_F32; DAB_F16 -> DAB_ERR_UNSUPPORTED: softmax gradients leave its
 *            range), rows ldh apart
 *   W        [V][D] of the same dtype, rows ldw apart.  T and V are below 2^30, ldh and ldw below 2^22, and T x V
 *            is below 2^25 tiles of 128 x 128, T x D below 2^21
 *   targets  [T] int64; ignore_index marks a token without a loss (its row of H may hold anything, infinities and NaN
 *            among it: loss 0, no part in any gradient).  A target that is neither that nor one of 0 .. V-1 gives a loss of
 *            NaN, and its token no part in any gradient.
 *   loss     [T] fp32 out, lse [T] fp32 out (0 for an ignored token)
 *   ws       dab_head_loss_workspace_bytes(...) bytes, 256-byte aligned
 * A NaN in a token's row of H, or in any row of W, gives that token (every token) a loss and an lse of NaN.  Words whose logits are minus
 * infinity have probability 0; but where fp32 inputs are multiplied as pieces an infinity in H or W may give NaN.
 */
size_t dab_head_loss_workspace_bytes(int32_t T, int32_t D, int32_t V, int32_t dtype, int64_t ldh, int64_t ldw);
int dab_head_loss(const void* H, int64_t ldh, const void* W, int64_t ldw, int32_t dtype, const int64_t* targets,
                  int64_t ignore_index, int32_t T, int32_t D, int32_t V, float* loss, float* lse, void* ws, size_t ws_bytes,
                  void* stream);

/*
 * dab_head_loss_gradient - its gradient.  With g_t the gradient with respect to loss_t,
 *     P_tv = g_t (exp(L_tv - lse_t) - [v = target(t)]),   dH = P W,   dW = P^T H,
 * the logits recomputed a piece of the vocabulary at a time.  Where H and W are bf16 P is rounded to bf16 (as those
 * are: the products stay on the matrix cores, and dH and dW are rounded to bf16 themselves), of up to 128 tokens to 16 bits and of
 * small heads not at all; for fp32 it is held as the operands are.  An entry of P is then off by up to 2^-8 of itself, a weight that all
 * tokens share aside (what is rounded is P over the significand of the first weight): the error of dH and dW is that of rounding them alone where
 * the weights are the same, about 1.4 times that where they differ, and more where the terms of a sum cancel (words with a large part in
 * common, which P's rows sum away; 16 times what sets them apart: dH 2.1 times).  A caller to whom that matters gives H and W
 * in fp32.  Sums are fp32; no atomics: the same inputs give the same bits.
 *
 *   lse      [T] fp32 of dab_head_loss for the same H, W, targets
 *   g        [T] fp32, or NULL for 1
 *   dH       [T][D] of dtype out (zero rows for tokens without a loss, whatever W holds), dW [V][D] of dtype out
 */
size_t dab_head_loss_gradient_workspace_bytes(int32_t T, int32_t D, int32_t V, int32_t dtype, int64_t ldh, int64_t ldw);
int dab_head_loss_gradient(const void* H, int64_t ldh, const void* W, int64_t ldw, int32_t dtype, const int64_t* targets,
                           int64_t ignore_index, const float* lse, const float* g, int32_t T, int32_t D, int32_t V, void* dH,
                           void* dW, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_w4_pack / dab_w4_unpack - weights of a real layer in 4 bits: groups of 32 neighbouring weights of a row
 * share a power of two, a weight is a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (codes 0 .. 7, the sign 8).
 * With a the largest magnitude of a group and f = floor(log2 a), the exponent is e = f - 2, or f - 1 where
 * a 2^-e would exceed 7 (further from 6 than half the step before it); values go to the nearest level, ties to the even
 * code, what lies above 6 to 6.  f - 2 is kept within -110 .. 120: weights beyond 6 * 2^121 are cut to that.
 *
 *   W   [F][K] of dtype, rows ldw apart.  F is at most 16 * 65535, K 2^31 - 513
 *   Q   uint8 [ceil(F/16)][ceil(K/128)][64][16] out: piece l of a block of 16 rows and 128 weights holds
 *       row l % 16, weights 32 (l / 16) .. + 31 of the block, two to a byte, the lower weight in the lower four bits.
 *       (What one lane of a wavefront takes; a block is one contiguous kilobyte.)  Zeros past F and K.
 *   S   uint8 [ceil(F/16)][ceil(K/512)][64][4] out: e + 127 of piece l of block 4 i + j at [.][i][l][j]; 17 for
 *       groups of zeros and past F and K.  A group with an infinity or a NaN has 255 and codes 7: it is restored as NaN.
 * unpack writes fp32 [F][K].
 */
int dab_w4_pack(const void* W, int32_t dtype, int32_t F, int32_t K, int64_t ldw, uint8_t* Q, uint8_t* S, void* stream);
int dab_w4_unpack(const uint8_t* Q, const uint8_t* S, int32_t F, int32_t K, float* W, void* stream);

/*
 * dab_w4_matvec - Y[b][f] = sum_k X[b][k] W[f][k] with packed weights, for one token or a few (B up to 65535, K up to 2^26; the
 * weights are read once for every 48 bf16, 24 f16 or 16 fp32 tokens).  On the matrix cores in bf16, which hold a 4-bit weight times its
 * scale exactly; f16 inputs are sums of two bf16 numbers, fp32 ones of three: only the fp32 accumulation
 * rounds, and a 16-bit Y once more.  Infinities and NaN in X come out as in the sum itself.
 *
 *   X   [B][K] of dtype, rows ldx apart;  Y  [B][F] of dtype out
 *   ws  dab_w4_matvec_workspace_bytes(...) bytes, 256-byte aligned (0 for up to 16 bf16
 *       tokens whose rows are 16-byte aligned)
 */
size_t dab_w4_matvec_workspace_bytes(int32_t B, int32_t K, int32_t F, int32_t dtype, int64_t ldx);
int dab_w4_matvec(const void* X, int32_t dtype, int64_t ldx, const uint8_t* Q, const uint8_t* S, int32_t B, int32_t K, int32_t F,
                  void* Y, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_rms_norm - the root-mean-square norm of a layer's input, with the residual's addition and, in the same pass, the output in 8 bits for
 * dab_ckpt8_weight_gradient of the layer behind it:
 *     h = x + r, rounded to dtype (x without a residual),   y_c = gain_c h_c rstd,  rstd = 1 / sqrt(mean_c(h_c^2) + eps).
 * Sums are fp32 (a row whose squares pass fp32's range has an rstd of 0, a row of zeros with an eps of 0 an infinite one); y is rounded once, to
 * dtype and, apart from that, to bytes.
 *
 *   X      [rows][cols] of dtype, rows ldx apart;  R  the same, rows ldr apart, or NULL.  cols is at most 2^26
 *   gain   [cols] fp32
 *   H      [rows][cols] of dtype out: h; written where R is given, else not touched and may be NULL.  May be X or R itself where their rows are cols apart
 *   Y      [rows][cols] of dtype out, or NULL.  May be X or R itself where their rows are cols apart
 *   Q, S   as dab_ckpt8_save writes them for y (in fp32), or both NULL.  One of Y and Q is given
 *   rstd   [rows] fp32 out, what the gradient takes
 * Errors: eps below 0 or a NaN -> DAB_ERR_SHAPE; Y or H over X or R in any other way, or over one another -> DAB_ERR_UNSUPPORTED, and so may a
 * call of more than 2^34 elements, or of 2^30 rows and more, be.
 */
int dab_rms_norm(const void* X, int32_t dtype, int64_t ldx, const void* R, int64_t ldr, const float* gain, float eps, int32_t rows, int32_t cols,
                 void* H, void* Y, int8_t* Q, uint8_t* S, float* rstd, void* stream);

/*
 * dab_rms_norm_gradient - its gradients.  With n = h rstd and w = gain dy:
 *     dx_c = rstd (w_c - n_c mean(w n)) + dh_c   (the gradient of x and of r alike),   dgain_c = sum over rows of dy_c n_c.
 * Sums are fp32, in an order that depends on the sizes alone: the same inputs give the same bits.
 *
 *   dY     [rows][cols] of dtype, rows lddy apart;  H  the h of dab_rms_norm (X without a residual), rows ldh apart;  rstd  its rstd
 *   dH     [rows][cols] of dtype, rows lddh apart, what arrives at h beside the norm, or NULL
 *   dX     [rows][cols] of dtype out.  May be dY, H or dH itself where their rows are cols apart (over them in another way:
 *          DAB_ERR_UNSUPPORTED);  dgain  [cols] fp32 out
 *   ws     dab_rms_norm_gradient_workspace_bytes(rows, cols) bytes, 256-byte aligned
 */
size_t dab_rms_norm_gradient_workspace_bytes(int32_t rows, int32_t cols);
int dab_rms_norm_gradient(const void* dY, int64_t lddy, const void* H, int64_t ldh, int32_t dtype, const float* gain, const float* rstd,
                          const void* dH, int64_t lddh, int32_t rows, int32_t cols, void* dX, float* dgain, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_adamw - a step of Adam with decoupled weight decay over many tensors at once, in one launch.  With g the gradient
 * times *grad_scale, every operation in fp32:
 *     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
 *     p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
 * Everything is updated in place.  m and v are held in fp32 (bits 32), or in 8 bits (bits 8), m and sqrt(v), groups of 32 neighbouring elements
 * sharing a scale 2^f, f = floor(log2(largest magnitude)), one more where that magnitude lies above the last code, kept within -100 .. 120
 * (-100 for zeros):
 *   m        a sign (128), four bits of exponent e, three of significand s: s 2^-17 2^f for e = 0, else (1 + s/8) 2^(e-15) 2^f
 *   sqrt(v)  four bits of exponent, four of significand: s 2^-18 2^f for e = 0, else (1 + s/16) 2^(e-15) 2^f
 * Both are rounded by chance, to the code above or below with the probabilities that keep the mean (with rounding to the nearest a
 * second moment, which changes by one part in a thousand a step, would never fall): the 23 bits of a magnitude's significand plus 16 random
 * bits at the top of those that go.  A sqrt(v) that is not zero keeps a code of at least 1.  The step itself takes m and v before they are rounded.
 * The random bits of element i: mix(lower word of place + i, plus mix(its upper word + key)), key = mix(seed's lower word + mix(its upper one +
 * mix(step))), the lower 16 bits for m, the upper for sqrt(v); mix(x): x ^= x >> 16, x *= 0x85A308D3, x ^= x >> 15, x *= 0x9E3779B1, x ^= x >> 16.
 * A group with an infinity or a NaN has scale byte 255 and is restored as NaN throughout.
 *
 *   P       [n] fp32;  G  [n] of grad_dtype;  copy  [n] of copy_dtype (DAB_BF16 or DAB_F16): the new p rounded to it, or NULL
 *   M, V    [n] fp32, MS and VS not used; or uint8 [32 ceil(n/32)] and MS, VS uint8 [ceil(n/32)]: f + 127
 *   place   of the tensor's first element in the sequence of random numbers, a multiple of 32: tensors that round apart from one another
 *           have places that lie their sizes apart
 * P, G, M, V and copy are 16-byte aligned; n is at most 2^34.  No tensor may overlap another one of the call.
 *   lr, step, grad_scale   in the structure, or in device memory (lr_dev, step_dev; grad_scale: NULL for 1), where a captured graph reads them anew at
 *           every replay.  A *grad_scale that is infinite or a NaN leaves everything as it was; step counts from 1
 * With an eps of 0 (in fp32) an element whose gradients were all 0 becomes 0/0, a NaN.
 * Errors: step < 1, a rate that is not finite, b1 or b2 outside 0 .. 1 (without 1), a negative eps, a place that is no multiple of 32 -> DAB_ERR_SHAPE.
 */
typedef struct dab_adamw_job {
    float* P;
    const void* G;
    void *M, *V;
    uint8_t *MS, *VS;
    void* copy;
    int64_t n;
    uint64_t place;
    int32_t grad_dtype, copy_dtype, bits;
    float weight_decay;
} dab_adamw_job;

typedef struct dab_adamw_step {
    double lr, beta1, beta2, eps;
    int64_t step;
    uint64_t seed;
    const float* lr_dev;            /* device memory, or NULL: lr                        */
    const int64_t* step_dev;        /* device memory, or NULL: step                      */
    const float* grad_scale;        /* device memory, or NULL: 1                         */
} dab_adamw_step;

/*
 * The tensors of a step are laid out once, in a table of the caller's device memory: dab_adamw_plan_of checks the jobs and says how large it is,
 * dab_adamw_table writes it (on `stream`, without reading host memory after it returns), and any number of dab_adamw calls take it as
 * long as the tensors, the gradients among them, stay where they are.  The plan is the caller's too; what another call than these wrote into plan or table is not supported.
 *   table   plan.table_bytes bytes, 256-byte aligned.  More than 2^23 workgroups (2^36 elements) -> DAB_ERR_UNSUPPORTED
 */
typedef struct dab_adamw_plan {
    int32_t n_jobs, turns, workgroups;
    int64_t table_bytes;
} dab_adamw_plan;

int dab_adamw_plan_of(const dab_adamw_job* jobs /* host */, int32_t n_jobs, dab_adamw_plan* plan /* host, out */);
int dab_adamw_table(const dab_adamw_job* jobs /* host */, const dab_adamw_plan* plan /* host */, void* table, size_t table_bytes, void* stream);
int dab_adamw(const void* table, size_t table_bytes, const dab_adamw_plan* plan /* host */, const dab_adamw_step* step /* host */, void* stream);

/*
 * dab_state8_restore / dab_state8_save - 8-bit states as numbers, and numbers as 8-bit states rounded to the nearest code (halves up): is_signed
 * for m, else sqrt(v) (what is negative counts as 0).  X [n] of dtype (save: fp32), Q uint8 [32 ceil(n/32)], zeros behind the last
 * element, S uint8 [ceil(n/32)].  X and Q are 16-byte aligned, n is at most 2^34.
 */
int dab_state8_restore(const uint8_t* Q, const uint8_t* S, int64_t n, int32_t is_signed, void* X, int32_t dtype, void* stream);
int dab_state8_save(const float* X, int64_t n, int32_t is_signed, uint8_t* Q, uint8_t* S, void* stream);

/*
 * dab_adapters - products of low rank beside a shared projection.  A token t has adapter i = ids[t] (none where that is not one of 0 .. n-1):
 *     U_t = A_i X_t,   Y_t = base_t + scale_i (U_t B_i),     Y_t = base_t and U_t = 0 without an adapter.
 * Both matrices of an adapter are r long rows.  Products are exact and sums fp32; Y is rounded once.  What an adapter that a token does
 * not have holds, infinities and NaN among it, does not reach the token; an infinity among a token's own numbers may come out as a NaN.
 *
 *   X       [T][K] of dtype, rows ldx apart;  ids  int32 [T], in any order;  scale  fp32 [n], or NULL for 1
 *   A       [n][r][K], B  [n][r][F] of dtype, contiguous.  r is at most 256, n 65535, T 2^25, K and F 2^21,
 *           the rows' distances (of dY and base too) 2^25
 *   base    [T][F] of dtype or fp32 (base_dtype), rows ldbase apart, or NULL for 0: any projection's output
 *   Y       [T][F] of dtype out.  May be base itself where that is of dtype and its rows are F apart (or T is 1); must not overlap base in
 *           another way, nor X, nor lie between their rows (DAB_ERR_UNSUPPORTED)
 *   U       fp32 [T][r] out: what the gradient takes
 */
int dab_adapters(const void* X, int32_t dtype, int64_t ldx, const int32_t* ids, const void* A, const void* B, const float* scale, int32_t T, int32_t K,
                 int32_t F, int32_t n, int32_t r, const void* base, int32_t base_dtype, int64_t ldbase, void* Y, float* U, void* stream);

/*
 * dab_adapters_gradient - its gradients.  With V_t = scale_i (B_i dY_t), 0 without an adapter:
 *     dX_t = base_t + V_t A_i,   dA_i = sum over t with ids[t] = i of V_t^T X_t,   dB_i = scale_i sum over the same t of U_t^T dY_t.
 * Sums are fp32, in an order that depends on the sizes and ids alone.  (base's gradient in dab_adapters is dY itself.)
 *
 *   dY      [T][F] of dtype, rows lddy apart;  X, ids, A, B, scale  as for dab_adapters, U  what it returned
 *   base    [T][K] of dtype or fp32, rows ldbase apart, or NULL for 0: what the shared projection's gradient gives
 *   dX      [T][K] of dtype out, or NULL where it is not needed (base is NULL then).  May be base itself where that is of dtype and its rows are K
 *           apart (or T is 1); must not overlap base in another way, nor X, nor dY, nor lie between their rows (DAB_ERR_UNSUPPORTED)
 *   dA      fp32 [n][r][K] out, dB  fp32 [n][r][F] out, zeros for an adapter without tokens
 *   ws      dab_adapters_gradient_workspace_bytes(T, K, F, n, r) bytes, 256-byte aligned
 */
size_t dab_adapters_gradient_workspace_bytes(int32_t T, int32_t K, int32_t F, int32_t n, int32_t r);
int dab_adapters_gradient(const void* dY, int64_t lddy, const void* X, int32_t dtype, int64_t ldx, const float* U, const int32_t* ids, const void* A,
                          const void* B, const float* scale, int32_t T, int32_t K, int32_t F, int32_t n, int32_t r, const void* base,
                          int32_t base_dtype, int64_t ldbase, void* dX, float* dA, float* dB, void* ws, size_t ws_bytes, void* stream);

/*
 * dab_w4_adapters - dab_w4_matvec and dab_adapters in one: Y_t = W X_t + scale_i (A_i X_t) B_i with the 4-bit weights Q, S that all tokens share, rounded
 * once.  Arguments as for those two; Bt is dab_adapters' B.  B tokens, up to 65535; Y must not overlap X (DAB_ERR_UNSUPPORTED).
 *
 *   ws      dab_w4_adapters_workspace_bytes(...) bytes, 256-byte aligned
 */
size_t dab_w4_adapters_workspace_bytes(int32_t B, int32_t K, int32_t F, int32_t r, int32_t dtype, int64_t ldx);
int dab_w4_adapters(const void* X, int32_t dtype, int64_t ldx, const uint8_t* Q, const uint8_t* S, const int32_t* ids, const void* A, const void* Bt,
                    const float* scale, int32_t B, int32_t K, int32_t F, int32_t n, int32_t r, void* Y, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DAB_H */
