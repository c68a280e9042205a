/*
 * gtp.h -- C ABI of the MI355X (gfx950) Gaunt Tensor Product library.
 *
 * The Gaunt Tensor Product (Luo, Chen, He, "Enabling efficient equivariant
 * operations in the Fourier basis via Gaunt Tensor Products", ICLR 2024) of
 * two real spherical-harmonic (SH) coefficient vectors x1 (degrees <= L1) and
 * x2 (degrees <= L2) is the SH expansion, truncated to degree Lout, of the
 * product of the two spherical functions they define (Sec. 3.1, eq.
 * tp-eq-mul):
 *
 *   y_l^m = sum G^{(l,m)}_{(l1,m1)(l2,m2)} x1_{l1}^{m1} x2_{l2}^{m2},
 *   G     = int_{S^2} Y_{l1}^{m1} Y_{l2}^{m2} Y_l^m dOmega   (real Gaunt coefficients).
 *
 * The library computes it the paper's way (Sec. 3.2): change of basis SH ->
 * 2D Fourier, product of the two functions as a 2D convolution of their Fourier
 * grids, projection back to SH.
 *
 * Conventions shared by every entry point
 *   - Real SH, z polar axis, no Condon-Shortley phase:
 *       Y_l^0 = Q_l^0(cos t), Y_l^{+m} = sqrt2 Q_l^m(cos t) cos(m p),
 *       Y_l^{-m} = sqrt2 Q_l^m(cos t) sin(m p),  Q_l^m = N_lm P_l^m,
 *     so Y_1 = sqrt(3/(4 pi)) (y, z, x).
 *   - Coefficient vectors are contiguous, index i = l*l + l + m, (L+1)^2 long.
 *     Batched tensors are row-major [B, C, (L+1)^2] (channel-wise products:
 *     product (b,c) uses channel c of both inputs, Appendix "Implementation
 *     Details", channel-wise combination).
 *   - Every data pointer is a DEVICE pointer on the current HIP device, owned
 *     by the caller; the library only reads inputs and writes outputs, never
 *     allocates or frees caller memory.  Pointers must be 4-byte aligned
 *     (2-byte for bf16 inputs).
 *   - `stream` is a hipStream_t (NULL = the default stream).  Calls are
 *     asynchronous on that stream; a launch failure returns GTP_ERR_HIP.
 *   - Every argument is validated on the host BEFORE any HIP call; invalid
 *     arguments return GTP_ERR_INVALID_ARG and touch nothing.
 *   - Functions never throw.  gtp_last_error() gives a thread-local message.
 *   - Floating point: tables are built in fp64 on the host; outputs and every
 *     accumulation are fp32, bf16 applies to inputs only.  Tables are rounded
 *     once to fp32 and products taken in fp32 except in two kernels that run on
 *     the 16-bit matrix instructions, with values and tables split: products of
 *     degrees 9..32 in two fp16 parts, 2^-23 of a value (of a row's norm where
 *     that is larger than 2^8 times the value) at worst, and channel mixing of
 *     degrees 1..8 in three bf16 parts, exact.  Against 64-bit results their
 *     errors measure no larger than those of the fp32 kernels they replaced
 *     (products 1.0e-7 to 1.4e-7, mixing 0.8e-7 to 1.9e-7, 2-norm).
 *   - Limits: 0 <= L1, L2, Lout <= 64.  Output degrees above L1 + L2 are
 *     written as zeros.
 */
#ifndef GTP_H
#define GTP_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  GTP_OK = 0,
  GTP_ERR_INVALID_ARG = 1, /* bad sizes, null pointers, overlap, bad enum */
  GTP_ERR_UNSUPPORTED = 2, /* valid request the library does not implement  */
  GTP_ERR_NO_DEVICE = 3,   /* no HIP device visible                          */
  GTP_ERR_HIP = 4,         /* a HIP runtime call or kernel launch failed      */
  GTP_ERR_ALLOC = 5        /* host or device allocation failed                */
} gtp_status;

typedef enum { GTP_F32 = 0, GTP_BF16 = 1 } gtp_dtype;

/* Plan flags (bitwise or).  The two low bits pick step 2 (eq. 2D-conv). */
#define GTP_CONV_AUTO 0u      /* the algorithm the measured crossover picks for the degrees */
#define GTP_CONV_DIRECT 1u    /* direct 2D convolution of the Fourier grids */
#define GTP_CONV_FFT 2u       /* convolution theorem, phi transforms by radix-2 FFTs where the library has such a
                                 kernel (L1 = L2 = Lout in {16, 32}), by the direct DFTs below otherwise */
#define GTP_CONV_DFT 3u       /* convolution theorem, phi transforms as direct DFTs over the 4-fold symmetric
                                 sample grid (unrolled at small degree, matrix-core contractions from 16 on) */
#define GTP_PLAN_HOST_ONLY 16u /* build the fp64 tables only; no HIP call (host-side checks) */

/* Many-body modes for gtp_selfproduct. */
#define GTP_SELF_STEPWISE 0u /* B_1 = A, B_{k+1} = P_Lout(B_k * A): truncate after every product */
#define GTP_SELF_FUSED 1u    /* P_Lout(A^nu): one multi-convolution, projected once */

/* Opaque plan: the SH <-> Fourier change-of-basis tables for one
 * (L1, L2, Lout), built in fp64 and uploaded once to the device that is
 * current at creation.  Use a plan only while that device is current. */
typedef struct gtp_plan_ *gtp_plan;

/* Create a plan (Sec. 3.2: the coefficients y^{l,m,*}_{u,v} of eq. sh-fs and
 * z^{l,m,*}_{u,v} of eq. fs-sh, plus the grids of the convolution).
 * out: receives the plan.  Returns GTP_ERR_NO_DEVICE without a device unless
 * GTP_PLAN_HOST_ONLY is set.  The plan owns its host and device tables.  A
 * triple whose product or rotated-frame convolution runs on an equal-degree
 * kernel of higher degree (16, 32 or 64; rows zero-padded) also gets that
 * degree's plan here, kept by the library until the process ends, so that
 * no later call needs to allocate. */
gtp_status gtp_plan_create(gtp_plan *out, int L1, int L2, int Lout, unsigned flags);

/* Destroy a plan and free its tables (NULL is a no-op).  Not stream-ordered:
 * the caller must make sure no launch using the plan is still pending. */
gtp_status gtp_plan_destroy(gtp_plan p);

/* Fused Gaunt tensor product (Sec. 3.1 eq. tp-eq-mul computed by Sec. 3.2):
 *   y[b,c,:] = GTP(x1[b,c,:], x2[b,c,:]) truncated to degree Lout.
 * x1: [B, C, (L1+1)^2], x2: [B, C, (L2+1)^2] of type in_dtype;
 * y: [B, C, (Lout+1)^2] fp32.  B*C == 0 is a successful no-op.  y must not
 * overlap x1 or x2.  The Fourier grids never leave the chip.  The plan's
 * GTP_CONV_* flag picks step 2 (eq. 2D-conv): the convolution theorem with
 * radix-2 FFTs (GTP_CONV_FFT) or direct DFTs (GTP_CONV_DFT) for the phi
 * transforms, or the direct real-form convolution (GTP_CONV_DIRECT;
 * GTP_ERR_UNSUPPORTED when its per-product working set exceeds 64 KB of LDS,
 * about L1 = L2 = 40); GTP_CONV_AUTO takes the measured fastest. */
gtp_status gtp_full(gtp_plan p, const void *x1, const void *x2, gtp_dtype in_dtype,
                    int64_t B, int64_t C, float *y, void *stream);

/* Channel mixing (Appendix, combination rules of features in different
 * channels, channel-mixing case):
 *   y[b, co] = sum_{c1 < C1, c2 < C2} W[co, c1, c2] GTP(x1[b, c1], x2[b, c2]),
 * O(C1 C2) full products per batch entry, in one of three ways:
 *   - L1 = L2 = Lout in 1..8, Co <= 128, C1 C2 >= 128 and sizes at which it is
 *     the fastest: in the sample domain, P_L(sum_{c2} F2[c2] (sum_{c1}
 *     W[co, c1, c2] F1[c1])) with each channel's function sampled once per
 *     entry, on the bf16 matrix cores with operands in three parts (exact fp32
 *     values).  A channel keeps its bits down to 2^-148 of the largest value of
 *     its batch entry, a weight down to 2^-110 of its output channel's largest;
 *   - the other sizes of those degrees: the pair products and their combination
 *     in one kernel per batch entry, fp32;
 *   - all else: the pair products by the fused product kernels (outer-product
 *     indexing) into a workspace, chunked over b, combined as y_b = W T_b (Co x
 *     C1C2 times C1C2 x (Lout+1)^2) on the fp32 matrix cores.
 * The weights in the kernel's layout (the first two) or the workspace are
 * stream-ordered allocations (hipMallocAsync; the first and the last at most
 * 256 MiB).
 * x1: [B, C1, (L1+1)^2], x2: [B, C2, (L2+1)^2] (in_dtype); W: [Co, C1, C2]
 * fp32; y: [B, Co, (Lout+1)^2] fp32, not overlapping the inputs or W.
 * C1 C2 == 0 writes zeros (x1, x2 and W may then be NULL); B Co == 0 is a
 * no-op. */
gtp_status gtp_channel_mix(gtp_plan p, const void *x1, const void *x2, gtp_dtype in_dtype, const float *W,
                           int64_t B, int64_t C1, int64_t C2, int64_t Co, float *y, void *stream);

/* Equivariant convolution with the SH filter of an edge (Sec. 3.3
 * "Equivariant Convolutions"; Appendix, eq. sh2fs-escn):
 *   y[b,c] = GTP(x[b,c], F[b,c]),  F[b,c,(l,m)] = h[b,c,l] Y_l^m(r_b / |r_b|),
 * the result of gtp_full(x, gtp_sh_filter(r, h)), computed in the frame in
 * which the edge points at the pole: x is rotated by the real-SH matrix D_b of
 * a rotation taking r_b / |r_b| to (0, 0, 1); there the filter has only the
 * m = 0 coefficients h_l Y_l^0(pole) (2D Fourier coefficients only at v = 0),
 * the product with it needs theta transforms only, and the result is rotated
 * back by D_b^T.  (The z pole is this library's polar axis; the paper uses
 * (0, 1, 0) in its y-up convention.)
 * x: [B, C, (L1+1)^2] (in_dtype); r: [B, 3] fp32 edge vectors (need not be
 * unit; a zero vector is taken as (0, 0, 1)); h: [B, C, L2+1] fp32 radial
 * weights; y: [B, C, (Lout+1)^2] fp32, not overlapping the inputs.  The
 * rotated-frame kernels cover L1 = L2 = Lout in 1..8 (one product per lane;
 * the per-edge rotation matrices go to a stream-ordered workspace,
 * hipMallocAsync) and 16 (the matrix cores, 16 channels per wave, the
 * rotation applied from the edge angles: no workspace), which also serves
 * every other triple whose highest degree is 9..16 (rows read zero-padded
 * to degree 16, outputs truncated: exact); both take one workgroup per edge
 * and 64 channels, so C >= 64 fills it.  Other degrees, and plans built with
 * GTP_CONV_DIRECT, build the filter in a stream-ordered workspace and take
 * gtp_full. */
gtp_status gtp_conv_escn(gtp_plan p, const void *x, gtp_dtype in_dtype, const float *r, const float *h, int64_t B,
                         int64_t C, float *y, void *stream);

/* gtp_conv_escn without any device allocation, for callers that cannot
 * allocate: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments, result and errors as gtp_conv_escn; no
 * hipMalloc / hipMallocAsync / hipFree / allocating library call is made.
 * The per-edge rotation matrices of L = 1..8 (or, for degrees without a
 * rotated-frame kernel, the filter rows; L = 16 needs none) go to a static
 * device scratch array of
 * GTP_NOALLOC_SCRATCH_BYTES (64 MiB) per device, which exists from the
 * library's load on that device until the process ends; the edges are
 * processed in chunks that fit it.  Returns GTP_ERR_UNSUPPORTED (before any
 * HIP call) when one edge alone needs more: C (L2+1)^2 4 bytes above 64 MiB
 * on the filter route.  Every call on a device shares that device's array
 * and leaves it holding the last chunk's values (each launch writes what it
 * reads, nothing has to start at zero): calls that may overlap on one device
 * (different streams, different host threads) race and must be serialised
 * by the caller.  The plan must have been created on the current device. */
#define GTP_NOALLOC_SCRATCH_BYTES (64ll << 20)
gtp_status gtp_conv_escn_noalloc(gtp_plan p, const void *x, gtp_dtype in_dtype, const float *r, const float *h,
                                 int64_t B, int64_t C, float *y, void *stream);

/* Weighted Gaunt tensor product (Sec. 3.1, eq. tp-eq-mul-weight; Appendix
 * "Feature Interaction" weights w^l_{l1,l2} reparameterized as
 * w_{l1} w_{l2} w_l):
 *   y[b,c,(l,m)] = wout[r,l] * sum_{l1,l2} w1[r,l1] w2[r,l2] (x1^(l1) (x) x2^(l2))^(l)_m,
 * computed as gtp_full of the degree-scaled inputs, scaled per output degree
 * (the weights are applied as the inputs are loaded and the output stored).
 * A degree mask (weights 0 / 1) gives the partial products x^(l1) (x) x^(l2).
 * r = c when per_channel = 1 (one weight row per channel), r = 0 when
 * per_channel = 0 (one row shared by every channel).
 * w1: [R, L1+1], w2: [R, L2+1], wout: [R, Lout+1] fp32 device arrays with
 * R = C or 1; any of them may be NULL (all ones).  Other arguments as in
 * gtp_full; y must not overlap the inputs or the weights.  Plans built with
 * GTP_CONV_DIRECT return GTP_ERR_UNSUPPORTED. */
gtp_status gtp_full_weighted(gtp_plan p, const void *x1, const void *x2, gtp_dtype in_dtype, const float *w1,
                             const float *w2, const float *wout, int per_channel, int64_t B, int64_t C, float *y,
                             void *stream);

/* Backward pass of gtp_full_weighted, weight gradients included (Sec. 3.1,
 * eq. tp-eq-mul-weight; the learnable weights of the feature-interaction
 * layers).  With y = wout GTP(w1 x1, w2 x2) and a loss gradient dy, writes
 *   dx1   = w1 P_L1 GTP(wout dy, w2 x2)                 [B, C, (L1+1)^2],
 *   dx2   = w2 P_L2 GTP(wout dy, w1 x1)                 [B, C, (L2+1)^2],
 *   dw1[r, l1] = sum over the products of weight row r of
 *                <x1, P_L1 GTP(wout dy, w2 x2)> on degree l1     [R, L1+1],
 *   dw2 likewise                                                 [R, L2+1],
 *   dwout[r, l] = sum over row r of <dy, GTP(w1 x1, w2 x2)> on degree l
 *                                                                [R, Lout+1],
 * R = C with per_channel = 1 (row c holds channel c's products), else 1.
 * Weights as in gtp_full_weighted (NULL = ones; the gradient is still that
 * of a weight of ones).  Any of dx1, dx2, dw1, dw2, dwout may be NULL (not
 * computed); the rest are written, not accumulated, and must not overlap an
 * input or each other.  The sums over the products are deterministic (fixed
 * order, no atomics).  Uses a stream-ordered workspace (hipMallocAsync) for
 * the partial sums and the products that are not outputs.  B*C == 0 writes
 * zero weight gradients.  GTP_ERR_UNSUPPORTED for GTP_CONV_DIRECT plans and
 * more than 65535 weight rows. */
gtp_status gtp_full_weighted_backward(gtp_plan p, const void *x1, const void *x2, gtp_dtype in_dtype,
                                      const float *w1, const float *w2, const float *wout, int per_channel,
                                      const float *dy, int64_t B, int64_t C, float *dx1, float *dx2, float *dw1,
                                      float *dw2, float *dwout, void *stream);

/* Backward pass (vector-Jacobian product) of gtp_full: given the gradient dy
 * of a scalar loss with respect to y = gtp_full(x1, x2), the gradients
 *   dx1[b,c,i] = sum_{j,k} G_{i j k} x2[b,c,j] dy[b,c,k]   (i over degrees <= L1),
 *   dx2[b,c,j] = sum_{i,k} G_{i j k} x1[b,c,i] dy[b,c,k]   (j over degrees <= L2),
 * with G the real Gaunt coefficients of Sec. 3.1 (eq. tp-eq-mul).  G is the
 * integral of a product of three real SH, symmetric in its three (l, m)
 * pairs, so dx1 is the Gaunt tensor product of dy and x2 truncated to degree
 * L1 (and dx2 that of dy and x1 truncated to L2); both are computed that way
 * (Sec. 3.2), with the plan's GTP_CONV_* choice.
 * x1, x2: the forward inputs (in_dtype); dy: [B, C, (Lout+1)^2] fp32;
 * dx1: [B, C, (L1+1)^2] fp32 or NULL (not computed); dx2: [B, C, (L2+1)^2]
 * fp32 or NULL.  x1 may be NULL when dx2 is, x2 when dx1 is.  The gradients
 * are written, not accumulated.  Neither may overlap an input or the other.
 * B*C == 0, or dx1 == dx2 == NULL, is a successful no-op.  Tables for
 * (Lout, L2, L1) and (Lout, L1, L2) are built on first use and cached per
 * device (that first call is synchronous); equal degrees reuse the plan's.
 * With L1 = L2 = Lout <= 7 and both gradients asked for, both come from one
 * launch that reads dy once (results equal bit for bit to asking for each
 * gradient alone). */
gtp_status gtp_full_backward(gtp_plan p, const void *x1, const void *x2, gtp_dtype in_dtype, const float *dy,
                             int64_t B, int64_t C, float *dx1, float *dx2, void *stream);

/* Step 1 (Sec. 3.2, eq. sh-fs): SH coefficients -> 2D Fourier coefficients
 * x*_{u,v}, |u|,|v| <= L, for L = L1 (which = 1) or L2 (which = 2).
 * The function is extended to theta in [-pi, pi) by F(-t, p) = F(t, p + pi).
 * x: [n, (L+1)^2] (in_dtype); grid: [n, 2L+1, 2L+1] complex64 interleaved
 * (re, im), element (u, v) at [(u+L)*(2L+1) + (v+L)]. */
gtp_status gtp_sh2fourier(gtp_plan p, int which, const void *x, gtp_dtype in_dtype, int64_t n,
                          float *grid, void *stream);

/* Step 2 (Sec. 3.2, eq. 2D-conv): f3_{u,v} = sum_{u1+u2=u, v1+v2=v} f1_{u1,v1} f2_{u2,v2}.
 * g1: [n, 2L1+1, 2L1+1], g2: [n, 2L2+1, 2L2+1], g3: [n, 2U+1, 2U+1] with
 * U = L1 + L2, all complex64 interleaved and centred as above.  Computed as a
 * direct convolution (the grids are the public, paper-layout grids). */
gtp_status gtp_fourier_conv(gtp_plan p, const float *g1, const float *g2, int64_t n, float *g3,
                            void *stream);

/* Step 3 (Sec. 3.2, eq. fs-sh): y_l^m = Re sum_{u,v} g3_{u,v} z^{l,m}_{u,v},
 * z^{l,m}_{u,v} = int_{S^2} exp(i(u t + v p)) Y_l^m dOmega (the projection of
 * the grid's function onto the SH basis), l <= Lout.
 * g3: [n, 2U+1, 2U+1] complex64; y: [n, (Lout+1)^2] fp32.  For grids of real
 * functions (anything made by gtp_sh2fourier and gtp_fourier_conv) the
 * discarded imaginary part is zero. */
gtp_status gtp_fourier2sh(gtp_plan p, const float *g3, int64_t n, float *y, void *stream);

/* Many-body self product (Sec. 3.3 "Equivariant Many-body Interactions";
 * Appendix "Implementation Details", generalized Gaunt coefficients and the
 * divide-and-conquer multi-convolution): the nu-fold product of A = x with
 * itself, nu >= 1.
 *   mode GTP_SELF_STEPWISE: B_1 = P_Lout(A), B_{k+1} = P_Lout(B_k * A).
 *   mode GTP_SELF_FUSED   : P_Lout(A^nu) with no intermediate truncation.
 * x: [B, C, (L+1)^2] (in_dtype); y: [B, C, (Lout+1)^2] fp32.  Plans for the
 * needed degrees are built and cached internally (per device).  The fused
 * mode needs nu * L <= 64 (GTP_ERR_UNSUPPORTED otherwise).  The stepwise
 * mode may take a stream-ordered device workspace (hipMallocAsync) when no
 * single-kernel path exists for (L, nu, Lout). */
gtp_status gtp_selfproduct(int L, int nu, int Lout, unsigned mode, const void *x,
                           gtp_dtype in_dtype, int64_t B, int64_t C, float *y, void *stream);

/* Spherical-harmonic filter of an equivariant convolution (Sec. 3.3
 * "Equivariant Convolutions"): out[b,c,(l,m)] = h[b,c,l] * Y_l^m(r_b / |r_b|).
 * r: [B, 3] fp32 edge vectors (need not be unit; zero vectors give the
 * direction (0,0,1)); h: [B, C, L+1] fp32 per-degree radial weights, or NULL
 * for h = 1 (then C must be 1); out: [B, C, (L+1)^2] fp32.  0 <= L <= 64. */
gtp_status gtp_sh_filter(int L, const float *r, const float *h, int64_t B, int64_t C, float *out,
                         void *stream);

/* ---- The layers around the product -------------------------------------
 * Normalisation, residual steps, dropout and attention of a block that holds Gaunt products.
 * Each commutes with rotations of the SH features: the normalisation scales a
 * degree as a whole, dropout drops a channel as a whole, and attention takes
 * dot products of whole heads, which a rotation leaves alone.
 *
 * Unlike the products these write results (y, dx, o, dq, dk, dv) in the type of
 * their inputs, rounded once; statistics and weight gradients are fp32, as is
 * every sum.  No device memory is allocated: what a call needs beside its
 * outputs is the caller's `work` (16-byte aligned, at least the bytes that the
 * _work function of the same arguments names, its contents of no interest
 * before or after), so every call can be captured in a graph.  No atomics: the
 * same call gives the same bits.  Data read on one stream and written on
 * another is the caller's to order. */

/* Normalisation of SH features by degree.  x: [N, C, (L+1)^2] of `dtype`; with
 *   mu = mean_c x[n, c, 0],  v_l = mean over (c, m) of (x[n, c, (l, m)] - mu [l = 0])^2:
 *   y[n, c, (l, m)] = (x[n, c, (l, m)] - mu [l = 0]) rstd_l w[l, c] + b[c] [l = 0],
 *   rstd_l = 1 / sqrt(v_l + eps).
 * L = 0 is the ordinary layer norm over C channels.  w: [L+1, C] fp32 or NULL
 * (ones); b: [C] fp32 or NULL (zeros); eps > 0; y: like x, may be x itself, else
 * not overlapping it; mean: [N] and rstd: [N, L+1] fp32, what the backward
 * reads, or NULL.  0 <= L <= 64; N C == 0 is a no-op.  GTP_ERR_UNSUPPORTED where N
 * or (L + 2) C is above 2^31 - 1. */
gtp_status gtp_layer_norm(int L, const void *x, gtp_dtype dtype, const float *w, const float *b, float eps, int64_t N,
                          int64_t C, void *y, float *mean, float *rstd, void *stream);

/* Bytes of `work` of gtp_layer_norm_backward (-1 on a bad argument); needed
 * only where dw or db is asked for. */
int64_t gtp_layer_norm_backward_work(int L, gtp_dtype dtype, int64_t N, int64_t C);

/* Gradient of gtp_layer_norm for dy (like x): with xh = (x - mu [l = 0]) rstd_l
 * and g = dy w,
 *   dx = rstd_l (g - xh mean_{c,m}(g xh) - [l = 0] mean_c g)   (like x; may be dy itself),
 *   dw[l, c] = sum_{n,m} dy xh   [L+1, C],   db[c] = sum_n dy[n, c, 0]   [C], fp32.
 * mean, rstd: as gtp_layer_norm wrote them.  dx, dw, db may each be NULL (not
 * computed); they are written, not accumulated.  N C == 0 writes zero weight
 * gradients. */
gtp_status gtp_layer_norm_backward(int L, const void *x, gtp_dtype dtype, const float *w, const float *mean,
                                   const float *rstd, const void *dy, int64_t N, int64_t C, void *dx, float *dw,
                                   float *db, void *work, int64_t work_bytes, void *stream);

/* The residual step between two parts of a block, with the norms around it: the
 * part's output a is normalised by degree (post = 1; or left as it is), scaled
 * per degree and channel and by a gate per channel, added to the residual stream
 * x, and the sum normalised for the next part:
 *   t = norm(a) w_post[l, c] + b_post[c] [l = 0]   (post = 0: t = a),
 *   r = x + scale[l, c] sigmoid(gate[n, c]) t,
 *   h = norm(r) w_pre[l, c] + b_pre[c] [l = 0],
 * norm as in gtp_layer_norm (statistics of r before its rounding).  A gate is one
 * number for all (L+1)^2 coefficients of a channel, so the step commutes with
 * rotations. */
typedef struct {
  int L;                            /* 0..64 */
  gtp_dtype dtype;                  /* of x, a, gate, r, h and their gradients */
  int64_t N, C;                     /* rows, channels; GTP_ERR_UNSUPPORTED as in gtp_layer_norm */
  int post;                         /* 0 or 1 */
  float eps;                        /* of both norms, positive */
  const float *scale;               /* [L+1, C] or NULL (ones) */
  const float *w_post, *b_post;     /* [L+1, C] and [C], each or NULL (ones, zeros); NULL without post */
  const float *w_pre, *b_pre;       /* [L+1, C] and [C], each or NULL */
  const void *gate;                 /* [N, C], before the sigmoid; or NULL (no gate) */
} gtp_residual;

/* Statistics of both norms, [N] and [N, L+1]: written by gtp_residual_norm (each may
 * be NULL there), read by its gradient (post's only with post). */
typedef struct {
  float *mean_post, *rstd_post, *mean_pre, *rstd_pre;
} gtp_residual_stats;

/* x, a, r, h: [N, C, (L+1)^2] of p->dtype; r may be x itself, else no output may
 * overlap an input or another.  stats may be NULL.  N C == 0 is a no-op. */
gtp_status gtp_residual_norm(const gtp_residual *p, const void *x, const void *a, void *r, void *h,
                             const gtp_residual_stats *stats, void *stream);

/* Gradients asked for, each or NULL. */
typedef struct {
  void *dx, *da;                    /* like x */
  void *dgate;                      /* [N, C] of p->dtype; with a gate only */
  float *dscale;                    /* [L+1, C] */
  float *dw_post, *db_post;         /* [L+1, C], [C]; with post only */
  float *dw_pre, *db_pre;           /* [L+1, C], [C] */
} gtp_residual_grads;

/* Bytes of `work` of gtp_residual_norm_backward (-1 on a bad argument). */
int64_t gtp_residual_norm_backward_work(const gtp_residual *p);

/* Gradient of gtp_residual_norm for dh and dr (like x; dr NULL: zeros), from r as it was
 * written, a and the statistics: dx = dr + the gradient of the norm of r; with u = dx
 * sigmoid(gate):
 *   dscale[l, c] = sum_{n,m} u t,  dgate[n, c] = sigmoid' sum_{l,m} dx scale t,
 *   dw_post, db_post, da: those of norm(a) w_post + b_post for u scale (post = 0: da = u scale).
 * dx may be dr itself, else no output may overlap an input or another.  Gradients are
 * written, not accumulated; N C == 0 writes zero weight gradients. */
gtp_status gtp_residual_norm_backward(const gtp_residual *p, const void *r, const void *a,
                                      const gtp_residual_stats *stats, const void *dh, const void *dr,
                                      const gtp_residual_grads *grads, void *work, int64_t work_bytes, void *stream);

/* Dropout of groups of K consecutive elements (all (L+1)^2 coefficients of a
 * channel, or K = 1) added to a residual:
 *   y = res + keep x / (1 - p),   keep = 0 with probability p, else 1,
 * one draw for each of `groups` groups.  The mask is never stored: the draw of
 * group g is halfword g mod 8 of the 128 bits that Philox4x32-10 (Salmon et al.,
 * SC 2011) gives for counter (g / 8, rng[1]) and key rng[0], kept where it is at
 * least round(65536 p) (at most 65535), so p counts in units of 2^-16 and 1 - p
 * above is that of the unit.  rng: two uint64 in device memory, seed and offset,
 * read when the call runs: a graph that is replayed draws anew where they were
 * changed between.  The gradient is the same call on dy, without res.
 * x, res (or NULL), y: [groups, K] of `dtype`; y may be x or res itself, else not
 * overlapping them.  0 <= p < 1.  groups K == 0 is a no-op.  GTP_ERR_UNSUPPORTED
 * above 2^37 - 8192 elements or K = 2^31 - 1. */
gtp_status gtp_dropout(const void *x, const void *res, gtp_dtype dtype, double p, const uint64_t *rng, int64_t groups,
                       int64_t K, void *y, void *stream);

/* Rows of a tensor [rows, heads, d]: element (t, h, i) at data[t row + h head + i]. */
typedef struct {
  void *data;
  int64_t row, head;
} gtp_rows;

/* What both directions of the attention share.  The rows of B segments (the
 * atoms of each molecule) lie one after the other: queries of segment b are rows
 * q_off[b] .. q_off[b+1] - 1 of q, its keys rows k_off[b] .. k_off[b+1] - 1 of k
 * and v.  Offsets are device arrays [B+1], ascending, read when the call runs;
 * NULL: equal segments of max_q (max_k) rows.  A segment longer than max_q
 * (max_k), and an offset outside the tensor, is cut there.  Rows of no segment are
 * not written. */
typedef struct {
  gtp_dtype dtype;          /* of q, k, v, o and the gradients */
  int H, Hk, d;             /* query heads, key heads (H a multiple of Hk: head h reads key head h / (H / Hk)),
                               head length 1..256 (c channels of degree L: c (L+1)^2) */
  int64_t B, Tq, Tk;        /* segments, rows of q, rows of k and v */
  int64_t max_q, max_k;     /* the longest segment's rows */
  const int64_t *q_off, *k_off;
  const uint8_t *key_mask;  /* [Tk]: 0 = absent key, as if its row were not there, whatever it holds; or NULL */
  float scale;              /* of the scores */
  double p;                 /* probabilities dropped with probability p, 0 <= p < 1 */
  const uint64_t *rng;      /* device {seed, offset}; may be NULL where p is 0 */
} gtp_attn;

/* Bytes of `work` of gtp_attention (backward = 0) or gtp_attention_backward (1);
 * -1 on a bad argument. */
int64_t gtp_attention_work(const gtp_attn *a, int backward);

/* Softmax attention over each segment:
 *   s = scale q k^T,  P = softmax(s) over the segment's present keys,
 *   o = (m P) v,  lse = log sum_j exp(s_j),
 * m the factors 0 or 1 / (1 - p) of dropped probabilities.  A row without a
 * present key (or whose every score is -infinity) has o = 0 and lse = -infinity.
 * q, o: [Tq, H, d]; k, v: [Tk, Hk, d]; lse: [Tq, H] fp32.  Any nonnegative strides
 * for inputs; outputs' rows must not overlap each other or an input (slices of one
 * buffer, side by side or interleaved, do not; where the strides of two tensors
 * differ, buffers that reach into each other count as overlapping).  The draws,
 * of the generator of gtp_dropout: the rows of a key head's G = H / Hk query heads
 * count together, R = i G + g for row i of the segment, in blocks of 4 rows x 4
 * keys; block ((b Hk + hk) ceil(max_q G / 4) + R / 4) ceil(max_k / 4) + j / 4 takes
 * calls 2 block (its first two rows) and 2 block + 1, element (R, j) halfword
 * 4 (R mod 2) + j mod 4.  Sums are fp32; with bf16 inputs P and (in the backward)
 * the scores' gradients enter the matrix products rounded to bf16.  What leaves
 * fp32's range: with fp32 inputs a product of q and k elements above 2^136 may make
 * its score NaN, whatever its sign; and values of v above 2^120 / (the number of keys) their
 * sum infinite before it is divided by the row's sum.  GTP_ERR_UNSUPPORTED for heads
 * longer than 256 and where rows, heads and segments are more than a launch holds
 * (some 2^25 tiles of 32 rows of a head, or keys of two). */
gtp_status gtp_attention(const gtp_attn *a, const gtp_rows *q, const gtp_rows *k, const gtp_rows *v, const gtp_rows *o,
                         float *lse, void *work, int64_t work_bytes, void *stream);

/* Gradient of gtp_attention for dout: the probabilities are made again from lse
 * and the draws from the generator, nothing of size rows x keys is stored:
 *   P = exp(s - lse),  dS = P (m (dout v^T) - delta),  delta = sum_i dout_i o_i,
 *   dq = scale dS k,  dk = scale dS^T q,  dv = (m P)^T dout,
 * dk and dv summed over the query heads of a key head.  o, lse: as gtp_attention
 * wrote them.  dq, or dk and dv, may be NULL (not computed).  Absent keys have
 * zero gradients, and so do rows with lse = -infinity, which add none to dk and dv.
 * GTP_ERR_INVALID_ARG where only one of dk and dv is NULL. */
gtp_status gtp_attention_backward(const gtp_attn *a, const gtp_rows *q, const gtp_rows *k, const gtp_rows *v,
                                  const gtp_rows *o, const gtp_rows *dout, const float *lse, const gtp_rows *dq,
                                  const gtp_rows *dk, const gtp_rows *dv, void *work, int64_t work_bytes, void *stream);

/* A learned bias of the scores by the distance of the atoms, for each query head and
 * bucket of the squared distance d2 of a query's and a key's position:
 *   bucket 0 where d2 < r0sq,  else 1 + (number(d2) - number(r0sq)) >> shift,  at most buckets - 1,
 * number(x) the place of a positive fp32 number among them (its bits as an integer), so
 * that each doubling of d2 has per_octave = 2^(23 - shift) buckets, evenly spaced between
 * powers of two; the last bucket is open.  d2 = dx^2 + dy^2 + dz^2 in fp32 with one rounding for
 * each difference, for dx^2 and for each of the two sums (fma), so a pair has the same bucket
 * everywhere.  A pair whose d2 is NaN is in the last bucket.  -infinity in the bias gives a
 * bucket's pairs probability zero (a cutoff).  Positions of absent keys may hold anything. */
typedef struct {
  const float *bias;                /* [H, buckets] */
  const float *q_pos, *k_pos;       /* [Tq, 3], [Tk, 3] */
  float r0sq;                       /* 2^-100 at least; the last bucket's edge must be finite */
  int buckets;                      /* 1..64 */
  int per_octave;                   /* 1, 2, 4, 8 or 16 */
} gtp_attn_bias;

/* The first squared distances of buckets 1 .. buckets - 1 (host memory, buckets - 1 floats). */
gtp_status gtp_attention_bias_edges(float r0sq, int buckets, int per_octave, float *edges);

/* gtp_attention with a bias: s = scale q k^T + bias[h, bucket] (b: not NULL; the bias's values are
 * multiplied by log2(e), within fp32's range).  GTP_ERR_UNSUPPORTED where a key head has more than 256
 * query heads, or they have more than 4096 biases in all.  Else as gtp_attention.
 * `work` of both directions, whichever gradients are asked for, may hold the buckets of all pairs
 * besides, a byte each for all heads: from 4 heads and segments of more than 256 rows and keys on, and
 * 1 GiB at most, B ceil64(max_q) ceil64(max_k) bytes (ceil64: rounded up to a multiple of 64); where they would
 * be more, each score makes its own, and nothing of size rows x keys is stored. */
int64_t gtp_attention_biased_work(const gtp_attn *a, const gtp_attn_bias *b, int backward);
gtp_status gtp_attention_biased(const gtp_attn *a, const gtp_attn_bias *b, const gtp_rows *q, const gtp_rows *k,
                                const gtp_rows *v, const gtp_rows *o, float *lse, void *work, int64_t work_bytes,
                                void *stream);

/* Its gradient: dq, dk, dv as gtp_attention_backward, and
 *   dbias[h, c] = sum of dS over the pairs of bucket c   [H, buckets] fp32, or NULL,
 * written, not accumulated, summed in a fixed order (`work` has a table [H / Hk, buckets] for each 64 to 256 rows of a key
 * head and segment besides).  Positions have no gradient: the bias is piecewise constant. */
gtp_status gtp_attention_biased_backward(const gtp_attn *a, const gtp_attn_bias *b, const gtp_rows *q,
                                         const gtp_rows *k, const gtp_rows *v, const gtp_rows *o, const gtp_rows *dout,
                                         const float *lse, const gtp_rows *dq, const gtp_rows *dk, const gtp_rows *dv,
                                         float *dbias, void *work, int64_t work_bytes, void *stream);

/* HBM streaming probe (measurement aid: the roof the HBM-bound kernels are
 * read against; each workgroup streams one contiguous chunk, the chunks
 * dealt to the XCDs in contiguous runs).  mode 0: read nbytes of src (dst: a
 * device float written only if the data holds a NaN); 1: write nbytes to dst
 * (non-temporal stores); 2: copy nbytes from src to dst (non-overlapping);
 * 3: dst = first half of src + second half (two read streams of nbytes / 2,
 * one written stream of nbytes / 2: the read/write mix of the pair
 * products; dst must not overlap src).  Device pointers 16-byte aligned,
 * nbytes >= 0 a multiple of 16 (32 for mode 3). */
gtp_status gtp_stream_probe(int mode, const void *src, void *dst, int64_t nbytes, void *stream);

/* Compute probe (measurement aid: the fp32 rates the chip delivers under
 * load, beside the published peak).  mode 0: fp32 VALU FMA chains (8
 * independent chains per lane); 1: fp32 v_mfma_f32_16x16x4f32 chains (4
 * independent accumulators per wave); 2048 workgroups of 256 lanes, iters
 * steps (1..2^30).  sink: one device float (4-byte aligned), written only if
 * a result is NaN; *flops (host) receives the flops the launch issues, for
 * the caller to divide by its own timing of the launch on stream. */
gtp_status gtp_compute_probe(int mode, int64_t iters, float *sink, double *flops, void *stream);

/* Number of floats of one per-product public grid: which = 1 or 2 gives the
 * input grids (2 * (2L+1)^2), which = 3 the product grid (2 * (2U+1)^2).
 * Returns -1 on a bad argument. */
int64_t gtp_grid_floats(gtp_plan p, int which);

/* Plan geometry: out[0..7] = {L1, L2, Lout, U = L1+L2, Le = min(Lout, U),
 * NT (theta intervals of the sampling grid on [0, pi]), NP (phi samples),
 * step-2 algorithm gtp_full actually runs: GTP_CONV_DIRECT, GTP_CONV_FFT or GTP_CONV_DFT}. */
gtp_status gtp_plan_info(gtp_plan p, int64_t *out8);

/* Copy one of the plan's fp64 host tables (test aid, host memory):
 *   which 0: T1   [tri(l,m)][u], u in [0, Lin]      theta-Fourier series of Q_l^m (step 1)
 *   which 1: Zc   [tri(l,m)][u], u in [0, U]        int cos(u t) Q sin t dt (step 3)
 *   which 2: Zs   [tri(l,m)][u], u in [0, U]        int sin(u t) Q sin t dt (step 3)
 *   which 3: S    [tri(l,m)][j], j in [0, NT]       synthesis at the theta nodes
 *   which 4: W    [tri(l,m)][j], j in [0, NT]       analysis weights at the theta nodes
 *   which 5: TWR  [lane][24]            phi-operand seeds of the matrix-core kernel
 *   which 6: SMP  [pass][s][u2][lane][4]  its lane-permuted theta synthesis values
 *   which 7: SM0P [pass][lane][v]         its m = 0 theta synthesis values (+ pole)
 *   which 8: WP   [pass][it][lane][8]     its lane-permuted theta analysis weights
 *   which 9: XMAP [lane][k]               its LDS slot of input coefficient lane + 64k
 *   which 10: J   per degree l, (2l+1)^2    real-SH matrix of the rotation R_x(90 deg)
 *   which 11: E   [pair][row]               theta-node rows of the rotated-frame convolution
 *   which 12: A   [m][lane][step]           its matrix-core operand images (theta tables)
 *   which 13: Z   [group][pair][l] + poles  its zonal-filter table
 *   which 14: JI  [l][tile][lane][step]     its operand images of J and J^T
 * with tri(l,m) = l(l+1)/2 + m, m >= 0.  Tables 5..9 exist only for
 * L1 = L2 = Lout = L in {16, 32, 64}, tables 10..11 for L1 = L2 = Lout in
 * 1..8 and 16, tables 12..14 for L1 = L2 = Lout = 16 (length 0 otherwise);
 * their layouts are internal to those kernels.  Pass buf = NULL to
 * get the length in *count; otherwise *count is the capacity in doubles. */
gtp_status gtp_plan_table(gtp_plan p, int which, double *buf, int64_t *count);

/* fp64 host evaluation of the plan's three-step transform pipeline on host
 * arrays (x1[n,(L1+1)^2], x2[n,(L2+1)^2] -> y[n,(Lout+1)^2]).  A CPU check of
 * the tables only; gtp_full never calls it and it is not a fallback. */
gtp_status gtp_debug_host_pipeline(gtp_plan p, const double *x1, const double *x2, int64_t n,
                                   double *y);

const char *gtp_status_str(gtp_status s);
const char *gtp_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* GTP_H */
