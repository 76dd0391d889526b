/*
 * afno.h -- C ABI of the MI355X (gfx950) AFNO spectral token-mixing filter.
 *
 * The filter is the spatial-mixing step of the FourCastNet AFNO transformer
 * (section "Model Innovations", the three steps: a 2-D FFT of the token grid, a
 * block-diagonal MLP applied to every token in Fourier space with weights shared by
 * all tokens, an inverse FFT), implemented with real-to-complex / complex-to-real
 * transforms batched over batch and channels, complex weights stored as real arrays
 * with (re, im) as the fastest index and activations acting on the real and
 * imaginary parts independently (section "Implementation Details" (b), "Spectral
 * convolution").  Softshrink, the hard mode cutoff and the residual come from the
 * AFNO layer the paper builds on.  Every step runs in hand-written HIP kernels.
 *
 * For one sample, with Wm = W/2 + 1, nb blocks of bs = C/nb channels, hs = bs:
 *   X[kh][kw][c] = (1/sqrt(HW)) sum_{h,w} x[h][w][c] exp(-2 pi i (kh h/H + kw w/W)),  kw <= W/2
 *   for every mode kept by the cutoff and every block k (true complex products):
 *     v[j] = b1[k][j] + sum_i X[k bs + i] w1[k][i][j];  h[j] = ReLU(Re v[j]) + i ReLU(Im v[j])
 *     o[i] = b2[k][i] + sum_j h[j] w2[k][j][i]
 *     Y[k bs + i] = S(Re o[i]) + i S(Im o[i]),  S(v) = v - lambda (v > lambda),
 *                                              v + lambda (v < -lambda), 0 otherwise
 *   modes outside the cutoff: Y = 0
 *   y[h][w][c] = (1/sqrt(HW)) sum_{kh, kw<=W/2} c_kw Re(Y[kh][kw][c] exp(+2 pi i (kh h/H + kw w/W))),
 *                c_kw = 1 for kw = 0 and kw = W/2, 2 otherwise
 *   out = x + y, rounded once to the storage dtype.
 * Hard mode cutoff (keep_fraction f): kept_h = floor((H/2+1) f) and
 * kept_w = floor((W/2+1) f), both evaluated in double; a mode (kh, kw) is kept when
 * |kh'| < kept_h, kh' = kh for kh <= H/2 and kh - H above, and kw < kept_w.
 * f = 1 keeps every mode; when either count is 0 nothing is kept and out = x.
 */
#ifndef AFNO_H_
#define AFNO_H_

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Storage dtype of x, the weights, the biases and out. */
typedef enum { AFNO_DTYPE_FP32 = 0, AFNO_DTYPE_BF16 = 1 } afno_dtype_t;

/* Return codes. */
enum {
  AFNO_OK = 0,
  AFNO_ERR_INVALID_ARG = -1, /* null pointer, non-positive size, C % nb != 0, bad lambda/keep/dtype */
  AFNO_ERR_UNSUPPORTED = -2, /* valid filter this library does not run: see afno_filter_forward */
  AFNO_ERR_ALIAS = -3,       /* out overlaps an input */
  AFNO_ERR_HIP = -4          /* a HIP allocation or launch failed; see afno_last_error() */
};

/*
 * afno_filter_forward -- out = x + filter(x) (the filter defined above).
 *
 *   x    [B][H][W][C]        dtype, row-major (channels fastest), device memory
 *   w1   [nb][bs][hs][2]     dtype, complex (re, im) fastest, input-major: x @ w1
 *   b1   [nb][hs][2]         dtype
 *   w2   [nb][hs][bs][2]     dtype
 *   b2   [nb][bs][2]         dtype
 *   B >= 0; H, W, C, num_blocks > 0; C % num_blocks == 0; hs = bs = C / num_blocks
 *   lambda         softshrink threshold, finite and >= 0
 *   keep_fraction  hard mode cutoff f, 0 < f <= 1
 *   dtype          an afno_dtype_t
 *   out  [B][H][W][C]        dtype, device memory, must not overlap any input
 *   stream         HIP stream the work is enqueued on (0 = the null stream)
 *
 * Ownership: the caller owns every array; all are contiguous device memory on the
 * current device and must stay valid until the stream has finished the work.  The
 * library allocates a spectrum workspace of B*H*kept_w*C complex values (8 bytes each
 * for fp32, 4 for bf16) stream-ordered on `stream` and frees it stream-ordered, from a
 * memory pool of its own per device that keeps freed memory for later calls (so the
 * largest workspaces in use at once stay allocated until the process ends).  Workspaces up to
 * 32 MB come, outside stream capture, from at most 8 pieces of 32 MB of that pool which the
 * library keeps per device; a stream takes over a piece of another one only when that one's work
 * in it has ended, and each user is ordered behind the last by an event.  Pieces no call is
 * using are given back when a workspace would not fit otherwise.  Under stream capture the workspace
 * is memory that the graph allocates and frees by itself, and a graph takes one call that does so, of all entry
 * points that allocate (this one, _hidden, _stage, _backward, afno_block_forward): the next one in the same
 * capture returns AFNO_ERR_UNSUPPORTED with nothing recorded, since a replay of several has
 * read memory that was not there any more.  A captured step takes afno_filter_forward_noalloc, as often
 * as it needs, one after another.
 * The call is asynchronous: it enqueues on `stream` and returns.
 * B == 0 returns AFNO_OK without touching the GPU (x and out may then be NULL).
 * Errors: arguments are validated before any HIP call; on a non-OK return nothing
 * has been enqueued, except for AFNO_ERR_HIP from a launch, after which out is
 * undefined.  AFNO_ERR_UNSUPPORTED: H or W not of the form 2^a 3^b 5^c, W odd,
 * bs not a multiple of 16 or above 128, or a grid too large for on-chip storage
 * (a column of H complex values x bs channels must fit the 160 KiB LDS of one CU,
 * H <= 192 for bs = 128, and W <= 1024), or a spectrum column (H * kept_w * C complex
 * values) or a grid row (W * C float32 values) larger than 4 GiB: the kernels address
 * them with 32-bit byte offsets.
 * Thread safety: calls from several host threads are safe; calls whose streams
 * overlap in time only share read-only inputs.
 */
int afno_filter_forward(const void* x, const void* w1, const void* b1, const void* w2,
                        const void* b2, int64_t B, int64_t H, int64_t W, int64_t C,
                        int64_t num_blocks, float lambda, float keep_fraction, int dtype,
                        void* out, hipStream_t stream);

/*
 * afno_filter_forward_noalloc -- afno_filter_forward for callers that cannot allocate device
 * memory: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, kernels and result (bitwise) as afno_filter_forward; the call allocates
 * nothing.  Its workspace (the spectrum, B*H*kept_w*C complex values of 4 bytes (bf16) or 8
 * (fp32), then the prepared block weights and the DFT table, about 1.2 MB for 8 blocks of 96)
 * is an array of AFNO_NOALLOC_MAX_WORKSPACE bytes in device memory that the library holds on
 * every GPU it runs on until the process ends (the 90 x 180 x 768 bf16 filter fits up to
 * B = 5).  AFNO_ERR_UNSUPPORTED, before any HIP call, when the workspace would be larger; the
 * size-generic column kernels do without the prepared weights where only those would not fit.
 * Every call on a GPU uses that GPU's one array, which keeps the last call's contents (each
 * call writes all it reads): calls whose work overlaps in time on one GPU (different streams
 * or host threads without ordering between them) race and leave out undefined; calls on one
 * stream are ordered and safe.  The first call on a device also resolves the array's address
 * there (hipGetSymbolAddress; AFNO_ERR_HIP if that fails).  Other errors as
 * afno_filter_forward.
 */
#define AFNO_NOALLOC_MAX_WORKSPACE (128u << 20)
int afno_filter_forward_noalloc(const void* x, const void* w1, const void* b1, const void* w2,
                                const void* b2, int64_t B, int64_t H, int64_t W, int64_t C,
                                int64_t num_blocks, float lambda, float keep_fraction, int dtype,
                                void* out, hipStream_t stream);

/*
 * afno_filter_forward_hidden -- the same filter with `hidden` hidden units per block in
 * the block MLP (the AFNO layer's hidden-size factor: hidden = factor * bs; the paper's
 * filter, "Model Innovations", uses hidden = bs, which afno_filter_forward assumes).
 *   w1 [nb][bs][hidden][2], b1 [nb][hidden][2], w2 [nb][hidden][bs][2], b2 [nb][bs][2]
 *   hidden > 0 (AFNO_ERR_INVALID_ARG otherwise); a multiple of 16 and <= 256, and the
 *   column's hidden layer (H x hidden complex values) must fit in LDS beside the column
 *   tile (AFNO_ERR_UNSUPPORTED otherwise).  hidden == bs runs exactly afno_filter_forward.
 * Other arguments, ownership and errors as afno_filter_forward.  hidden == 2 * bs with bf16
 * storage, H <= 96 and bs 32, 64 or 96 runs a matrix-core column kernel (the workspace holds
 * its weight fragments and the DFT table besides the spectrum); other hidden sizes run the
 * size-generic column kernel.
 */
int afno_filter_forward_hidden(const void* x, const void* w1, const void* b1, const void* w2,
                               const void* b2, int64_t B, int64_t H, int64_t W, int64_t C,
                               int64_t num_blocks, int64_t hidden, float lambda,
                               float keep_fraction, int dtype, void* out, hipStream_t stream);

/*
 * afno_block_forward -- one AFNO transformer block around the filter: the paper's layer
 * mixes tokens with the spectral filter and channels with a single-hidden-layer MLP of four
 * times the embedding width shared by all tokens ("Model Innovations"; "Implementation
 * Details" (c)).  With per-token LayerNorms (the paper states none; the AFNO layer's pre-norm
 * arrangement is taken) and the exact GELU:
 *   t = LN1(x);  v = x + filter(t)  (the filter includes its own residual: filter(t) = t + y);
 *   w = LN2(v);  out = v + GELU(w wa + ba) wb + bb
 *   LN(z) = (z - mean) / sqrt(var + 1e-6) * gamma + beta over the C channels of a token,
 *   biased variance.
 *   x, out       [B][H][W][C] bf16; tokens are the rows of x viewed as [B*H*W][C]
 *   ln1_g, ln1_b, ln2_g, ln2_b  [C] bf16, 16-byte aligned
 *   w1, b1, w2, b2              the filter's weights, as afno_filter_forward
 *   wa [C][4C], ba [4C], wb [4C][C], bb [C]   bf16, input-major (z wa)
 * dtype must be AFNO_DTYPE_BF16 (fp32: AFNO_ERR_UNSUPPORTED); C a multiple of 128 and
 * <= 2048; the filter's limits as afno_filter_forward.  out must not overlap any input
 * (AFNO_ERR_ALIAS).  The library allocates one stream-ordered workspace (four token grids,
 * the B*H*W x 4C hidden layer in bf16, the transposed MLP weights and the filter's spectrum)
 * and frees it stream-ordered.  Intermediates (t, the filter output, v, w, the hidden layer)
 * are rounded to bf16; products accumulate in fp32.  Other arguments, ownership, errors and
 * asynchrony as afno_filter_forward.
 */
int afno_block_forward(const void* x, const void* ln1_g, const void* ln1_b, const void* w1,
                       const void* b1, const void* w2, const void* b2, const void* ln2_g,
                       const void* ln2_b, const void* wa, const void* ba, const void* wb,
                       const void* bb, int64_t B, int64_t H, int64_t W, int64_t C,
                       int64_t num_blocks, float lambda, float keep_fraction, int dtype,
                       void* out, hipStream_t stream);

/*
 * afno_filter_stage -- diagnostic entry point: runs the filter's kernels up to a stage
 * and writes that stage's result in float32, for per-stage parity checks.
 *   stage AFNO_STAGE_SPECTRUM  dst [B][H][Wm][C][2] float32: the forward spectrum X
 *                              (both axes, ortho-normalised); columns kw >= kept_w
 *                              are not computed and are written as 0.
 *   stage AFNO_STAGE_MIXED     dst [B][H][Wm][C][2] float32: Y after the block MLP,
 *                              softshrink and the cutoff.
 *   stage AFNO_STAGE_DELTA     dst [B][H][W][C] float32: y = filter(x) before the
 *                              residual add and before rounding to dtype.
 * Other arguments, ownership and errors as afno_filter_forward, with dst in place of
 * out.  The values are what the kernels hold at that point (for bf16 storage the
 * spectra are bf16-rounded).
 */
enum { AFNO_STAGE_SPECTRUM = 1, AFNO_STAGE_MIXED = 2, AFNO_STAGE_DELTA = 3 };
int afno_filter_stage(const void* x, const void* w1, const void* b1, const void* w2,
                      const void* b2, int64_t B, int64_t H, int64_t W, int64_t C,
                      int64_t num_blocks, float lambda, float keep_fraction, int dtype,
                      int stage, float* dst, hipStream_t stream);

/*
 * afno_filter_stage_hidden -- afno_filter_stage for the block MLP with `hidden` units per
 * block (weights as afno_filter_forward_hidden).  AFNO_STAGE_DELTA runs the same kernels as
 * afno_filter_forward_hidden up to the inverse W-axis transform; AFNO_STAGE_SPECTRUM and
 * AFNO_STAGE_MIXED stop inside the column pass, which for hidden != bs is the size-generic
 * column kernel.  Arguments, ownership and errors as afno_filter_stage and
 * afno_filter_forward_hidden (hidden <= 0: AFNO_ERR_INVALID_ARG).
 */
int afno_filter_stage_hidden(const void* x, const void* w1, const void* b1, const void* w2,
                             const void* b2, int64_t B, int64_t H, int64_t W, int64_t C,
                             int64_t num_blocks, int64_t hidden, float lambda,
                             float keep_fraction, int dtype, int stage, float* dst,
                             hipStream_t stream);

/*
 * afno_filter_backward -- gradients of a loss L through out = x + filter(x), given
 * gout = dL/dout: the transpose of the filter's forward map (the paper trains through it:
 * "Implementation Details" (a), (e)), step by step in reverse order.  With X the forward
 * spectrum, v = X w1 + b1, h = relu(v), o = h w2 + b2 per kept mode and block as above:
 *   dz  = c_kw F(gout)            (F the forward 2-D transform, c_kw its inverse's weights)
 *   do  = dz where |o| > lambda on that component and the mode is kept, else 0
 *   dh  = do w2^H (conjugate transpose),  dv = dh where v > 0 on that component, else 0
 *   dx  = gout + F^T(dv w1^H)     (F^T: the inverse with unit weights c_kw = 1)
 *   dw1 = sum over kept modes of conj(X)^T dv,  db1 = sum of dv
 *   dw2 = sum over kept modes of conj(h)^T do,  db2 = sum of do
 * (re, im pairs hold d/d re and d/d im; relu'(0) = 0 and the softshrink slope is 0 on
 * [-lambda, lambda]).
 *   x, w1, b1, w2, b2, sizes, lambda, keep_fraction, dtype   as afno_filter_forward
 *   gout [B][H][W][C]        dtype, device memory
 *   dx   [B][H][W][C]        dtype, device memory
 *   dw1, dw2 [nb][bs][bs][2]  float32, device memory, overwritten (not accumulated)
 *   db1, db2 [nb][bs][2]      float32, device memory, overwritten
 * No output may overlap an input or another output (AFNO_ERR_ALIAS).  The library
 * allocates stream-ordered workspace on `stream`: two spectra, the prepared
 * weights, four per-mode factor tensors of nb * 2 bs * B * kept_w * ceil32(ceil16(H)) values
 * in dtype, and float32 chunk sums (2 nb 2 bs (2 bs + 1) per chunk of modes, at most 128
 * chunks).  B == 0 or nothing kept: dx = gout and zero weight and bias gradients.  Errors as
 * afno_filter_forward; AFNO_ERR_UNSUPPORTED also when a column of the backward kernel (one
 * tile of H x bs complex values plus two bit masks) does not fit the LDS.  Reproducibility:
 * no atomics; the weight and bias gradients are chunk sums stored by the weight-product
 * kernels and added in a fixed order, so repeated calls give the same bits.
 */
int afno_filter_backward(const void* x, const void* w1, const void* b1, const void* w2,
                         const void* b2, const void* gout, int64_t B, int64_t H, int64_t W,
                         int64_t C, int64_t num_blocks, float lambda, float keep_fraction,
                         int dtype, void* dx, float* dw1, float* db1, float* dw2, float* db2,
                         hipStream_t stream);

/*
 * Training around the filter: linear products, LayerNorm and dropout, each with its gradient --
 * the rest of an AFNO block (LayerNorm, the channel MLP, the residual adds) as operators of their
 * own.  Arrays are rows of channels, [M][C] with the channels fastest (a [B][H][W][C] grid: M = B H W),
 * contiguous device memory on the current device, aligned to their element (16 bytes take the wider
 * kernels).  Any M from 0 to 2^25, any width up to 2^20, up to 2^34 values an array
 * (AFNO_ERR_UNSUPPORTED beyond).  No output may overlap an input or another output
 * (AFNO_ERR_ALIAS).  Ownership, asynchrony and errors as afno_filter_forward; sums are held in float32
 * and added in a fixed order, so repeated calls give the same bits.
 *
 * Workspace.  afno_*_workspace gives the bytes that a call of these sizes may need (0: none; an error
 * code for sizes that the call refuses); aligned non-zero: for arrays that are all 16-byte aligned,
 * which may need less (rows at other addresses are copied).  With workspace non-NULL the call uses
 * the caller's memory: at least that many bytes, 16-byte aligned, apart from every array, the call's
 * alone until its work has ended, so that captured graphs that may run at the same time need one each.  With NULL the
 * library takes one of its own as afno_filter_forward does, except under stream capture, where a
 * call that needs one returns AFNO_ERR_UNSUPPORTED.
 *
 * Dropout.  Element e (its flat index) is kept where number e % 8 of group e / 8 is at least
 * T = 65536 p rounded to a whole number, and scaled by 65536 / (65536 - T); else it becomes 0,
 * whatever it was.  A group's eight 16-bit numbers are the words of Philox4x32 with seven rounds, low
 * halves first, of the counter (group low, group high, place low, place high) with the seed as key;
 * place = offset + *counter modulo 2^64 (counter NULL: offset).  counter is a device address that
 * is read when the kernel runs, so that a captured training step draws anew in each replay.  The
 * mask is a function of these numbers alone and is never stored.  0 <= p < 1, and T < 65536.
 */
enum { AFNO_ACT_NONE = 0, AFNO_ACT_RELU = 1, AFNO_ACT_GELU = 2 };

/*
 * afno_linear_forward -- out = drop(act(x w + b)) + residual.
 *   x [M][K], w [K][N] (input-major: x w), b [N] or NULL, residual [M][N] or NULL    dtype
 *   activation  none, ReLU, or the exact GELU z Phi(z)
 *   out [M][N]           dtype; one rounding from the float32 sum
 *   pre [M][N] or NULL   dtype: x w + b, which the gradient of an activation takes
 * M == 0 returns AFNO_OK without touching the GPU.
 */
int afno_linear_forward(const void* x, const void* w, const void* b, const void* residual, int64_t M,
                        int64_t K, int64_t N, int activation, float p, uint64_t seed,
                        uint64_t offset, const uint64_t* counter, int dtype, void* out, void* pre,
                        void* workspace, int64_t workspace_bytes, hipStream_t stream);
int64_t afno_linear_forward_workspace(int64_t M, int64_t K, int64_t N, int dtype, int aligned);

/*
 * afno_linear_backward -- gradients of afno_linear_forward for g = dL/dout (the residual's is g):
 *   dz = act'(pre) drop(g);  dx = dz w^T [M][K],  dw = x^T dz [K][N],  db = sum of dz's rows [N]
 * With ReLU, dz = drop(g) where pre > 0 and 0 elsewhere (where pre is NaN too), whatever g is there.
 * dx, dw and db are in dtype and overwritten; each may be NULL, at least one is not.
 * pre is not read where the activation is none, w only for dx, x only for dw.  dz is rounded to dtype
 * before the products; db sums the unrounded values.  dw and db are each rounded once from their float32
 * sums: a caller that adds up several bf16 batches' adds their roundings.  M == 0: dw and db are 0.
 */
int afno_linear_backward(const void* g, const void* x, const void* w, const void* pre, int64_t M,
                         int64_t K, int64_t N, int activation, float p, uint64_t seed,
                         uint64_t offset, const uint64_t* counter, int dtype, void* dx, void* dw,
                         void* db, void* workspace, int64_t workspace_bytes, hipStream_t stream);
int64_t afno_linear_backward_workspace(int64_t M, int64_t K, int64_t N, int dtype, int aligned);

/*
 * afno_layer_norm_forward -- v = x + residual rounded to dtype (residual NULL: v = x);
 *   out = (v - mean) / sqrt(var + eps) * gamma + beta over the C channels of a row, biased variance.
 *   x, residual, out [M][C], gamma, beta [C]   dtype;  eps finite and >= 0
 *   sum [M][C] or NULL   dtype: v, the residual stream and what the gradient takes
 */
int afno_layer_norm_forward(const void* x, const void* residual, const void* gamma, const void* beta,
                            int64_t M, int64_t C, float eps, int dtype, void* out, void* sum,
                            hipStream_t stream);

/*
 * afno_layer_norm_backward -- gradients of the norm of x (the v above) for g = dL/dout:
 *   with a = g gamma and h = (x - mean) / sqrt(var + eps):
 *   dx = (a - mean(a) - h mean(a h)) / sqrt(var + eps) + gsum
 *   dgamma = sum over the rows of g h,  dbeta = sum over the rows of g
 *   gsum [M][C] or NULL  dtype: the gradient that reaches v along the residual stream
 *   dx [M][C] dtype; dgamma, dbeta [C] float32, overwritten.  M == 0: dgamma and dbeta are 0.
 */
int afno_layer_norm_backward(const void* g, const void* x, const void* gamma, const void* gsum,
                             int64_t M, int64_t C, float eps, int dtype, void* dx, float* dgamma,
                             float* dbeta, void* workspace, int64_t workspace_bytes,
                             hipStream_t stream);
int64_t afno_layer_norm_backward_workspace(int64_t M, int64_t C, int dtype);

/*
 * afno_dropout_forward -- out = drop(x) + residual (NULL: none) over n elements of dtype;
 * afno_dropout_backward -- dx = drop(g) with the same numbers (the residual's gradient is g).
 */
int afno_dropout_forward(const void* x, const void* residual, int64_t n, float p, uint64_t seed,
                         uint64_t offset, const uint64_t* counter, int dtype, void* out,
                         hipStream_t stream);
int afno_dropout_backward(const void* g, int64_t n, float p, uint64_t seed, uint64_t offset,
                          const uint64_t* counter, int dtype, void* dx, hipStream_t stream);

/*
 * The channel MLP in eight bits: rows kept and multiplied in half the memory of bf16, and the
 * root-mean-square norm that makes them.  Arrays, workspaces, dropout, ownership and errors as for the
 * operators above.
 *
 * Eight bits ("mx8", the Open Compute Project's microscaling layout with E4M3 values): rows of C channels are
 *   values [M][32 ceil(C / 32)]  uint8, E4M3 (largest 448, no infinity), 0 behind the C channels
 *   scales [M][ceil(C / 32)]     uint8, s + 127 for every 32 neighbouring channels: a value is 2^s E4M3
 * with values 16-byte aligned.  Writing, s is the smallest with which no finite value of the block is above
 * 448 2^s, kept in -117 .. 119 (every value is then a normal bf16 number or 0, and finite: a block with larger
 * ones has them at 448 2^119), values are rounded to nearest, ties to even, once from float32, and a NaN
 * or an infinity becomes NaN.  What the calls read has its scales in that range and zeros behind the C.
 */

/*
 * afno_mx8_pack -- x [M][C] of dtype to eight bits;  afno_mx8_unpack -- out [M][C] of dtype from
 * eight bits, exact in either dtype.
 */
int afno_mx8_pack(const void* x, int64_t M, int64_t C, int dtype, void* values, void* scales,
                  hipStream_t stream);
int afno_mx8_unpack(const void* values, const void* scales, int64_t M, int64_t C, int dtype, void* out,
                    hipStream_t stream);

/*
 * afno_rms_norm_forward -- v = x + residual rounded to dtype (residual NULL: v = x);
 *   out = v / sqrt(mean(v^2) + eps) * gamma over the C channels of a row.
 *   x, residual [M][C], gamma [C]   dtype;  eps finite and >= 0
 *   out [M][C] or NULL   dtype;  out_values, out_scales: out in eight bits, or NULL; one of the two at least
 *   sum [M][C] or NULL   dtype: v, the residual stream and what the gradient takes
 * The sum of v^2 is float32's: in a row where it passes 2^128 the results are 0 (the gradient's, too, but for
 * gsum); rows as small as the type holds keep their digits whatever eps is.  eps 0: a row of zeros gives NaN.
 */
int afno_rms_norm_forward(const void* x, const void* residual, const void* gamma, int64_t M, int64_t C,
                          float eps, int dtype, void* out, void* sum, void* out_values,
                          void* out_scales, hipStream_t stream);

/*
 * afno_rms_norm_backward -- gradients of the norm of x (the v above) for g = dL/dout (one in eight bits passes
 * its gradient on as it is):
 *   with a = g gamma, r = 1 / sqrt(mean(x^2) + eps), h = x r:  dx = r (a - h mean(a h)) + gsum
 *   dgamma = sum over the rows of g h
 *   gsum [M][C] or NULL  dtype: the gradient that reaches v along the residual stream
 *   dx [M][C] dtype; dgamma [C] float32, overwritten.  M == 0: dgamma is 0.
 */
int afno_rms_norm_backward(const void* g, const void* x, const void* gamma, const void* gsum, int64_t M,
                           int64_t C, float eps, int dtype, void* dx, float* dgamma, void* workspace,
                           int64_t workspace_bytes, hipStream_t stream);
int64_t afno_rms_norm_backward_workspace(int64_t M, int64_t C, int dtype);

/*
 * afno_mx8_linear_forward -- out = drop(act(x w^T + b)) + residual for rows in eight bits.
 *   x [M][K], w [N][K] (output-major: the transpose of afno_linear_forward's)   eight bits
 *   b [N] or NULL, residual [M][N] or NULL   dtype
 *   out [M][N] or NULL   dtype;  out_values, out_scales: out in eight bits, or NULL; one of the two at
 *                        least, each one rounding from the float32 sum
 *   pre_values, pre_scales   x w^T + b in eight bits, which the gradient of an activation takes, or NULL
 * dtype AFNO_DTYPE_FP32: products and sums are float32's.  AFNO_DTYPE_BF16: the matrix cores' eight-bit
 * instruction, at twice the rate, whose sums are off by 1.7e-5 (relative 2-norm; a result in eight bits is
 * now and then the neighbouring E4M3 value), and a GELU within 1.3e-5 of its own size down to -9.
 */
int afno_mx8_linear_forward(const void* x_values, const void* x_scales, const void* w_values,
                            const void* w_scales, const void* b, const void* residual, int64_t M,
                            int64_t K, int64_t N, int activation, float p, uint64_t seed,
                            uint64_t offset, const uint64_t* counter, int dtype, void* out,
                            void* out_values, void* out_scales, void* pre_values, void* pre_scales,
                            void* workspace, int64_t workspace_bytes, hipStream_t stream);
int64_t afno_mx8_linear_forward_workspace(int64_t M, int64_t K, int64_t N, int dtype);

/*
 * afno_mx8_linear_backward -- afno_linear_backward from rows kept in eight bits: x and the value before the
 * activation are what their eight bits stand for, g, w [K][N] (as afno_linear_forward's) and the gradients are
 * of dtype, the products as afno_linear_backward's.  Where the forward product's w was in eight bits, too, its
 * rounding passes the gradient on as it is.
 */
int afno_mx8_linear_backward(const void* g, const void* x_values, const void* x_scales, const void* w,
                             const void* pre_values, const void* pre_scales, int64_t M, int64_t K,
                             int64_t N, int activation, float p, uint64_t seed, uint64_t offset,
                             const uint64_t* counter, int dtype, void* dx, void* dw, void* db,
                             void* workspace, int64_t workspace_bytes, hipStream_t stream);
int64_t afno_mx8_linear_backward_workspace(int64_t M, int64_t K, int64_t N, int dtype, int aligned);

/*
 * Diagnostic per-kernel timing.  afno_profile_begin(max_calls) creates HIP events for
 * up to max_calls filter calls (process-wide); each later afno_filter_forward call
 * records an event before its first kernel and after each of its four phases, on the
 * call's stream.  afno_profile_end waits for those events, writes the summed
 * milliseconds of each phase to kernel_ms[0..3] (0: operand preparation as a launch of its
 * own -- the block weights in MFMA fragment order and the H-axis DFT table; exactly 0 where
 * there is no such launch, the column kernel taking none or the preparation running as extra
 * workgroups of the size-specialised W-axis forward launch; 1: W-axis forward transform; 2: column kernel,
 * H transforms + block MLP; 3: W-axis inverse transform + residual) and the number of timed calls to *calls, and
 * frees the events.  Calls beyond max_calls are not timed.
 * Returns AFNO_OK, AFNO_ERR_INVALID_ARG (max_calls <= 0, null output, or end without
 * begin) or AFNO_ERR_HIP.  Not for concurrent use with calls on other streams.
 */
int afno_profile_begin(int max_calls);
int afno_profile_end(double* kernel_ms, int64_t* calls);

/*
 * Diagnostic kernel selection, process-wide.  AFNO_PATH_AUTO (the default) runs the
 * specialised kernels where the library has them and the size-generic kernels elsewhere:
 * W-axis kernels for every even W = 2^a 3^b 5^c from 12 to 576; for bf16 with H <= 96 and bs in {32, 64, 96}
 * the column kernel that computes the H-axis DFTs as bf16 matrix-core products against a
 * DFT table (and its hidden-size variant for hidden = 2 bs); else column kernels with
 * vector-ALU FFTs for H x bs in {16 x 16, 90 x 96, 180 x 32, and for bf16 180 x 64 and
 * 180 x 128}.  AFNO_PATH_VALU_DFT is AUTO without the matrix-core DFT column kernels;
 * AFNO_PATH_GENERIC runs the size-generic kernels for every shape.  All compute the same
 * filter (the matrix-core DFT rounds its table to bf16: one more bf16-sized error per H
 * transform).  Returns AFNO_OK or AFNO_ERR_INVALID_ARG.  Safe while other threads enqueue
 * calls: a call reads the setting once, when it sizes its workspace, and runs that path
 * throughout.
 */
enum { AFNO_PATH_AUTO = 0, AFNO_PATH_GENERIC = 1, AFNO_PATH_VALU_DFT = 2 };
int afno_set_kernel_path(int path);

/* Message of the calling thread's last non-OK return ("" if none).  The pointer
 * stays valid until the thread's next call into the library. */
const char* afno_last_error(void);

/* Library version as major*10000 + minor*100 + patch. */
int afno_version(void);

#ifdef __cplusplus
}
#endif
#endif /* AFNO_H_ */
