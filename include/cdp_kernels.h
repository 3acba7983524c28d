/* libcdp kernel-level entry points: the contractions a CDP tick is made of, callable on
 * their own (unit parity tests against the CPU oracle, roofline micro-benchmarks).
 * All pointers are HIP device pointers owned by the caller; work is enqueued on
 * `stream` (hipStream_t, may be NULL) and the call returns without waiting.
 * Return value: 0 or a negative status code of cdp.h. */
#ifndef CDP_KERNELS_H
#define CDP_KERNELS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* C[M][N] (fp32, row-major, ldc = N) = A * B^T with fp32 accumulation, the tile
 * contraction used by every stage forward / backward of a tick (Sec. 3.1: the forward and
 * backward computation of a stage on one micro-batch).
 *   dtype      0 fp32, 1 bf16 (operand element type)
 *   tile_shape 0: 128x128, 1: 64x128, 2: 64x64 workgroup tile of the generic kernel (with a_kmajor =
 *              b_kmajor = 0, a weight gradient, all three run the tiles the Linear stages use for it
 *              where those are faster: in fp32 not for large results in odd layouts or of very few rows);
 *              3: 64x64, 4: 64x128 tile of the weight-streaming kernel the Linear stages
 *              use; 5: what is fastest for a Linear layer on its own: a kernel for one problem of few
 *              rows and 16-byte-chunked operands, else the tiles the engine launches; 6: those tiles, which for
 *              at most 32 rows and 16-byte-chunked operands are 32x32 with waves that split the reduction
 *              (3..6 need a_kmajor = b_kmajor = 1); 7, 8, 9: the generic kernel of 0, 1, 2 in every layout
 *   a_kmajor   1: A[m][k] at A[m*lda + k]   0: A[m][k] at A[k*lda + m]
 *   b_kmajor   1: B[n][k] at B[n*ldb + k]   0: B[n][k] at B[k*ldb + n] */
int cdp_k_gemm(int dtype, int tile_shape, int a_kmajor, int b_kmajor, const void* A, const void* B,
               float* C, int M, int N, int K, int lda, int ldb, void* stream);

/* One NHWC convolution contraction as implicit GEMM (no affine, no activation).
 *   which 0: forward        y[B][Ho][Wo][Cout] (elem type) = conv(x, w),  w[Cout][k][k][Cin]
 *         1: data gradient  dx[B][H][W][Cin]   (elem type) from dy and wt[Cin][k][k][Cout]
 *         2: weight gradient dw[Cout][k][k][Cin] (fp32, overwritten) from dy and x
 *         3, 4: as 0, 1 on the direct-to-LDS kernel's 256 x 256 tile whatever the size (the engine and which =
 *               0, 1 choose by launch size); 5, 6: the same kernel's 256 x 128 tile; CDP_EINVAL unless bf16 with
 *               channel counts that are multiples of 64
 *         7, 8: as 0, 1 the way the engine launches them, with a workspace in which workgroups share the reductions
 *               of a launch of few tiles: CDP_CONV_SHARE_BYTES, the last 8192 of them zero before the first call (every
 *               call leaves them zero); CDP_EINVAL without it or for channel counts that are not whole 16-byte chunks
 *         9: as 2, but added to dw instead of overwriting it; needs the workspace of the two-phase path
 *         10, 11: as 0, 1 before and after a GELU, as the engine launches them: 10 also stores the GELU of y, 11 multiplies dx by the GELU's
 *               derivative at its input; that other tensor, of the size and type of the result and 16-byte aligned, is
 *               `workspace`; CDP_EINVAL unless bf16, more than 64 columns and channel counts that are whole 16-byte chunks
 * in0/in1: (x, w) | (dy, wt) | (dy, x).  `out` must not alias the inputs.
 * workspace (device, may be NULL): scratch for the split weight-gradient kernel.  Where the shape allows and it holds
 * at least one partial sum (4 * Cout*k*k*Cin bytes) the two-phase path is used; without, the generic single-pass kernel
 * runs.  How many ranges the reduction is cut into, and with it the order of the sums, depends on the shape alone where the
 * workspace holds B*Ho*Wo / 512 + 4 partial sums; a smaller one may mean fewer ranges (other roundings, slower). */
#define CDP_CONV_SHARE_BYTES ((32u << 20) + 8192u)
int cdp_k_conv(int dtype, int which, const void* in0, const void* in1, void* out, int B, int H, int W,
               int Cin, int Cout, int ksize, int stride, int pad, void* workspace,
               size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc): the weight gradient of cdp_k_conv (which = 2, two-phase path) with the
 * partial sums of its reduction ranges in a device array that is part of the library image
 * (CDP_STATIC_SCRATCH_BYTES per GPU, held until the process ends) instead of a caller's workspace.
 * dw[Cout][k][k][Cin] (fp32, overwritten) from dy[B][Ho][Wo][Cout] and x[B][H][W][Cin] (element type by
 * dtype).  Calls no hipMalloc / hipFree and no allocating library routine.
 * Errors: CDP_EINVAL for shapes the two-phase kernels do not take (channel counts that are not whole
 * 16-byte chunks, more than 32 taps); CDP_ENOMEM when the partial sums (4 * Cout*k*k*Cin * ranges bytes)
 * exceed the array - cdp_last_error(NULL) then says how many bytes were needed; CDP_EHIP.
 * All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (different streams,
 * different threads) race.  Nothing in the array has to be cleared between calls. */
#define CDP_STATIC_SCRATCH_BYTES (16u << 20)
int cdp_k_conv_wgrad_static(int dtype, const void* dy, const void* x, float* dw, int B, int H, int W, int Cin,
                            int Cout, int ksize, int stride, int pad, void* stream);

/* The kernels of ViT-shaped stages (the homogeneous stages of Sec. 5 "Memory") on their own.
 * Element type of x / dy / out / qkv / P / dout by `dtype`; gamma, beta and their gradients fp32.
 *
 * LayerNorm over the last axis of x[rows][C] (C <= 1024, eps 1e-5, biased variance):
 *   backward 0: out = y = (x - mean) * rstd * gamma + beta       (dy, add, dgamma, dbeta, workspace unused)
 *   backward 1: out = dx (+ add, may be NULL); dgamma[C] += sum dy * xhat; dbeta[C] += sum dy;
 *               workspace: 8 * rows + 8 * C * ceil(rows / 32) + 256 bytes (CDP_EINVAL if smaller). */
int cdp_k_layernorm(int dtype, int backward, const void* x, const void* dy, const void* add, const float* gamma,
                    const float* beta, void* out, float* dgamma, float* dbeta, void* workspace,
                    size_t workspace_bytes, int rows, int C, void* stream);

/* Exact GELU on n elements: backward 0: out = x * Phi(x); backward 1: out = dy * (Phi(x) + x * phi(x)). */
int cdp_k_gelu(int dtype, int backward, const void* x, const void* dy, void* out, int64_t n, void* stream);

/* Multi-head self-attention core on qkv[B][T][3*D] (q | k | v per token, head h in columns
 * h*D/heads..; T <= 1024):
 *   backward 0: P[B][heads][T][T] = softmax(q k^T / sqrt(D/heads)) (written), out[B][T][D] = P v
 *   backward 1: out = dqkv[B][T][3*D] from P (read) and dout[B][T][D]
 * workspace: 4 * B*heads*T*T bytes (forward), (4 + element size) * B*heads*T*T + 256 bytes (backward). */
int cdp_k_attention(int dtype, int backward, const void* qkv, void* P, const void* dout, void* out, void* workspace,
                    size_t workspace_bytes, int B, int T, int D, int heads, void* stream);

/* ---- token models on packed batches ----------------------------------------------------------------------------
 * Rows are tokens.  Tensors are row-major and packed; nothing but what is said to be written is touched.  Outputs must not alias
 * inputs except where it is said.  Sizes of zero are CDP_EINVAL like negative ones, and so
 * are scales that are not finite, and sizes whose launch would have 2^32 threads (none of less than 2^22 rows, 2^29 words, 2^34
 * elements of a table, 2^23 heads times tokens and sequences).  The device of the pointers and of `stream` has to be the current one.  Every call may be captured into a graph; calls that overlap in time need workspaces of their own.  The same inputs give
 * the same bits.
 *
 * Embedding: rows of table[vocab][C] (C <= 2^24) by ids[rows].  A token whose id is outside [0, vocab) (padding) has a row of zeros and no gradient.
 *   backward 0: out[rows][C] (elem type) = scale * table[ids]   (dout, workspace unused)
 *   backward 1: out = dtable[vocab][C] (fp32) = scale * sum over the tokens of a row of dout[rows][C] (table unused), zero for
 *               rows without a token; the tokens of a row are summed in a fixed order
 *   backward 2: as 1, but added to dtable; rows without a token are not touched
 * workspace (backward): 16 * rows + 8 * C * ceil(rows / 32) + 512 bytes (CDP_EINVAL if smaller). */
int cdp_k_embedding(int dtype, int backward, const void* table, const int32_t* ids, const void* dout, void* out, float scale,
                    void* workspace, size_t workspace_bytes, int rows, int vocab, int C, void* stream);

/* The end of one block and the start of the next, over rows of C <= 16384 channels, norm(v) = v / sqrt(mean(v^2) + eps),
 * for rows whose squares have a sum that fp32 holds (rms up to 1e17):
 *   u = norm(h) * gamma_post       h[rows][C]: what the block computed; gamma_post NULL: u = h
 *   r = x + scale * sigmoid(gate) * u       gate[rows][C]; NULL: no gate.  h NULL: r = x, and gate and gamma_post are NULL
 *   y = norm(r) * gamma_pre        gamma_pre NULL: no y
 * x, h, gate, r, y in the element type, gamma_* fp32[C].  r may be NULL (not wanted) if y is not; r may be x, which the
 * backward of y reads, however: not where that is to follow. */
int cdp_k_residual_norm(int dtype, const void* x, const void* h, const void* gate, const float* gamma_post, const float* gamma_pre,
                        void* r, void* y, float scale, float eps, int rows, int C, void* stream);

/* Its gradients from dr[rows][C] (the gradient of r beside the one through y; NULL: none) and dy[rows][C] (with gamma_pre; NULL without):
 *   dx = d r in all, dh, dgate (elem type, written; dh and dgate with h and gate);
 *   dgamma_post[C], dgamma_pre[C] (fp32, with gamma_post and gamma_pre): overwritten, with accumulate != 0 added to.
 * x, h, gate, gammas: as the forward had them (x NULL without gamma_pre); r and y are made again.  dx may be dr.
 * workspace: 8 * C * min(rows, 512) + 256 bytes (CDP_EINVAL if smaller). */
int cdp_k_residual_norm_backward(int dtype, int accumulate, const void* x, const void* h, const void* gate, const float* gamma_post,
                                 const float* gamma_pre, const void* dr, const void* dy, void* dx, void* dh, void* dgate,
                                 float* dgamma_post, float* dgamma_pre, float scale, float eps, void* workspace, size_t workspace_bytes,
                                 int rows, int C, void* stream);

/* Causal self-attention of sequences of different lengths packed behind each other: sequence s is the rows offsets[s] ..
 * offsets[s + 1] - 1 (device int32 [sequences + 1], ascending, within [0, tokens]; a length may be zero), and a token sees its own
 * sequence up to itself.  qkv[tokens][(heads + 2 * kv_heads) * width]: q heads | k heads | v heads per token; query head h goes with key
 * head h / (heads / kv_heads).  width: a multiple of 8 up to 128; heads a multiple of kv_heads, heads + 2 * kv_heads up to 4096; tensors 16-byte
 * aligned.
 *   backward 0: out[tokens][heads * width] = softmax(scale * q k^T) v, lse[heads][tokens] (fp32) = log of the sum that the softmax divides
 *               by, sum exp(scale * q k^T)   (dout, dqkv, workspace unused)
 *   backward 1: dqkv from dout[tokens][heads * width] and the forward's out and lse
 * Sums are fp32.  fp32 products leave out less than 2^-21 of themselves (2^-24.5 on average).  bf16: between two products P and dS are
 * rounded to the element type, but held in two of it where one launch does the backward of few rows.  That and the order of sums go by
 * all sizes of a call: what a sequence is packed with may change its results by their roundings.
 * The backward makes probabilities from lse, with its rounding: |lse| * 2^-22 of themselves.
 * What is infinite or NaN in a row of qkv or dout may reach every row of its sequence, earlier and later ones (0 * NaN), as NaN in fp32, and no other
 * sequence.
 * Rows outside all sequences are neither read for another's sake nor written.  Offsets that are not as said give wrong results, within
 * the tensors.
 * workspace (backward): 4 * heads * tokens + 512 bytes (CDP_EINVAL if smaller).  Where it holds P times 8 * kv_heads * tokens * width
 * bytes more, launches of few key tiles share the query heads of a key head over up to P workgroups: faster, other roundings. */
int cdp_k_attention_packed(int dtype, int backward, const void* qkv, const int32_t* offsets, void* out, float* lse, const void* dout,
                           void* dqkv, void* workspace, size_t workspace_bytes, int tokens, int sequences, int heads, int kv_heads,
                           int width, float scale, void* stream);

/* The norm over all elements of `tensors` gradients, and the gradients scaled so that it is at most max_norm:
 *   norm[0] (device fp32) = sqrt(sum of squares), summed in 64 bits
 *   outs[i][0 .. counts[i]) = norm > max_norm ? grads[i] * (max_norm / norm) : grads[i]   (elem type; outs[i] may be grads[i])
 * grads, outs, counts: HOST arrays of device pointers and element counts (0: nothing there; up
 * to 2^40 in all), read during the call.  outs NULL: the norm alone.
 * A norm that is NaN leaves the gradients as they are; that of an infinite gradient scales by zero.  That of finite ones may be too large for norm[0],
 * which reads infinite then; they are scaled by what it is.
 * workspace: CDP_CLIP_BYTES, 8-byte aligned; nothing in it has to be cleared. */
#define CDP_CLIP_BYTES 65536u
int cdp_k_grad_clip(int dtype, int tensors, const void* const* grads, void* const* outs, const int64_t* counts, float max_norm,
                    float* norm, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CDP_KERNELS_H */
