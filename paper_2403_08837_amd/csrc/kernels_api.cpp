// C ABI of the kernel-level entry points (include/cdp_kernels.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "../../include/cdp.h"
#include "../../include/cdp_kernels.h"
#include "kernels.h"

using namespace cdp;

// Both operands run along the output (a weight gradient): the weight-gradient tiles of the Linear launch read them as they lie and
// transpose on the way out of LDS, where the generic kernel scatters 2- or 4-byte elements into LDS.  Against the generic kernel's
// best tile over outputs of 64 x 64 to 4096 x 4096, 8 to 4096 rows: fp32 64 x 64 x 8 13 -> 7 us, bf16 4096 x 4096 x 64 52 -> 16 us,
// 4096^3 1124 -> 271 us.  Not so in fp32 for large results on the generic kernel's 128 x 128 tile, where what counts is how the result
// leaves: if rows of an operand are not whole 16-byte chunks (us, generic / these: 4001 x 3003 x 16 29 / 40, x 64 55 / 50, x 2000 830 / 945), and for
// up to one slab of 16 if rows of the result are not whole 128-byte lines (4672 x 2320 x 16 24 / 28, x 17 35 / 28, 4096 x 4096 x 8 40 / 30).  At
// 512 tiles of 64 x 128 these are 1.5 times as fast, at 1025 they are not.
bool cdp::gemm_wgrad_tiles_wanted(int tile_shape, int M, int N, int K, int lda, int ldb, int dtype) {
  if (dtype != DT_F32 || tile_shape != TILE_128x128) return true;
  if ((int64_t)((M + 63) / 64) * ((N + 127) / 128) < 768) return true;
  const bool whole = M % 4 == 0 && N % 4 == 0 && lda % 4 == 0 && ldb % 4 == 0;
  return whole && (K > 16 || N % 32 == 0);
}

static_assert((int64_t)CDP_CONV_SHARE_BYTES == CONV_SPLIT_WS_BYTES + CONV_SPLIT_SLOTS * 4, "partial tiles, then counters");

static bool aligned_to(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// What the head norms' two entry points check alike.
static bool head_rotary(HeadRotary& a, int dtype, const void* qkv, const int32_t* positions, const float* freqs, const float* gamma_q, const float* gamma_k,
                        float eps, int interleaved, int tokens, int heads, int kv_heads, int width, int rotary) {
  if (tokens <= 0 || heads <= 0 || kv_heads <= 0 || heads > 4096 || (int64_t)heads + 2ll * kv_heads > 4096 || width <= 0 || width % 8 || width > 128 || rotary < 0 ||
      rotary % 2 || rotary > width || !(eps > 0.f) || (dtype != DT_F32 && dtype != DT_BF16))
    return false;
  if ((rotary && (!positions || !freqs)) || (!rotary && !gamma_q && !gamma_k)) return false;
  if (!aligned_to(qkv, 16)) return false;
  for (const void* p : {(const void*)positions, (const void*)freqs, (const void*)gamma_q, (const void*)gamma_k})
    if (!aligned_to(p, 4)) return false;
  memset(&a, 0, sizeof(a));
  a.qkv = qkv; a.positions = positions; a.freqs = freqs; a.gamma_q = gamma_q; a.gamma_k = gamma_k; a.eps = eps; a.interleaved = interleaved != 0;
  a.tokens = tokens; a.heads = heads; a.kv_heads = kv_heads; a.width = width; a.rotary = rotary;
  return true;
}
static bool linear_sizes(int dtype, int act, int rows, int in, int hidden) {
  return rows > 0 && rows <= LINEAR_MAX_ROWS && in > 0 && hidden > 0 && in % 8 == 0 && hidden % 8 == 0 && in <= LINEAR_MAX_WIDTH && hidden <= LINEAR_MAX_WIDTH && act >= TOKEN_SILU &&
         act <= TOKEN_NONE && (dtype == DT_F32 || dtype == DT_BF16);
}
static bool logprob_sizes(int dtype, const void* logits, int64_t ld, const int32_t* targets, float scale, int rows, int vocab) {
  return (dtype == DT_F32 || dtype == DT_BF16) && logits && aligned_to(logits, dtype == DT_BF16 ? 2 : 4) && aligned_to(targets, 4) && rows > 0 && vocab > 0 &&
         vocab <= LOGPROB_MAX_VOCAB && ld >= vocab && ld <= (1ll << 31) && scale >= LOGPROB_MIN_SCALE && scale <= LOGPROB_MAX_SCALE;
}

extern "C" {

int cdp_k_gemm(int dtype, int tile_shape, int a_kmajor, int b_kmajor, const void* A, const void* B, float* C, int M, int N,
               int K, int lda, int ldb, void* stream) {
  // tile shapes: 0 .. 2 generic kernel, 3, 4 tick launch with 64 / 128 columns, 5 fastest, 6 tick launch as the engine makes it, 7 .. 9 generic
  // kernel in every layout
  constexpr int FASTEST = TILE_COUNT + 2, AS_ENGINE = TILE_COUNT + 3, GENERIC = TILE_COUNT + 4;
  if (!A || !B || !C || M <= 0 || N <= 0 || K <= 0 || tile_shape < 0 || tile_shape >= GENERIC + TILE_COUNT) return CDP_EINVAL;
  if (tile_shape >= TILE_COUNT && tile_shape < GENERIC && !(a_kmajor && b_kmajor)) return CDP_EINVAL;
  if (dtype != DT_F32 && dtype != DT_BF16) return CDP_EINVAL;
  GemmBatch b;
  memset(&b, 0, sizeof(b));
  b.n = 1;
  GemmProb& p = b.p[0];
  p.A = A; p.B = B; p.out = C;
  p.M = M; p.N = N; p.K = K; p.lda = lda; p.ldb = ldb; p.ldo = N;
  p.a_mode = a_kmajor ? OP_PLAIN_K : OP_PLAIN_R;
  p.b_mode = b_kmajor ? OP_PLAIN_K : OP_PLAIN_R;
  p.epi = EPI_FWD;
  p.flags = GF_OUT_F32;
  p.splits = 1;
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (tile_shape >= GENERIC) {
    e = launch_gemm_batch(b, dtype, tile_shape - GENERIC, st);
  } else if (!a_kmajor && !b_kmajor && gemm_wgrad_tiles_wanted(tile_shape, M, N, K, lda, ldb, dtype)) {
    p.epi = EPI_WGRAD;
    p.flags = 0;
    e = launch_linear_tick(b, dtype, false, false, st);
  } else if (tile_shape == FASTEST && gemm_stream_wanted(A, B, M, N, K, lda, ldb, dtype)) {
    e = launch_gemm_stream(A, B, C, M, N, K, lda, ldb, dtype, st);
  } else if (tile_shape >= TILE_COUNT) {
    e = launch_linear_tick(b, dtype, tile_shape == TILE_COUNT + 1, tile_shape == FASTEST || tile_shape == AS_ENGINE, st);
  } else {
    e = launch_gemm_batch(b, dtype, tile_shape, st);
  }
  return e == hipSuccess ? CDP_OK : CDP_EHIP;
}

int cdp_k_conv(int dtype, int which, const void* in0, const void* in1, void* out, int B, int H, int W, int Cin, int Cout,
               int ks, int stride, int pad, void* workspace, size_t workspace_bytes, void* stream) {
  if (!in0 || !in1 || !out || B <= 0 || H <= 0 || W <= 0 || Cin <= 0 || Cout <= 0 || ks <= 0 || stride <= 0 || pad < 0)
    return CDP_EINVAL;
  if (dtype != DT_F32 && dtype != DT_BF16) return CDP_EINVAL;
  if (H + 2 * pad < ks || W + 2 * pad < ks) return CDP_EINVAL;
  const int Ho = (H + 2 * pad - ks) / stride + 1, Wo = (W + 2 * pad - ks) / stride + 1;
  GemmBatch b;
  memset(&b, 0, sizeof(b));
  b.n = 1;
  GemmProb& p = b.p[0];
  p.splits = 1;
  p.A = in0; p.B = in1; p.out = out;
  ConvGeom& g = p.g;
  g.KH = ks; g.KW = ks; g.stride = stride; g.pad = pad;
  const bool force256 = which >= 3 && which <= 6;  // the direct-to-LDS tile regardless of the launch heuristic
  const int forced_tile = which >= 5 ? DL_256x128 : DL_256x256;
  const bool shared = which == 7 || which == 8, accumulate = which == 9, gelu = which == 10 || which == 11;
  if (force256) which -= which >= 5 ? 5 : 3;
  if (shared) which -= 7;
  if (accumulate) which = 2;
  if (gelu) which -= 10;
  if (which == 0) {
    p.M = B * Ho * Wo; p.N = Cout; p.K = ks * ks * Cin;
    p.a_mode = OP_CONV_FWD; p.b_mode = OP_PLAIN_K; p.ldb = p.K; p.ldo = Cout;
    g.H = H; g.W = W; g.C = Cin; g.OH = Ho; g.OW = Wo;
    p.epi = EPI_FWD;
  } else if (which == 1) {
    p.M = B * H * W; p.N = Cin; p.K = ks * ks * Cout;
    p.a_mode = OP_CONV_DGRAD; p.b_mode = OP_PLAIN_K; p.ldb = p.K; p.ldo = Cin;
    g.H = Ho; g.W = Wo; g.C = Cout; g.OH = H; g.OW = W;
    p.epi = EPI_DGRAD;
  } else if (which == 2) {
    p.M = Cout; p.N = ks * ks * Cin; p.K = B * Ho * Wo;
    p.a_mode = OP_PLAIN_R; p.lda = Cout; p.b_mode = OP_CONV_WGRAD; p.ldo = p.N;
    g.H = H; g.W = W; g.C = Cin; g.OH = Ho; g.OW = Wo;
    p.epi = EPI_WGRAD;
  } else {
    return CDP_EINVAL;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (shared && (!conv_fast_eligible(p, dtype) || !workspace || workspace_bytes < (size_t)CDP_CONV_SHARE_BYTES)) return CDP_EINVAL;
  if (gelu) {
    if (dtype != DT_BF16 || p.N <= 64 || !conv_fast_eligible(p, dtype) || !workspace || workspace_bytes / 2 < (size_t)p.M * p.N) return CDP_EINVAL;
    if (which == 0) p.aux2 = workspace;
    else p.aux1 = workspace;
    p.flags |= GF_GELU;
    if (!conv_gelu_valid(b, dtype)) return CDP_EINVAL;
  }
  // the fast implicit-GEMM paths where the shape allows, as in the engine; what is different for a call on its own: no workspace to share
  // reductions in (which = 7, 8 have one), ranges of the weight gradient for a launch of its own, and a fold that overwrites
  if (which == 2) {
    const size_t range_bytes = (size_t)p.M * p.N * 4;
    const int room = (int)std::min<size_t>(INT_MAX, workspace ? workspace_bytes / range_bytes : 0);
    if (conv_fast_eligible(p, dtype) && room >= 1) {
      const int splits = conv_wgrad_splits_alone(p, dtype, room);
      // two phases: partial sums per reduction range, then the fold
      WReduceBatch rb;
      memset(&rb, 0, sizeof(rb));
      rb.n = 1;
      rb.p[0].part = static_cast<const float*>(workspace);
      rb.p[0].G = static_cast<float*>(out);
      rb.p[0].Cout = p.M; rb.p[0].Ncol = p.N; rb.p[0].splits = splits;
      rb.p[0].overwrite = !accumulate;
      p.out = workspace;
      p.splits = splits;
      if (launch_conv_wgrad(b, dtype, p.M >= 128, st) != hipSuccess) return CDP_EHIP;
      return launch_wgrad_reduce(rb, dtype, st) == hipSuccess ? CDP_OK : CDP_EHIP;
    }
    if (accumulate) return CDP_EINVAL;
  } else if (force256) {
    if (!conv_gemm256_eligible(p, dtype)) return CDP_EINVAL;
    return launch_conv_dl(b, dtype, forced_tile, st) == hipSuccess ? CDP_OK : CDP_EHIP;
  } else if (conv_fast_eligible(p, dtype)) {
    if (shared) {
      b.thin_ws = static_cast<float*>(workspace);
      b.thin_cnt = reinterpret_cast<unsigned int*>(static_cast<char*>(workspace) + CONV_SPLIT_WS_BYTES);
    }
    if (conv_gemm256_wanted(&p, 1, dtype)) return launch_conv_dl(b, dtype, DL_256x256, st) == hipSuccess ? CDP_OK : CDP_EHIP;
    int bm, bn;
    conv_gemm_tile(&p, 1, &bm, &bn);
    return launch_conv_gemm(b, dtype, bm, bn, st) == hipSuccess ? CDP_OK : CDP_EHIP;
  }
  const int shape = p.M <= 64 ? (p.N >= 128 ? TILE_64x128 : TILE_64x64) : (p.N <= 64 ? TILE_64x64 : TILE_128x128);
  return launch_gemm_batch(b, dtype, shape, st) == hipSuccess ? CDP_OK : CDP_EHIP;
}

int cdp_k_layernorm(int dtype, int backward, const void* x, const void* dy, const void* add, const float* gamma,
                    const float* beta, void* out, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                    int rows, int C, void* stream) {
  if (!x || !gamma || !out || rows <= 0 || C <= 0 || C > 1024 || (dtype != DT_F32 && dtype != DT_BF16)) return CDP_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (!backward) {
    if (!beta) return CDP_EINVAL;
    return launch_layernorm_fwd(x, gamma, beta, out, rows, C, dtype, st) == hipSuccess ? CDP_OK : CDP_EHIP;
  }
  if (!dy || !dgamma || !dbeta || !workspace || (int64_t)workspace_bytes < layernorm_bwd_workspace_bytes(rows, C)) return CDP_EINVAL;
  return launch_layernorm_bwd(x, dy, add, gamma, out, dgamma, dbeta, static_cast<float*>(workspace), rows, C, dtype, st) == hipSuccess
             ? CDP_OK : CDP_EHIP;
}

int cdp_k_gelu(int dtype, int backward, const void* x, const void* dy, void* out, int64_t n, void* stream) {
  if (!x || !out || n <= 0 || (backward && !dy) || (dtype != DT_F32 && dtype != DT_BF16)) return CDP_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = backward ? launch_gelu_bwd(x, dy, out, n, dtype, st) : launch_gelu_fwd(x, out, n, dtype, st);
  return e == hipSuccess ? CDP_OK : CDP_EHIP;
}

int cdp_k_attention(int dtype, int backward, const void* qkv, void* P, const void* dout, void* out, void* workspace,
                    size_t workspace_bytes, int B, int T, int D, int heads, void* stream) {
  if (!qkv || !P || !out || !workspace || B <= 0 || T <= 0 || T > 1024 || D <= 0 || heads <= 0 || D % heads ||
      (dtype != DT_F32 && dtype != DT_BF16))
    return CDP_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t tt = (int64_t)B * heads * T * T;
  if (!backward) {
    if ((int64_t)workspace_bytes < 4 * tt) return CDP_EINVAL;
    return launch_attention_fwd(qkv, P, out, static_cast<float*>(workspace), B, T, D, heads, dtype, st) == hipSuccess ? CDP_OK : CDP_EHIP;
  }
  const int64_t dp_bytes = (4 * tt + 255) / 256 * 256;
  if (!dout || (int64_t)workspace_bytes < dp_bytes + tt * (dtype == DT_BF16 ? 2 : 4)) return CDP_EINVAL;
  return launch_attention_bwd(qkv, P, dout, out, static_cast<float*>(workspace), static_cast<char*>(workspace) + dp_bytes, B, T, D,
                              heads, dtype, st) == hipSuccess ? CDP_OK : CDP_EHIP;
}

static int launched(hipError_t e) { return e == hipSuccess ? CDP_OK : e == hipErrorInvalidConfiguration ? CDP_EINVAL : CDP_EHIP; }

int cdp_k_embedding(int dtype, int backward, const void* table, const int32_t* ids, const void* dout, void* out, float scale,
                    void* workspace, size_t workspace_bytes, int rows, int vocab, int C, void* stream) {
  if (!ids || !out || rows <= 0 || vocab <= 0 || C <= 0 || C > (1 << 24) || !std::isfinite(scale) || backward < 0 || backward > 2 || (dtype != DT_F32 && dtype != DT_BF16)) return CDP_EINVAL;
  const int eb = dtype == DT_BF16 ? 2 : 4;
  if (!aligned_to(ids, 4) || !aligned_to(out, backward ? 4 : eb)) return CDP_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (!backward) {
    if (!table || !aligned_to(table, eb)) return CDP_EINVAL;
    return launched(launch_embedding_fwd(table, ids, out, scale, rows, vocab, C, dtype, st));
  }
  if (!dout || !aligned_to(dout, eb) || !workspace || !aligned_to(workspace, 16) ||
      workspace_bytes < (size_t)embedding_bwd_workspace_bytes(rows, C))
    return CDP_EINVAL;
  return launched(launch_embedding_bwd(ids, dout, static_cast<float*>(out), scale, workspace, backward == 2, rows, vocab, C, dtype, st));
}

int cdp_k_residual_norm(int dtype, const void* x, const void* h, const void* gate, const float* gamma_post, const float* gamma_pre,
                        void* r, void* y, float scale, float eps, int rows, int C, void* stream) {
  if (!x || (!r && !y) || rows <= 0 || C <= 0 || C > RNORM_MAX_C || !(eps > 0.f) || !std::isfinite(scale) || (dtype != DT_F32 && dtype != DT_BF16)) return CDP_EINVAL;
  if (!y != !gamma_pre || (!h && (gate || gamma_post))) return CDP_EINVAL;
  const int eb = dtype == DT_BF16 ? 2 : 4;
  if (!aligned_to(x, eb) || !aligned_to(h, eb) || !aligned_to(gate, eb) || !aligned_to(r, eb) || !aligned_to(y, eb) ||
      !aligned_to(gamma_post, 4) || !aligned_to(gamma_pre, 4))
    return CDP_EINVAL;
  ResidualNorm a;
  memset(&a, 0, sizeof(a));
  a.x = x; a.h = h; a.gate = gate; a.gamma_post = gamma_post; a.gamma_pre = gamma_pre;
  a.r = r; a.y = y; a.rows = rows; a.C = C; a.scale = scale; a.eps = eps;
  return launched(launch_residual_norm_fwd(a, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_residual_norm_backward(int dtype, int accumulate, const void* x, const void* h, const void* gate, const float* gamma_post,
                                 const float* gamma_pre, const void* dr, const void* dy, void* dx, void* dh, void* dgate,
                                 float* dgamma_post, float* dgamma_pre, float scale, float eps, void* workspace, size_t workspace_bytes,
                                 int rows, int C, void* stream) {
  if (!dx || (!dr && !dy) || rows <= 0 || C <= 0 || C > RNORM_MAX_C || !(eps > 0.f) || !std::isfinite(scale) || (dtype != DT_F32 && dtype != DT_BF16)) return CDP_EINVAL;
  if (!dy != !gamma_pre || !dgamma_pre != !gamma_pre || !x != !gamma_pre) return CDP_EINVAL;
  if (!h != !dh || !gate != !dgate || !gamma_post != !dgamma_post || (!h && (gate || gamma_post))) return CDP_EINVAL;
  const int eb = dtype == DT_BF16 ? 2 : 4;
  for (const void* p : {x, h, gate, dr, dy, (const void*)dx, (const void*)dh, (const void*)dgate})
    if (!aligned_to(p, eb)) return CDP_EINVAL;
  for (const float* p : {gamma_post, gamma_pre, (const float*)dgamma_post, (const float*)dgamma_pre})
    if (!aligned_to(p, 4)) return CDP_EINVAL;
  if ((gamma_post || gamma_pre) &&
      (!workspace || !aligned_to(workspace, 16) || workspace_bytes < (size_t)residual_norm_bwd_workspace_bytes(rows, C)))
    return CDP_EINVAL;
  ResidualNorm a;
  memset(&a, 0, sizeof(a));
  a.x = x; a.h = h; a.gate = gate; a.gamma_post = gamma_post; a.gamma_pre = gamma_pre;
  a.dr = dr; a.dy = dy; a.dx = dx; a.dh = dh; a.dgate = dgate; a.dgamma_post = dgamma_post; a.dgamma_pre = dgamma_pre;
  a.part = static_cast<float*>(workspace);
  a.rows = rows; a.C = C; a.accumulate = accumulate != 0; a.scale = scale; a.eps = eps;
  return launched(launch_residual_norm_bwd(a, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_attention_packed(int dtype, int backward, const void* qkv, const int32_t* offsets, void* out, float* lse, const void* dout,
                           void* dqkv, void* workspace, size_t workspace_bytes, int tokens, int sequences, int heads, int kv_heads,
                           int width, float scale, void* stream) {
  if (!qkv || !offsets || !out || !lse || tokens <= 0 || sequences <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || width <= 0 ||
      width % 8 || width > 128 || !std::isfinite(scale) || (dtype != DT_F32 && dtype != DT_BF16))
    return CDP_EINVAL;
  // a tile of rows within 32-bit offsets of its first; tiles of 32 rows at least, and one more for every sequence, within what a launch can number
  if (heads > 4096 || (int64_t)heads + 2ll * kv_heads > 4096 || ((int64_t)tokens / 32 + sequences + 1) * heads > INT_MAX / 2) return CDP_EINVAL;
  if (!aligned_to(qkv, 16) || !aligned_to(out, 16) || !aligned_to(lse, 4) || !aligned_to(offsets, 4)) return CDP_EINVAL;
  PackedAttention a;
  memset(&a, 0, sizeof(a));
  a.qkv = qkv; a.offsets = offsets; a.out = out; a.lse = lse;
  a.tokens = tokens; a.sequences = sequences; a.heads = heads; a.kv_heads = kv_heads; a.width = width; a.scale = scale;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (!backward) return launched(launch_packed_attention_fwd(a, dtype, st));
  const size_t rows = (size_t)heads * tokens, need = 4 * rows + 512;
  if (!dout || !dqkv || !aligned_to(dout, 16) || !aligned_to(dqkv, 16) || !workspace || !aligned_to(workspace, 16) || workspace_bytes < need)
    return CDP_EINVAL;
  a.dout = dout; a.dqkv = dqkv;
  a.delta = static_cast<float*>(workspace);
  a.parts = a.delta + (rows + 63) / 64 * 64;
  a.max_parts = (int64_t)((workspace_bytes - need) / (8 * (size_t)kv_heads * tokens * width));
  return launched(launch_packed_attention_bwd(a, dtype, st));
}

int cdp_k_grad_clip(int dtype, int tensors, const void* const* grads, void* const* outs, const int64_t* counts, float max_norm,
                    float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (tensors <= 0 || !grads || !counts || !norm || !(max_norm >= 0.f) || (dtype != DT_F32 && dtype != DT_BF16)) return CDP_EINVAL;
  if (!workspace || workspace_bytes < CDP_CLIP_BYTES || !aligned_to(workspace, 8) || !aligned_to(norm, 4)) return CDP_EINVAL;
  const int eb = dtype == DT_BF16 ? 2 : 4;
  int64_t total = 0;
  for (int i = 0; i < tensors; ++i) {
    if (counts[i] < 0 || counts[i] > (1ll << 40) - total) return CDP_EINVAL;
    total += counts[i];
    if (counts[i] && (!grads[i] || !aligned_to(grads[i], eb) || (outs && (!outs[i] || !aligned_to(outs[i], eb))))) return CDP_EINVAL;
  }
  return launched(launch_grad_clip(tensors, grads, outs, counts, max_norm, norm, workspace, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_head_norm_rotary(int dtype, const void* qkv, const int32_t* positions, const float* freqs, const float* gamma_q, const float* gamma_k, void* out,
                           float eps, int interleaved, int tokens, int heads, int kv_heads, int width, int rotary, void* stream) {
  if (!out) return CDP_EINVAL;
  HeadRotary a;
  if (!head_rotary(a, dtype, qkv, positions, freqs, gamma_q, gamma_k, eps, interleaved, tokens, heads, kv_heads, width, rotary) || !qkv || !aligned_to(out, 16))
    return CDP_EINVAL;
  a.out = out;
  a.in_place = out == qkv;
  return launched(launch_head_rotary(a, false, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_head_norm_rotary_backward(int dtype, int accumulate, const void* qkv, const int32_t* positions, const float* freqs, const float* gamma_q,
                                    const float* gamma_k, const void* dout, void* dqkv, float* dgamma_q, float* dgamma_k, float eps, int interleaved,
                                    void* workspace, size_t workspace_bytes, int tokens, int heads, int kv_heads, int width, int rotary, void* stream) {
  HeadRotary a;
  if (!head_rotary(a, dtype, qkv, positions, freqs, gamma_q, gamma_k, eps, interleaved, tokens, heads, kv_heads, width, rotary)) return CDP_EINVAL;
  if (!dout || !dqkv || !aligned_to(dout, 16) || !aligned_to(dqkv, 16) || !gamma_q != !dgamma_q || !gamma_k != !dgamma_k || !aligned_to(dgamma_q, 4) ||
      !aligned_to(dgamma_k, 4))
    return CDP_EINVAL;
  if ((gamma_q || gamma_k) && (!qkv || !workspace || !aligned_to(workspace, 16) || workspace_bytes < (size_t)head_rotary_bwd_workspace_bytes(tokens, width)))
    return CDP_EINVAL;
  a.dout = dout; a.dqkv = dqkv; a.dgamma_q = dgamma_q; a.dgamma_k = dgamma_k;
  a.part = static_cast<float*>(workspace);
  a.accumulate = accumulate != 0;
  a.in_place = dout == dqkv;
  return launched(launch_head_rotary(a, true, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_gated_linear(int dtype, int act, const void* x, const void* wg, const void* wu, void* h, void* g, void* u, void* workspace, size_t workspace_bytes,
                       int rows, int in, int hidden, void* stream) {
  if (!linear_sizes(dtype, act, rows, in, hidden) || !x || !wg || !wu || !h || !g != !u) return CDP_EINVAL;
  for (const void* p : {x, wg, wu, (const void*)h, (const void*)g, (const void*)u, (const void*)workspace})
    if (!aligned_to(p, 16)) return CDP_EINVAL;
  GatedLinear a;
  memset(&a, 0, sizeof(a));
  a.x = x; a.wg = wg; a.wu = wu; a.h = h; a.g = g; a.u = u;
  a.workspace = workspace; a.workspace_bytes = workspace ? (int64_t)std::min<size_t>(workspace_bytes, INT64_MAX / 2) : 0;
  a.rows = rows; a.in = in; a.hidden = hidden; a.act = act;
  return launched(launch_gated_linear(a, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_gated_linear_backward(int dtype, int act, const void* x, const void* wg, const void* wu, const void* g, const void* u, const void* dh, void* dx,
                                void* dwg, void* dwu, void* workspace, size_t workspace_bytes, int rows, int in, int hidden, void* stream) {
  if (!linear_sizes(dtype, act, rows, in, hidden) || !x || !wg || !wu || !g || !u || !dh || !dwg != !dwu || (!dx && !dwg)) return CDP_EINVAL;
  for (const void* p : {x, wg, wu, g, u, dh, (const void*)dx, (const void*)dwg, (const void*)dwu, (const void*)workspace})
    if (!aligned_to(p, 16)) return CDP_EINVAL;
  if (!workspace || workspace_bytes < (size_t)gated_linear_bwd_workspace_bytes(rows, hidden, dtype)) return CDP_EINVAL;
  GatedLinear a;
  memset(&a, 0, sizeof(a));
  a.x = x; a.wg = wg; a.wu = wu; a.g = const_cast<void*>(g); a.u = const_cast<void*>(u); a.dh = dh; a.dx = dx; a.dwg = dwg; a.dwu = dwu;
  a.workspace = workspace; a.workspace_bytes = (int64_t)std::min<size_t>(workspace_bytes, INT64_MAX / 2);
  a.rows = rows; a.in = in; a.hidden = hidden; a.act = act;
  return launched(launch_gated_linear_bwd(a, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_linear(int dtype, int act, const void* x, const void* w, const void* bias, const void* residual, void* y, void* z, void* workspace,
                 size_t workspace_bytes, int rows, int in, int out, void* stream) {
  if (!linear_sizes(dtype, act, rows, in, out) || !x || !w || !y) return CDP_EINVAL;
  for (const void* p : {x, w, bias, residual, (const void*)y, (const void*)z, (const void*)workspace})
    if (!aligned_to(p, 16)) return CDP_EINVAL;
  TokenLinear a;
  memset(&a, 0, sizeof(a));
  a.x = x; a.w = w; a.bias = bias; a.residual = residual; a.y = y; a.z = z;
  a.workspace = workspace; a.workspace_bytes = workspace ? (int64_t)std::min<size_t>(workspace_bytes, INT64_MAX / 2) : 0;
  a.rows = rows; a.in = in; a.out = out; a.act = act;
  return launched(launch_token_linear(a, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_linear_backward(int dtype, int act, const void* x, const void* w, const void* z, const void* dy, void* dx, void* dw, void* dbias, void* workspace,
                          size_t workspace_bytes, int rows, int in, int out, void* stream) {
  if (!linear_sizes(dtype, act, rows, in, out) || !dy || (!z && act != TOKEN_NONE) || (!dx && !dw && !dbias)) return CDP_EINVAL;
  if ((dx && !w) || (dw && !x)) return CDP_EINVAL;
  for (const void* p : {x, w, z, dy, (const void*)dx, (const void*)dw, (const void*)dbias, (const void*)workspace})
    if (!aligned_to(p, 16)) return CDP_EINVAL;
  if (!workspace || workspace_bytes < (size_t)token_linear_bwd_workspace_bytes(rows, out, dtype)) return CDP_EINVAL;
  TokenLinear a;
  memset(&a, 0, sizeof(a));
  a.x = x; a.w = w; a.z = const_cast<void*>(z); a.dy = dy; a.dx = dx; a.dw = dw; a.dbias = dbias;
  a.workspace = workspace; a.workspace_bytes = (int64_t)std::min<size_t>(workspace_bytes, INT64_MAX / 2);
  a.rows = rows; a.in = in; a.out = out; a.act = act;
  return launched(launch_token_linear_bwd(a, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_token_logprob(int dtype, const void* logits, int64_t ld, const int32_t* targets, float scale, float* logprob, float* entropy, float* lse,
                        int32_t* top_ids, float* top_logprobs, int top, void* workspace, size_t workspace_bytes, int rows, int vocab, void* stream) {
  if (!logprob_sizes(dtype, logits, ld, targets, scale, rows, vocab) || !lse || (logprob && !targets)) return CDP_EINVAL;
  if (top < 0 || top > LOGPROB_MAX_TOP || top > vocab || (top && (!top_ids || !top_logprobs))) return CDP_EINVAL;
  for (const void* p : {(const void*)logprob, (const void*)entropy, (const void*)lse, (const void*)top_ids, (const void*)top_logprobs})
    if (!aligned_to(p, 4)) return CDP_EINVAL;
  if (workspace && (!aligned_to(workspace, 16) || workspace_bytes < CDP_LOGPROB_BYTES)) return CDP_EINVAL;
  static_assert(CDP_LOGPROB_BYTES == LOGPROB_BYTES, "");
  TokenLogprob a;
  memset(&a, 0, sizeof(a));
  a.logits = logits; a.ld = ld; a.targets = targets; a.logprob = logprob; a.entropy = entropy; a.lse = lse;
  a.top_ids = top_ids; a.top_logprobs = top_logprobs;
  a.rows = rows; a.vocab = vocab; a.top = top; a.scale = scale;
  return launched(launch_token_logprob(a, workspace, dtype, static_cast<hipStream_t>(stream)));
}

int cdp_k_token_logprob_backward(int dtype, const void* logits, int64_t ld, const int32_t* targets, float scale, const float* lse, const float* entropy,
                                 const float* dlogprob, const float* dentropy, void* dlogits, int rows, int vocab, void* stream) {
  if (!logprob_sizes(dtype, logits, ld, targets, scale, rows, vocab) || !lse || !dlogits || !aligned_to(dlogits, dtype == DT_BF16 ? 2 : 4)) return CDP_EINVAL;
  if ((dlogprob && !targets) || (dentropy && !entropy) || (!dlogprob && !dentropy)) return CDP_EINVAL;
  for (const float* p : {lse, entropy, dlogprob, dentropy})
    if (!aligned_to(p, 4)) return CDP_EINVAL;
  TokenLogprob a;
  memset(&a, 0, sizeof(a));
  a.logits = logits; a.ld = ld; a.targets = targets; a.lse = const_cast<float*>(lse); a.entropy = const_cast<float*>(entropy);
  a.dlogprob = dlogprob; a.dentropy = dentropy; a.dlogits = dlogits;
  a.rows = rows; a.vocab = vocab; a.scale = scale;
  return launched(launch_token_logprob_bwd(a, dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
