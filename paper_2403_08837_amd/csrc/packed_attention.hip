// Causal attention over packed sequences of different lengths, with grouped heads.
//   S = scale q k^T, P = softmax(S) over the keys of the own sequence up to the query itself, out = P v, lse = log sum exp S;
//   backward: P = exp(S - lse), delta = rowsum(dout out), dP = dout v^T, dS = P (dP - delta), dq = scale dS k, dk = scale dS^T q, dv = P^T dout.
#include "elem.h"
#include "kernels.h"

namespace cdp {

namespace {

__device__ __forceinline__ float wave_sum(float v) {
  for (int n = 32; n > 0; n >>= 1) v += __shfl_xor(v, n, 64);
  return v;
}
struct Span { int begin, end; };
// The sequence that holds row t (none: an empty one): offsets that are not as they should be give rows within the tensor all the same.
__device__ __forceinline__ Span find_span(const PackedAttention& a, int t) {
  int lo = 0, hi = a.sequences;  // the first offset past t is at lo + 1 ..
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.offsets[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  if (lo == a.sequences || a.offsets[lo] > t) return Span{0, 0};
  return Span{max(a.offsets[lo], 0), min(a.offsets[lo + 1], a.tokens)};
}

// One wavefront per row and head; a lane holds columns lane and lane + 64.
template <typename T> struct Lanes {
  const PackedAttention& a;
  int lane;
  __device__ void load(const void* base, int64_t row, int ld, int col, float (&v)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = lane + 64 * i < a.width ? ld_f32<T>(static_cast<const T*>(base), row * ld + col + lane + 64 * i) : 0.f;
  }
  __device__ void store(void* base, int64_t row, int ld, int col, const float (&v)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (lane + 64 * i < a.width) st_f32<T>(static_cast<T*>(base), row * ld + col + lane + 64 * i, v[i]);
  }
};
__device__ __forceinline__ float dot(const float (&x)[2], const float (&y)[2]) { return wave_sum(x[0] * y[0] + x[1] * y[1]); }

template <typename T> __global__ __launch_bounds__(64) void packed_fwd_kernel(const PackedAttention a) {
  const int t = blockIdx.x, head = blockIdx.y, kv = head / (a.heads / a.kv_heads), W = a.width, ld = (a.heads + 2 * a.kv_heads) * W;
  const Span s = find_span(a, t);
  if (s.end <= s.begin) return;
  const Lanes<T> L{a, (int)threadIdx.x};
  float q[2], k[2], v[2], o[2] = {0.f, 0.f}, m = -INFINITY, z = 0.f;
  L.load(a.qkv, t, ld, head * W, q);
  for (int j = s.begin; j <= t; ++j) {
    L.load(a.qkv, j, ld, (a.heads + kv) * W, k);
    L.load(a.qkv, j, ld, (a.heads + a.kv_heads + kv) * W, v);
    const float x = a.scale * dot(q, k), mn = fmaxf(m, x), c = expf(m - mn), p = expf(x - mn);
    z = z * c + p;
    o[0] = o[0] * c + p * v[0];
    o[1] = o[1] * c + p * v[1];
    m = mn;
  }
  o[0] /= z;
  o[1] /= z;
  L.store(a.out, t, a.heads * W, head * W, o);
  if (threadIdx.x == 0) a.lse[(int64_t)head * a.tokens + t] = m + logf(z);
}

template <typename T> __global__ __launch_bounds__(64) void packed_bwd_q_kernel(const PackedAttention a) {
  const int t = blockIdx.x, head = blockIdx.y, kv = head / (a.heads / a.kv_heads), W = a.width, ld = (a.heads + 2 * a.kv_heads) * W;
  const Span s = find_span(a, t);
  if (s.end <= s.begin) return;
  const Lanes<T> L{a, (int)threadIdx.x};
  float q[2], k[2], v[2], o[2], g[2], dq[2] = {0.f, 0.f};
  L.load(a.qkv, t, ld, head * W, q);
  L.load(a.out, t, a.heads * W, head * W, o);
  L.load(a.dout, t, a.heads * W, head * W, g);
  const float delta = dot(o, g), lse = a.lse[(int64_t)head * a.tokens + t];
  if (threadIdx.x == 0) a.delta[(int64_t)head * a.tokens + t] = delta;
  for (int j = s.begin; j <= t; ++j) {
    L.load(a.qkv, j, ld, (a.heads + kv) * W, k);
    L.load(a.qkv, j, ld, (a.heads + a.kv_heads + kv) * W, v);
    const float ds = a.scale * expf(a.scale * dot(q, k) - lse) * (dot(g, v) - delta);
    dq[0] += ds * k[0];
    dq[1] += ds * k[1];
  }
  L.store(a.dqkv, t, ld, head * W, dq);
}
template <typename T> __global__ __launch_bounds__(64) void packed_bwd_kv_kernel(const PackedAttention a) {
  const int t = blockIdx.x, kv = blockIdx.y, group = a.heads / a.kv_heads, W = a.width, ld = (a.heads + 2 * a.kv_heads) * W;
  const Span s = find_span(a, t);
  if (s.end <= s.begin) return;
  const Lanes<T> L{a, (int)threadIdx.x};
  float q[2], k[2], v[2], g[2], dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
  L.load(a.qkv, t, ld, (a.heads + kv) * W, k);
  L.load(a.qkv, t, ld, (a.heads + a.kv_heads + kv) * W, v);
  for (int head = kv * group; head < (kv + 1) * group; ++head)
    for (int i = t; i < s.end; ++i) {
      L.load(a.qkv, i, ld, head * W, q);
      L.load(a.dout, i, a.heads * W, head * W, g);
      const int64_t at = (int64_t)head * a.tokens + i;
      const float p = expf(a.scale * dot(q, k) - a.lse[at]), ds = a.scale * p * (dot(g, v) - a.delta[at]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        dk[e] += ds * q[e];
        dv[e] += p * g[e];
      }
    }
  L.store(a.dqkv, t, ld, (a.heads + kv) * W, dk);
  L.store(a.dqkv, t, ld, (a.heads + a.kv_heads + kv) * W, dv);
}

}  // namespace

hipError_t launch_packed_attention_fwd(const PackedAttention& a, int dtype, hipStream_t stream) {
  if (dtype == DT_BF16) hipLaunchKernelGGL((packed_fwd_kernel<uint16_t>), dim3(a.tokens, a.heads), dim3(64), 0, stream, a);
  else hipLaunchKernelGGL((packed_fwd_kernel<float>), dim3(a.tokens, a.heads), dim3(64), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_packed_attention_bwd(const PackedAttention& a, int dtype, hipStream_t stream) {
  if (dtype == DT_BF16) hipLaunchKernelGGL((packed_bwd_q_kernel<uint16_t>), dim3(a.tokens, a.heads), dim3(64), 0, stream, a);
  else hipLaunchKernelGGL((packed_bwd_q_kernel<float>), dim3(a.tokens, a.heads), dim3(64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dtype == DT_BF16) hipLaunchKernelGGL((packed_bwd_kv_kernel<uint16_t>), dim3(a.tokens, a.kv_heads), dim3(64), 0, stream, a);
  else hipLaunchKernelGGL((packed_bwd_kv_kernel<float>), dim3(a.tokens, a.kv_heads), dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace cdp
