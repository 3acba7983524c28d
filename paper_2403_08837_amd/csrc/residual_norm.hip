// Norm after a block, its gate and residual scale, and the norm before the next block (root mean square norms), with their gradients:
//   n = h eta, eta = 1 / sqrt(mean h^2 + eps);  u = n gamma_post (or h);  r = x + scale sigmoid(gate) u;  y = r rho gamma_pre, rho likewise of r.
// Backward, with rhat = r rho and a = dy gamma_pre:  d = dr + rho (a - rhat mean(a rhat)) is dx;  du = scale sig d;  dgate = scale u d sig (1 - sig);
//   b = du gamma_post, dh = eta (b - n mean(b n)) (or du);  dgamma_post = sum du n;  dgamma_pre = sum dy rhat.
#include "elem.h"
#include "kernels.h"

#include <algorithm>

namespace cdp {

namespace {

// Sum over the 256 threads, in every one of them.
__device__ __forceinline__ float group_sum(float v, float* lds) {
  lds[threadIdx.x] = v;
  __syncthreads();
  for (int n = 128; n > 0; n >>= 1) {
    if ((int)threadIdx.x < n) lds[threadIdx.x] += lds[threadIdx.x + n];
    __syncthreads();
  }
  v = lds[0];
  __syncthreads();
  return v;
}
__device__ __forceinline__ float sigmoid(float g) { return 1.f / (1.f + expf(-g)); }

template <typename T> struct Row {
  const ResidualNorm& a;
  int64_t at;
  float eta;
  __device__ float u(int c) const {
    const float h = ld_f32<T>(static_cast<const T*>(a.h), at + c);
    return a.gamma_post ? h * eta * a.gamma_post[c] : h;
  }
  __device__ float sig(int c) const { return a.gate ? sigmoid(ld_f32<T>(static_cast<const T*>(a.gate), at + c)) : 1.f; }
};

template <typename T> __global__ __launch_bounds__(256) void residual_norm_fwd_kernel(const ResidualNorm a) {
  __shared__ float lds[256];
  Row<T> row{a, (int64_t)blockIdx.x * a.C, 1.f};
  const T* x = static_cast<const T*>(a.x) + row.at;
  if (a.gamma_post) {
    float s = 0.f;
    for (int c = threadIdx.x; c < a.C; c += 256) { const float h = ld_f32<T>(static_cast<const T*>(a.h), row.at + c); s += h * h; }
    row.eta = rsqrtf(group_sum(s, lds) / a.C + a.eps);
  }
  float s = 0.f;
  constexpr int MAX = RNORM_MAX_C / 256;
  float r[MAX];
#pragma unroll
  for (int i = 0; i < MAX; ++i) {
    const int c = threadIdx.x + 256 * i;
    if (c >= a.C) break;
    r[i] = ld_f32<T>(x, c) + (a.h ? a.scale * row.sig(c) * row.u(c) : 0.f);
    s += r[i] * r[i];
  }
  const float rho = rsqrtf(group_sum(s, lds) / a.C + a.eps);
#pragma unroll
  for (int i = 0; i < MAX; ++i) {
    const int c = threadIdx.x + 256 * i;
    if (c >= a.C) break;
    if (a.r) st_f32<T>(static_cast<T*>(a.r), row.at + c, r[i]);
    if (a.y) st_f32<T>(static_cast<T*>(a.y), row.at + c, r[i] * rho * a.gamma_pre[c]);
  }
}

// Workgroup b takes the rows b, b + gridDim.x, ..; its column sums are part[0][b][C] (post) and part[1][b][C] (pre).
template <typename T> __global__ __launch_bounds__(256) void residual_norm_bwd_kernel(const ResidualNorm a) {
  __shared__ float lds[256];
  float* post = a.part + (int64_t)blockIdx.x * a.C;
  float* pre = post + (int64_t)gridDim.x * a.C;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    Row<T> row{a, i * a.C, 1.f};
    auto ld = [&](const void* p, int c) { return p ? ld_f32<T>(static_cast<const T*>(p), row.at + c) : 0.f; };
    float rho = 0.f, mean = 0.f;
    if (a.gamma_pre) {
      float s = 0.f, t = 0.f;
      for (int c = threadIdx.x; c < a.C; c += 256) {
        const float r = ld(a.rin, c);
        s += r * r;
        t += r * ld(a.dy, c) * a.gamma_pre[c];
      }
      rho = rsqrtf(group_sum(s, lds) / a.C + a.eps);
      mean = group_sum(t, lds) * rho / a.C;
    }
    auto d = [&](int c) {
      float v = ld(a.dr, c);
      if (a.gamma_pre) v += rho * (ld(a.dy, c) * a.gamma_pre[c] - ld(a.rin, c) * rho * mean);
      return v;
    };
    float dot = 0.f;
    if (a.gamma_post) {
      float s = 0.f, t = 0.f;
      for (int c = threadIdx.x; c < a.C; c += 256) {
        const float h = ld(a.h, c);
        s += h * h;
        t += h * a.scale * row.sig(c) * d(c) * a.gamma_post[c];
      }
      row.eta = rsqrtf(group_sum(s, lds) / a.C + a.eps);
      dot = group_sum(t, lds) * row.eta / a.C;
    }
    const bool first = i == blockIdx.x;
    for (int c = threadIdx.x; c < a.C; c += 256) {
      const float dc = d(c);
      if (a.h) {
        const float sig = row.sig(c), du = a.scale * sig * dc, h = ld(a.h, c);
        if (a.gate) st_f32<T>(static_cast<T*>(a.dgate), row.at + c, du * row.u(c) * (1.f - sig));
        st_f32<T>(static_cast<T*>(a.dh), row.at + c, a.gamma_post ? row.eta * (du * a.gamma_post[c] - h * row.eta * dot) : du);
        if (a.gamma_post) post[c] = (first ? 0.f : post[c]) + du * h * row.eta;
      }
      if (a.gamma_pre) pre[c] = (first ? 0.f : pre[c]) + ld(a.dy, c) * ld(a.rin, c) * rho;
      st_f32<T>(static_cast<T*>(a.dx), row.at + c, dc);
    }
    __syncthreads();
  }
}
__global__ __launch_bounds__(256) void residual_norm_fold_kernel(const ResidualNorm a, int parts) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.C) return;
  for (int k = 0; k < 2; ++k) {
    float* g = k ? a.dgamma_pre : a.dgamma_post;
    if (!g) continue;
    float s = a.accumulate ? g[c] : 0.f;
    for (int p = 0; p < parts; ++p) s += a.part[((int64_t)k * parts + p) * a.C + c];
    g[c] = s;
  }
}

}  // namespace

int64_t residual_norm_bwd_workspace_bytes(int rows, int C) { return 8ll * C * std::min(rows, RNORM_MAX_PARTS) + 256; }

hipError_t launch_residual_norm_fwd(const ResidualNorm& a, int dtype, hipStream_t stream) {
  if (dtype == DT_BF16) hipLaunchKernelGGL((residual_norm_fwd_kernel<uint16_t>), dim3(a.rows), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((residual_norm_fwd_kernel<float>), dim3(a.rows), dim3(256), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_residual_norm_bwd(const ResidualNorm& a, int dtype, hipStream_t stream) {
  const int parts = std::min(a.rows, RNORM_MAX_PARTS);
  if (dtype == DT_BF16) hipLaunchKernelGGL((residual_norm_bwd_kernel<uint16_t>), dim3(parts), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((residual_norm_bwd_kernel<float>), dim3(parts), dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !(a.dgamma_post || a.dgamma_pre)) return e;
  hipLaunchKernelGGL(residual_norm_fold_kernel, dim3((a.C + 255) / 256), dim3(256), 0, stream, a, parts);
  return hipGetLastError();
}

}  // namespace cdp
