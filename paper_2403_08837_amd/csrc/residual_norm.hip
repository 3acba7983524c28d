// Norm after a block, its gate and residual scale, and the norm before the next block (root mean square norms), with their gradients:
//   n = h eta, eta = 1 / sqrt(mean h^2 + eps);  u = n gamma_post (or h);  r = x + scale sig u, sig = sigmoid(gate);  y = r rho gamma_pre, rho likewise of r.
// Backward, with rhat = r rho and a = dy gamma_pre:  d = dr + rho (a - rhat mean(a rhat)) is dx;  du = scale sig d;  dgate = du u (1 - sig);
//   b = du gamma_post, dh = eta (b - n mean(b n)) (or du);  dgamma_post = sum du n;  dgamma_pre = sum dy rhat.
//
// Bound by memory: five tensors forward, eight backward, each once.  A row stays in the registers of the lanes that share it (8 to 1024 of them, eight values
// in each, sixteen past 8192 channels), read in one round of buffer loads: a tensor that is not there is a buffer of no bytes, which reads zeros and drops stores,
// so that one kernel without branches serves every form.  Forward a row needs two sums, one after the other (eta, then rho of what it makes).  So does backward:
// r is made again from x, in fp32 as the forward had it (from the rounded r the gradient of gamma_pre would be off by half a step of bf16), and
// mean(b n) falls into sums that do not wait for rho,
//   sum b h = sum sg dr h + rho sum sg a h - rho^2 mean(a rhat) sum sg r h,   sg = scale sig gamma_post.
// us and TB/s, bf16, all tensors: 16384 x 4096 forward 124 and 5.4, backward 223 and 4.8; 6272 x 768 9.4 and 5.1, 26.4 and 2.9 (the fold is 4.4 of it); fp32
// 8192 x 4096 118 and 5.7, 219 and 4.9.  Past 8192 channels a lane's 16 values of five tensors are more than the 128 registers of a workgroup of 1024:
// backward 28 to 61 of them are spilled, 4096 x 12288 119 and 4.2, 356 and 2.3, fp32 2048 x 16384 119 and 5.6, 308 and 3.5.
// Column sums stay in registers over a workgroup's rows; what the workgroups have is added up by residual_norm_fold_kernel in a fixed order.
#include "elem.h"
#include "kernels.h"

#include <algorithm>

namespace cdp {

namespace {

// Sum over groups of L neighbouring lanes, in every one of them, without LDS.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
  v += dpp<0xB1>(v);                           // neighbours
  if constexpr (L >= 4) v += dpp<0x4E>(v);     // pairs
  if constexpr (L >= 8) v += dpp<0x141>(v);    // the other four of eight (mirrored)
  if constexpr (L >= 16) v += dpp<0x140>(v);
  if constexpr (L >= 32) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  if constexpr (L >= 64) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  return v;
}
// Sum over the lanes that are a multiple of L apart, in every one of them.
template <int L> __device__ __forceinline__ float groups_sum(float v) {
  if constexpr (L <= 8) v += dpp<0x128>(v);  // (eight on, around sixteen)
  if constexpr (L <= 16) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  if constexpr (L <= 32) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  return v;
}
// Sums over the LR lanes of a row, n of them at once; rows of more than a wavefront through LDS (`lds`: not in use by the sums before).
template <int LR, int NS> __device__ __forceinline__ void row_sums(float (&v)[NS], float* lds) {
#pragma unroll
  for (int i = 0; i < NS; ++i) v[i] = lanes_sum<LR < 64 ? LR : 64>(v[i]);
  if constexpr (LR > 64) {
    constexpr int W = LR / 64;
    const int wave = threadIdx.x >> 6, first = wave / W * W;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < NS; ++i) lds[wave * NS + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      v[i] = lanes_sum<W>(lds[(first + threadIdx.x % W) * NS + i]);  // (every lane its wavefront's share, then as above)
    }
  }
}
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }

// K groups of V neighbouring values of a row per lane (V = 1: rows that are not whole 16-byte pieces).
template <typename T, int V, int K, int LR> struct Lay {
  static constexpr int N = V * K, THREADS = LR > 256 ? LR : 256, SLOTS = THREADS / LR;  // values of a lane; rows that a workgroup has at once
  static constexpr bool HEAVY = N > 8;                            // 128 registers a lane do not hold the channel vectors and the column sums too
  static constexpr bool AHEAD = sizeof(T) == 2 && V > 1 && LR <= 512;  // registers for the next row's values
  typedef typename std::conditional<V == 1, T, uint4>::type Group;
};
template <typename Group> __device__ __forceinline__ Group buffer_load(__amdgpu_buffer_rsrc_t b, unsigned off) {
  if constexpr (sizeof(Group) == 16) return __builtin_bit_cast(Group, __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0));
  else if constexpr (sizeof(Group) == 4) return __builtin_bit_cast(Group, __builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0));
  else return __builtin_bit_cast(Group, __builtin_amdgcn_raw_buffer_load_b16(b, off, 0, 0));
}
template <typename Group> __device__ __forceinline__ void buffer_store(__amdgpu_buffer_rsrc_t b, unsigned off, Group g) {
  if constexpr (sizeof(Group) == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(__attribute__((ext_vector_type(4))) unsigned, g), b, off, 0, 0);
  else if constexpr (sizeof(Group) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, g), b, off, 0, 0);
  else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, g), b, off, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p) + (p ? bytes : 0)), 0, p ? 0xfffffff0u : 0u, 0x00020000);
}
template <typename T, typename Group, int K> struct Values {
  static constexpr int V = sizeof(Group) / sizeof(T);
  Group g[K];
  __device__ __forceinline__ void load(const void* p, int64_t bytes, const unsigned (&off)[K]) {
    const __amdgpu_buffer_rsrc_t b = buffer_at(p, bytes);
#pragma unroll
    for (int k = 0; k < K; ++k) g[k] = buffer_load<Group>(b, off[k]);
  }
  __device__ __forceinline__ float operator[](int i) const {
    union { Group g; T e[V]; } c;
    c.g = g[i / V];
    return Elem<T>::to_f32(c.e[i % V]);
  }
};
template <typename T, typename Group, int K, int N>
__device__ __forceinline__ void store_row(void* p, int64_t bytes, const unsigned (&off)[K], const float (&v)[N]) {
  constexpr int V = N / K;
  const __amdgpu_buffer_rsrc_t b = buffer_at(p, bytes);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    union { Group g; T e[V]; } c;
#pragma unroll
    for (int e = 0; e < V; ++e) c.e[e] = Elem<T>::from_f32(v[V * k + e]);
    buffer_store<Group>(b, off[k], c.g);
  }
}
// Channel vectors (fp32, aligned to 4 bytes): `none` where there is none.
template <int V, int K> __device__ __forceinline__ void load_gamma(float (&v)[V * K], const float* p, const int (&col)[K], int C, float none) {
  const __amdgpu_buffer_rsrc_t b = buffer_at(p, 0);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const unsigned off = col[k] < C ? 4u * col[k] : ~0u;
#pragma unroll
    for (int e = 0; e < V; e += V == 1 ? 1 : 4) {
      if constexpr (V == 1) v[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0));
      else {
        const auto x = __builtin_amdgcn_raw_buffer_load_b128(b, off == ~0u ? off : off + 4 * e, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[V * k + e + i] = __uint_as_float(x[i]);
      }
    }
  }
  if (!p)
#pragma unroll
    for (int i = 0; i < V * K; ++i) v[i] = none;
}

template <typename T, int V, int K, int LR>
__global__ __launch_bounds__(LR > 256 ? LR : 256) void residual_norm_fwd_kernel(const ResidualNorm a) {
  using Ly = Lay<T, V, K, LR>;
  using Vals = Values<T, typename Ly::Group, K>;
  constexpr int N = Ly::N;
  __shared__ float lds[2][Ly::THREADS / 64];
  const int slot = threadIdx.x / LR, idx = threadIdx.x % LR;
  const int64_t row0 = (int64_t)blockIdx.x * Ly::SLOTS, at = row0 * a.C * (int)sizeof(T);
  unsigned off[K];
  int col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    col[k] = (k * LR + idx) * V;
    off[k] = col[k] < a.C && row0 + slot < a.rows ? (unsigned)(slot * a.C + col[k]) * (unsigned)sizeof(T) : ~0u;
  }
  Vals x, h, g;
  x.load(a.x, at, off);
  h.load(a.h, at, off);
  g.load(a.gate, at, off);
  float post[N], pre[N], r[N];
  load_gamma<V, K>(post, a.gamma_post, col, a.C, 1.f);
  load_gamma<V, K>(pre, a.gamma_pre, col, a.C, 0.f);
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < N; ++i) s[0] += h[i] * h[i];
  row_sums<LR>(s, lds[0]);
  const float inv = 1.f / a.C, f = a.scale * (a.gamma_post ? rsqrtf(s[0] * inv + a.eps) : 1.f);
  s[0] = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    r[i] = x[i] + f * (h[i] * post[i]) * (a.gate ? sigmoid(g[i]) : 1.f);  // (as the backward makes it)
    s[0] += r[i] * r[i];
  }
  store_row<T, typename Ly::Group, K>(a.r, at, off, r);
  row_sums<LR>(s, lds[1]);
  const float rho = rsqrtf(s[0] * inv + a.eps);
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = r[i] * rho * pre[i];
  store_row<T, typename Ly::Group, K>(a.y, at, off, r);
}

// Workgroup b takes the row groups b, b + gridDim.x, ..; its column sums are part[0][b][C] (post) and part[1][b][C] (pre), or, where it is the only one, the
// gradients.
template <typename T, int V, int K, int LR>
__global__ __launch_bounds__(LR > 256 ? LR : 256) void residual_norm_bwd_kernel(const ResidualNorm a) {
  using Ly = Lay<T, V, K, LR>;
  using Vals = Values<T, typename Ly::Group, K>;
  typedef typename Ly::Group Group;
  constexpr int N = Ly::N, NS = 5;
  __shared__ float lds[2][Ly::THREADS / 64 * NS], lds_eta[2][Ly::THREADS / 64];
  const int slot = threadIdx.x / LR, idx = threadIdx.x % LR, C = a.C;
  const int64_t groups = ((int64_t)a.rows + Ly::SLOTS - 1) / Ly::SLOTS;
  int col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) col[k] = (k * LR + idx) * V;
  // HEAVY: a thread's column sums in LDS, the channel vectors read again for every row
  __shared__ float held[Ly::HEAVY ? 2 * N : 1][Ly::HEAVY ? Ly::THREADS : 1];
  float post[N], pre[N], dpost[Ly::HEAVY ? 1 : N], dpre[Ly::HEAVY ? 1 : N];
  auto sum_of = [&](int which, int i) -> float& {
    if constexpr (Ly::HEAVY) return held[which * N + i][threadIdx.x];
    else return which ? dpre[i] : dpost[i];
  };
  auto gammas = [&] {
    load_gamma<V, K>(post, a.gamma_post, col, C, 1.f);
    load_gamma<V, K>(pre, a.gamma_pre, col, C, 0.f);
  };
  if constexpr (!Ly::HEAVY) gammas();
#pragma unroll
  for (int i = 0; i < N; ++i) sum_of(0, i) = sum_of(1, i) = 0.f;
  struct Row { Vals x, h, g, dr, dy; };
  auto offsets = [&](int64_t group, unsigned (&off)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) off[k] = col[k] < C && group * Ly::SLOTS + slot < a.rows ? (unsigned)(slot * C + col[k]) * (unsigned)sizeof(T) : ~0u;
  };
  auto request = [&](int64_t group, Row& w) {
    const int64_t at = group * Ly::SLOTS * C * (int)sizeof(T);
    unsigned off[K];
    offsets(group, off);
    w.x.load(a.x, at, off);
    w.h.load(a.h, at, off);
    w.g.load(a.gate, at, off);
    w.dr.load(a.dr, at, off);
    w.dy.load(a.dy, at, off);
  };
  const float inv = 1.f / C;
  auto step = [&](int64_t group, const Row& w, int parity) {
    const int64_t at = group * Ly::SLOTS * C * (int)sizeof(T);
    unsigned off[K];
    offsets(group, off);
    float e[1] = {0.f}, s[NS] = {}, sig[N], away[Ly::HEAVY ? 1 : N], r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[0] += w.h[i] * w.h[i];
    row_sums<LR>(e, lds_eta[parity]);
    const float eta = a.gamma_post ? rsqrtf(e[0] * inv + a.eps) : 1.f, f = a.scale * eta;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float x = __expf(-w.g[i]);
      sig[i] = a.gate ? __builtin_amdgcn_rcpf(1.f + x) : 1.f;
      if constexpr (!Ly::HEAVY) away[i] = x;
      const float hp = w.h[i] * post[i], ad = w.dy[i] * pre[i], sgh = a.scale * sig[i] * hp;
      r[i] = w.x[i] + f * hp * sig[i];
      s[0] += r[i] * r[i];
      s[1] += r[i] * ad;
      s[2] += sgh * w.dr[i];
      s[3] += sgh * ad;
      s[4] += sgh * r[i];
    }
    row_sums<LR>(s, lds[parity]);
    const float rho = a.gamma_pre ? rsqrtf(s[0] * inv + a.eps) : 0.f;
    // mean(a rhat) and mean(b n), each factor next to the sum that it brings back to size: a reciprocal's square or cube would leave fp32 first
    const float mean_a = rho * (s[1] * inv);
    const float mean_b = a.gamma_post ? eta * (inv * (s[2] + rho * (s[3] - mean_a * (rho * s[4])))) : 0.f;
    // (branches, not factors of zero: without the norms what is infinite in h is not met)
    float d[N];
    if (a.gamma_pre) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float dy = w.dy[i], rhat = r[i] * rho;
        d[i] = w.dr[i] + rho * (dy * pre[i] - rhat * mean_a);
        sum_of(1, i) += dy * rhat;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] = w.dr[i];
    }
    store_row<T, Group, K>(a.dx, at, off, d);
    float dg[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float h = w.h[i], du = a.scale * sig[i] * d[i], n = h * eta;
      sum_of(0, i) += du * n;
      // 1 - sigmoid(g), not as a difference: of an open gate that has no bits left (g = 10: 1e-3 off, from 17 on zero).  exp(-g) sigmoid(g), and 1 where that
      // is inf * 0; where the register for it would be spilled sigmoid(-g) is faster (us, backward, 4096 x 12288 in bf16 448 / 373; 16384 x 4096 223 / 226)
      float shut;
      if constexpr (Ly::HEAVY) shut = sigmoid(-w.g[i]);
      else shut = fminf(away[i] * sig[i], 1.f);
      dg[i] = du * (n * post[i]) * shut;
      d[i] = eta * (du * post[i]);
    }
    if (a.gamma_post)
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] -= eta * (w.h[i] * eta * mean_b);
    store_row<T, Group, K>(a.dgate, at, off, dg);
    store_row<T, Group, K>(a.dh, at, off, d);
  };
  int64_t group = blockIdx.x;
  if constexpr (Ly::AHEAD) {
    Row w[2];
    request(group, w[0]);
    for (;;) {
      const int64_t second = group + gridDim.x, third = second + gridDim.x;
      if (second < groups) request(second, w[1]);
      step(group, w[0], 0);
      if (second >= groups) break;
      if (third < groups) request(third, w[0]);
      step(second, w[1], 1);
      if (third >= groups) break;
      group = third;
    }
  } else {
    for (int parity = 0; group < groups; group += gridDim.x, parity ^= 1) {
      Row w;
      request(group, w);
      if constexpr (Ly::HEAVY) gammas();
      step(group, w, parity);
    }
  }
  if (!a.dgamma_post && !a.dgamma_pre) return;
  // the sums of the rows that the workgroup has at once, one vector after the other: those of a wavefront between its lanes, the others through LDS
  constexpr int SHARES = LR < 64 ? Ly::THREADS / 64 : Ly::SLOTS;
  const int share = LR < 64 ? (int)threadIdx.x >> 6 : slot;
  __shared__ float join[SHARES > 1 ? SHARES * LR * N : 1];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* const out = which ? a.dgamma_pre : a.dgamma_post;
    if (!out) continue;
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = groups_sum<LR>(sum_of(which, i));
    if constexpr (SHARES > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) join[(i * SHARES + share) * LR + idx] = v[i];  // (the same from every group of a wavefront)
      __syncthreads();
      if (slot) continue;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = 0.f;
#pragma unroll
        for (int q = 0; q < SHARES; ++q) v[i] += join[(i * SHARES + q) * LR + idx];
      }
    }
    float* const to = gridDim.x == 1 ? out : a.part + ((int64_t)which * gridDim.x + blockIdx.x) * C;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = col[i / V] + i % V;
      if (c < C) to[c] = v[i] + (gridDim.x == 1 && a.accumulate ? to[c] : 0.f);
    }
  }
}
// 64 columns of one of the two vectors per workgroup, its 16 wavefronts share the parts.
__global__ __launch_bounds__(1024) void residual_norm_fold_kernel(const ResidualNorm a, int parts) {
  __shared__ float shares[16][64];
  float* const g = blockIdx.y ? a.dgamma_pre : a.dgamma_post;
  if (!g) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const float* const p = a.part + (int64_t)blockIdx.y * parts * a.C + min(c, a.C - 1);
  float s = 0.f;
#pragma unroll 8
  for (int k = wave; k < parts; k += 16) s += p[(int64_t)k * a.C];
  shares[wave][lane] = s;
  __syncthreads();
  if (wave || c >= a.C) return;
  s = a.accumulate ? g[c] : 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += shares[w][lane];
  g[c] = s;
}

template <typename T, int V, int K, int LR> hipError_t launch(const ResidualNorm& a, bool backward, hipStream_t stream) {
  using Ly = Lay<T, V, K, LR>;
  const int64_t groups = ((int64_t)a.rows + Ly::SLOTS - 1) / Ly::SLOTS;
  if (!backward) {
    if (!launchable(groups, Ly::THREADS)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((residual_norm_fwd_kernel<T, V, K, LR>), dim3((unsigned)groups), dim3(Ly::THREADS), 0, stream, a);
    return hipGetLastError();
  }
  // (a few row groups are one workgroup's: a second launch for the sums costs more than it saves)
  const int parts = groups <= 4 ? 1 : (int)std::min<int64_t>(groups, RNORM_MAX_PARTS);
  hipLaunchKernelGGL((residual_norm_bwd_kernel<T, V, K, LR>), dim3(parts), dim3(Ly::THREADS), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1 || !(a.dgamma_post || a.dgamma_pre)) return e;
  hipLaunchKernelGGL(residual_norm_fold_kernel, dim3((a.C + 63) / 64, 2), dim3(1024), 0, stream, a, parts);
  return hipGetLastError();
}
// The fewest lanes whose K groups of V hold a row.
template <typename T, int V, int K, int LR = 8> hipError_t dispatch(const ResidualNorm& a, bool backward, hipStream_t stream) {
  if constexpr (LR < 1024)
    if ((int64_t)LR * K * V < a.C) return dispatch<T, V, K, LR * 2>(a, backward, stream);
  return launch<T, V, K, LR>(a, backward, stream);
}
template <typename T> hipError_t any(const ResidualNorm& a, bool backward, hipStream_t stream) {
  uintptr_t all = (uintptr_t)(a.C % Elem<T>::VEC);
  for (const void* p : {a.x, a.h, a.gate, (const void*)a.r, (const void*)a.y, a.dr, a.dy, (const void*)a.dx, (const void*)a.dh, (const void*)a.dgate})
    all |= reinterpret_cast<uintptr_t>(p) & 15;
  if (all == 0)
    return a.C <= 8192 ? dispatch<T, Elem<T>::VEC, 8 / Elem<T>::VEC>(a, backward, stream) : launch<T, Elem<T>::VEC, 16 / Elem<T>::VEC, 1024>(a, backward, stream);
  if (a.C <= 4096) return dispatch<T, 1, 4>(a, backward, stream);
  return a.C <= 8192 ? launch<T, 1, 8, 1024>(a, backward, stream) : launch<T, 1, 16, 1024>(a, backward, stream);
}

}  // namespace

int64_t residual_norm_bwd_workspace_bytes(int rows, int C) { return 8ll * C * std::min(rows, RNORM_MAX_PARTS) + 256; }

hipError_t launch_residual_norm_fwd(const ResidualNorm& a, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? any<uint16_t>(a, false, stream) : any<float>(a, false, stream);
}
hipError_t launch_residual_norm_bwd(const ResidualNorm& a, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? any<uint16_t>(a, true, stream) : any<float>(a, true, stream);
}

}  // namespace cdp
