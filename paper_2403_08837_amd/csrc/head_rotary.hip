// Norms of query and key heads and the rotation of their pairs by position, in one pass over qkv[tokens][heads + 2 kv_heads][width], with the gradients:
//   n = x rho gamma, rho = 1 / sqrt(mean x^2 + eps);  a pair (p, q) of n becomes (p cos - q sin, q cos + p sin), angle = position * freq;  v heads are copied.
// Backward: the pairs of dout turned back are dn;  a = dn gamma, hat = x rho:  dx = rho (a - hat mean(a hat)),  dgamma = sum dn hat.
//
// Bound by memory: a head is read and written once (backward: x and dout read, dx written).  A lane holds V pairs of a head, as two vectors of V neighbouring
// values (16 bytes each where the sizes allow), so that a pair never crosses lanes and the norm is one sum over the G lanes of a head, backward two at once.  The
// angles of a workgroup's tokens are made once, by all of its lanes, and kept as cosine and sine in LDS for all heads.  They are position * freq / 2 pi in 64
// bits and more, taken into an eighth of a turn before they become fp32: a far position costs no exactness.
// Column sums (dgamma) stay in registers over a workgroup's tokens; what the workgroups have is added up by head_rotary_fold_kernel in a fixed order.
#include "elem.h"
#include "kernels.h"
#include "lane_sums.h"

#include <algorithm>

namespace cdp {

namespace {

constexpr int THREADS = 256, MAX_TOKENS = 8, MAX_PAIRS = 64;

template <typename T, int V> struct alignas(V * sizeof(T)) Vec { T e[V]; };

// Cosine and sine of position * freq.  freq / 2 pi as a sum of two doubles, its product with the position exact up to 2^-106 of it, the eighths of a turn taken
// off before anything is rounded: the angle is as exact at 2^31 as at 1.
__device__ __forceinline__ float2 turned(int position, float freq) {
  constexpr double I = 0.15915494309189535, I_LOW = -9.839338337591243e-18;  // 1 / 2 pi
  const double f = (double)freq * I, f_low = fma((double)freq, I, -f) + (double)freq * I_LOW;
  const double n = position, t = n * f, t_low = fma(n, f, -t) + n * f_low;  // turns
  const double q = rint(4.0 * t);
  const float r = (float)((t - 0.25 * q) + t_low);  // |r| <= 1/8
  float s, c;
  sincospif(2.f * r, &s, &c);
  const int k = (int)(q - 4.0 * floor(0.25 * q));
  const float c2 = k & 1 ? s : c, s2 = k & 1 ? c : s;
  return make_float2(k == 1 || k == 2 ? -c2 : c2, k >= 2 ? -s2 : s2);
}

struct Place { int o0, o1; };  // where a lane's two vectors begin in a head
template <int V, bool INTER> __device__ __forceinline__ Place place(int c, int W, int R) {
  if (INTER) return {2 * V * c, 2 * V * c + V};
  const int rotated = R / (2 * V);
  if (c < rotated) return {V * c, R / 2 + V * c};
  return {R + V * (c - rotated), R + (W - R) / 2 + V * (c - rotated)};
}
// Values of pair j among the 2 V of a lane.
template <int V, bool INTER> constexpr int first_of(int j) { return INTER ? 2 * j : j; }
template <int V, bool INTER> constexpr int second_of(int j) { return INTER ? 2 * j + 1 : V + j; }

// Workgroups take `per` tokens at once; forward one such group each, backward b, b + gridDim.x, ..
template <typename T, int V, bool INTER, int G, bool BACKWARD>
__global__ __launch_bounds__(THREADS) void head_rotary_kernel(const HeadRotary a, int per) {
  using Values = Vec<T, V>;
  constexpr int SLOTS = THREADS / G;
  __shared__ __attribute__((aligned(16))) float2 turn[MAX_TOKENS * MAX_PAIRS];
  const int W = a.width, R = a.rotary, pairs = W / 2, c = threadIdx.x % G, slot = threadIdx.x / G;
  const int normed = a.heads + a.kv_heads, all = normed + a.kv_heads;
  const bool has = c * V < pairs;
  const Place at = place<V, INTER>(has ? c : 0, W, R);
  const float inv = 1.f / W;
  float gq[2 * V], gk[2 * V], sq[BACKWARD ? 2 * V : 1], sk[BACKWARD ? 2 * V : 1];
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    const int o = i < V ? at.o0 + i : at.o1 + i - V;
    gq[i] = a.gamma_q ? a.gamma_q[o] : 1.f;
    gk[i] = a.gamma_k ? a.gamma_k[o] : 1.f;
    if constexpr (BACKWARD) sq[i] = sk[i] = 0.f;
  }
  const int64_t groups = ((int64_t)a.tokens + per - 1) / per;
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
    const int64_t token0 = group * per;
    const int tokens = (int)min((int64_t)per, a.tokens - token0);
    if (BACKWARD && group != blockIdx.x) __syncthreads();  // the angles before have been used
    for (int i = threadIdx.x; i < tokens * pairs; i += THREADS) {
      const int t = i / pairs, p = i - t * pairs;
      turn[t * MAX_PAIRS + p] = 2 * p < R ? turned(a.positions[token0 + t], a.freqs[p]) : make_float2(1.f, 0.f);
    }
    __syncthreads();
    int t = slot / all, h = slot - t * all;
    for (; t < tokens; h += SLOTS) {
      while (h >= all) {
        h -= all;
        ++t;
      }
      if (t >= tokens) break;
      if (a.in_place && h >= normed) continue;  // (heads go to lanes alike in place or not, and sums have one order)
      const int64_t base = ((token0 + t) * all + h) * W;
      const T* const from = static_cast<const T*>(BACKWARD ? a.dout : a.qkv) + base;
      T* const to = static_cast<T*>(BACKWARD ? a.dqkv : a.out) + base;
      Values lo, hi;
      if (has) {
        lo = *reinterpret_cast<const Values*>(from + at.o0);
        hi = *reinterpret_cast<const Values*>(from + at.o1);
      }
      if (h >= normed) {
        if (has) {
          *reinterpret_cast<Values*>(to + at.o0) = lo;
          *reinterpret_cast<Values*>(to + at.o1) = hi;
        }
        continue;
      }
      const bool is_q = h < a.heads, norm = is_q ? a.gamma_q != nullptr : a.gamma_k != nullptr;
      float v[2 * V], x[BACKWARD ? 2 * V : 1], cs[V], sn[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[i] = has ? Elem<T>::to_f32(lo.e[i]) : 0.f;
        v[V + i] = has ? Elem<T>::to_f32(hi.e[i]) : 0.f;
        const float2 w = turn[t * MAX_PAIRS + (has ? c : 0) * V + i];
        cs[i] = w.x;
        sn[i] = w.y;
      }
      if constexpr (!BACKWARD) {
        if (norm) {
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) s += v[i] * v[i];
          const float rho = rsqrtf(lanes_sum<G>(s) * inv + a.eps);
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) v[i] = v[i] * rho * (is_q ? gq[i] : gk[i]);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float p = v[first_of<V, INTER>(j)], q = v[second_of<V, INTER>(j)];
          v[first_of<V, INTER>(j)] = p * cs[j] - q * sn[j];
          v[second_of<V, INTER>(j)] = q * cs[j] + p * sn[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float p = v[first_of<V, INTER>(j)], q = v[second_of<V, INTER>(j)];
          v[first_of<V, INTER>(j)] = p * cs[j] + q * sn[j];
          v[second_of<V, INTER>(j)] = q * cs[j] - p * sn[j];
        }
        if (norm) {
          if (has) {
            const T* const was = static_cast<const T*>(a.qkv) + base;
            lo = *reinterpret_cast<const Values*>(was + at.o0);
            hi = *reinterpret_cast<const Values*>(was + at.o1);
          }
          float ss = 0.f, sa = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            x[i] = has ? Elem<T>::to_f32(i < V ? lo.e[i] : hi.e[i - V]) : 0.f;
            ss += x[i] * x[i];
            sa += v[i] * (is_q ? gq[i] : gk[i]) * x[i];
          }
          const float rho = rsqrtf(lanes_sum<G>(ss) * inv + a.eps), mean = rho * (lanes_sum<G>(sa) * inv);
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            const float hat = x[i] * rho, g = v[i] * hat;
            if (is_q) sq[i] += g;
            else sk[i] += g;
            v[i] = rho * (v[i] * (is_q ? gq[i] : gk[i]) - hat * mean);
          }
        }
      }
      if (has) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          lo.e[i] = Elem<T>::from_f32(v[i]);
          hi.e[i] = Elem<T>::from_f32(v[V + i]);
        }
        *reinterpret_cast<Values*>(to + at.o0) = lo;
        *reinterpret_cast<Values*>(to + at.o1) = hi;
      }
    }
  }
  if constexpr (BACKWARD) {
    if (!a.dgamma_q && !a.dgamma_k) return;
    // the heads that a wavefront has at once between its lanes, its four wavefronts through LDS
    __shared__ float join[4][2 * MAX_PAIRS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float* const out = which ? a.dgamma_k : a.dgamma_q;
      if (!out) continue;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) {
        const float s = groups_sum<G>(which ? sk[i] : sq[i]);
        if (lane < G && has) join[wave][i < V ? at.o0 + i : at.o1 + i - V] = s;
      }
      __syncthreads();
      const int col = threadIdx.x;
      if (col < W) {
        const float s = (join[0][col] + join[1][col]) + (join[2][col] + join[3][col]);
        if (gridDim.x == 1) out[col] = s + (a.accumulate ? out[col] : 0.f);
        else a.part[((int64_t)which * gridDim.x + blockIdx.x) * W + col] = s;
      }
    }
  }
}

// 8 columns of one of the two vectors per workgroup, 32 lanes share the parts of a column.
__global__ __launch_bounds__(THREADS) void head_rotary_fold_kernel(const HeadRotary a, int parts) {
  __shared__ float shares[32][8];
  float* const out = blockIdx.y ? a.dgamma_k : a.dgamma_q;
  if (!out) return;
  const int c = threadIdx.x & 7, share = threadIdx.x >> 3, col = blockIdx.x * 8 + c;  // (widths are multiples of 8)
  const float* const p = a.part + (int64_t)blockIdx.y * parts * a.width + col;
  float s = 0.f;
#pragma unroll 8
  for (int k = share; k < parts; k += 32) s += p[(int64_t)k * a.width];
  shares[share][c] = s;
  __syncthreads();
  if (share) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) s += shares[k][c];
  out[col] = s + (a.accumulate ? out[col] : 0.f);
}

template <typename T, int V, bool INTER, int G> hipError_t launch(const HeadRotary& a, bool backward, hipStream_t stream) {
  constexpr int SLOTS = THREADS / G;
  // tokens at once: enough heads to fill a workgroup a few times, fewer where that leaves less than two workgroups a CU
  const int heads = a.heads + 2 * a.kv_heads;
  int per = std::max(1, std::min(MAX_TOKENS, 4 * SLOTS / heads));
  while (per > 1 && (a.tokens + per - 1) / per < 512) per /= 2;
  const int64_t groups = ((int64_t)a.tokens + per - 1) / per;
  if (!backward) {
    if (!launchable(groups, THREADS)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((head_rotary_kernel<T, V, INTER, G, false>), dim3((unsigned)groups), dim3(THREADS), 0, stream, a, per);
    return hipGetLastError();
  }
  const bool sums = a.dgamma_q || a.dgamma_k;
  // a few groups are one workgroup's: a second launch for the sums costs more than it saves
  const int parts = sums && groups <= 4 ? 1 : (int)std::min<int64_t>(groups, HEAD_ROTARY_MAX_PARTS);
  hipLaunchKernelGGL((head_rotary_kernel<T, V, INTER, G, true>), dim3(parts), dim3(THREADS), 0, stream, a, per);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1 || !sums) return e;
  hipLaunchKernelGGL(head_rotary_fold_kernel, dim3(a.width / 8, 2), dim3(THREADS), 0, stream, a, parts);
  return hipGetLastError();
}
template <typename T> hipError_t any(const HeadRotary& a, bool backward, hipStream_t stream) {
  const int W = a.width, both = a.rotary / 2 | (W - a.rotary) / 2;  // vectors begin at multiples of what divides both
  if (a.interleaved) return W <= 64 ? launch<T, 4, true, 8>(a, backward, stream) : launch<T, 4, true, 16>(a, backward, stream);
  if constexpr (sizeof(T) == 2)
    if (both % 8 == 0) return W <= 64 ? launch<T, 8, false, 4>(a, backward, stream) : launch<T, 8, false, 8>(a, backward, stream);
  if (both % 4 == 0) return W <= 64 ? launch<T, 4, false, 8>(a, backward, stream) : launch<T, 4, false, 16>(a, backward, stream);
  if (both % 2 == 0) return launch<T, 2, false, 32>(a, backward, stream);
  return launch<T, 1, false, 64>(a, backward, stream);
}

}  // namespace

int64_t head_rotary_bwd_workspace_bytes(int tokens, int width) { return 8ll * width * std::min(tokens, HEAD_ROTARY_MAX_PARTS) + 256; }

hipError_t launch_head_rotary(const HeadRotary& a, bool backward, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? any<uint16_t>(a, backward, stream) : any<float>(a, backward, stream);
}

}  // namespace cdp
