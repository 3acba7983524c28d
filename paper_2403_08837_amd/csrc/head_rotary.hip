// Norms of query and key heads and the rotation of their pairs by position, in one pass over qkv[tokens][heads + 2 kv_heads][width], with the gradients:
//   n = x rho gamma, rho = 1 / sqrt(mean x^2 + eps);  a pair (p, q) of n becomes (p cos - q sin, q cos + p sin), angle = position * freq;  v heads are copied.
// Backward: the pairs of dout turned back are dn;  a = dn gamma, hat = x rho:  dx = rho (a - hat mean(a hat)),  dgamma = sum dn hat.  Without norms that is the forward,
// turned the other way.
//
// Bound by memory: a head is read and written once (backward: x and dout read, dx written).  A lane holds V pairs of a head, as two vectors of V neighbouring
// values (16 bytes each where the sizes allow), so that a pair never crosses lanes and the norm is one sum over the G lanes of a head, backward two at once.  The
// angles of a workgroup's tokens are made once, by all of its lanes, and kept as cosine and sine in LDS for all heads.  They are position * freq / 2 pi in 64
// bits and more, taken into an eighth of a turn before they become fp32: a far position costs no exactness.
// us of 16384 tokens of 48 heads of 128 in bf16: forward 70 (5.8 TB/s), backward 115 to 124 (5.2 to 5.6 TB/s) and 5 for the sums of dgamma; 2501 tokens of 24 x 80 in fp32,
// interleaved, 7.3 to 9, 11.5 to 13.6 and 4; the shortest 3.4, 4.7 and 1.7.
// Column sums (dgamma) stay in registers over a workgroup's tokens; what the workgroups have is added up by head_rotary_fold_kernel in a fixed order.
#include "elem.h"
#include "kernels.h"
#include "lane_sums.h"

#include <algorithm>

namespace cdp {

namespace {

constexpr int THREADS = 256, MAX_TOKENS = 16, MAX_PAIRS = 64;

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
  constexpr int SLOTS = THREADS / G, AT_ONCE = BACKWARD ? 2 : 1;  // heads of a lane that are on their way together
  __shared__ __attribute__((aligned(16))) float2 turns[BACKWARD ? 2 : 1][MAX_TOKENS * MAX_PAIRS];
  const int W = a.width, R = a.rotary, pairs = W / 2, c = threadIdx.x % G, slot = threadIdx.x / G;
  const int normed = a.heads + a.kv_heads, all = normed + a.kv_heads;
  const bool has = c * V < pairs;
  const Place at = place<V, INTER>(has ? c : 0, W, R);
  const float inv = 1.f / W;
  __shared__ __attribute__((aligned(16))) float gammas[2][2 * MAX_PAIRS];  // of q and k heads; ones where there is none
  if ((int)threadIdx.x < W) {
    gammas[0][threadIdx.x] = a.gamma_q ? a.gamma_q[threadIdx.x] : 1.f;
    gammas[1][threadIdx.x] = a.gamma_k ? a.gamma_k[threadIdx.x] : 1.f;
  }
  float sq[BACKWARD ? 2 * V : 1], sk[BACKWARD ? 2 * V : 1];
  if constexpr (BACKWARD)
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) sq[i] = sk[i] = 0.f;
  const int64_t groups = ((int64_t)a.tokens + per - 1) / per;
  // backward the next group's angles are made ahead of this one's heads, into the other half
  auto angles_of = [&](int64_t group, float2* turn) {
    const int64_t token0 = group * per;
    const int n = (int)min((int64_t)per, a.tokens - token0) * pairs;
    for (int i = threadIdx.x; i < n; i += THREADS) {
      const int t = i / pairs, p = i - t * pairs;
      float2 w = 2 * p < R ? turned(a.positions[token0 + t], a.freqs[p]) : make_float2(1.f, 0.f);
      if (a.back) w.y = -w.y;
      turn[t * MAX_PAIRS + p] = w;
    }
  };
  int half = 0;
  angles_of(blockIdx.x, turns[0]);
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
    const int64_t token0 = group * per;
    const int tokens = (int)min((int64_t)per, a.tokens - token0);
    __syncthreads();
    const float2* const turn = turns[half];
    if (BACKWARD) {
      half ^= 1;
      if (group + gridDim.x < groups) angles_of(group + gridDim.x, turns[half]);
    }
    struct Item {
      int t, h;
      Values lo, hi, x_lo, x_hi;
    };
    auto request = [&](Item& w) {
      if (!has || w.t >= tokens || (a.in_place && w.h >= normed)) return;
      const int64_t base = ((token0 + w.t) * all + w.h) * W;
      const T* const from = static_cast<const T*>(BACKWARD ? a.dout : a.qkv) + base;
      w.lo = *reinterpret_cast<const Values*>(from + at.o0);
      w.hi = *reinterpret_cast<const Values*>(from + at.o1);
      if (BACKWARD && w.h < normed) {  // (both at once: one round trip)
        const T* const was = static_cast<const T*>(a.qkv) + base;
        w.x_lo = *reinterpret_cast<const Values*>(was + at.o0);
        w.x_hi = *reinterpret_cast<const Values*>(was + at.o1);
      }
    };
    auto finish = [&](Item& w) {
      const int t = w.t, h = w.h;
      if (t >= tokens || (a.in_place && h >= normed)) return;  // (heads go to lanes alike in place or not, and sums have one order)
      T* const to = static_cast<T*>(BACKWARD ? a.dqkv : a.out) + ((token0 + t) * all + h) * W;
      Values &lo = w.lo, &hi = w.hi, &x_lo = w.x_lo, &x_hi = w.x_hi;
      if (h >= normed) {
        if (has) {
          *reinterpret_cast<Values*>(to + at.o0) = lo;
          *reinterpret_cast<Values*>(to + at.o1) = hi;
        }
        return;
      }
      const bool is_q = h < a.heads, norm = is_q ? a.gamma_q != nullptr : a.gamma_k != nullptr;
      const float* const gamma = gammas[is_q ? 0 : 1];
      const float2* const angles = turn + t * MAX_PAIRS + (has ? c : 0) * V;
      float v[2 * V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[i] = has ? Elem<T>::to_f32(lo.e[i]) : 0.f;
        v[V + i] = has ? Elem<T>::to_f32(hi.e[i]) : 0.f;
      }
      if constexpr (!BACKWARD) {
        if (norm) {
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) s += v[i] * v[i];
          const float rho = rsqrtf(lanes_sum<G>(s) * inv + a.eps);
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) v[i] = v[i] * rho * gamma[i < V ? at.o0 + i : at.o1 + i - V];
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float2 w = angles[j];
          const float p = v[first_of<V, INTER>(j)], q = v[second_of<V, INTER>(j)];
          const bool here = c * V + j < R / 2;  // (what is behind stays as it is: times a sine of zero, an infinite value would reach the one beside it)
          v[first_of<V, INTER>(j)] = here ? p * w.x - q * w.y : p;
          v[second_of<V, INTER>(j)] = here ? q * w.x + p * w.y : q;
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float2 w = angles[j];
          const float p = v[first_of<V, INTER>(j)], q = v[second_of<V, INTER>(j)];
          const bool here = c * V + j < R / 2;
          v[first_of<V, INTER>(j)] = here ? p * w.x - q * w.y : p;
          v[second_of<V, INTER>(j)] = here ? q * w.x + p * w.y : q;
        }
        if (norm) {
          float x[2 * V], ss = 0.f, sa = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            x[i] = has ? Elem<T>::to_f32(i < V ? x_lo.e[i] : x_hi.e[i - V]) : 0.f;
            ss += x[i] * x[i];
            sa += v[i] * gamma[i < V ? at.o0 + i : at.o1 + i - V] * x[i];
          }
          const float rho = rsqrtf(lanes_sum<G>(ss) * inv + a.eps), mean = rho * (lanes_sum<G>(sa) * inv);
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            const float hat = x[i] * rho, g = v[i] * hat;
            if (is_q) sq[i] += g;
            else sk[i] += g;
            v[i] = rho * (v[i] * gamma[i < V ? at.o0 + i : at.o1 + i - V] - hat * mean);
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
    };
    Item w[AT_ONCE];
    for (int t = slot / all, h = slot - t * all; t < tokens;) {
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        w[u].t = t;
        w[u].h = h;
        request(w[u]);
        for (h += SLOTS; h >= all; h -= all) ++t;
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) finish(w[u]);
    }
  }
  if constexpr (BACKWARD) {
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
  int per = std::max(1, std::min(MAX_TOKENS, (backward ? 8 : 4) * SLOTS / heads));
  while (per > 1 && (a.tokens + per - 1) / per < 512) per /= 2;
  const int64_t groups = ((int64_t)a.tokens + per - 1) / per;
  if (!backward) {
    if (!launchable(groups, THREADS)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((head_rotary_kernel<T, V, INTER, G, false>), dim3((unsigned)groups), dim3(THREADS), 0, stream, a, per);
    return hipGetLastError();
  }
  if constexpr (V == 8) return hipErrorInvalidValue;  // (`any` takes fewer values at once: 131 us instead of 114 for 16384 tokens of 48 x 128, for want of registers)
  else {
    // a few groups are one workgroup's: a second launch for the sums costs more than it saves
    const int parts = groups <= 4 ? 1 : (int)std::min<int64_t>(groups, HEAD_ROTARY_MAX_PARTS);
    hipLaunchKernelGGL((head_rotary_kernel<T, V, INTER, G, true>), dim3(parts), dim3(THREADS), 0, stream, a, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    hipLaunchKernelGGL(head_rotary_fold_kernel, dim3(a.width / 8, 2), dim3(THREADS), 0, stream, a, parts);
    return hipGetLastError();
  }
}
template <typename T> hipError_t any(const HeadRotary& a, bool backward, hipStream_t stream) {
  const int W = a.width, both = a.rotary / 2 | (W - a.rotary) / 2;  // vectors begin at multiples of what divides both
  if (a.interleaved) return W <= 64 ? launch<T, 4, true, 8>(a, backward, stream) : launch<T, 4, true, 16>(a, backward, stream);
  if constexpr (sizeof(T) == 2)
    if (both % 8 == 0 && !backward) return W <= 64 ? launch<T, 8, false, 4>(a, backward, stream) : launch<T, 8, false, 8>(a, backward, stream);
  if (both % 4 == 0) return W <= 64 ? launch<T, 4, false, 8>(a, backward, stream) : launch<T, 4, false, 16>(a, backward, stream);
  if (both % 2 == 0) return launch<T, 2, false, 32>(a, backward, stream);
  return launch<T, 1, false, 64>(a, backward, stream);
}

}  // namespace

int64_t head_rotary_bwd_workspace_bytes(int tokens, int width) { return 8ll * width * std::min(tokens, HEAD_ROTARY_MAX_PARTS) + 256; }

hipError_t launch_head_rotary(const HeadRotary& given, bool backward, int dtype, hipStream_t stream) {
  HeadRotary a = given;
  a.back = backward;
  if (backward && !a.dgamma_q && !a.dgamma_k) {  // without norms: forward, turned the other way
    a.qkv = a.dout;
    a.out = a.dqkv;
    backward = false;
  }
  return dtype == DT_BF16 ? any<uint16_t>(a, backward, stream) : any<float>(a, backward, stream);
}

}  // namespace cdp
