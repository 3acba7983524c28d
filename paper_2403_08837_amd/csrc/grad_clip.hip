// The norm over all gradients of a model, and the gradients scaled to at most a given norm.
//
// Two passes, bound by memory: every gradient is read for the norm, and read and written for the result.  The tensors are cut into units of 32 KB, which workgroups
// take in strides: eight 16-byte loads in flight in every thread.  Squares are summed in 64 bits (any fp32 value's square is there, and the
// order hardly matters), the workgroups' sums go to the workspace, and every workgroup of the second pass adds them up for itself in the same
// order: no third launch, no atomics.  The second pass goes through the units backwards: what the first read last is still cached.
// fp32, 400 million elements in 300 tensors: 0.88 ms, 5.5 TB/s over the two reads and the write.
// Sets of up to 64 pieces of 4 KB are one launch of one workgroup, whose wavefronts keep their pieces in registers between the two.
// The tensors' addresses travel in the kernel arguments, 160 of them a launch (160 tensors of 100 elements 9.3 us, 161 15.1); a wavefront finds the
// tensor of a unit by comparing all of them at once.
#include "elem.h"
#include "kernels.h"

#include <algorithm>
#include <cstring>

namespace cdp {

namespace {

constexpr int CLIP_TENSORS = 160, CLIP_GROUPS = 2048, UNIT_BYTES = 32768;
// one workgroup: threads, bytes of a piece, pieces of a wavefront, of all
constexpr int SOLE = 1024, SOLE_BYTES = 4096, SOLE_EACH = 4, SOLE_UNITS = SOLE / 64 * SOLE_EACH;

struct ClipTable {
  const void* g[CLIP_TENSORS];
  void* out[CLIP_TENSORS];
  uint16_t last[CLIP_TENSORS];  // elements of its last unit
  int32_t units[CLIP_TENSORS];  // of the tensors before it; past the last tensor all units (2^31 of them are 64 TB)
  int32_t total;
};
static_assert(sizeof(ClipTable) <= 3600, "kernel arguments are 4 KB at most");

// 16 bytes at a word's address: gradients are often slices of one vector, and what is not 16-byte aligned loses nothing (us, 300 slices, 400 million fp32
// elements: element by element 912, so 875; 30 million in bf16 47, 41).
typedef unsigned Words __attribute__((ext_vector_type(4), aligned(4)));

template <typename T, int BYTES = UNIT_BYTES> struct Unit {
  static constexpr int V = Elem<T>::VEC, SIZE = BYTES / (int)sizeof(T);
  const T* g;
  T* out;
  int n;        // elements, up to SIZE
  bool whole;   // 16-byte pieces, at addresses of words
  __device__ __forceinline__ Unit(const ClipTable& t, int u, bool scaling) {
    const int lane = threadIdx.x & 63;
    int i = -1;
#pragma unroll
    for (int k = 0; k < CLIP_TENSORS; k += 64) i += __popcll(__ballot(k + lane < CLIP_TENSORS && t.units[min(k + lane, CLIP_TENSORS - 1)] <= u));
    const int behind = i + 1 < CLIP_TENSORS ? t.units[i + 1] : t.total;
    const int64_t first = (int64_t)(u - t.units[i]) * SIZE;
    g = static_cast<const T*>(t.g[i]) + first;
    out = scaling ? static_cast<T*>(t.out[i]) + first : nullptr;
    n = u + 1 < behind ? SIZE : t.last[i];
    whole = ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(out)) & 3) == 0;
  }
};

template <int THREADS> __device__ __forceinline__ double group_sum(double s, double* lds) {
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
  return s;
}
// A thread's part of the sum of squares of a unit.
template <typename T, int THREADS> __device__ __forceinline__ double unit_squares(const Unit<T>& w) {
  constexpr int L = UNIT_BYTES / 16 / THREADS;
  const int t = threadIdx.x, pieces = w.whole ? w.n / Unit<T>::V : 0;
  double s = 0;
  Chunk16<T> c[L];
  const T behind = w.g[min(pieces * Unit<T>::V + t, w.n - 1)];  // what is behind the pieces, its first round
#pragma unroll
  for (int k = 0; k < L; ++k)
    if (pieces) c[k].v = __builtin_bit_cast(uint4, reinterpret_cast<const Words*>(w.g)[min(t + THREADS * k, pieces - 1)]);
#pragma unroll
  for (int k = 0; k < L; ++k)
    if (t + THREADS * k < pieces)
#pragma unroll
      for (int e = 0; e < Unit<T>::V; ++e) {
        const double v = Elem<T>::to_f32(c[k].e[e]);
        s += v * v;
      }
  if (pieces * Unit<T>::V + t < w.n) {
    const double v = Elem<T>::to_f32(behind);
    s += v * v;
  }
  for (int e = pieces * Unit<T>::V + t + THREADS; e < w.n; e += THREADS) {
    const double v = Elem<T>::to_f32(w.g[e]);
    s += v * v;
  }
  return s;
}
// What gradients are multiplied by.  Two factors, as one would be subnormal where gradients are large: 2^-100 or less, and what is left.
struct Factor {
  bool over;  // (a norm that is not a number: no)
  float first, rest;
  __device__ __forceinline__ Factor(double norm, float max_norm) {
    const double f = max_norm / norm;
    over = norm > max_norm;
    first = f >= 0x1p-100 ? 1.f : f >= 0x1p-200 ? 0x1p-100f : 0x1p-140f;
    rest = (float)(f * (f >= 0x1p-100 ? 1. : f >= 0x1p-200 ? 0x1p100 : 0x1p140));
  }
  template <typename T> __device__ __forceinline__ T operator()(T v) const { return Elem<T>::from_f32(rest * (first * Elem<T>::to_f32(v))); }
};
template <typename T, int THREADS> __device__ __forceinline__ void unit_scale(const Unit<T>& w, const Factor& f) {
  if (!f.over && w.out == w.g) return;  // in place, nothing to do
  constexpr int L = UNIT_BYTES / 16 / THREADS;
  const int t = threadIdx.x, pieces = w.whole ? w.n / Unit<T>::V : 0;
  Chunk16<T> c[L];
  const T behind = w.g[min(pieces * Unit<T>::V + t, w.n - 1)];
#pragma unroll
  for (int k = 0; k < L; ++k)
    if (pieces) c[k].v = __builtin_bit_cast(uint4, reinterpret_cast<const Words*>(w.g)[min(t + THREADS * k, pieces - 1)]);
#pragma unroll
  for (int k = 0; k < L; ++k) {
    if (t + THREADS * k >= pieces) continue;
    if (f.over)
#pragma unroll
      for (int e = 0; e < Unit<T>::V; ++e) c[k].e[e] = f(c[k].e[e]);
    reinterpret_cast<Words*>(w.out)[t + THREADS * k] = __builtin_bit_cast(Words, c[k].v);
  }
  if (pieces * Unit<T>::V + t < w.n) w.out[pieces * Unit<T>::V + t] = f.over ? f(behind) : behind;
  for (int e = pieces * Unit<T>::V + t + THREADS; e < w.n; e += THREADS) w.out[e] = f.over ? f(w.g[e]) : w.g[e];
}

// Sum of squares of a workgroup's units, written to part[workgroup], or, past the first table, added to it.
template <typename T> __global__ __launch_bounds__(256) void grad_norm_kernel(const ClipTable t, double* part, int first) {
  __shared__ double lds[4];
  double s = 0;
  for (int u = blockIdx.x; u < t.total; u += gridDim.x) s += unit_squares<T, 256>(Unit<T>(t, u, false));
  s = group_sum<256>(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = first ? s : part[blockIdx.x] + s;
}
template <typename T> __global__ __launch_bounds__(256) void grad_scale_kernel(const ClipTable t, const double* part, int parts, float* norm, float max_norm, int scaling) {
  __shared__ double lds[4];
  double s = 0;
#pragma unroll
  for (int k = 0; k < CLIP_GROUPS / 256; ++k) {
    const int i = threadIdx.x + 256 * k;
    const double v = part[min(i, parts - 1)];
    s += i < parts ? v : 0.0;
  }
  const double r = sqrt(group_sum<256>(s, lds));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r;
  if (!scaling) return;
  const Factor f(r, max_norm);
  for (int v = blockIdx.x; v < t.total; v += gridDim.x) unit_scale<T, 256>(Unit<T>(t, t.total - 1 - v, true), f);
}
// Both for a set of one table and few pieces; a wavefront has the pieces wave, wave + 16, ..
template <typename T> __global__ __launch_bounds__(SOLE) void grad_sole_kernel(const ClipTable t, float* norm, float max_norm, int scaling) {
  typedef Unit<T, SOLE_BYTES> U;
  constexpr int L = SOLE_BYTES / 16 / 64;
  __shared__ double lds[SOLE / 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Chunk16<T> c[SOLE_EACH][L];
  T behind[SOLE_EACH];
  double s = 0;
  // (a piece past the last: the last one, of nothing)
  auto piece = [&](int k) {
    const int u = wave + k * (SOLE / 64);
    U w(t, min(u, max(t.total - 1, 0)), scaling);
    if (u >= t.total) w.n = 0;
    return w;
  };
  const U w[SOLE_EACH] = {piece(0), piece(1), piece(2), piece(3)};
  static_assert(SOLE_EACH == 4, "pieces");
  auto wholes = [&](int k) { return w[k].whole ? w[k].n / U::V : 0; };
#pragma unroll
  for (int k = 0; k < SOLE_EACH; ++k) {
    const int pieces = wholes(k);
    if (w[k].n) behind[k] = w[k].g[min(pieces * U::V + lane, w[k].n - 1)];
    if (pieces)
#pragma unroll
      for (int l = 0; l < L; ++l) c[k][l].v = __builtin_bit_cast(uint4, reinterpret_cast<const Words*>(w[k].g)[min(lane + 64 * l, pieces - 1)]);
  }
#pragma unroll
  for (int k = 0; k < SOLE_EACH; ++k) {
    const int pieces = wholes(k);
#pragma unroll
    for (int l = 0; l < L; ++l)
      if (lane + 64 * l < pieces)
#pragma unroll
        for (int e = 0; e < U::V; ++e) {
          const double v = Elem<T>::to_f32(c[k][l].e[e]);
          s += v * v;
        }
    if (pieces * U::V + lane < w[k].n) {
      const double v = Elem<T>::to_f32(behind[k]);
      s += v * v;
    }
    for (int e = pieces * U::V + lane + 64; e < w[k].n; e += 64) {
      const double v = Elem<T>::to_f32(w[k].g[e]);
      s += v * v;
    }
  }
  const double r = sqrt(group_sum<SOLE>(s, lds));
  if (threadIdx.x == 0) *norm = (float)r;
  if (!scaling) return;
  const Factor f(r, max_norm);
#pragma unroll
  for (int k = 0; k < SOLE_EACH; ++k) {
    if (!f.over && w[k].out == w[k].g) continue;
    const int pieces = wholes(k);
#pragma unroll
    for (int l = 0; l < L; ++l) {
      if (lane + 64 * l >= pieces) continue;
      if (f.over)
#pragma unroll
        for (int e = 0; e < U::V; ++e) c[k][l].e[e] = f(c[k][l].e[e]);
      reinterpret_cast<Words*>(w[k].out)[lane + 64 * l] = __builtin_bit_cast(Words, c[k][l].v);
    }
    if (pieces * U::V + lane < w[k].n) w[k].out[pieces * U::V + lane] = f.over ? f(behind[k]) : behind[k];
    for (int e = pieces * U::V + lane + 64; e < w[k].n; e += 64) w[k].out[e] = f.over ? f(w[k].g[e]) : w[k].g[e];
  }
}

template <typename T>
hipError_t clip(int tensors, const void* const* grads, void* const* outs, const int64_t* counts, float max_norm, float* norm, double* part, hipStream_t stream) {
  auto table = [&](int i0, int size) {
    ClipTable t;
    int32_t units = 0;
    for (int i = 0; i < CLIP_TENSORS; ++i) {
      const bool there = i0 + i < tensors && counts[i0 + i] > 0;
      t.g[i] = there ? grads[i0 + i] : nullptr;
      t.out[i] = there && outs ? outs[i0 + i] : nullptr;
      t.last[i] = there ? (uint16_t)((counts[i0 + i] - 1) % size + 1) : 0;
      t.units[i] = units;  // (of tensors with the same one, only the last has units)
      if (there) units += (int32_t)((counts[i0 + i] + size - 1) / size);
    }
    t.total = units;
    return t;
  };
  int64_t most = 1;
  for (int i0 = 0; i0 < tensors; i0 += CLIP_TENSORS) {
    int64_t units = 0;
    for (int i = i0; i < std::min(tensors - i0, CLIP_TENSORS) + i0; ++i) units += (counts[i] + Unit<T>::SIZE - 1) / Unit<T>::SIZE;
    most = std::max(most, units);
  }
  if (tensors <= CLIP_TENSORS && most <= SOLE_UNITS) {
    const ClipTable t = table(0, Unit<T, SOLE_BYTES>::SIZE);
    if (t.total <= SOLE_UNITS) {
      hipLaunchKernelGGL((grad_sole_kernel<T>), dim3(1), dim3(SOLE), 0, stream, t, norm, max_norm, outs != nullptr);
      return hipGetLastError();
    }
  }
  const int groups = (int)std::min<int64_t>(most, CLIP_GROUPS);
  for (int i0 = 0; i0 < tensors; i0 += CLIP_TENSORS) {
    hipLaunchKernelGGL((grad_norm_kernel<T>), dim3(groups), dim3(256), 0, stream, table(i0, Unit<T>::SIZE), part, i0 == 0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  for (int i0 = (tensors - 1) / CLIP_TENSORS * CLIP_TENSORS; i0 >= 0; i0 -= CLIP_TENSORS) {
    hipLaunchKernelGGL((grad_scale_kernel<T>), dim3(outs ? groups : 1), dim3(256), 0, stream, table(i0, Unit<T>::SIZE), part, groups, norm, max_norm, outs != nullptr);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !outs) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_grad_clip(int tensors, const void* const* grads, void* const* outs, const int64_t* counts, float max_norm, float* norm,
                            void* workspace, int dtype, hipStream_t stream) {
  double* part = static_cast<double*>(workspace);
  return dtype == DT_BF16 ? clip<uint16_t>(tensors, grads, outs, counts, max_norm, norm, part, stream)
                          : clip<float>(tensors, grads, outs, counts, max_norm, norm, part, stream);
}

}  // namespace cdp
