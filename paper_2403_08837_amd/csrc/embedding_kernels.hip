// Embedding: rows of a table by token ids, scaled, and the gradient of the table.
//
// Forward: a gather in 16-byte pieces.  Bound by memory: every token's row read (a repeated one from cache) and written.
//
// Backward: dtable[v] = scale * sum of the rows of dout whose token is v, in fp32 and in a fixed order, without atomics.  The least it has to do is to read dout
// and write the table; what makes it more than a copy is that a few words are a large part of a text, so that a row of the table is the sum
// of anything from none to thousands of rows.  The tokens are sorted by word (stably: a word's tokens stay in order):
//   1. runs of 2048 in LDS; in the same launch, under the sort, all other workgroups write the zeros of the table;
//   2. sixteen runs to one, repeated: a token's place is the sum of its ranks in the sixteen, each a binary search;
//   3. a wavefront per 32 sorted tokens and 64 pieces of their rows: words that begin and end among them are finished there; of one
//      that goes on, the sums before the first and after the last border go to the workspace;
//   4. those sums, a workgroup per word that crosses a border.
// Up to 256 tokens are looked for by comparison instead: every row of the table is matched against all ids, which are in registers, in one launch.
#include "elem.h"
#include "kernels.h"

#include <algorithm>

namespace cdp {

namespace {

constexpr int RUN = 2048, WAYS = 16, CHUNK = 32, FEW = 256;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// What a lane of a wavefront holds of a row: piece `p` of 64 pieces of V neighbouring columns, or (V = 1, rows that are not whole 16-byte
// pieces) eight columns 64 apart.
template <typename T, int V> struct Piece {
  static constexpr int K = V == 1 ? 8 : 1, N = V * K, SPAN = 64 * N;
  __device__ static __forceinline__ int col(int p, int k, int lane) { return p * SPAN + (V == 1 ? 64 * k + lane : lane * V); }
  // the bits: a conversion is a use, which waits for the load
  struct Bits { uint4 v; uint32_t e[K]; };
  __device__ static __forceinline__ void load(Bits& b, const T* row, int p, int lane, int C) {
    if constexpr (V > 1) b.v = *reinterpret_cast<const uint4*>(row + min(col(p, 0, lane), C - V));
    else
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const T x = row[min(col(p, k, lane), C - 1)];
        if constexpr (sizeof(T) == 2) b.e[k] = x;
        else b.e[k] = __float_as_uint(x);
      }
  }
  __device__ static __forceinline__ void values(const Bits& b, float (&x)[N]) {
    if constexpr (V > 1) {
      Chunk16<T> c;
      c.v = b.v;
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = Elem<T>::to_f32(c.e[e]);
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) x[k] = __uint_as_float(sizeof(T) == 2 ? b.e[k] << 16 : b.e[k]);
    }
  }
  // fp32 rows of the table and of the workspace
  __device__ static __forceinline__ void load32(float (&x)[N], const float* row, int p, int lane, int C) {
    if constexpr (V > 1) {
      const float* r = row + min(col(p, 0, lane), C - V);
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const float4 f = *reinterpret_cast<const float4*>(r + e);
        x[e] = f.x; x[e + 1] = f.y; x[e + 2] = f.z; x[e + 3] = f.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) x[k] = row[min(col(p, k, lane), C - 1)];
    }
  }
  __device__ static __forceinline__ void store32(const float (&x)[N], float* row, int p, int lane, int C) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (col(p, k, lane) < C) {
        if constexpr (V > 1) {
#pragma unroll
          for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(row + col(p, 0, lane) + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        } else row[col(p, k, lane)] = x[k];
      }
  }
};
template <typename T, int V, int N>
__device__ __forceinline__ void finish_row(float (&x)[N], float* row, float scale, int accumulate, int p, int lane, int C) {
  float old[N];
  if (accumulate) Piece<T, V>::load32(old, row, p, lane, C);
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = accumulate ? old[e] + scale * x[e] : scale * x[e];
  Piece<T, V>::store32(x, row, p, lane, C);
}

// ---- forward ----------------------------------------------------------------------------------------------------------
// `per` rows of n units (16-byte pieces, or elements) each per workgroup, units 1024 blockIdx.y .. of them.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const T* table, const int32_t* ids, T* out, float scale, int rows, int vocab, int n, int per) {
  const int64_t row0 = (int64_t)blockIdx.x * per;
  const int here = (int)min((int64_t)per, rows - row0), first = 1024 * blockIdx.y, units = min(n - first, 1024), total = here * units;
  typedef typename std::conditional<VEC, uint4, T>::type Unit;
  const Unit* const from = reinterpret_cast<const Unit*>(table);
  Unit* const to = reinterpret_cast<Unit*>(out);
  Unit x[4];
  int r[4], c[4];
  bool in[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int e = min((int)threadIdx.x + 256 * u, total - 1);
    r[u] = e / units;
    c[u] = first + e - r[u] * units;
    const int id = ids[row0 + r[u]];
    in[u] = (unsigned)id < (unsigned)vocab;
    x[u] = from[(int64_t)(in[u] ? id : 0) * n + c[u]];
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if ((int)threadIdx.x + 256 * u >= total) break;
    if constexpr (VEC) {
      Chunk16<T> k;
      k.v = x[u];
#pragma unroll
      for (int e = 0; e < Elem<T>::VEC; ++e) k.e[e] = in[u] ? Elem<T>::from_f32(scale * Elem<T>::to_f32(k.e[e])) : T(0);
      to[(row0 + r[u]) * n + c[u]] = k.v;
    } else {
      to[(row0 + r[u]) * n + c[u]] = in[u] ? Elem<T>::from_f32(scale * Elem<T>::to_f32(x[u])) : T(0);
    }
  }
}

// ---- backward, up to FEW tokens -----------------------------------------------------------------------------------------
// A wavefront's rows of the table are blockIdx.x * 4 * per + wave, + 4, ..: matched against all ids, their tokens listed in LDS in order, summed.
template <typename T, int V>
__global__ __launch_bounds__(256) void embedding_bwd_few_kernel(const int32_t* ids, const T* dout, float* dtable, float scale, int accumulate, int rows, int vocab,
                                                                int C, int per) {
  using P = Piece<T, V>;
  __shared__ int list[4][FEW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = blockIdx.y;
  int id[FEW / 64];
#pragma unroll
  for (int k = 0; k < FEW / 64; ++k) id[k] = lane + 64 * k < rows ? ids[lane + 64 * k] : -1;
  for (int i = 0; i < per; ++i) {
    const int64_t v = (blockIdx.x * (int64_t)per + i) * 4 + wave;
    if (v >= vocab) return;
    int n = 0;
#pragma unroll
    for (int k = 0; k < FEW / 64; ++k) {
      const bool hit = id[k] == (int)v;
      const uint64_t mask = __ballot(hit);
      if (hit) list[wave][n + __popcll(mask & ((1ull << lane) - 1))] = lane + 64 * k;
      n += __popcll(mask);
    }
    if (n == 0 && accumulate) continue;
    float sum[P::N] = {};
    for (int j0 = 0; j0 < n; j0 += 8) {
      typename P::Bits b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) P::load(b[j], dout + (int64_t)list[wave][min(j0 + j, n - 1)] * C, p, lane, C);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float x[P::N];
        P::values(b[j], x);
        if (j0 + j < n)
#pragma unroll
          for (int e = 0; e < P::N; ++e) sum[e] += x[e];
      }
    }
    finish_row<T, V>(sum, dtable + v * C, scale, accumulate, p, lane, C);
  }
}

// ---- backward, sorted ---------------------------------------------------------------------------------------------------
// Workgroups 0 .. runs - 1 sort a run each (ids that are no word come last, as ~0); the others clear the table, 64 KB each.
__global__ __launch_bounds__(1024) void embedding_sort_kernel(const int32_t* ids, uint32_t* word, int* token, float* dtable, int64_t elements, int rows, int vocab, int runs) {
  const int t = threadIdx.x;
  if ((int)blockIdx.x >= runs) {
    const int64_t head = min((int64_t)((16 - reinterpret_cast<uintptr_t>(dtable) % 16) % 16 / 4), elements), pieces = (elements - head) / 4;
    float4* const to = reinterpret_cast<float4*>(dtable + head);
    const int64_t e = (int64_t)(blockIdx.x - runs) * 4096 + t;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (e + 1024 * u < pieces) to[e + 1024 * u] = make_float4(0.f, 0.f, 0.f, 0.f);
    if ((int)blockIdx.x == runs) {
      if (t < head) dtable[t] = 0.f;
      const int64_t tail = head + 4 * pieces + t;
      if (tail < elements) dtable[tail] = 0.f;
    }
    return;
  }
  __shared__ uint64_t key[RUN];
  const uint32_t base = blockIdx.x * RUN;
#pragma unroll
  for (int i = t; i < RUN; i += 1024) {
    const uint32_t at = base + i;
    const uint32_t id = at < (uint32_t)rows ? (uint32_t)ids[at] : ~0u;
    key[i] = ((uint64_t)(id < (uint32_t)vocab ? id : ~0u) << 32) | at;
  }
  for (int size = 2; size <= RUN; size <<= 1)
    for (int stride = size >> 1; stride > 0; stride >>= 1) {
      __syncthreads();
      const int i = 2 * t - (t & (stride - 1)), j = i + stride;
      const uint64_t x = key[i], y = key[j];
      if ((x > y) == ((i & size) == 0)) {
        key[i] = y;
        key[j] = x;
      }
    }
  __syncthreads();
#pragma unroll
  for (int i = t; i < RUN; i += 1024)
    if (base + i < (uint32_t)rows) {
      word[base + i] = (uint32_t)(key[i] >> 32);
      token[base + i] = (int)(uint32_t)key[i];
    }
}
// Sorted runs of `run` (a power of two) to runs of WAYS times that.  Equal words: an earlier run's come first.
__global__ __launch_bounds__(256) void embedding_merge_kernel(const uint32_t* word, const int* token, uint32_t* word_out, int* token_out, int rows, int run) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= rows) return;
  const int64_t own = e / run, group = own / WAYS * WAYS;
  const uint32_t w = word[e];
  int below[WAYS] = {};
  for (int s = run; s > 0; s >>= 1) {
    uint32_t x[WAYS];
#pragma unroll
    for (int q = 0; q < WAYS; ++q) x[q] = word[min((group + q) * run + below[q] + s - 1, (int64_t)rows - 1)];
#pragma unroll
    for (int q = 0; q < WAYS; ++q) {
      const bool inside = below[q] + s <= run && (group + q) * run + below[q] + s <= rows;
      if (inside && (group + q < own ? x[q] <= w : x[q] < w)) below[q] += s;
    }
  }
  int64_t to = group * run + (e - own * run);
#pragma unroll
  for (int q = 0; q < WAYS; ++q)
    if (group + q != own) to += below[q];
  word_out[to] = w;
  token_out[to] = token[e];
}
// part[chunk][0]: of a word that began before the chunk; [1]: of one that began in it and goes on.
template <typename T, int V>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const uint32_t* word, const int* token, const T* dout, float* dtable, float* part, float scale, int accumulate,
                                                            int rows, int C) {
  using P = Piece<T, V>;
  const int lane = threadIdx.x & 63, p = blockIdx.y;
  const int64_t chunk = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), e0 = chunk * CHUNK;
  if (e0 >= rows) return;
  const int there = (int)min((int64_t)CHUNK, rows - e0);
  const uint32_t w = lane < there ? word[e0 + lane] : ~0u;
  const int at = lane < there ? token[e0 + lane] : 0;
  const uint32_t before = e0 > 0 ? word[e0 - 1] : ~0u, after = e0 + there < rows ? word[e0 + there] : ~0u;
  const int n = __popcll(__ballot(w != ~0u));
  if (n == 0) return;
  const uint32_t next = __shfl_down(w, 1, 64);
  const uint64_t ends = __ballot(lane == n - 1 || (lane < n && next != w));
  float sum[P::N] = {};
  bool first = true;
  for (int j0 = 0; j0 < n; j0 += 8) {
    typename P::Bits b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) P::load(b[j], dout + (int64_t)__builtin_amdgcn_readlane(at, min(j0 + j, n - 1)) * C, p, lane, C);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j0 + j >= n) break;
      float x[P::N];
      P::values(b[j], x);
#pragma unroll
      for (int e = 0; e < P::N; ++e) sum[e] += x[e];
      if ((ends >> (j0 + j)) & 1) {
        const uint32_t here = __builtin_amdgcn_readlane(w, j0 + j);
        if (first && here == before) P::store32(sum, part + 2 * chunk * C, p, lane, C);
        else if (j0 + j == there - 1 && here == after) P::store32(sum, part + (2 * chunk + 1) * C, p, lane, C);
        else finish_row<T, V>(sum, dtable + (int64_t)here * C, scale, accumulate, p, lane, C);
#pragma unroll
        for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
        first = false;
      }
    }
  }
}
template <typename T, int V>
__global__ __launch_bounds__(256) void embedding_join_kernel(const uint32_t* word, float* dtable, const float* part, float scale, int accumulate, int rows, int C) {
  using P = Piece<T, V>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = blockIdx.y;
  const int64_t chunk = blockIdx.x, e0 = chunk * CHUNK;
  // (the last chunk is not launched: nothing goes on behind it)
  const uint32_t w = word[e0 + CHUNK - 1];
  if (w == ~0u || word[e0 + CHUNK] != w || (word[e0] == w && e0 > 0 && word[e0 - 1] == w)) return;
  // tokens of the word behind the chunk: the last of them by a search of 64 ways
  int64_t lo = e0 + CHUNK, n = rows - lo;  // word[lo] is w
  while (n > 1) {
    const int64_t step = (n + 63) / 64, i = lane * step;
    const int64_t is = __popcll(__ballot(i < n && word[lo + min(i, n - 1)] == w)) - 1;
    lo += is * step;
    n = min(step, n - is * step);
  }
  const int64_t last = lo / CHUNK;
  float sum[P::N];
  if (wave == 0) P::load32(sum, part + (2 * chunk + 1) * C, p, lane, C);
  else
#pragma unroll
    for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
  for (int64_t k0 = chunk + 1 + wave; k0 <= last; k0 += 16) {
    float x[4][P::N];
#pragma unroll
    for (int j = 0; j < 4; ++j) P::load32(x[j], part + 2 * min(k0 + 4 * j, last) * C, p, lane, C);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (k0 + 4 * j <= last)
#pragma unroll
        for (int e = 0; e < P::N; ++e) sum[e] += x[j][e];
  }
  __shared__ float shares[3][P::N][64];
  if (wave)
#pragma unroll
    for (int e = 0; e < P::N; ++e) shares[wave - 1][e][lane] = sum[e];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int e = 0; e < P::N; ++e) sum[e] = (sum[e] + shares[0][e][lane]) + (shares[1][e][lane] + shares[2][e][lane]);
  finish_row<T, V>(sum, dtable + (int64_t)w * C, scale, accumulate, p, lane, C);
}

template <typename T> hipError_t forward(const T* table, const int32_t* ids, T* out, float scale, int rows, int vocab, int C, hipStream_t stream) {
  const bool vec = C % Elem<T>::VEC == 0 && aligned16(table) && aligned16(out);
  const int n = vec ? C / Elem<T>::VEC : C, per = std::max(1, 1024 / n);
  const dim3 grid((unsigned)((rows + (int64_t)per - 1) / per), (n + 1023) / 1024);
  if (vec) hipLaunchKernelGGL((embedding_fwd_kernel<T, true>), grid, dim3(256), 0, stream, table, ids, out, scale, rows, vocab, n, per);
  else hipLaunchKernelGGL((embedding_fwd_kernel<T, false>), grid, dim3(256), 0, stream, table, ids, out, scale, rows, vocab, n, per);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t backward(const int32_t* ids, const T* dout, float* dtable, float scale, void* workspace, int accumulate, int rows, int vocab, int C, hipStream_t stream) {
  const unsigned pieces = (C + Piece<T, V>::SPAN - 1) / Piece<T, V>::SPAN;
  if (rows <= FEW) {
    const int per = 8;
    hipLaunchKernelGGL((embedding_bwd_few_kernel<T, V>), dim3((unsigned)((vocab + 4ll * per - 1) / (4 * per)), pieces), dim3(256), 0, stream, ids, dout, dtable, scale,
                       accumulate, rows, vocab, C, per);
    return hipGetLastError();
  }
  uint32_t* word[2] = {static_cast<uint32_t*>(workspace), static_cast<uint32_t*>(workspace) + rows};
  int* token[2] = {reinterpret_cast<int*>(word[1] + rows), reinterpret_cast<int*>(word[1] + rows) + rows};
  float* part = static_cast<float*>(workspace) + (4ll * rows + 63) / 64 * 64;
  const int runs = (int)((rows + (int64_t)RUN - 1) / RUN);
  const int64_t elements = (int64_t)vocab * C, clear = accumulate ? 0 : (elements + 16383) / 16384;
  hipLaunchKernelGGL(embedding_sort_kernel, dim3((unsigned)(runs + clear)), dim3(1024), 0, stream, ids, word[0], token[0], dtable, elements, rows, vocab, runs);
  hipError_t e = hipGetLastError();
  int at = 0;
  for (int64_t run = RUN; run < rows && e == hipSuccess; run *= WAYS, at ^= 1) {
    hipLaunchKernelGGL(embedding_merge_kernel, dim3((unsigned)((rows + 255ll) / 256)), dim3(256), 0, stream, word[at], token[at], word[at ^ 1], token[at ^ 1], rows, (int)run);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  const int64_t chunks = (rows + (int64_t)CHUNK - 1) / CHUNK;
  hipLaunchKernelGGL((embedding_sum_kernel<T, V>), dim3((unsigned)((chunks + 3) / 4), pieces), dim3(256), 0, stream, word[at], token[at], dout, dtable, part, scale, accumulate,
                     rows, C);
  if ((e = hipGetLastError()) != hipSuccess || chunks == 1) return e;
  hipLaunchKernelGGL((embedding_join_kernel<T, V>), dim3((unsigned)(chunks - 1), pieces), dim3(256), 0, stream, word[at], dtable, part, scale, accumulate, rows, C);
  return hipGetLastError();
}
template <typename T>
hipError_t backward(const int32_t* ids, const T* dout, float* dtable, float scale, void* workspace, int accumulate, int rows, int vocab, int C, hipStream_t stream) {
  const bool vec = C % Elem<T>::VEC == 0 && aligned16(dout) && aligned16(dtable);
  return vec ? backward<T, Elem<T>::VEC>(ids, dout, dtable, scale, workspace, accumulate, rows, vocab, C, stream)
             : backward<T, 1>(ids, dout, dtable, scale, workspace, accumulate, rows, vocab, C, stream);
}

}  // namespace

hipError_t launch_embedding_fwd(const void* table, const int32_t* ids, void* out, float scale, int rows, int vocab, int C, int dtype,
                                hipStream_t stream) {
  return dtype == DT_BF16 ? forward(static_cast<const uint16_t*>(table), ids, static_cast<uint16_t*>(out), scale, rows, vocab, C, stream)
                          : forward(static_cast<const float*>(table), ids, static_cast<float*>(out), scale, rows, vocab, C, stream);
}

int64_t embedding_bwd_workspace_bytes(int rows, int C) { return 16ll * rows + 8ll * C * ((rows + 31ll) / 32) + 512; }

hipError_t launch_embedding_bwd(const int32_t* ids, const void* dout, float* dtable, float scale, void* workspace, bool accumulate, int rows, int vocab, int C,
                                int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? backward(ids, static_cast<const uint16_t*>(dout), dtable, scale, workspace, accumulate, rows, vocab, C, stream)
                          : backward(ids, static_cast<const float*>(dout), dtable, scale, workspace, accumulate, rows, vocab, C, stream);
}

}  // namespace cdp
