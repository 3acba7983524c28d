// Embedding: rows of a table by token ids, scaled, and the gradient of the table.
//
// Forward: a gather in 16-byte pieces.  Bound by memory: every token's row read (a repeated one from cache) and written (32768 tokens, 2048 columns, bf16:
// 33 us, 8.2 TB/s of rows in and out).
//
// Backward: dtable[v] = scale * sum of the rows of dout whose token is v, in fp32 and in a fixed order, without atomics.  The least it has to do is to read dout
// and write the table; what makes it more than a copy is that a few words are a large part of a text, so that a row of the table is the sum
// of anything from none to thousands of rows.  The tokens are sorted by word (stably: a word's tokens stay in order):
//   1. runs of 2048 in registers and LDS; in the same launch, under the sort, all other workgroups write the zeros of the table (two thirds of them under 2.);
//   2. sixteen runs to one, repeated: a token's place is the sum of its ranks in the sixteen, each a binary search;
//   3. a workgroup per 32 sorted tokens and 512 columns of their rows (fp32: 256): words that begin and end among them are finished there; of one
//      that goes on, the sums before the first and after the last border go to the workspace;
//   4. those sums, a workgroup per word that crosses a border.
// Bound by the writes of the table (us, bf16: 8192 tokens, 50257 x 768 38; 32768 tokens, 128000 x 2048 258, of which writing zeros alone is 151 at the rate
// of a fill, 6.9 TB/s) and, for small tables, by four dependent launches (2000 tokens, 257 x 768 11).
// Up to 256 tokens are looked for by comparison instead: every row of the table is matched against all ids, which are in registers, in one launch.
#include "elem.h"
#include "kernels.h"

#include <algorithm>

namespace cdp {

namespace {

constexpr int RUN = 2048, WAYS = 16, CHUNK = 32, FEW = 256;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// What a lane of a wavefront holds of a row, columns p * SPAN ..: K groups of V neighbouring columns, 64 V apart (V = 4: what makes 16 bytes of the table
// per lane, so that a wavefront writes whole lines; V = 1 for rows that are not whole groups).
template <typename T, int V> struct Piece {
  static constexpr int K = V == 1 ? 8 : 4 / (int)sizeof(T), N = V * K, SPAN = 64 * N;
  __device__ static __forceinline__ int col(int p, int k, int lane) { return p * SPAN + (64 * k + lane) * V; }
  // the bits: a conversion is a use, which waits for the load
  typedef typename std::conditional<V == 1, T, typename std::conditional<sizeof(T) == 2, uint2, uint4>::type>::type Group;
  struct Bits { Group g[K]; };
  __device__ static __forceinline__ void load(Bits& b, const T* row, int p, int lane, int C) {
#pragma unroll
    for (int k = 0; k < K; ++k) b.g[k] = *reinterpret_cast<const Group*>(row + min(col(p, k, lane), C - V));
  }
  __device__ static __forceinline__ void add(float (&sum)[N], const Bits& b) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      union { Group g; T e[V]; } c;
      c.g = b.g[k];
#pragma unroll
      for (int e = 0; e < V; ++e) sum[V * k + e] += Elem<T>::to_f32(c.e[e]);
    }
  }
  // fp32 rows of the table and of the workspace
  typedef typename std::conditional<V == 1, float, float4>::type Group32;
  __device__ static __forceinline__ void load32(float (&x)[N], const float* row, int p, int lane, int C) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      union { Group32 g; float e[V]; } c;
      c.g = *reinterpret_cast<const Group32*>(row + min(col(p, k, lane), C - V));
#pragma unroll
      for (int e = 0; e < V; ++e) x[V * k + e] = c.e[e];
    }
  }
  __device__ static __forceinline__ void store32(const float (&x)[N], float* row, int p, int lane, int C) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (col(p, k, lane) < C) {
        union { Group32 g; float e[V]; } c;
#pragma unroll
        for (int e = 0; e < V; ++e) c.e[e] = x[V * k + e];
        *reinterpret_cast<Group32*>(row + col(p, k, lane)) = c.g;
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
      for (int j = 0; j < 8; ++j)
        if (j0 + j < n) P::add(sum, b[j]);
    }
    finish_row<T, V>(sum, dtable + v * C, scale, accumulate, p, lane, C);
  }
}

// ---- backward, sorted ---------------------------------------------------------------------------------------------------
// Zeros to a workgroup's part of the table, one 16-byte piece a thread (1 GB so 152 us in workgroups of 256 and 166 in workgroups of 1024, four pieces a
// thread 171 and 190, a grid that walks the table 208 and more).  Pieces are counted from `first`.
__device__ __forceinline__ void clear_table(float* table, int64_t elements, int64_t first) {
  const int64_t head = min((int64_t)((16 - reinterpret_cast<uintptr_t>(table) % 16) % 16 / 4), elements), pieces = (elements - head) / 4, e = first + threadIdx.x;
  if (e < pieces) reinterpret_cast<float4*>(table + head)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (first == 0) {
    if ((int)threadIdx.x < head) table[threadIdx.x] = 0.f;
    const int64_t tail = head + 4 * pieces + threadIdx.x;
    if (tail < elements) table[tail] = 0.f;
  }
}
// The value of lane `lane ^ M`.
template <int M> __device__ __forceinline__ uint32_t across_lanes(uint32_t v, int lane) {
  if constexpr (M == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);
  else if constexpr (M == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);
  else if constexpr (M == 4) {  // four on for the lower four of eight, four back for the upper
    const uint32_t x = __builtin_amdgcn_update_dpp(0, v, 0x104, 0xf, 0x5, false);
    return __builtin_amdgcn_update_dpp(x, v, 0x114, 0xf, 0xa, false);
  } else if constexpr (M == 8) return __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false);
  else if constexpr (M == 16) {
    const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return lane & 16 ? x[0] : x[1];
  } else {
    const auto x = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane & 32 ? x[0] : x[1];
  }
}
template <int M> __device__ __forceinline__ uint64_t across_lanes(uint64_t v, int lane) {
  return (uint64_t)across_lanes<M>((uint32_t)(v >> 32), lane) << 32 | across_lanes<M>((uint32_t)v, lane);
}
// Workgroups 0 .. runs - 1 sort a run each (ids that are no word come last); the others clear the table.  A key is the word and the place in the run,
// two neighbours a thread; keys less than 128 apart are exchanged between lanes without LDS, ten steps of 66 go through LDS (every one of them 14 us; eight keys
// a thread of 256, where three steps are left, 11).
constexpr int SORTERS = 1024;
template <typename Key>
__global__ __launch_bounds__(SORTERS) void embedding_sort_kernel(const int32_t* ids, uint32_t* word, int* token, float* dtable, int64_t elements, int rows, int vocab, int runs) {
  if ((int)blockIdx.x >= runs) return clear_table(dtable, elements, (int64_t)(blockIdx.x - runs) * SORTERS);
  constexpr int BITS = 11, K = RUN / SORTERS;
  static_assert(RUN == 1 << BITS, "a place in the run");
  __shared__ Key keys[RUN];
  const int lane = threadIdx.x & 63, i = K * threadIdx.x;
  const uint32_t base = blockIdx.x * RUN;
  Key k[K];
#pragma unroll
  for (int u = 0; u < K; ++u) {
    const uint32_t at = base + i + u, id = at < (uint32_t)rows ? (uint32_t)ids[at] : ~0u;
    k[u] = ((Key)min(id, (uint32_t)vocab) << BITS) | (i + u);
  }
  auto keep = [](Key mine, Key other, bool low) { return low == (mine < other) ? mine : other; };
  static_for<BITS>([&](auto s) {
    constexpr int size = 2 << decltype(s)::value;
    static_for<decltype(s)::value + 1>([&](auto d) {
      constexpr int stride = size >> (decltype(d)::value + 1);
      if constexpr (stride >= K) {
        const bool low = ((i & stride) == 0) == ((i & size) == 0);
        if constexpr (stride < 64 * K) {
#pragma unroll
          for (int u = 0; u < K; ++u) k[u] = keep(k[u], across_lanes<stride / K>(k[u], lane), low);
        } else {
          __syncthreads();
#pragma unroll
          for (int u = 0; u < K; ++u) keys[u * SORTERS + threadIdx.x] = k[u];
          __syncthreads();
#pragma unroll
          for (int u = 0; u < K; ++u) k[u] = keep(k[u], keys[u * SORTERS + (threadIdx.x ^ (stride / K))], low);
        }
      } else {
#pragma unroll
        for (int u = 0; u < K; ++u)
          if (!(u & stride)) {
            const bool up = size < K ? (u & size) == 0 : (i & size) == 0;
            const Key x = k[u], y = k[u | stride];
            k[u] = keep(x, y, up);
            k[u | stride] = keep(y, x, !up);
          }
      }
    });
  });
#pragma unroll
  for (int u = 0; u < K; ++u) {
    const uint32_t w = (uint32_t)(k[u] >> BITS);
    if (base + i + u < (uint32_t)rows) {
      word[base + i + u] = w < (uint32_t)vocab ? w : ~0u;
      token[base + i + u] = (int)(base + (uint32_t)(k[u] & (RUN - 1)));
    }
  }
}
// Sorted runs of `run` (a power of two) to runs of WAYS times that: sixteen lanes search an element's place in sixteen runs, which is equal words of
// earlier runs and smaller ones of later runs before it.  Workgroups past `merging` clear the rest of the table.
__global__ __launch_bounds__(256) void embedding_merge_kernel(const uint32_t* word, const int* token, uint32_t* word_out, int* token_out, int rows, int run, float* dtable,
                                                              int64_t elements, int64_t merging, int64_t cleared) {
  if (blockIdx.x >= merging) return clear_table(dtable, elements, (blockIdx.x - merging) * 256 + cleared);
  const int64_t e = (int64_t)blockIdx.x * (256 / WAYS) + threadIdx.x / WAYS;
  if (e >= rows) return;
  const int q = threadIdx.x % WAYS;
  const int64_t own = e / run, other = own / WAYS * WAYS + q, start = other * run;
  const uint32_t w = word[e];
  const int len = (int)max(min((int64_t)run, rows - start), (int64_t)0);
  int below = 0;
  if (other == own) below = (int)(e - start);
  else
    for (int s = run; s > 0; s >>= 1) {
      if (below + s > len) continue;
      const uint32_t x = word[start + below + s - 1];
      if (x < w || (x == w && other < own)) below += s;
    }
#pragma unroll
  for (int s = 1; s < WAYS; s <<= 1) below += __shfl_xor(below, s, 64);
  if (q) return;
  word_out[start + below] = w;  // (start of the group's first run)
  token_out[start + below] = token[e];
}
// A workgroup per 32 sorted tokens and piece of their rows, eight tokens a wavefront, all of them requested at once.  What a word has in a wavefront goes to the
// table where it begins and ends there, else to LDS: heads (it began before) and tails (it began here and goes on), which the wavefront where it
// began adds up.  part[chunk][0]: of a word that began before the chunk; [1]: of one that began in it and goes on.
template <typename T, int V>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const uint32_t* word, const int* token, const T* dout, float* dtable, float* part, float scale, int accumulate,
                                                            int rows, int C) {
  using P = Piece<T, V>;
  constexpr int U = CHUNK / 4;
  __shared__ float heads[4][P::N][64], tails[4][P::N][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = blockIdx.y;
  const int64_t chunk = blockIdx.x, e0 = chunk * CHUNK;
  const int there = (int)min((int64_t)CHUNK, rows - e0);
  const uint32_t w = lane < there ? word[e0 + lane] : ~0u;
  const int at = lane < there ? token[e0 + lane] : 0;
  const uint32_t before = e0 > 0 ? word[e0 - 1] : ~0u, after = e0 + there < rows ? word[e0 + there] : ~0u;
  const int n = __popcll(__ballot(w != ~0u)), j0 = wave * U;
  if (n == 0) return;
  typename P::Bits b[U];
  if (j0 < n)
#pragma unroll
    for (int j = 0; j < U; ++j) P::load(b[j], dout + (int64_t)__builtin_amdgcn_readlane(at, min(j0 + j, n - 1)) * C, p, lane, C);
  uint32_t next = __shfl_down(w, 1, 64), previous = __shfl_up(w, 1, 64);
  if (lane == there - 1) next = after;
  if (lane == 0) previous = before;
  const uint32_t begins = (uint32_t)__ballot(lane < n && previous != w), ends = (uint32_t)__ballot(lane < n && next != w);
  float sum[P::N] = {};
  bool began = (begins >> j0) & 1, going = false;  // this wavefront's last word begins in it and goes on
  if (j0 < n)
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (j0 + j >= n) break;
      P::add(sum, b[j]);
      const bool end = (ends >> (j0 + j)) & 1;
      if (!end && j < U - 1 && j0 + j < n - 1) continue;
      going = began && !end;
      if (began && end) finish_row<T, V>(sum, dtable + (int64_t)__builtin_amdgcn_readlane(w, j0 + j) * C, scale, accumulate, p, lane, C);
      else {
        float(*const to)[64] = began ? tails[wave] : heads[wave];
#pragma unroll
        for (int e = 0; e < P::N; ++e) to[e][lane] = sum[e];
      }
#pragma unroll
      for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
      began = true;
    }
  __syncthreads();
  const bool lead = wave == 0 && !(begins & 1);  // the chunk's first word began before it
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {  // the word that began before the chunk, the one that began in this wavefront
    if (k ? !going : !lead) continue;
    bool open = true;
#pragma unroll
    for (int e = 0; e < P::N; ++e) sum[e] = k ? tails[wave][e][lane] : 0.f;
    for (int u = k ? wave + 1 : 0; open && u * U < n; ++u) {
#pragma unroll
      for (int e = 0; e < P::N; ++e) sum[e] += heads[u][e][lane];
      open = !((ends >> (u * U)) & ((1u << U) - 1));
    }
    if (!k) P::store32(sum, part + 2 * chunk * C, p, lane, C);
    else if (open) P::store32(sum, part + (2 * chunk + 1) * C, p, lane, C);
    else finish_row<T, V>(sum, dtable + (int64_t)__builtin_amdgcn_readlane(w, j0 + U - 1) * C, scale, accumulate, p, lane, C);
  }
}
constexpr int JOIN = 8;  // wavefronts that share a word's chunks
template <typename T, int V>
__global__ __launch_bounds__(64 * JOIN) void embedding_join_kernel(const uint32_t* word, float* dtable, const float* part, float scale, int accumulate, int rows, int C) {
  using P = Piece<T, V>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = blockIdx.y;
  const int64_t chunk = blockIdx.x, e0 = chunk * CHUNK;
  // (the last chunk is not launched: nothing goes on behind it)
  const uint32_t w = word[e0 + CHUNK - 1], next = word[e0 + CHUNK], first = word[e0], before = word[max(e0 - 1, (int64_t)0)];
  if (w == ~0u || next != w || (first == w && e0 > 0 && before == w)) return;
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
  for (int64_t k0 = chunk + 1 + wave; k0 <= last; k0 += 8 * JOIN) {
    float x[8][P::N];
#pragma unroll
    for (int j = 0; j < 8; ++j) P::load32(x[j], part + 2 * min(k0 + JOIN * j, last) * C, p, lane, C);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k0 + JOIN * j <= last)
#pragma unroll
        for (int e = 0; e < P::N; ++e) sum[e] += x[j][e];
  }
  __shared__ float shares[JOIN][P::N][64];
#pragma unroll
  for (int e = 0; e < P::N; ++e) shares[wave][e][lane] = sum[e];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int e = 0; e < P::N; ++e) {
    sum[e] = 0.f;
#pragma unroll
    for (int k = 0; k < JOIN; ++k) sum[e] += shares[k][e][lane];
  }
  finish_row<T, V>(sum, dtable + (int64_t)w * C, scale, accumulate, p, lane, C);
}

template <typename T> hipError_t forward(const T* table, const int32_t* ids, T* out, float scale, int rows, int vocab, int C, hipStream_t stream) {
  const bool vec = C % Elem<T>::VEC == 0 && aligned16(table) && aligned16(out);
  const int n = vec ? C / Elem<T>::VEC : C, per = std::max(1, 1024 / n);
  const dim3 grid((unsigned)((rows + (int64_t)per - 1) / per), (n + 1023) / 1024);
  if (!launchable(grid.x, 256)) return hipErrorInvalidConfiguration;
  if (vec) hipLaunchKernelGGL((embedding_fwd_kernel<T, true>), grid, dim3(256), 0, stream, table, ids, out, scale, rows, vocab, n, per);
  else hipLaunchKernelGGL((embedding_fwd_kernel<T, false>), grid, dim3(256), 0, stream, table, ids, out, scale, rows, vocab, n, per);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t backward(const int32_t* ids, const T* dout, float* dtable, float scale, void* workspace, int accumulate, int rows, int vocab, int C, hipStream_t stream) {
  const unsigned pieces = (C + Piece<T, V>::SPAN - 1) / Piece<T, V>::SPAN;
  // (a large table is cleared faster by itself: 200 tokens, 100000 x 2048 177 us here)
  if (rows <= FEW && (accumulate || (int64_t)vocab * C <= (8 << 20))) {
    const int per = 8;
    if (!launchable((vocab + 4ll * per - 1) / (4 * per), 256)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((embedding_bwd_few_kernel<T, V>), dim3((unsigned)((vocab + 4ll * per - 1) / (4 * per)), pieces), dim3(256), 0, stream, ids, dout, dtable, scale,
                       accumulate, rows, vocab, C, per);
    return hipGetLastError();
  }
  uint32_t* word[2] = {static_cast<uint32_t*>(workspace), static_cast<uint32_t*>(workspace) + rows};
  int* token[2] = {reinterpret_cast<int*>(word[1] + rows), reinterpret_cast<int*>(word[1] + rows) + rows};
  float* part = static_cast<float*>(workspace) + (4ll * rows + 63) / 64 * 64;
  const int runs = (int)((rows + (int64_t)RUN - 1) / RUN);
  // the table is cleared beside the sort and, where there is one, the first merge, whose workgroups are smaller: a third and two thirds
  const int64_t elements = (int64_t)vocab * C, clear = accumulate ? 0 : elements / 4 + 1, beside_sort = (runs > 1 ? (clear + 2) / 3 : clear) + SORTERS - 1;
  const int64_t first = beside_sort / SORTERS * SORTERS * (clear > 0);  // pieces
  const int64_t chunks = (rows + (int64_t)CHUNK - 1) / CHUNK;
  const int64_t merging = ((int64_t)rows * WAYS + 255) / 256, rest = runs > 1 ? (std::max<int64_t>(clear - first, 0) + 255) / 256 : 0;
  if (!launchable(runs + first / SORTERS, SORTERS) || !launchable(merging + rest, 256) || !launchable(chunks, 64 * JOIN)) return hipErrorInvalidConfiguration;
  const dim3 sorting((unsigned)(runs + first / SORTERS));
  if (vocab < (1 << 20)) hipLaunchKernelGGL((embedding_sort_kernel<uint32_t>), sorting, dim3(SORTERS), 0, stream, ids, word[0], token[0], dtable, elements, rows, vocab, runs);
  else hipLaunchKernelGGL((embedding_sort_kernel<uint64_t>), sorting, dim3(SORTERS), 0, stream, ids, word[0], token[0], dtable, elements, rows, vocab, runs);
  hipError_t e = hipGetLastError();
  int at = 0;
  for (int64_t run = RUN; run < rows && e == hipSuccess; run *= WAYS, at ^= 1) {
    const int64_t clearing = run == RUN ? rest : 0;
    hipLaunchKernelGGL(embedding_merge_kernel, dim3((unsigned)(merging + clearing)), dim3(256), 0, stream, word[at], token[at], word[at ^ 1], token[at ^ 1], rows, (int)run, dtable,
                       elements, merging, first);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((embedding_sum_kernel<T, V>), dim3((unsigned)chunks, pieces), dim3(256), 0, stream, word[at], token[at], dout, dtable, part, scale, accumulate,
                     rows, C);
  if ((e = hipGetLastError()) != hipSuccess || chunks == 1) return e;
  hipLaunchKernelGGL((embedding_join_kernel<T, V>), dim3((unsigned)(chunks - 1), pieces), dim3(64 * JOIN), 0, stream, word[at], dtable, part, scale, accumulate, rows, C);
  return hipGetLastError();
}
template <typename T>
hipError_t backward(const int32_t* ids, const T* dout, float* dtable, float scale, void* workspace, int accumulate, int rows, int vocab, int C, hipStream_t stream) {
  const bool vec = C % 4 == 0 && reinterpret_cast<uintptr_t>(dout) % (4 * sizeof(T)) == 0 && aligned16(dtable);
  return vec ? backward<T, 4>(ids, dout, dtable, scale, workspace, accumulate, rows, vocab, C, stream)
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
