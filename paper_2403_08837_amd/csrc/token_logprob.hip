// Log probabilities of given tokens, the entropy and the likeliest tokens of rows of logits, and the gradient.  With z = scale * logits, of a row:
//   lse = log sum exp z,  p = exp(z - lse),  logprob = z[target] - lse,  entropy = lse - sum p z;
//   dlogits[j] = scale * (dlogprob * ((j == target) - p[j]) - dentropy * p[j] * (log p[j] + entropy)).
//
// Bound by memory: a row is read once forward, read and written once backward.  us of 4096 x 128000 in bf16, a quarter
// not wanted: forward 154 by itself (5.1 TB/s; without t 149), 193 to 209 right behind the backward, whose results are still on their way to memory, with the 8 likeliest 31
// more; backward 350 (5.2 TB/s); 1500 x 50257 in fp32, rows that begin anywhere: 48 by itself (5.6 TB/s), with the 8 likeliest 61, backward 92 to 95.
// A lane keeps the maximum m of what it has seen with s = sum 2^y and
// t = sum 2^y y, y = (logit - m) scale log2(e): a new maximum multiplies s by f = 2^d and makes t = f (t + d s).  That maximum is raised once for eight values at most.
// entropy = log s - (t / s) log 2 over the row.
//
// The likeliest tokens come from the same pass: a border that k of the lanes' maxima (ordered by value, then by place) are not below is one that the k-th token is
// not below either, and only lanes whose maximum is not below it, little more than k of 256, can hold better ones.  Their share of the row is read again, and
// what is not below the border, little more than k tokens, is ranked.
#include "elem.h"
#include "kernels.h"
#include "lane_sums.h"

#include <algorithm>
#include <climits>

namespace cdp {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64, UNROLL = 4;
constexpr int MAX_FOUND = 1024;  // tokens not below the border that LDS holds at once; where there are more (it takes ordered rows) the border is raised
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;
typedef unsigned long long u64;

// A row as 16-byte pieces of aligned memory: piece k has the elements k * V - lead .. k * V - lead + V - 1, the first and the last of them perhaps not all.
template <typename T> struct Row {
  static constexpr int V = Elem<T>::VEC;
  const T* at;     // of element 0
  int lead, size;  // elements that piece 0 lacks; elements
  __device__ __forceinline__ Row(const T* p, int n) : at(p), lead((int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T))), size(n) {}
  __device__ __forceinline__ int pieces() const { return (int)(((unsigned)size + lead + V - 1) / V); }
  __device__ __forceinline__ bool whole(int k) const { return (k > 0 || !lead) && (int64_t)(k + 1) * V - lead <= size; }
  __device__ __forceinline__ uint4 get(int k) const { return *reinterpret_cast<const uint4*>(at + ((int64_t)k * V - lead)); }
  // elements outside the row read as `none`
  __device__ __forceinline__ void values(int k, float none, float (&v)[V]) const {
    Chunk16<T> c;
    if (whole(k)) {
      c.v = get(k);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = Elem<T>::to_f32(c.e[i]);
      return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t j = (int64_t)k * V - lead + i;
      v[i] = j >= 0 && j < size ? Elem<T>::to_f32(at[j]) : none;
    }
  }
};

// 32 bits that order floats (-0 as 0, NaN as the lowest), and with a place 64 bits: larger values first, then lower places.  0: nothing.
__device__ __forceinline__ unsigned ordered(float v) {
  v = v != v ? -INFINITY : v + 0.f;
  const unsigned u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ u64 key_of(float v, unsigned place) { return (u64)ordered(v) << 32 | (0xffffffffu - place); }
__device__ __forceinline__ int place_of(u64 key) { return (int)(0xffffffffu - (unsigned)key); }

// (fmaxf of values that come out of shifts and masks makes each canonical first: an instruction more for every one)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float v;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(v) : "v"(a), "v"(b), "v"(c));
  return v;
}
struct Sums {
  float m = -INFINITY, s = 0.f, t = 0.f;
  static __device__ __forceinline__ Sums of(float4 q) {
    Sums w;
    w.m = q.x;
    w.s = q.y;
    w.t = q.z;
    return w;
  }
  __device__ __forceinline__ float4 all() const { return make_float4(m, s, t, 0.f); }
  // the values so far relative to another maximum, not below m
  __device__ __forceinline__ void raise(float to, float c) {
    const float d = fmaxf((m - to) * c, -256.f), f = __builtin_amdgcn_exp2f(d);  // (0 from there on)
    const bool some = m > -INFINITY;  // (else s and t are zero, or NaN)
    t = some ? f * (t + d * s) : t;
    s = some ? f * s : s;
    m = to;
  }
  __device__ __forceinline__ void join(Sums b, float c) {
    const float to = fmaxf(m, b.m);
    if (m != to) raise(to, c);
    if (b.m != to) b.raise(to, c);
    s += b.s;
    t += b.t;
  }
  template <int V> __device__ __forceinline__ void add(const float (&v)[V], float c) {
    const float from = m > -INFINITY ? m : 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      // (the difference first: the product's rounding would be an exponent for logits of 1e9 and more)
      const float y = (v[i] - from) * c, e = __builtin_amdgcn_exp2f(y);
      s += e;
      t += e * fmaxf(y, -256.f);  // (a value of -infinity has e = 0; one that is NaN is in s)
    }
  }
};
// The sums of a wavefront's lanes, in every lane: their maximum first, then one exponential each.
__device__ __forceinline__ void join_lanes(Sums& w, float c) {
  const float to = lanes_max<64>(w.m);
  if (w.m != to) w.raise(to, c);
  w.s = lanes_sum<64>(w.s);
  w.t = lanes_sum<64>(w.t);
}

// The key of the wanted-th largest of a wavefront's lanes by value, then by place; 0 where there are fewer.
__device__ __forceinline__ u64 border_of(float v, int place, bool there, int wanted) {
  if (v != v) v = -INFINITY;
  unsigned long long left = __builtin_amdgcn_ballot_w64(there);
  const int lane = threadIdx.x & 63;
  while (left) {
    const bool mine = left >> lane & 1;
    const float most = lanes_max<64>(mine ? v : -INFINITY);
    const unsigned long long ties = __builtin_amdgcn_ballot_w64(mine && v == most);
    const int n = __builtin_popcountll(ties);
    if (n < wanted) {
      wanted -= n;
      left &= ~ties;
      continue;
    }
    // of those of one value the wanted-th by place
    unsigned long long equal = ties;
    int at = 0;
    for (; wanted > 0; --wanted) {
      int first = equal >> lane & 1 ? place : INT_MAX;
#pragma unroll
      for (int mask = 1; mask < 64; mask *= 2) first = min(first, __shfl_xor(first, mask, 64));
      at = first;
      equal &= ~__builtin_amdgcn_ballot_w64((equal >> lane & 1) && place == first);
    }
    return key_of(most, (unsigned)at);
  }
  return 0;
}

struct Found {
  float4 sums[WAVES];
  u64 found[MAX_FOUND];
  int lanes[THREADS];
  u64 border, borders[WAVES];
  int count, chosen;
};

// The `top` largest of keys[0 .. n) in order, out(rank, key); by all of a workgroup, for which the keys have been written, with room for a power of two of them.  A few by
// their ranks, more sorted (us, by ranks / sorted: 400 keys 10 / 14, 906 48 / 18).
template <typename F> __device__ __forceinline__ void ranked(u64* keys, int n, int top, F&& out) {
  if (n <= 512) {
    for (int i = threadIdx.x; i < n; i += THREADS) {
      const u64 key = keys[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += keys[j] > key;
      if (rank < top) out(rank, key);
    }
    return;
  }
  int all = 256;
  while (all < n) all *= 2;
  for (int i = n + threadIdx.x; i < all; i += THREADS) keys[i] = 0;
  for (int size = 2; size <= all; size *= 2)
    for (int apart = size / 2; apart > 0; apart /= 2) {
      __syncthreads();
      for (int t = threadIdx.x; t < all / 2; t += THREADS) {
        const int i = 2 * t - (t & (apart - 1)), j = i + apart;
        const u64 x = keys[i], y = keys[j];
        if ((x < y) == ((i & size) == 0)) {
          keys[i] = y;
          keys[j] = x;
        }
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < min(n, top); i += THREADS) out(i, keys[i]);
}

// scale * (l - m) - ls, in 64 bits where the difference is past fp32 (logits of either sign near its end), which the product need not be.
__device__ __forceinline__ float log_of(float scale, float l, float m, float ls) {
  const float d = l - m;
  return fabsf(d) < INFINITY ? fmaf(scale, d, -ls) : (float)((double)scale * ((double)l - (double)m) - (double)ls);
}
// What a row is, from its sums.
__device__ __forceinline__ void write_row(const TokenLogprob& a, int64_t row, const Sums& w, float l) {  // l: the target's logit
  const bool none = w.m == -INFINITY && w.s == 0.f;  // everything masked
  const float ls = logf(w.s), lse = none ? -INFINITY : fmaf(a.scale, w.m, ls);
  a.lse[row] = lse;
  if (a.entropy) a.entropy[row] = none ? 0.f : ls - LN2 * (w.t / w.s);
  if (a.logprob) {
    a.logprob[row] = none || l == -INFINITY ? (w.s != w.s ? w.s : -INFINITY) : log_of(a.scale, l, w.m, ls);
  }
}
__device__ __forceinline__ float top_logprob(const TokenLogprob& a, const Sums& w, float l) {
  if (w.m == -INFINITY && w.s == 0.f) return -INFINITY;
  return l == -INFINITY && w.s == w.s ? -INFINITY : log_of(a.scale, l, w.m, logf(w.s));
}
// A row that is not wanted: nothing of it is read.
__device__ __forceinline__ void write_none(const TokenLogprob& a, int64_t row) {
  if (threadIdx.x == 0) {
    a.lse[row] = 0.f;
    if (a.entropy) a.entropy[row] = 0.f;
    if (a.logprob) a.logprob[row] = 0.f;
  }
  for (int i = threadIdx.x; i < a.top; i += THREADS) {
    a.top_ids[row * a.top + i] = -1;
    a.top_logprobs[row * a.top + i] = 0.f;
  }
}

// Part blockIdx.x % parts of row blockIdx.x / parts: with parts > 1 its sums and its `top` largest go to the workspace.
template <typename T, bool TOP> __global__ __launch_bounds__(THREADS) void token_logprob_kernel(const TokenLogprob a) {
  constexpr int V = Elem<T>::VEC;
  __shared__ Found f;
  const int64_t row = (int64_t)(blockIdx.x / (unsigned)a.parts);
  const int part = blockIdx.x % (unsigned)a.parts, tid = threadIdx.x;
  const int target = a.targets ? a.targets[row] : 0;
  if (target < 0 || target >= a.vocab) {
    if (part == 0) write_none(a, row);
    return;
  }
  const T* const logits = static_cast<const T*>(a.logits) + row * a.ld;
  const Row<T> r(logits, a.vocab);
  const float c = a.scale * LOG2E, l_target = Elem<T>::to_f32(logits[target]);
  const int all = r.pieces(), share = (all + a.parts - 1) / a.parts;
  const int begin = min(part * share, all), end = min(begin + share, all);
  int inner = begin, whole_end = end;  // the pieces that are whole
  if (begin < end) {
    if (!r.whole(begin)) ++inner;
    if (end - 1 >= inner && !r.whole(end - 1)) --whole_end;
  }
  Sums w;
  int best_piece = begin + tid;  // that of the lane's maximum, the first of several
  auto take = [&](const float (&v)[V], int k) {
    float most = max3(v[0], v[1], v[2]);
#pragma unroll
    for (int i = 3; i < V; i += 2) most = max3(most, v[i], v[i + 1 < V ? i + 1 : i]);
    if (most > w.m) {
      w.raise(most, c);
      best_piece = k;
    }
    w.add<V>(v, c);
  };
  // lane l takes the pieces begin + l, begin + l + THREADS, ..
  int k = begin + tid;
  if (k < inner && k < end) {
    float v[V];
    r.values(k, -INFINITY, v);
    take(v, k);
    k += THREADS;
  }
  const uint4* from = reinterpret_cast<const uint4*>(r.at - r.lead) + k;
  for (; k + (UNROLL - 1) * THREADS < whole_end; k += UNROLL * THREADS) {
    Chunk16<T> q[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) q[u].v = from[u * THREADS];
    from += UNROLL * THREADS;
    __builtin_amdgcn_sched_barrier(0);  // all of them before the first is waited for
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = Elem<T>::to_f32(q[u].e[i]);
      take(v, k + u * THREADS);
    }
  }
  for (; k < end; k += THREADS) {
    float v[V];
    r.values(k, -INFINITY, v);
    take(v, k);
  }
  const float best = w.m;
  if constexpr (TOP) {
    // the first `of` wavefronts have a share of the border each: those that have the lanes for it, and half of theirs at least (the best of a few lanes is no border)
    int of = WAVES;
    while (of > 1 && end - begin - 64 * (of - 1) < 32) --of;
    if (end - begin < (a.top + of - 1) / of) of = 0;
    u64 border = of ? ~0ull : 0;
    if (tid >> 6 < of) border = border_of(best, best_piece, begin + tid < end, (a.top + of - 1) / of);
    if ((tid & 63) == 0) f.borders[tid >> 6] = border;
  }
  join_lanes(w, c);
  if ((tid & 63) == 0) f.sums[tid >> 6] = w.all();
  if (tid == 0) f.count = f.chosen = 0;
  __syncthreads();
  w = Sums::of(f.sums[0]);
#pragma unroll
  for (int i = 1; i < WAVES; ++i) w.join(Sums::of(f.sums[i]), c);
  if (tid == 0) {
    if (a.parts == 1) write_row(a, row, w, l_target);
    else a.part_sums[blockIdx.x] = w.all();
  }
  if constexpr (TOP) {
    // as many lanes as `top` are not below the least of the wavefronts' borders (~0: no say)
    u64 border = f.borders[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) border = f.borders[i] < border ? f.borders[i] : border;
    if (begin + tid < end && key_of(best, (unsigned)best_piece) >= border) f.lanes[atomicAdd(&f.chosen, 1)] = tid;
    // (of places of pieces one of places of elements: anything in that piece)
    if (tid == 0) f.border = border ? (border >> 32) << 32 | (0xffffffffu - (unsigned)((int64_t)(place_of(border) + 1) * V - 1 - r.lead)) : 0;
    __syncthreads();
    const int chosen = f.chosen, steps = (share + THREADS - 1) / THREADS, shift = min(6, 32 - __builtin_clz(steps) - (steps & (steps - 1) ? 0 : 1));  // 2^shift lanes for the pieces of one
    int n;
    for (;;) {
      const u64 least = f.border;
      for (int i = tid >> shift; i < chosen; i += THREADS >> shift) {
        for (int piece = begin + f.lanes[i] + (tid & ((1 << shift) - 1)) * THREADS; piece < end; piece += THREADS << shift) {
          float v[V];
          r.values(piece, 0.f, v);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const int64_t j = (int64_t)piece * V - r.lead + e;
            const u64 key = key_of(v[e], (unsigned)j);
            if (j >= 0 && j < a.vocab && key >= least) {
              const int at = atomicAdd(&f.count, 1);
              // of more than there is room for a sample stays (the at-th with a chance of MAX_FOUND / at), whatever their order: of the first ones the border may hardly rise
              // (us, 2^20 fp32 logits of which 64 lanes have ascending large ones, 64 wanted: 3040 with the first, 996 so)
              if (at < MAX_FOUND) f.found[at] = key;
              else if (const unsigned to = __umulhi((unsigned)key * 2654435769u, (unsigned)at + 1); to < MAX_FOUND) atomicMax(&f.found[to], key);
            }
          }
        }
      }
      __syncthreads();
      n = f.count;
      if (n <= MAX_FOUND) break;
      // the border of those that were kept; what is below it is not among the `top` largest of all
      __syncthreads();
      if (tid == 0) f.count = 0;
      ranked(f.found, MAX_FOUND, a.top, [&](int rank, u64 key) {
        if (rank == a.top - 1) f.border = key;
      });
      __syncthreads();
    }
    if (a.parts == 1) {
      ranked(f.found, n, a.top, [&](int rank, u64 key) {
        a.top_ids[row * a.top + rank] = place_of(key);
        a.top_logprobs[row * a.top + rank] = top_logprob(a, w, value_of((unsigned)(key >> 32)));
      });
    } else {
      u64* const to = a.part_keys + (int64_t)blockIdx.x * a.top;
      ranked(f.found, n, a.top, [&](int rank, u64 key) { to[rank] = key; });
      for (int i = n + tid; i < a.top; i += THREADS) to[i] = 0;
    }
  }
}

// Joins the parts of a row: 4.1 to 4.8 us, 16 x 16 x 20 tokens; beside 10 for the parts, all of it round trips.
template <typename T> __global__ __launch_bounds__(THREADS) void token_logprob_join_kernel(const TokenLogprob a) {
  __shared__ u64 found[LOGPROB_MAX_SPLIT * LOGPROB_MAX_TOP];
  __shared__ int count;
  const int64_t row = blockIdx.x;
  const int target = a.targets ? a.targets[row] : 0, tid = threadIdx.x;
  if (target < 0 || target >= a.vocab) return;
  const float c = a.scale * LOG2E, l_target = Elem<T>::to_f32(static_cast<const T*>(a.logits)[row * a.ld + target]);
  // (at most 32 parts: a lane each, of every wavefront)
  Sums w;
  if ((tid & 63) < a.parts) w = Sums::of(a.part_sums[row * a.parts + (tid & 63)]);
  const u64* const keys = a.part_keys + row * a.parts * a.top;
  const int each = (a.top + a.parts - 1) / a.parts;
  u64 border = a.top && (tid & 63) < a.parts ? keys[(tid & 63) * a.top + each - 1] : ~0ull;
  u64 mine[LOGPROB_MAX_SPLIT * LOGPROB_MAX_TOP / THREADS];
#pragma unroll
  for (int i = 0; i < LOGPROB_MAX_SPLIT * LOGPROB_MAX_TOP / THREADS; ++i) mine[i] = tid + i * THREADS < a.parts * a.top ? keys[tid + i * THREADS] : 0;
  join_lanes(w, c);
  if (tid == 0) write_row(a, row, w, l_target);
  if (!a.top) return;
  // each part's list is in order: the least of their each's-th keys is not above the `top`-th of all
#pragma unroll
  for (int mask = 1; mask < 64; mask *= 2) {
    const u64 other = __shfl_xor(border, mask, 64);
    border = other < border ? other : border;
  }
  if (tid == 0) count = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < LOGPROB_MAX_SPLIT * LOGPROB_MAX_TOP / THREADS; ++i)
    if (mine[i] && mine[i] >= border) found[atomicAdd(&count, 1)] = mine[i];
  __syncthreads();
  ranked(found, count, a.top, [&](int rank, u64 key) {
    a.top_ids[row * a.top + rank] = place_of(key);
    a.top_logprobs[row * a.top + rank] = top_logprob(a, w, value_of((unsigned)(key >> 32)));
  });
}

// Pieces blockIdx.y * share .. of row blockIdx.x, each value's exponential made again from lse.
template <typename T> __global__ __launch_bounds__(THREADS) void token_logprob_bwd_kernel(const TokenLogprob a, int share) {
  constexpr int V = Elem<T>::VEC;
  const int64_t row = blockIdx.x;
  const int target = a.targets ? a.targets[row] : 0;
  const Row<T> r(static_cast<const T*>(a.logits) + row * a.ld, a.vocab);
  T* const out = static_cast<T*>(a.dlogits) + row * a.ld;
  const bool alike = (reinterpret_cast<uintptr_t>(out) & 15) == (reinterpret_cast<uintptr_t>(r.at) & 15);
  const int begin = (int)min((int64_t)blockIdx.y * share, (int64_t)r.pieces()), end = min(begin + share, r.pieces());
  const bool wanted = target >= 0 && target < a.vocab;
  float lse = 0.f, A = 0.f, B = 0.f, at_target = 0.f;
  bool some = wanted;
  if (wanted) {
    lse = a.lse[row];
    const float dl = a.dlogprob ? a.dlogprob[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f;
    some = lse != -INFINITY;  // (a row with everything masked has no gradient)
    A = a.scale * (dl + (a.dentropy ? dh * a.entropy[row] : 0.f));
    if (lse != lse) A = lse;
    B = a.scale * dh * LN2;
    at_target = a.scale * dl;
  }
  auto store = [&](int k, const float (&v)[V]) {
    const int64_t j = (int64_t)k * V - r.lead;
    if (alike && r.whole(k)) {
      Chunk16<T> q;
#pragma unroll
      for (int i = 0; i < V; ++i) q.e[i] = Elem<T>::from_f32(v[i]);
      *reinterpret_cast<uint4*>(out + j) = q.v;
      return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (j + i >= 0 && j + i < r.size) out[j + i] = Elem<T>::from_f32(v[i]);
  };
  auto gradient = [&](int k, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      // a product rounded as lse was, so that the largest of far apart logits has p = 1; not over 1 by lse's rounding; where it is NaN, A is
      const float z = a.scale * v[i], y = __builtin_amdgcn_fmed3f((z - lse) * LOG2E, -256.f, 0.f);
      v[i] = -(__builtin_amdgcn_exp2f(y) * fmaf(B, y, A));
    }
    const int64_t at = (int64_t)target - ((int64_t)k * V - r.lead);
    if (at >= 0 && at < V && a.targets)
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += i == (int)at ? at_target : 0.f;
  };
  int k = begin + threadIdx.x;
  if (!some) {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.f;
    for (; k < end; k += THREADS) store(k, v);
    return;
  }
  for (; k + (UNROLL - 1) * THREADS < end; k += UNROLL * THREADS) {
    float v[UNROLL][V];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) r.values(k + u * THREADS, 0.f, v[u]);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      gradient(k + u * THREADS, v[u]);
      store(k + u * THREADS, v[u]);
    }
  }
  for (; k < end; k += THREADS) {
    float v[V];
    r.values(k, 0.f, v);
    gradient(k, v);
    store(k, v);
  }
}

template <typename T> hipError_t forward(TokenLogprob a, void* workspace, hipStream_t stream) {
  // parts of a row of at least 16 KB, up to 1024 workgroups in all.  (Of more rows, whose last round of workgroups may be short, parts gain what joining them
  // costs: us with parts of 64 KB / whole rows, 1100 x 128000 bf16 46.7 + 4.8 / 53.0, with the 5 likeliest 63.6 + 5.0 / 68.5, 4096 rows 146 + 6 / 157.)
  const int64_t bytes = (int64_t)a.vocab * (int)sizeof(T), room = LOGPROB_BYTES / (16 + 8 * a.top);
  a.parts = workspace ? (int)std::max<int64_t>(1, std::min<int64_t>({LOGPROB_MAX_SPLIT, room / a.rows, 1024 / a.rows, bytes >> 14})) : 1;
  a.part_sums = static_cast<float4*>(workspace);
  a.part_keys = reinterpret_cast<u64*>(a.part_sums + (int64_t)a.rows * a.parts);
  const int64_t groups = (int64_t)a.rows * a.parts;
  if (!launchable(groups, THREADS)) return hipErrorInvalidConfiguration;
  if (a.top) hipLaunchKernelGGL((token_logprob_kernel<T, true>), dim3((unsigned)groups), dim3(THREADS), 0, stream, a);
  else hipLaunchKernelGGL((token_logprob_kernel<T, false>), dim3((unsigned)groups), dim3(THREADS), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  hipLaunchKernelGGL((token_logprob_join_kernel<T>), dim3(a.rows), dim3(THREADS), 0, stream, a);
  return hipGetLastError();
}
template <typename T> hipError_t backward(const TokenLogprob& a, hipStream_t stream) {
  constexpr int V = Elem<T>::VEC;
  const int64_t pieces = ((int64_t)a.vocab + V - 1) / V + 1;
  // 64 KB of a row a workgroup, down to 4 KB where that leaves fewer than four a CU (us so / with 64 KB, 20 x 20803 bf16 3.8 / 8.9)
  int share = 4 * UNROLL * THREADS;
  while (share > THREADS && a.rows * ((pieces + share - 1) / share) < 1024) share /= 2;
  const int64_t segments = (pieces + share - 1) / share;
  if (!launchable(a.rows * segments, THREADS)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((token_logprob_bwd_kernel<T>), dim3(a.rows, (unsigned)segments), dim3(THREADS), 0, stream, a, share);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprob(const TokenLogprob& a, void* workspace, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? forward<uint16_t>(a, workspace, stream) : forward<float>(a, workspace, stream);
}
hipError_t launch_token_logprob_bwd(const TokenLogprob& a, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? backward<uint16_t>(a, stream) : backward<float>(a, stream);
}

}  // namespace cdp
