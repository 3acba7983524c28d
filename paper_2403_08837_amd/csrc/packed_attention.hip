// Causal attention over packed sequences of different lengths, with grouped heads.
//   S = scale q k^T, P = softmax(S) over the keys of the own sequence up to the query itself, out = P v, lse = log sum exp S;
//   backward: P = exp(S - lse), delta = rowsum(dout out), dP = dout v^T, dS = P (dP - delta), dq = scale dS k, dk = scale dS^T q, dv = P^T dout.
//
// One pass over the keys with the running maximum and sum of the softmax; nothing of S or P goes through memory.  A workgroup is four wavefronts
// of 32 rows each (queries forward and for dq, keys for dk and dv) of one head of one sequence and walks tiles of the other side, which two
// stages of LDS hold: the next tile's loads (straight into LDS, zeros past the sequence from the buffer's bounds) are in flight under the products
// of the current one.  Score blocks are contracted so that a lane holds one of the wavefront's own rows, 16 rows of the other side in its
// registers: row sums and maxima stay in the lane (and lane +- 32), and the probabilities are, in the registers they are in, the column operand of the next
// product, whose row operand is read from LDS across rows (bf16: transposing reads) in that same order.
// Work is found on the device: sequence s takes offsets[s + 1] / ROWS - offsets[s] / ROWS + 1 workgroups per head, which is what it needs or one more, so
// that workgroup t's sequence is the last with offsets[s] / ROWS + s <= t: no table, no launch ahead.
// fp32: the same on 32x32x2 products, tiles of 32 rows instead of 64.
#include "elem.h"
#include "kernels.h"

namespace cdp {

namespace {

typedef short att_v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int OWN = 128;  // rows of a workgroup
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// Tile of `OTHER` rows of one head, DW columns (the width rounded up, zeros behind it), in LDS.  16-byte chunk c of row r sits in slot c ^ swz(r) of the
// row: 16 consecutive rows' chunk c are 16 different slots modulo 256 bytes, and so are the pieces that a read across rows takes.
template <typename T, int DW> struct Tile {
  static constexpr int E = sizeof(T), VEC = 16 / E, CPR = DW / VEC, STEPS = CPR / 2;  // steps: 16-byte reads of a row by either lane half
  static constexpr int OTHER = E == 2 ? 64 : 32, NB = OTHER / 32, OB = DW / 32;
  static constexpr int BYTES = OTHER * DW * E, LOADS = BYTES / 1024 / 4;              // per wavefront
  static_assert(LOADS * 4 * 1024 == BYTES, "tiles are dealt to the wavefronts in 1 KB blocks");
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (E == 2) return CPR == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : CPR == 8 ? ((r & 2) << 1) | ((r >> 2) & 3) : (r >> 2) & 3;
    else return CPR % 16 == 0 ? (r & 3) | ((r & 4) << 1) | ((r & 8) >> 1) : (r >> 1) & 7;
  }
  __device__ static __forceinline__ int slot(int r, int c) { return (r * CPR + (c ^ swz(r))) * 16; }  // bytes
};

// Operand rows r0 .. r0 + 31 of the tile, 16-byte step ks of them.
template <typename T, int DW> __device__ __forceinline__ uint4 rows_frag(const char* tile, int r0, int ks, int l31, int hi) {
  return *reinterpret_cast<const uint4*>(tile + Tile<T, DW>::slot(r0 + l31, 2 * ks + hi));
}
// acc += rows x columns over one 16-byte step of both.
template <typename T> __device__ __forceinline__ v16f_t step_product(uint4 a, uint4 b, v16f_t c) {
  if constexpr (sizeof(T) == 2) return mfma_bf16(a, b, c);
  else {
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
  }
}
__device__ __forceinline__ v16f_t zero16() {
  v16f_t a;
#pragma unroll
  for (int v = 0; v < 16; ++v) a[v] = 0.f;
  return a;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) { return (uint32_t)f32_to_bf16(lo) | ((uint32_t)f32_to_bf16(hi) << 16); }

// out[ob] += (columns 32 ob .. of the tile's rows r0 .. r0 + 31)^T x p, p as a score block's accumulator holds it (rounded to the element type).
template <typename T, int DW>
__device__ __forceinline__ void across_product(const char* tile, int r0, const v16f_t& p, v16f_t (&out)[DW / 32], int lane) {
  using Tl = Tile<T, DW>;
  const int hi = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    const int rho = lane & 15, cl = 16 * ((lane >> 4) & 1) + 4 * (rho & 3);
    typedef __attribute__((address_space(3))) att_v4s* v4s_ptr;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint4 w = make_uint4(pack2(p[8 * t], p[8 * t + 1]), pack2(p[8 * t + 2], p[8 * t + 3]), pack2(p[8 * t + 4], p[8 * t + 5]), pack2(p[8 * t + 6], p[8 * t + 7]));
      const int r = r0 + 16 * t + 4 * hi + (rho >> 2);
#pragma unroll
      for (int ob = 0; ob < Tl::OB; ++ob) {
        const int c = 32 * ob + cl;
        union { att_v4s v[2]; uint4 u; } f;
        f.v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s_ptr)(tile + Tl::slot(r, c >> 3) + 2 * (c & 7)));
        f.v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s_ptr)(tile + Tl::slot(r + 8, c >> 3) + 2 * (c & 7)));
        out[ob] = mfma_bf16(f.u, w, out[ob]);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int r = r0 + 8 * (v >> 2) + 4 * hi + (v & 3);
#pragma unroll
      for (int ob = 0; ob < Tl::OB; ++ob) {
        const int c = 32 * ob + (lane & 31);
        const float x = *reinterpret_cast<const float*>(tile + Tl::slot(r, c >> 2) + 4 * (c & 3));
        out[ob] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p[v], out[ob], 0, 0, 0);
      }
    }
  }
}

// A tile's loads into LDS.  Lane offsets are the same for every tile; the buffer's base and bounds move.  Where 4 KB of the tile are whole rows whose
// swizzle repeats, load i differs from load 0 by rows alone, which go into the base: one offset register instead of one per load.
template <typename T, int DW> struct TileLoads {
  using Tl = Tile<T, DW>;
  static constexpr int STEP_ROWS = 256 / Tl::CPR;  // rows of 4 KB
  static constexpr bool BY_ROWS = Tl::E == 2 && 256 % Tl::CPR == 0;
  unsigned off[BY_ROWS ? 1 : Tl::LOADS];
  __device__ __forceinline__ void start(int wave, int lane, unsigned row_bytes, int width) {
#pragma unroll
    for (int i = 0; i < (BY_ROWS ? 1 : Tl::LOADS); ++i) {
      const int e = (4 * i + wave) * 64 + lane, r = e / Tl::CPR, c = (e % Tl::CPR) ^ Tl::swz(r);
      off[i] = c * Tl::VEC < width ? r * row_bytes + 16 * c : ~0u;  // past the width: out of bounds, zero
    }
  }
  // Rows base, base + row_bytes, .. (`rows` of them are there, fewer than none count as none) into the tile at LDS address `at`.
  __device__ __forceinline__ void issue(unsigned at, int wave, const char* base, int rows, unsigned row_bytes, int width) const {
    typedef unsigned v4u __attribute__((ext_vector_type(4)));
    rows = min(rows, Tl::OTHER);
    auto uniform = [](unsigned x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)x); };
#pragma unroll
    for (int i = 0; i < Tl::LOADS; ++i) {
      const int skip = BY_ROWS ? i * STEP_ROWS : 0;
      const unsigned records = rows > skip ? (rows - 1 - skip) * row_bytes + width * Tl::E : 0u;
      const uintptr_t p = (uintptr_t)base + (uintptr_t)skip * row_bytes;
      const v4u buffer = {uniform((unsigned)p), uniform((unsigned)(p >> 32)), uniform(records), 0x00020000u};
      const unsigned lds = at + (4 * i + wave) * 1024;
      // the wait states of this are ours: one between the write of m0 and the load, five between a write of a descriptor word by the vector unit
      // (the readfirstlane above) and the load; s_mov_b32 is one, s_nop 3 four
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off[BY_ROWS ? 0 : i]), "s"(buffer) : "m0");
#pragma clang diagnostic pop
    }
  }
};
// This wavefront's loads have landed and its LDS reads and writes are done; then everyone's, and everyone has left the other stage.
__device__ __forceinline__ void tile_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(7 << 4);  // vmcnt(0) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

struct Span { int begin, len, first; };  // rows of a sequence, and the workgroup's first row in it; len 0: nothing to do
// Offsets that are not as they should be give some span within the tensor.
__device__ __forceinline__ Span find_span(const PackedAttention& a, int t, int lane) {
  auto at = [&](int s) { return min(max(a.offsets[s], 0), a.tokens); };
  int lo = 0, n = a.sequences;
  for (;;) {
    const int step = (n + 63) >> 6;
    const bool before = lane * step < n && at(lo + lane * step) / OWN + lo + lane * step <= t;
    const int count = __popcll(__ballot(before));
    lo += max(count - 1, 0) * step;
    if (step == 1) break;
    n = min(step, a.sequences - lo);
  }
  Span s;
  s.begin = __builtin_amdgcn_readfirstlane(at(lo));
  s.len = max(__builtin_amdgcn_readfirstlane(at(lo + 1)) - s.begin, 0);
  s.first = (t - (s.begin / OWN + lo)) * OWN;
  if (s.first < 0 || s.first >= s.len) s.len = 0;
  return s;
}

template <typename T> __device__ __forceinline__ uint4 flip(uint4 u) {
  const uint32_t m = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
  return make_uint4(u.x ^ m, u.y ^ m, u.z ^ m, u.w ^ m);
}
// One of the wavefront's own rows as a column operand: a lane half's chunks of it, zeros past the width.
template <typename T, int STEPS> __device__ __forceinline__ void load_own(uint4 (&f)[STEPS], const char* row, int hi, int width) {
#pragma unroll
  for (int ks = 0; ks < STEPS; ++ks) {
    const int c = 2 * ks + hi;
    f[ks] = c * Elem<T>::VEC < width ? *reinterpret_cast<const uint4*>(row + 16 * c) : make_uint4(0, 0, 0, 0);
  }
}
// A transposed result (rows = columns 32 ob .., column = the lane's own row) times f -> the row.
template <typename T, int DW> __device__ __forceinline__ void store_own(T* row, const v16f_t (&acc)[DW / 32], float f, int hi, int width) {
#pragma unroll
  for (int ob = 0; ob < DW / 32; ++ob)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int j = 32 * ob + 8 * g + 4 * hi;
      if (j >= width) continue;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(row + j) = make_uint2(pack2(acc[ob][4 * g] * f, acc[ob][4 * g + 1] * f), pack2(acc[ob][4 * g + 2] * f, acc[ob][4 * g + 3] * f));
      else
        *reinterpret_cast<float4*>(row + j) = make_float4(acc[ob][4 * g] * f, acc[ob][4 * g + 1] * f, acc[ob][4 * g + 2] * f, acc[ob][4 * g + 3] * f);
    }
}
__device__ __forceinline__ float both_halves(float v, bool maximum) {
  auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float lo = __uint_as_float(x[0]), hi = __uint_as_float(x[1]);
  return maximum ? fmaxf(lo, hi) : lo + hi;
}
// log2 of what a score is multiplied by to be exponentiated; a scale of zero as the smallest factor that leaves masked scores -inf.  A negative scale
// is taken by turning the sign of one operand, so that the largest product is the largest score.
__device__ __forceinline__ float score_factor(float scale) { return fmaxf(fabsf(scale) * LOG2E, 1.17549435e-38f); }

// ---- forward ----------------------------------------------------------------------------------------------------------
template <typename T, int DW> __global__ __launch_bounds__(256, 2) void packed_fwd_kernel(const PackedAttention a) {
  using Tl = Tile<T, DW>;
  __shared__ __attribute__((aligned(1024))) char smem[4 * Tl::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l31 = lane & 31, hi = lane >> 5;
  const int head = blockIdx.x % a.heads, kv = head / (a.heads / a.kv_heads), W = a.width;
  const Span span = find_span(a, gridDim.x / a.heads - 1 - blockIdx.x / a.heads, lane);
  if (span.len == 0) return;
  const unsigned row_bytes = (a.heads + 2 * a.kv_heads) * W * Tl::E;
  const char* base = static_cast<const char*>(a.qkv) + (int64_t)span.begin * row_bytes;
  const char* kbase = base + (int64_t)(a.heads + kv) * W * Tl::E;
  const char* vbase = kbase + (int64_t)a.kv_heads * W * Tl::E;
  const int q = span.first + 32 * wave + l31, last = span.first + 32 * wave + 31;
  uint4 qf[Tl::STEPS];
  load_own<T>(qf, base + (int64_t)min(q, span.len - 1) * row_bytes + (int64_t)head * W * Tl::E, hi, W);
  if (a.scale < 0.f) {
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks) qf[ks] = flip<T>(qf[ks]);
  }
  const float c = score_factor(a.scale);
  TileLoads<T, DW> loads;
  loads.start(wave, lane, row_bytes, W);
  const unsigned lds = (unsigned)(uintptr_t)(lds_ptr)smem;
  auto issue = [&](int i) {
    const int k0 = i * Tl::OTHER;
    const unsigned at = lds + (i & 1) * 2 * Tl::BYTES;
    loads.issue(at, wave, kbase + (int64_t)k0 * row_bytes, span.len - k0, row_bytes, W);
    loads.issue(at + Tl::BYTES, wave, vbase + (int64_t)k0 * row_bytes, span.len - k0, row_bytes, W);
  };
  const int tiles = (min(span.len, span.first + OWN) + Tl::OTHER - 1) / Tl::OTHER;
  v16f_t o[Tl::OB];
#pragma unroll
  for (int ob = 0; ob < Tl::OB; ++ob) o[ob] = zero16();
  float m = -INFINITY, z = 0.f;
  issue(0);
  for (int i = 0; i < tiles; ++i) {
    tile_barrier();
    if (i + 1 < tiles) issue(i + 1);
    const int k0 = i * Tl::OTHER;
    if (k0 > last) continue;
    const char* Ks = smem + (i & 1) * 2 * Tl::BYTES;
    v16f_t s[Tl::NB];
#pragma unroll
    for (int b = 0; b < Tl::NB; ++b) s[b] = zero16();
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks)
#pragma unroll
      for (int b = 0; b < Tl::NB; ++b) s[b] = step_product<T>(rows_frag<T, DW>(Ks, 32 * b, ks, l31, hi), qf[ks], s[b]);
    if (k0 + Tl::OTHER - 1 > last - 31) {
#pragma unroll
      for (int b = 0; b < Tl::NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (k0 + 32 * b + 8 * (v >> 2) + 4 * hi + (v & 3) > q) s[b][v] = -INFINITY;
    }
    float mt = s[0][0];
#pragma unroll
    for (int b = 0; b < Tl::NB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) mt = fmaxf(mt, s[b][v]);
    mt = both_halves(mt, true) * c;
    // the running maximum only has to be near enough that nothing overflows: probabilities up to 2^8 (any maximum gives the same quotient)
    if (__any(mt > m + 8.f)) {
      const float mn = fmaxf(m, mt), f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      z *= f;
#pragma unroll
      for (int ob = 0; ob < Tl::OB; ++ob)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[ob][v] *= f;
    }
#pragma unroll
    for (int b = 0; b < Tl::NB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[b][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][v], c, -m));
        z += s[b][v];
      }
#pragma unroll
    for (int b = 0; b < Tl::NB; ++b) across_product<T, DW>(Ks + Tl::BYTES, 32 * b, s[b], o, lane);
  }
  if (q >= span.len) return;
  z = both_halves(z, false);
  store_own<T, DW>(static_cast<T*>(a.out) + ((int64_t)(span.begin + q) * a.heads + head) * W, o, 1.f / z, hi, W);
  if (hi == 0) a.lse[(int64_t)head * a.tokens + span.begin + q] = (m + __builtin_amdgcn_logf(z)) * LN2;
}

// ---- backward: dq, and delta for the other kernel ---------------------------------------------------------------------
template <typename T, int DW> __global__ __launch_bounds__(256, sizeof(T) == 2 || DW < 96 ? 2 : 1) void packed_bwd_q_kernel(const PackedAttention a) {
  using Tl = Tile<T, DW>;
  __shared__ __attribute__((aligned(1024))) char smem[4 * Tl::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l31 = lane & 31, hi = lane >> 5;
  const int head = blockIdx.x % a.heads, kv = head / (a.heads / a.kv_heads), W = a.width;
  const Span span = find_span(a, gridDim.x / a.heads - 1 - blockIdx.x / a.heads, lane);
  if (span.len == 0) return;
  const unsigned row_bytes = (a.heads + 2 * a.kv_heads) * W * Tl::E;
  const char* base = static_cast<const char*>(a.qkv) + (int64_t)span.begin * row_bytes;
  const char* kbase = base + (int64_t)(a.heads + kv) * W * Tl::E;
  const char* vbase = kbase + (int64_t)a.kv_heads * W * Tl::E;
  const int q = span.first + 32 * wave + l31, last = span.first + 32 * wave + 31, qc = min(q, span.len - 1);
  uint4 qf[Tl::STEPS], df[Tl::STEPS];
  load_own<T>(qf, base + (int64_t)qc * row_bytes + (int64_t)head * W * Tl::E, hi, W);
  if (a.scale < 0.f) {
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks) qf[ks] = flip<T>(qf[ks]);
  }
  const int64_t orow = ((int64_t)(span.begin + qc) * a.heads + head) * W, at = (int64_t)head * a.tokens + span.begin + qc;
  load_own<T>(df, static_cast<const char*>(a.dout) + orow * Tl::E, hi, W);
  float delta = 0.f;
  {
    uint4 of[Tl::STEPS];
    load_own<T>(of, static_cast<const char*>(a.out) + orow * Tl::E, hi, W);
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks) {
      Chunk16<T> x, y;
      x.v = of[ks];
      y.v = df[ks];
#pragma unroll
      for (int e = 0; e < Tl::VEC; ++e) delta += Elem<T>::to_f32(x.e[e]) * Elem<T>::to_f32(y.e[e]);
    }
    delta = both_halves(delta, false);
  }
  const float lse = a.lse[at] * LOG2E;
  if (hi == 0 && q < span.len) a.delta[at] = delta;
  const float c = score_factor(a.scale);
  TileLoads<T, DW> loads;
  loads.start(wave, lane, row_bytes, W);
  const unsigned lds = (unsigned)(uintptr_t)(lds_ptr)smem;
  auto issue = [&](int i) {
    const int k0 = i * Tl::OTHER;
    const unsigned to = lds + (i & 1) * 2 * Tl::BYTES;
    loads.issue(to, wave, kbase + (int64_t)k0 * row_bytes, span.len - k0, row_bytes, W);
    loads.issue(to + Tl::BYTES, wave, vbase + (int64_t)k0 * row_bytes, span.len - k0, row_bytes, W);
  };
  const int tiles = (min(span.len, span.first + OWN) + Tl::OTHER - 1) / Tl::OTHER;
  v16f_t dq[Tl::OB];
#pragma unroll
  for (int ob = 0; ob < Tl::OB; ++ob) dq[ob] = zero16();
  issue(0);
  for (int i = 0; i < tiles; ++i) {
    tile_barrier();
    if (i + 1 < tiles) issue(i + 1);
    const char* Ks = smem + (i & 1) * 2 * Tl::BYTES;
#pragma unroll
    for (int b = 0; b < Tl::NB; ++b) {
      const int k0 = i * Tl::OTHER + 32 * b;
      if (k0 > last) continue;
      v16f_t s = zero16(), dp = zero16();
#pragma unroll
      for (int ks = 0; ks < Tl::STEPS; ++ks) {
        s = step_product<T>(rows_frag<T, DW>(Ks, 32 * b, ks, l31, hi), qf[ks], s);
        dp = step_product<T>(rows_frag<T, DW>(Ks + Tl::BYTES, 32 * b, ks, l31, hi), df[ks], dp);
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -lse)) * (dp[v] - delta);
      if (k0 + 31 > last - 31) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (k0 + 8 * (v >> 2) + 4 * hi + (v & 3) > q) s[v] = 0.f;
      }
      across_product<T, DW>(Ks, 32 * b, s, dq, lane);
    }
  }
  if (q < span.len) store_own<T, DW>(static_cast<T*>(a.dqkv) + (int64_t)(span.begin + q) * (a.heads + 2 * a.kv_heads) * W + head * W, dq, a.scale, hi, W);
}

// ---- backward: dk and dv ------------------------------------------------------------------------------------------------
// The tiles are those of the query heads of the key head, one head after the other, each from the workgroup's first key on.  Where that leaves
// the chip short of workgroups the heads are shared by `shares` of them, whose sums (fp32, in the workspace) packed_bwd_fold_kernel adds in a fixed order.
template <typename T, int DW> __global__ __launch_bounds__(256, sizeof(T) == 2 || DW < 64 ? 2 : 1) void packed_bwd_kv_kernel(const PackedAttention a, const int shares) {
  using Tl = Tile<T, DW>;
  __shared__ __attribute__((aligned(1024))) char smem[4 * Tl::BYTES];
  __shared__ __attribute__((aligned(16))) float stats[2][2][Tl::OTHER];  // per stage: lse (in log2), delta
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l31 = lane & 31, hi = lane >> 5;
  const int share = blockIdx.x % shares, kv = blockIdx.x / shares % a.kv_heads, group = a.heads / a.kv_heads, W = a.width;
  const Span span = find_span(a, blockIdx.x / (shares * a.kv_heads), lane);
  if (span.len == 0) return;
  const unsigned row_bytes = (a.heads + 2 * a.kv_heads) * W * Tl::E, out_bytes = a.heads * W * Tl::E;
  const char* base = static_cast<const char*>(a.qkv) + (int64_t)span.begin * row_bytes;
  const char* obase = static_cast<const char*>(a.dout) + (int64_t)span.begin * out_bytes;
  const int key = span.first + 32 * wave + l31, first = span.first + 32 * wave, kc = min(key, span.len - 1);
  uint4 kf[Tl::STEPS], vf[Tl::STEPS];
  const char* krow = base + (int64_t)kc * row_bytes + (int64_t)(a.heads + kv) * W * Tl::E;
  load_own<T>(kf, krow, hi, W);
  load_own<T>(vf, krow + (int64_t)a.kv_heads * W * Tl::E, hi, W);
  if (a.scale < 0.f) {
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks) kf[ks] = flip<T>(kf[ks]);
  }
  const float c = score_factor(a.scale);
  TileLoads<T, DW> qloads, oloads;
  qloads.start(wave, lane, row_bytes, W);
  oloads.start(wave, lane, out_bytes, W);
  const unsigned lds = (unsigned)(uintptr_t)(lds_ptr)smem;
  const int per_head = (span.len - span.first + Tl::OTHER - 1) / Tl::OTHER, tiles = per_head * (group / shares);
  // the next tile: head and first query; what its statistics were
  int head = kv * group + share * (group / shares), q0 = span.first;
  float stat = 0.f;
  auto issue = [&](int i) {
    const unsigned to = lds + (i & 1) * 2 * Tl::BYTES;
    const int64_t col = (int64_t)head * W * Tl::E;
    qloads.issue(to, wave, base + (int64_t)q0 * row_bytes + col, span.len - q0, row_bytes, W);
    oloads.issue(to + Tl::BYTES, wave, obase + (int64_t)q0 * out_bytes + col, span.len - q0, out_bytes, W);
    if (threadIdx.x < 2 * Tl::OTHER) {
      // rows past the sequence: exp(score - inf) is a probability of zero
      const bool is_lse = threadIdx.x < Tl::OTHER;
      const int q = q0 + threadIdx.x % Tl::OTHER;
      const float* from = (is_lse ? a.lse : a.delta) + (int64_t)head * a.tokens + span.begin;
      const float x = from[min(q, span.len - 1)];
      stat = is_lse ? (q < span.len ? x * LOG2E : INFINITY) : (q < span.len ? x : 0.f);
    }
    q0 += Tl::OTHER;
    if (q0 >= span.len) {
      q0 = span.first;
      ++head;
    }
  };
  auto put = [&](int i) {
    if (threadIdx.x < 2 * Tl::OTHER) stats[i & 1][threadIdx.x / Tl::OTHER][threadIdx.x % Tl::OTHER] = stat;
  };
  v16f_t dk[Tl::OB], dv[Tl::OB];
#pragma unroll
  for (int ob = 0; ob < Tl::OB; ++ob) dk[ob] = dv[ob] = zero16();
  issue(0);
  int t0 = span.first;  // first query of the current tile
  for (int i = 0; i < tiles; ++i) {
    put(i);
    tile_barrier();
    if (i + 1 < tiles) issue(i + 1);
    const char* Qs = smem + (i & 1) * 2 * Tl::BYTES;
#pragma unroll 1
    for (int b = 0; b < Tl::NB; ++b) {
      const int b0 = t0 + 32 * b;
      if (b0 + 31 < first || b0 >= span.len) continue;
      v16f_t s = zero16(), dp = zero16();
#pragma unroll
      for (int ks = 0; ks < Tl::STEPS; ++ks) {
        s = step_product<T>(rows_frag<T, DW>(Qs, 32 * b, ks, l31, hi), kf[ks], s);
        dp = step_product<T>(rows_frag<T, DW>(Qs + Tl::BYTES, 32 * b, ks, l31, hi), vf[ks], dp);
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 lse = *reinterpret_cast<const float4*>(&stats[i & 1][0][32 * b + 8 * g + 4 * hi]);
        const float4 delta = *reinterpret_cast<const float4*>(&stats[i & 1][1][32 * b + 8 * g + 4 * hi]);
        const float l[4] = {lse.x, lse.y, lse.z, lse.w}, d[4] = {delta.x, delta.y, delta.z, delta.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[4 * g + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * g + e], c, -l[e]));
          dp[4 * g + e] = s[4 * g + e] * (dp[4 * g + e] - d[e]);
        }
      }
      if (b0 < first + 31) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (b0 + 8 * (v >> 2) + 4 * hi + (v & 3) < key) s[v] = dp[v] = 0.f;
      }
      across_product<T, DW>(Qs + Tl::BYTES, 32 * b, s, dv, lane);
      across_product<T, DW>(Qs, 32 * b, dp, dk, lane);
    }
    t0 += Tl::OTHER;
    if (t0 >= span.len) t0 = span.first;
  }
  if (key >= span.len) return;
  if (shares > 1) {
    float* row = a.parts + (((int64_t)share * 2 * a.tokens + span.begin + key) * a.kv_heads + kv) * W;
    store_own<float, DW>(row, dk, a.scale, hi, W);
    store_own<float, DW>(row + (int64_t)a.tokens * a.kv_heads * W, dv, 1.f, hi, W);
    return;
  }
  T* row = static_cast<T*>(a.dqkv) + (int64_t)(span.begin + key) * (a.heads + 2 * a.kv_heads) * W + (a.heads + kv) * W;
  store_own<T, DW>(row, dk, a.scale, hi, W);
  store_own<T, DW>(row + a.kv_heads * W, dv, 1.f, hi, W);
}

// Sums of the shares: [share][dk, dv][tokens][kv_heads][width] -> the rows of dqkv that belong to a sequence, eight columns a thread.
template <typename T> __global__ __launch_bounds__(256) void packed_bwd_fold_kernel(const PackedAttention a, const int shares) {
  const int n8 = a.kv_heads * a.width / 8, begin = min(max(a.offsets[0], 0), a.tokens), end = min(max(a.offsets[a.sequences], 0), a.tokens);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / n8;
  if (row < begin || row >= end) return;
  const int64_t stride = (int64_t)a.tokens * a.kv_heads * a.width;
  const int col = (int)(i - row * n8) * 8;
  const float* p = a.parts + row * a.kv_heads * a.width + col + blockIdx.y * stride;
  float s[8] = {};
  for (int k = 0; k < shares; ++k, p += 2 * stride) {
    const float4 x = *reinterpret_cast<const float4*>(p), y = *reinterpret_cast<const float4*>(p + 4);
    s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
  }
  T* out = static_cast<T*>(a.dqkv) + row * (a.heads + 2 * a.kv_heads) * a.width + (a.heads + blockIdx.y * a.kv_heads) * a.width + col;
  Chunk16<T> c[8 / Elem<T>::VEC];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e / Elem<T>::VEC].e[e % Elem<T>::VEC] = Elem<T>::from_f32(s[e]);
#pragma unroll
  for (int e = 0; e < 8 / Elem<T>::VEC; ++e) reinterpret_cast<uint4*>(out)[e] = c[e].v;
}

#define CDP_WIDTHS(CALL)                                 \
  do {                                                   \
    if (a.width <= 32) { constexpr int DW = 32; CALL; }  \
    else if (a.width <= 64) { constexpr int DW = 64; CALL; } \
    else if (a.width <= 96) { constexpr int DW = 96; CALL; } \
    else { constexpr int DW = 128; CALL; }               \
  } while (0)

int tiles_of(const PackedAttention& a) { return a.tokens / OWN + a.sequences; }

// Workgroups that share a key tile's query heads: as few as make 2048 workgroups, four rounds of two per CU (a causal launch's workgroups differ in
// length by as much as their tiles are many, and the longest, which start first, have to be short against the whole).
int shares_of(const PackedAttention& a) {
  const int group = a.heads / a.kv_heads;
  const int64_t have = (int64_t)tiles_of(a) * a.kv_heads;
  int shares = 1;
  for (int n = 2; n <= group && have * shares < 2048; ++n)
    if (group % n == 0 && n <= a.max_parts) shares = n;
  return shares;
}

template <typename T> hipError_t forward(const PackedAttention& a, hipStream_t stream) {
  const dim3 grid((unsigned)tiles_of(a) * a.heads);
  CDP_WIDTHS(hipLaunchKernelGGL((packed_fwd_kernel<T, DW>), grid, dim3(256), 0, stream, a));
  return hipGetLastError();
}
template <typename T> hipError_t backward(const PackedAttention& a, hipStream_t stream) {
  const dim3 qgrid((unsigned)tiles_of(a) * a.heads);
  const unsigned kgrid = (unsigned)tiles_of(a) * a.kv_heads;
  CDP_WIDTHS(hipLaunchKernelGGL((packed_bwd_q_kernel<T, DW>), qgrid, dim3(256), 0, stream, a));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int shares = shares_of(a);
  CDP_WIDTHS(hipLaunchKernelGGL((packed_bwd_kv_kernel<T, DW>), dim3(kgrid * shares), dim3(256), 0, stream, a, shares));
  if ((e = hipGetLastError()) != hipSuccess || shares == 1) return e;
  const int64_t n = (int64_t)a.tokens * a.kv_heads * a.width / 8;
  hipLaunchKernelGGL((packed_bwd_fold_kernel<T>), dim3((unsigned)((n + 255) / 256), 2), dim3(256), 0, stream, a, shares);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_attention_fwd(const PackedAttention& a, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? forward<uint16_t>(a, stream) : forward<float>(a, stream);
}
hipError_t launch_packed_attention_bwd(const PackedAttention& a, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? backward<uint16_t>(a, stream) : backward<float>(a, stream);
}

}  // namespace cdp
