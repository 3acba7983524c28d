// Causal attention over packed sequences of different lengths, with grouped heads.
//   S = scale q k^T, P = softmax(S) over the keys of the own sequence up to the query itself, out = P v, lse = log sum exp S;
//   backward: P = exp(S - lse), delta = rowsum(dout out), dP = dout v^T, dS = P (dP - delta), dq = scale dS k, dk = scale dS^T q, dv = P^T dout.
//
// One pass over the keys with the running maximum and sum of the softmax; nothing of S or P goes through memory.  A workgroup is four wavefronts
// of 32 rows (ROWS = 128) each (queries forward and for dq, keys for dk and dv) of one head of one sequence and walks tiles of the other side, which two
// stages of LDS hold: the next tile's loads (straight into LDS, zeros past the sequence from the buffer's bounds) are in flight under the products
// of the current one.  Score blocks are contracted so that a lane holds one of the wavefront's own rows, 16 rows of the other side in its
// registers: row sums and maxima stay in the lane (and lane +- 32), and the probabilities are, in the registers they are in, the column operand of the next
// product, whose row operand is read from LDS across rows (bf16: transposing reads) in that same order.
// SPLIT, for launches of few workgroups: all four wavefronts have the same 32 rows, each walks every fourth tile of the other side, filled by itself
// into LDS of its own (no barrier), and they join their sums at the end.
// Work is found on the device (find_span): a sequence needs at most offsets[s + 1] / ROWS - offsets[s] / ROWS + 1 workgroups per head, which bounds the grid by
// tokens / ROWS + sequences: no table, no launch ahead.
// fp32: the same with every operand as three bf16 planes (Part), tiles of 32 rows instead of 64.
//
// Bound by the matrix cores for long sequences, with the exponentials and the LDS reads between the products: 8192 tokens, 32 heads of 128 over 8, bf16: forward
// 530 us, 1040 TFLOP/s (a large matrix product: 1339), backward 1800 us, 765; fp32 4096 tokens, 16 heads of 128 over 4: 452 us, 153 TFLOP/s, and
// 1655, 104 (its kernel for keys has all 512 registers of a lane and spills 40 more: k and v in planes are 192, the sums 128; at width 112 16; where
// wavefronts share rows 67 and 43, in the launch for both 69 and 49).  For short ones by a workgroup's own way: its span, its rows, its tiles, one memory
// round trip after the other: 8192 tokens in 24 sequences, 12 heads of 64 over 4, bf16: 22 us and 65, of which bytes and products would be 7 and 14.
#include "elem.h"
#include "kernels.h"

#include <type_traits>

namespace cdp {

namespace {

typedef short att_v4s __attribute__((ext_vector_type(4)));
typedef float att_v4f __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// Tile of `OTHER` rows of one head, DW columns (zeros past the width; products along a row take SW of them), in LDS.  16-byte chunk c of row r sits in slot
// c ^ swz(r) of the row: 16 consecutive rows' chunk c are 16 different slots modulo 256 bytes, and so are the pieces that a read across rows takes.
constexpr int columns(int sw) { return (sw + 31) / 32 * 32; }
template <typename T, int SW, bool SPLIT> struct Tile {
  static constexpr int DW = columns(SW);
  static constexpr int E = sizeof(T), VEC = 16 / E, CPR = DW / VEC;
  static constexpr int STEPS = SW / 16, CHUNKS = SW * E / 32;  // products along a row; 16-byte reads of it by either lane half
  static constexpr int OWN = SPLIT ? 32 : 128, OTHER = SPLIT || E == 4 ? 32 : 64, NB = OTHER / 32, OB = DW / 32;
  static constexpr int BYTES = OTHER * DW * E, FILLERS = SPLIT ? 1 : 4, LOADS = BYTES / 1024 / FILLERS;  // wavefronts that fill a tile, loads of each
  static_assert(LOADS * FILLERS * 1024 == BYTES, "tiles are dealt to the wavefronts in 1 KB blocks");
  static constexpr int LDS = (SPLIT ? 4 : 2) * 2 * BYTES;                             // two stages, or one for each wavefront, of two tiles
  static_assert(!SPLIT || LDS >= 4 * 32 * DW * 4, "room for what the wavefronts join");
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (E == 2) return CPR == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : CPR == 8 ? ((r & 2) << 1) | ((r >> 2) & 3) : (r >> 2) & 3;
    else return CPR % 16 == 0 ? (r & 3) | ((r & 4) << 1) | ((r & 8) >> 1) : (r >> 1) & 7;
  }
  __device__ static __forceinline__ int slot(int r, int c) { return (r * CPR + (c ^ swz(r))) * 16; }  // bytes
  // Where chunk c + `more` is, given where chunk c is: the bits of a chunk's number that the swizzle turns are turned in the address (tile rows are
  // aligned to them), the others are added.  (more: a constant that c has no bits of)
  static constexpr int TURNED = (CPR & (CPR - 1)) == 0 ? CPR - 1 : E == 2 ? 3 : 7;
  __device__ static __forceinline__ unsigned chunk(unsigned at, int more) { return (at ^ ((more & TURNED) << 4)) + ((more & ~TURNED) << 4); }
};
template <typename V> __device__ __forceinline__ V lds_at(unsigned at) { return *(__attribute__((address_space(3))) const V*)(uintptr_t)at; }
__device__ __forceinline__ void lds_put(unsigned at, float v) { *(__attribute__((address_space(3))) float*)(uintptr_t)at = v; }
// The lane's place in what it reads of a tile, kept where it is: the addresses that a loop reads from differ from it by a constant turn, made
// where they are used (all of them at hand, as the compiler would have it, are registers that wide heads need for data).
struct Lane {
  unsigned at;
  __device__ __forceinline__ Lane(unsigned a) : at(a) { asm volatile("" : "+v"(at)); }
};

// Eight values of a lane as an operand of 32x32x16 products.  fp32: three bf16 planes, the upper 8 bits of the significand, the next 8, the last 8,
// cut and not rounded, so that their sum is the value.  A product of two such operands is six of planes, from the smallest; the three that are left
// out make it smaller by less than 2^-21 of itself, the largest when both significands are 1 and next to 2^-7 more, and by 2^-24.5 on average: of a long sum less
// than its own roundings.  (Planes rounded to nearest would leave out 2^-24 at most, of either sign: their conversions cost 2 to 10 %, us, 4096 tokens, 16 heads of
// 128 over 4, forward 452 -> 459, backward 1655 -> 1816; 2500 tokens, 8 heads of 80, 38 -> 40 and 112 -> 115; and values from 2^128 - 2^119 on would be infinite.)
// Six products at the rate of bf16 are 192 cycles, one on 32x32x2 in fp32 512.  (What is infinite has no planes: it gives NaN.)
template <typename T> struct Part {
  uint4 v;
  __device__ __forceinline__ Part() {}
  __device__ __forceinline__ explicit Part(const uint4* raw) : v(raw[0]) {}
};
template <> struct Part<float> {
  uint32_t w[3][4];
  __device__ __forceinline__ Part() {}
  __device__ __forceinline__ explicit Part(const uint4* raw) {
    const uint32_t x[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
    for (int i = 0; i < 8; i += 2) set(i / 2, __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
  }
  __device__ __forceinline__ void set(int pair, float a, float b) {
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      w[p][pair] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);  // both upper halves
      a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
      b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
    }
  }
  __device__ __forceinline__ uint4 plane(int p) const { return make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]); }
};
// Operand rows r0 .. r0 + 31 (r0 a multiple of 32) of the tile at LDS address `at`, columns 16 ks .. of them.
template <typename Tl> __device__ __forceinline__ unsigned rows_place(int l31, int hi) { return Tl::slot(l31, Tl::E == 2 ? hi : 2 * hi); }
template <typename T, typename Tl> __device__ __forceinline__ Part<T> rows_frag(Lane at, int r0, int ks) {
  typedef unsigned v4u __attribute__((ext_vector_type(4)));
  constexpr int N = Tl::E / 2;
  uint4 raw[N];
#pragma unroll
  for (int i = 0; i < N; ++i) raw[i] = __builtin_bit_cast(uint4, lds_at<v4u>(Tl::chunk(at.at, 2 * N * ks + i) + r0 * Tl::CPR * 16));
  return Part<T>(raw);
}
// acc += rows x columns over 16 of both.
template <typename T> __device__ __forceinline__ v16f_t step_product(const Part<T>& a, const Part<T>& b, v16f_t c) {
  if constexpr (sizeof(T) == 2) return mfma_bf16(a.v, b.v, c);
  else {
    constexpr int order[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
#pragma unroll
    for (int i = 0; i < 6; ++i) c = mfma_bf16(a.plane(order[i][0]), b.plane(order[i][1]), c);
    return c;
  }
}
__device__ __forceinline__ v16f_t zero16() {
  v16f_t a;
#pragma unroll
  for (int v = 0; v < 16; ++v) a[v] = 0.f;
  return a;
}
// Both halves in one conversion (to nearest even); put together from two it is four instructions.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef float v2f __attribute__((ext_vector_type(2)));
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){lo, hi}, v2bf));
}

// out[ob] += (columns 32 ob .. of the tile's rows r0 .. r0 + 31)^T x p, p as a score block's accumulator holds it.
// bf16: a 16-lane group's addresses are 4 rows by 16 columns, and lane i gets column i of them; `at` of rows 4 hi + .. and `at8` of those 8 on.
template <typename Tl> __device__ __forceinline__ unsigned across_place(int lane, int rows_on) {
  const int hi = lane >> 5;
  if constexpr (Tl::E == 2) {
    const int rho = lane & 15, c = 16 * ((lane >> 4) & 1) + 4 * (rho & 3);
    return Tl::slot(4 * hi + (rho >> 2) + rows_on, c >> 3) + 2 * (c & 7);
  } else {
    return Tl::slot(4 * hi, (lane & 31) >> 2) + 4 * (lane & 3);
  }
}
// bf16: p is rounded to the operand's type, as the matrix instruction has no other: half a step of every term, in a sum of terms of either sign as
// much again as the result's own rounding.  FINE: p in two planes, its rounding and what that leaves, a second product for each.  Errors of out and of
// dqkv, of their norm, rounded / FINE (1.6e-3 is the rounding of the results themselves): 8192 tokens in 24 sequences, 12 heads of 64 over 4 2.0e-3 /
// 1.6e-3 and 2.4e-3 / 1.8e-3; us, forward and backward: 22.6 / 27.1 and 66 / 75, one sequence, 32 heads of 128 over 8 533 / 691 and 1811 / 2371.  So it is
// for the launches that have the time.
template <typename T, typename Tl, bool FINE, int OB>
__device__ __forceinline__ void across_product(Lane at, Lane at8, int r0, const v16f_t& p, v16f_t (&out)[OB]) {
  constexpr int PITCH = Tl::CPR * 16;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    Part<T> w, rest;
    if constexpr (sizeof(T) == 2) {
      uint32_t x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = p[8 * t + 2 * i], b = p[8 * t + 2 * i + 1];
        x[i] = pack2(a, b);
        y[i] = FINE ? pack2(a - __uint_as_float(x[i] << 16), b - __uint_as_float(x[i] & 0xffff0000u)) : 0u;
      }
      w.v = make_uint4(x[0], x[1], x[2], x[3]);
      rest.v = make_uint4(y[0], y[1], y[2], y[3]);
    } else
#pragma unroll
      for (int i = 0; i < 4; ++i) w.set(i, p[8 * t + 2 * i], p[8 * t + 2 * i + 1]);
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) {
      Part<T> f;
      if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) att_v4s* v4s_ptr;
        union { att_v4s v[2]; uint4 u; } x;
        x.v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s_ptr)(uintptr_t)(Tl::chunk(at.at, 4 * ob) + (r0 + 16 * t) * PITCH));
        x.v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s_ptr)(uintptr_t)(Tl::chunk(at8.at, 4 * ob) + (r0 + 16 * t) * PITCH));
        f.v = x.u;
      } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = 16 * t + 8 * (i >> 2) + (i & 3);  // + 4 hi: bits of their own
          x[i] = lds_at<float>((Tl::chunk(at.at, 8 * ob) ^ (Tl::swz(r) << 4)) + (r0 + r) * PITCH);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) f.set(i, x[2 * i], x[2 * i + 1]);
      }
      if constexpr (FINE && sizeof(T) == 2) out[ob] = step_product<T>(f, rest, out[ob]);
      out[ob] = step_product<T>(f, w, out[ob]);
    }
  }
}

// A tile's loads into LDS.  Lane offsets are the same for every tile; the buffer's base and bounds move.  Where one load of every wavefront is whole rows whose
// swizzle repeats, load i differs from load 0 by rows alone, which go into the base: one offset register instead of one per load.
template <typename Tl> struct TileLoads {
  static constexpr int STEP = Tl::FILLERS * 64, STEP_ROWS = STEP / Tl::CPR;  // chunks and rows of a load by every filler
  static constexpr bool BY_ROWS = Tl::E == 2 && STEP % Tl::CPR == 0 && STEP_ROWS % 16 == 0;
  unsigned off[BY_ROWS ? 1 : Tl::LOADS];
  // wave: of the wavefronts that fill the tile
  __device__ __forceinline__ void start(int wave, int lane, unsigned row_bytes, int width) {
#pragma unroll
    for (int i = 0; i < (BY_ROWS ? 1 : Tl::LOADS); ++i) {
      const int e = i * STEP + wave * 64 + lane, r = e / Tl::CPR, c = (e % Tl::CPR) ^ Tl::swz(r);
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
      const unsigned lds = at + i * STEP * 16 + wave * 1024;
      // the wait states of this are ours: one between the write of m0 and the load, five between a write of a descriptor word by the vector unit
      // (the readfirstlane above) and the load; s_mov_b32 is one, s_nop 3 four
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off[BY_ROWS ? 0 : i]), "s"(buffer) : "m0");
#pragma clang diagnostic pop
    }
  }
};
// Up to 64 floats from `from` (`rows` of them are there) to LDS address `at`; what is not there is zero.
__device__ __forceinline__ void issue_floats(unsigned at, const float* from, int rows, int lane) {
  typedef unsigned v4u __attribute__((ext_vector_type(4)));
  auto uniform = [](unsigned x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)x); };
  const uintptr_t p = (uintptr_t)from;
  const v4u buffer = {uniform((unsigned)p), uniform((unsigned)(p >> 32)), uniform(4u * max(rows, 0)), 0x00020000u};
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(at), "v"(4u * lane), "s"(buffer) : "m0");
#pragma clang diagnostic pop
}
// This wavefront's loads but for the newest N have landed (63: no matter), and its LDS reads and writes are done.
template <int N> __device__ __forceinline__ void wait_newest() {
  static_assert(N < 64, "vmcnt");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));  // vmcnt(N) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// Shared tiles: everyone's loads have landed, and everyone has left the other stage.
__device__ __forceinline__ void tile_barrier() {
  wait_newest<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Sum, or largest, of a wavefront's values (none below zero).
template <bool LARGEST> __device__ __forceinline__ int of_wave(int x) {
  auto with = [&](int y) { x = LARGEST ? max(x, y) : x + y; };
  with(__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, false));   // neighbours, pairs, and the other halves of 8 and of 16 lanes
  with(__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, false));
  with(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, false));
  with(__builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, false));
  const int a = __builtin_amdgcn_readlane(x, 0), b = __builtin_amdgcn_readlane(x, 16), c = __builtin_amdgcn_readlane(x, 32), d = __builtin_amdgcn_readlane(x, 48);
  return LARGEST ? max(max(a, b), max(c, d)) : a + b + c + d;
}

struct Span { int begin, len, first; };  // rows of a sequence, and the workgroup's first row in it; len 0: nothing to do
// The work of the workgroup that starts as the t-th of `all`, without a table.  Two to 63 sequences, one a lane: the longest work starts first, as the
// launch lasts until it ends.  (A level is how many workgroups of its sequence have less to do; they start from the highest level on, those of one
// level by sequence.  us, 8192 tokens in 24 sequences, 12 heads of 64 over 4, in their own order / so: forward 28.0 / 22.3, backward 90 / 76; 25 sequences
// of 32 5.0 / 5.0.)  One has that order anyway; more take their workgroups in their own order, the longest of each first.
// Offsets that are not as they should be give some span within the tensor.
template <int OWN, bool KEYS> __device__ __forceinline__ Span find_span(const PackedAttention& a, int t, int all, int lane) {
  auto at = [&](int s) { return min(max(a.offsets[s], 0), a.tokens); };
  Span s{0, 0, 0};
  if (a.sequences > 1 && a.sequences < 64) {
    const int begin = at(min(lane, a.sequences)), len = max(at(min(lane + 1, a.sequences)) - begin, 0), n = (len + OWN - 1) / OWN;
    if (of_wave<false>(n) <= t) return s;
    // the lowest level that has no more than t workgroups above it; `above`: how many
    int low = 0, high = of_wave<true>(n), above = 0;
    while (high - low > 1) {
      const int middle = (low + high) >> 1, from = of_wave<false>(max(n - middle, 0));
      if (from > t) low = middle;
      else high = middle, above = from;
    }
    const uint64_t there = __ballot(n > low);
    const bool mine = n > low && __builtin_amdgcn_mbcnt_hi((uint32_t)(there >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)there, 0)) == (unsigned)(t - above);
    const int of = __ffsll((unsigned long long)__ballot(mine)) - 1;
    s.begin = __builtin_amdgcn_readlane(begin, of);
    s.len = __builtin_amdgcn_readlane(len, of);
    s.first = (KEYS ? __builtin_amdgcn_readlane(n, of) - 1 - low : low) * OWN;
    if (s.first < 0 || s.first >= s.len) s.len = 0;
    return s;
  }
  // sequence s has its workgroups from offsets[s] / OWN + s on: the last one with that at or below `place`
  const int place = KEYS ? t : all - 1 - t;
  int lo = 0, n = a.sequences;
  for (;;) {
    const int step = (n + 62) / 63, i = min(lo + lane * step, a.sequences), from = at(i);
    const bool before = lane * step < n && from / OWN + i <= place;
    const int count = max(__popcll(__ballot(before)), 1);
    lo += (count - 1) * step;
    if (step == 1) {
      s.begin = __builtin_amdgcn_readlane(from, count - 1);
      s.len = max(__builtin_amdgcn_readlane(from, count) - s.begin, 0);
      break;
    }
    n = min(step, a.sequences - lo);
  }
  s.first = (place - (s.begin / OWN + lo)) * OWN;
  if (s.first < 0 || s.first >= s.len) s.len = 0;
  return s;
}

template <typename T> __device__ __forceinline__ uint4 flip(uint4 u) {
  const uint32_t m = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
  return make_uint4(u.x ^ m, u.y ^ m, u.z ^ m, u.w ^ m);
}
// One of the wavefront's own rows, a lane half's chunks of it, zeros past the width; and as column operands.
template <typename Tl> struct Own {
  uint4 raw[Tl::CHUNKS];
  __device__ __forceinline__ Own(const char* row, int hi, int width) {
    constexpr int N = Tl::E / 2;
#pragma unroll
    for (int k = 0; k < Tl::CHUNKS; ++k) {
      const int c = 2 * N * (k / N) + N * hi + k % N;
      raw[k] = c * Tl::VEC < width ? *reinterpret_cast<const uint4*>(row + 16 * c) : make_uint4(0, 0, 0, 0);
    }
  }
  template <typename T> __device__ __forceinline__ void parts(Part<T> (&f)[Tl::STEPS], bool turned) const {
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks) {
      constexpr int N = Tl::E / 2;
      uint4 x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = turned ? flip<T>(raw[N * ks + i]) : raw[N * ks + i];
      f[ks] = Part<T>(x);
    }
  }
};
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

// SPLIT: four wavefronts' accumulators of the same 32 rows through LDS, [wavefront][column][row], and the sum of them for DW / 8 columns of a lane's row.
// `mine`, `shares`: LDS addresses of [column][row] and of four of those.
template <int OB> __device__ __forceinline__ void put_share(unsigned mine, const v16f_t (&acc)[OB], float f, int l31, int hi) {
#pragma unroll
  for (int ob = 0; ob < OB; ++ob)
#pragma unroll
    for (int v = 0; v < 16; ++v) lds_put(mine + 4 * ((32 * ob + 8 * (v >> 2) + 4 * hi + (v & 3)) * 32 + l31), acc[ob][v] * f);
}
template <typename T, int DW> __device__ __forceinline__ void join_shares(T* row, unsigned shares, float f, int wave, int l31, int hi, int width) {
  const int d0 = (2 * wave + hi) * (DW / 8);
#pragma unroll
  for (int d = d0; d < d0 + DW / 8; d += 4) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned p = shares + 4 * ((d + e) * 32 + l31);
      v[e] = ((lds_at<float>(p) + lds_at<float>(p + DW * 128)) + (lds_at<float>(p + 2 * DW * 128) + lds_at<float>(p + 3 * DW * 128))) * f;
    }
    if (d >= width) continue;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(row + d) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    else *reinterpret_cast<float4*>(row + d) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

// ---- forward ----------------------------------------------------------------------------------------------------------
template <typename T, int SW, bool SPLIT>
__global__ __launch_bounds__(256, sizeof(T) == 4 && SW > (SPLIT ? 64 : 96) ? 1 : 2) void packed_fwd_kernel(const PackedAttention a) {
  using Tl = Tile<T, SW, SPLIT>;
  constexpr int DW = Tl::DW;
  __shared__ __attribute__((aligned(1024))) char memory[Tl::LDS];
  const unsigned smem = (unsigned)(uintptr_t)(lds_ptr)memory;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l31 = lane & 31, hi = lane >> 5;
  // which of the workgroup's 32-row groups is the wavefront's; its place among those that fill a tile
  const int rows_of = SPLIT ? 0 : wave, filler = SPLIT ? 0 : wave;
  const int head = blockIdx.x % a.heads, kv = head / (a.heads / a.kv_heads), W = a.width;
  const Span span = find_span<Tl::OWN, false>(a, blockIdx.x / a.heads, gridDim.x / a.heads, lane);
  if (span.len == 0) return;
  const unsigned row_bytes = (a.heads + 2 * a.kv_heads) * W * Tl::E;
  const char* base = static_cast<const char*>(a.qkv) + (int64_t)span.begin * row_bytes;
  const char* kbase = base + (int64_t)(a.heads + kv) * W * Tl::E;
  const char* vbase = kbase + (int64_t)a.kv_heads * W * Tl::E;
  const int q = span.first + 32 * rows_of + l31, last = span.first + 32 * rows_of + 31;
  Part<T> qf[Tl::STEPS];
  Own<Tl>(base + (int64_t)min(q, span.len - 1) * row_bytes + (int64_t)head * W * Tl::E, hi, W).parts(qf, a.scale < 0.f);
  const float c = score_factor(a.scale);
  TileLoads<Tl> loads;
  loads.start(filler, lane, row_bytes, W);
  const unsigned lds = smem + (SPLIT ? wave * (Tl::LDS / 4) : 0);
  const unsigned rows_of_tile = lds + rows_place<Tl>(l31, hi), across_tile = lds + across_place<Tl>(lane, 0), across_tile8 = lds + across_place<Tl>(lane, 8);
  auto issue = [&](int i, int stage, bool v) {  // tiles of k, then of v
    const int k0 = i * Tl::OTHER;
    loads.issue(lds + (2 * stage + v) * Tl::BYTES, filler, (v ? vbase : kbase) + (int64_t)k0 * row_bytes, span.len - k0, row_bytes, W);
  };
  const int tiles = (min(span.len, span.first + Tl::OWN) + Tl::OTHER - 1) / Tl::OTHER;
  v16f_t o[Tl::OB], s[Tl::NB];
#pragma unroll
  for (int ob = 0; ob < Tl::OB; ++ob) o[ob] = zero16();
  float m = -INFINITY, z = 0.f;
  auto scores = [&](int i, int stage) {
    const int k0 = i * Tl::OTHER;
    const Lane rows(rows_of_tile + 2 * stage * Tl::BYTES);
#pragma unroll
    for (int b = 0; b < Tl::NB; ++b) s[b] = zero16();
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks)
#pragma unroll
      for (int b = 0; b < Tl::NB; ++b) s[b] = step_product<T>(rows_frag<T, Tl>(rows, 32 * b, ks), qf[ks], s[b]);
    if (k0 + Tl::OTHER - 1 > last - 31) {
#pragma unroll
      for (int b = 0; b < Tl::NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (k0 + 32 * b + 8 * (v >> 2) + 4 * hi + (v & 3) > q) s[b][v] = -INFINITY;
    }
  };
  auto probabilities = [&] {
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
    for (int b = 0; b < Tl::NB; ++b) {
      float y[4] = {};
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[b][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][v], c, -m));
        y[v & 3] += s[b][v];
      }
      z += (y[0] + y[1]) + (y[2] + y[3]);
    }
  };
  auto values = [&](int stage) {
    const unsigned to = (2 * stage + 1) * Tl::BYTES;
    const Lane across(across_tile + to), across8(across_tile8 + to);
#pragma unroll
    for (int b = 0; b < Tl::NB; ++b) across_product<T, Tl, false>(across, across8, 32 * b, s[b], o);
  };
  if constexpr (SPLIT) {
    // one tile of each in LDS: the next one of k is under way from the scores on, the next one of v from their product on
    if (wave < tiles) {
      issue(wave, 0, false);
      issue(wave, 0, true);
    }
    for (int i = wave; i < tiles; i += 4) {
      const bool more = i + 4 < tiles;
      wait_newest<Tl::LOADS>();
      scores(i, 0);
      wait_newest<63>();
      if (more) issue(i + 4, 0, false);
      probabilities();
      if (more) wait_newest<Tl::LOADS>();
      else wait_newest<0>();
      values(0);
      wait_newest<63>();
      if (more) issue(i + 4, 0, true);
    }
  } else {
    issue(0, 0, false);
    issue(0, 0, true);
    for (int i = 0, stage = 0; i < tiles; ++i, stage ^= 1) {
      tile_barrier();
      if (i + 1 < tiles) {
        issue(i + 1, stage ^ 1, false);
        issue(i + 1, stage ^ 1, true);
      }
      if (i * Tl::OTHER > last || last - 31 >= span.len) continue;
      scores(i, stage);
      probabilities();
      values(stage);
    }
  }
  z = both_halves(z, false);
  T* const out = static_cast<T*>(a.out) + ((int64_t)(span.begin + q) * a.heads + head) * W;
  if constexpr (SPLIT) {
    // every wavefront's maximum, then its sums relative to the largest (one without tiles has a maximum of -inf and a factor of 0)
    __shared__ float ms[4][32], zs[4][32];
    if (hi == 0) ms[wave][l31] = m;
    __syncthreads();
    const float top = fmaxf(fmaxf(ms[0][l31], ms[1][l31]), fmaxf(ms[2][l31], ms[3][l31])), f = __builtin_amdgcn_exp2f(m - top);
    if (hi == 0) zs[wave][l31] = z * f;
    put_share(smem + wave * DW * 128, o, f, l31, hi);
    __syncthreads();
    if (q >= span.len) return;
    z = (zs[0][l31] + zs[1][l31]) + (zs[2][l31] + zs[3][l31]);
    m = top;
    join_shares<T, DW>(out, smem, 1.f / z, wave, l31, hi, W);
    if (wave) return;
  } else {
    if (q >= span.len) return;
    store_own<T, DW>(out, o, 1.f / z, hi, W);
  }
  if (hi == 0) a.lse[(int64_t)head * a.tokens + span.begin + q] = (m + __builtin_amdgcn_logf(z)) * LN2;
}

// ---- backward: dq, and delta for the other kernel ---------------------------------------------------------------------
// id: of the workgroups for queries, of which there are `all`.
template <typename T, int SW, bool SPLIT, bool FINE>
__device__ __forceinline__ void bwd_q(const PackedAttention& a, unsigned smem, unsigned id, unsigned all, bool write_delta) {
  using Tl = Tile<T, SW, SPLIT>;
  constexpr int DW = Tl::DW;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l31 = lane & 31, hi = lane >> 5;
  // which of the workgroup's 32-row groups is the wavefront's; its place among those that fill a tile
  const int rows_of = SPLIT ? 0 : wave, filler = SPLIT ? 0 : wave;
  const int head = id % a.heads, kv = head / (a.heads / a.kv_heads), W = a.width;
  const Span span = find_span<Tl::OWN, false>(a, id / a.heads, all / a.heads, lane);
  if (span.len == 0) return;
  const unsigned row_bytes = (a.heads + 2 * a.kv_heads) * W * Tl::E;
  const char* base = static_cast<const char*>(a.qkv) + (int64_t)span.begin * row_bytes;
  const char* kbase = base + (int64_t)(a.heads + kv) * W * Tl::E;
  const char* vbase = kbase + (int64_t)a.kv_heads * W * Tl::E;
  const int q = span.first + 32 * rows_of + l31, last = span.first + 32 * rows_of + 31, qc = min(q, span.len - 1);
  Part<T> qf[Tl::STEPS], df[Tl::STEPS];
  Own<Tl>(base + (int64_t)qc * row_bytes + (int64_t)head * W * Tl::E, hi, W).parts(qf, a.scale < 0.f);
  const int64_t orow = ((int64_t)(span.begin + qc) * a.heads + head) * W, at = (int64_t)head * a.tokens + span.begin + qc;
  float delta = 0.f;
  {
    const Own<Tl> d(static_cast<const char*>(a.dout) + orow * Tl::E, hi, W), o(static_cast<const char*>(a.out) + orow * Tl::E, hi, W);
    d.parts(df, false);
#pragma unroll
    for (int k = 0; k < Tl::CHUNKS; ++k) {
      Chunk16<T> x, y;
      x.v = o.raw[k];
      y.v = d.raw[k];
#pragma unroll
      for (int e = 0; e < Tl::VEC; ++e) delta += Elem<T>::to_f32(x.e[e]) * Elem<T>::to_f32(y.e[e]);
    }
    delta = both_halves(delta, false);
  }
  const float lse = a.lse[at] * LOG2E;
  if (write_delta && hi == 0 && q < span.len && (!SPLIT || wave == 0)) a.delta[at] = delta;
  const float c = score_factor(a.scale);
  TileLoads<Tl> loads;
  loads.start(filler, lane, row_bytes, W);
  const unsigned lds = smem + (SPLIT ? wave * (Tl::LDS / 4) : 0);
  const unsigned rows_of_tile = lds + rows_place<Tl>(l31, hi), across_tile = lds + across_place<Tl>(lane, 0), across_tile8 = lds + across_place<Tl>(lane, 8);
  auto issue = [&](int i, int stage, bool v) {  // tiles of k, then of v
    const int k0 = i * Tl::OTHER;
    loads.issue(lds + (2 * stage + v) * Tl::BYTES, filler, (v ? vbase : kbase) + (int64_t)k0 * row_bytes, span.len - k0, row_bytes, W);
  };
  const int tiles = (min(span.len, span.first + Tl::OWN) + Tl::OTHER - 1) / Tl::OTHER;
  v16f_t dq[Tl::OB];
#pragma unroll
  for (int ob = 0; ob < Tl::OB; ++ob) dq[ob] = zero16();
  auto dprobabilities = [&](v16f_t& dp, int b, int stage) {
    const Lane rows(rows_of_tile + (2 * stage + 1) * Tl::BYTES);
    dp = zero16();
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks) dp = step_product<T>(rows_frag<T, Tl>(rows, 32 * b, ks), df[ks], dp);
  };
  auto scores = [&](v16f_t& s, int b, int stage) {
    const Lane rows(rows_of_tile + 2 * stage * Tl::BYTES);
    s = zero16();
#pragma unroll
    for (int ks = 0; ks < Tl::STEPS; ++ks) s = step_product<T>(rows_frag<T, Tl>(rows, 32 * b, ks), qf[ks], s);
  };
  auto finish = [&](v16f_t& s, const v16f_t& dp, int k0, int b, int stage) {  // dS, and dq from it
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -lse)) * (dp[v] - delta);
    if (k0 + 31 > last - 31) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (k0 + 8 * (v >> 2) + 4 * hi + (v & 3) > q) s[v] = 0.f;
    }
    const unsigned to = 2 * stage * Tl::BYTES;
    across_product<T, Tl, FINE>(Lane(across_tile + to), Lane(across_tile8 + to), 32 * b, s, dq);
  };
  if constexpr (SPLIT) {
    // v's tile is read first and given back first: the next one of it is under way while k's is in use, and k's under the next product with v
    if (wave < tiles) {
      issue(wave, 0, true);
      issue(wave, 0, false);
    }
    for (int i = wave; i < tiles; i += 4) {
      const bool more = i + 4 < tiles;
      v16f_t s, dp;
      wait_newest<Tl::LOADS>();
      dprobabilities(dp, 0, 0);
      wait_newest<63>();
      if (more) issue(i + 4, 0, true);
      if (more) wait_newest<Tl::LOADS>();
      else wait_newest<0>();
      scores(s, 0, 0);
      finish(s, dp, 32 * i, 0, 0);
      wait_newest<63>();
      if (more) issue(i + 4, 0, false);
    }
  } else {
    issue(0, 0, false);
    issue(0, 0, true);
    for (int i = 0, stage = 0; i < tiles; ++i, stage ^= 1) {
      tile_barrier();
      if (i + 1 < tiles) {
        issue(i + 1, stage ^ 1, false);
        issue(i + 1, stage ^ 1, true);
      }
#pragma unroll
      for (int b = 0; b < Tl::NB; ++b) {
        const int k0 = i * Tl::OTHER + 32 * b;
        if (k0 > last || last - 31 >= span.len) continue;
        v16f_t s, dp;
        scores(s, b, stage);
        dprobabilities(dp, b, stage);
        finish(s, dp, k0, b, stage);
      }
    }
  }
  T* const row = static_cast<T*>(a.dqkv) + (int64_t)(span.begin + q) * (a.heads + 2 * a.kv_heads) * W + head * W;
  if constexpr (SPLIT) {
    __syncthreads();
    put_share(smem + wave * DW * 128, dq, 1.f, l31, hi);
    __syncthreads();
    if (q < span.len) join_shares<T, DW>(row, smem, a.scale, wave, l31, hi, W);
  } else if (q < span.len) {
    store_own<T, DW>(row, dq, a.scale, hi, W);
  }
}
template <typename T, int SW, bool SPLIT>
__global__ __launch_bounds__(256, sizeof(T) == 2 || SW <= 64 ? 2 : 1) void packed_bwd_q_kernel(const PackedAttention a) {
  __shared__ __attribute__((aligned(1024))) char memory[Tile<T, SW, SPLIT>::LDS];
  const unsigned smem = (unsigned)(uintptr_t)(lds_ptr)memory;
  bwd_q<T, SW, SPLIT, false>(a, smem, blockIdx.x, gridDim.x, true);
}

// ---- backward: dk and dv ------------------------------------------------------------------------------------------------
// The tiles are those of the query heads of the key head, one head after the other, each from the workgroup's first key on.  Where that leaves
// the chip short of workgroups the heads are shared by `shares` of them, whose sums (fp32, in the workspace) packed_bwd_fold_kernel adds in a fixed order.
// OWN: delta is not in memory yet; the workgroup makes that of all the rows it will meet first (up to OWN_ROWS of them: no span is longer than the tensor).
constexpr int OWN_ROWS = 512;
template <typename T, int SW, bool SPLIT, bool OWN> __device__ __forceinline__ void bwd_kv(const PackedAttention& a, unsigned smem, unsigned wg, int shares) {
  using Tl = Tile<T, SW, SPLIT>;
  constexpr int DW = Tl::DW;
  __shared__ __attribute__((aligned(16))) float stats[SPLIT ? 4 : 2][2][64];  // per wavefront or stage: lse and delta of the tile's rows
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l31 = lane & 31, hi = lane >> 5;
  // which of the workgroup's 32-row groups is the wavefront's; its place among those that fill a tile
  const int rows_of = SPLIT ? 0 : wave, filler = SPLIT ? 0 : wave;
  const int share = wg % shares, kv = wg / shares % a.kv_heads, group = a.heads / a.kv_heads, W = a.width;
  const Span span = find_span<Tl::OWN, true>(a, wg / (shares * a.kv_heads), 0, lane);
  if (span.len == 0) return;
  const unsigned row_bytes = (a.heads + 2 * a.kv_heads) * W * Tl::E, out_bytes = a.heads * W * Tl::E;
  const char* base = static_cast<const char*>(a.qkv) + (int64_t)span.begin * row_bytes;
  const char* obase = static_cast<const char*>(a.dout) + (int64_t)span.begin * out_bytes;
  const int key = span.first + 32 * rows_of + l31, first = span.first + 32 * rows_of, kc = min(key, span.len - 1);
  Part<T> kf[Tl::STEPS], vf[Tl::STEPS];
  const char* krow = base + (int64_t)kc * row_bytes + (int64_t)(a.heads + kv) * W * Tl::E;
  Own<Tl>(krow, hi, W).parts(kf, a.scale < 0.f);
  Own<Tl>(krow + (int64_t)a.kv_heads * W * Tl::E, hi, W).parts(vf, false);
  const float c = score_factor(a.scale);
  TileLoads<Tl> qloads, oloads;
  qloads.start(filler, lane, row_bytes, W);
  oloads.start(filler, lane, out_bytes, W);
  const unsigned lds = smem + (SPLIT ? wave * (Tl::LDS / 4) : 0);
  const unsigned rows_of_tile = lds + rows_place<Tl>(l31, hi), across_tile = lds + across_place<Tl>(lane, 0), across_tile8 = lds + across_place<Tl>(lane, 8);
  const int per_head = (span.len - span.first + Tl::OTHER - 1) / Tl::OTHER, tiles = per_head * (group / shares);
  const int head0 = kv * group + share * (group / shares);
  __shared__ float own_memory[OWN ? OWN_ROWS : 1];  // [head of the group][query - first]
  const unsigned own = (unsigned)(uintptr_t)(lds_ptr)own_memory;
  const int own_rows = span.len - span.first;
  if constexpr (OWN) {
    // eight lanes a row
    const int n = group * own_rows, l8 = threadIdx.x & 7;
    for (int r = threadIdx.x >> 3; r < n; r += 32) {
      const int64_t row = ((int64_t)(span.begin + span.first + r % own_rows) * a.heads + head0 + r / own_rows) * W * Tl::E;
      const char* const o = static_cast<const char*>(a.out) + row;
      const char* const d = static_cast<const char*>(a.dout) + row;
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < (Tl::CPR + 7) / 8; ++k) {
        const int c = l8 + 8 * k;
        if (c * Tl::VEC >= W) continue;
        Chunk16<T> p, g;
        p.v = *reinterpret_cast<const uint4*>(o + 16 * c);
        g.v = *reinterpret_cast<const uint4*>(d + 16 * c);
#pragma unroll
        for (int e = 0; e < Tl::VEC; ++e) x += Elem<T>::to_f32(p.e[e]) * Elem<T>::to_f32(g.e[e]);
      }
#pragma unroll
      for (int k = 4; k > 0; k >>= 1) x += __shfl_xor(x, k, 64);
      if (l8 == 0) lds_put(own + 4 * r, x);
    }
    __syncthreads();
  }
  const unsigned stats_at = (unsigned)(uintptr_t)(lds_ptr)stats + (SPLIT ? 512 * wave : 0);
  // tiles of q, then of dout, with it what is kept of its rows.  Rows past the sequence are zeros in all of them, which add nothing.
  auto issue = [&](int i, int stage, bool o) {
    const unsigned to = lds + (2 * stage + o) * Tl::BYTES;
    const int head = head0 + i / per_head, q0 = span.first + i % per_head * Tl::OTHER, rows = span.len - q0;
    const int64_t col = (int64_t)head * W * Tl::E;
    if (!o) return qloads.issue(to, filler, base + (int64_t)q0 * row_bytes + col, rows, row_bytes, W);
    const int64_t at = (int64_t)head * a.tokens + span.begin + q0;
    const unsigned st = stats_at + 512 * stage;
    if (SPLIT || wave == 0) issue_floats(st, a.lse + at, min(rows, Tl::OTHER), lane);
    if constexpr (OWN) {
      if (lane < Tl::OTHER) lds_put(st + 256 + 4 * lane, lane < rows ? lds_at<float>(own + 4 * ((head - head0) * own_rows + q0 - span.first + lane)) : 0.f);
    } else if (SPLIT || wave == 1) {
      issue_floats(st + 256, a.delta + at, min(rows, Tl::OTHER), lane);
    }
    oloads.issue(to, filler, obase + (int64_t)q0 * out_bytes + col, rows, out_bytes, W);
  };
  v16f_t dk[Tl::OB], dv[Tl::OB];
#pragma unroll
  for (int ob = 0; ob < Tl::OB; ++ob) dk[ob] = dv[ob] = zero16();
  auto statistics = [&](int which, int row, int stage) { return lds_at<att_v4f>(stats_at + 512 * stage + 256 * which + 4 * row); };
  // P from the scores, dS from dP
  auto finish = [&](v16f_t& s, v16f_t& dp, int b0, int b, int stage) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const att_v4f l = statistics(0, 32 * b + 8 * g + 4 * hi, stage), d = statistics(1, 32 * b + 8 * g + 4 * hi, stage);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[4 * g + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * g + e], c, -LOG2E * l[e]));
        dp[4 * g + e] = s[4 * g + e] * (dp[4 * g + e] - d[e]);
      }
    }
    if (b0 < first + 31) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (b0 + 8 * (v >> 2) + 4 * hi + (v & 3) < key) s[v] = dp[v] = 0.f;
    }
  };
  if constexpr (SPLIT) {
    // dout's tile is read first and given back first, as v's in the kernel for queries
    if (wave < tiles) {
      issue(wave, 0, true);
      issue(wave, 0, false);
    }
    for (int i = wave; i < tiles; i += 4) {
      const bool more = i + 4 < tiles;
      const Lane rows(rows_of_tile), across(across_tile), across8(across_tile8);
      v16f_t s = zero16(), dp = zero16();
      wait_newest<Tl::LOADS>();
#pragma unroll
      for (int ks = 0; ks < Tl::STEPS; ++ks) dp = step_product<T>(rows_frag<T, Tl>(rows, Tl::OTHER, ks), vf[ks], dp);
      wait_newest<0>();
#pragma unroll
      for (int ks = 0; ks < Tl::STEPS; ++ks) s = step_product<T>(rows_frag<T, Tl>(rows, 0, ks), kf[ks], s);
      finish(s, dp, span.first + i % per_head * 32, 0, 0);
      across_product<T, Tl, OWN>(across, across8, Tl::OTHER, s, dv);
      wait_newest<63>();
      if (more) issue(i + 4, 0, true);
      across_product<T, Tl, OWN>(across, across8, 0, dp, dk);
      wait_newest<63>();
      if (more) issue(i + 4, 0, false);
    }
  } else {
    issue(0, 0, false);
    issue(0, 0, true);
    for (int i = 0, stage = 0; i < tiles; ++i, stage ^= 1) {
      tile_barrier();
      if (i + 1 < tiles) {
        issue(i + 1, stage ^ 1, false);
        issue(i + 1, stage ^ 1, true);
      }
      const int t0 = span.first + i % per_head * Tl::OTHER;
#pragma unroll 1
      for (int b = 0; b < Tl::NB; ++b) {
        const int b0 = t0 + 32 * b;
        if (b0 + 31 < first || b0 >= span.len || first >= span.len) continue;
        v16f_t s = zero16(), dp = zero16();
        const unsigned to = 2 * stage * Tl::BYTES + 32 * b * Tl::CPR * 16;
        const Lane rows(rows_of_tile + to);
#pragma unroll
        for (int ks = 0; ks < Tl::STEPS; ++ks) {
          s = step_product<T>(rows_frag<T, Tl>(rows, 0, ks), kf[ks], s);
          dp = step_product<T>(rows_frag<T, Tl>(rows, Tl::OTHER, ks), vf[ks], dp);  // (dout's tile lies behind q's)
        }
        finish(s, dp, b0, b, stage);
        const Lane across(across_tile + to), across8(across_tile8 + to);
        across_product<T, Tl, OWN>(across, across8, Tl::OTHER, s, dv);
        across_product<T, Tl, OWN>(across, across8, 0, dp, dk);
      }
    }
  }
  // to dqkv, or to the share's sums
  auto write = [&](auto* row, int64_t v_from_k) {
    using R = std::remove_reference_t<decltype(*row)>;
    if constexpr (SPLIT) {
      __syncthreads();
      put_share(smem + wave * DW * 128, dk, 1.f, l31, hi);
      __syncthreads();
      if (key < span.len) join_shares<R, DW>(row, smem, a.scale, wave, l31, hi, W);
      __syncthreads();
      put_share(smem + wave * DW * 128, dv, 1.f, l31, hi);
      __syncthreads();
      if (key < span.len) join_shares<R, DW>(row + v_from_k, smem, 1.f, wave, l31, hi, W);
    } else {
      if (key >= span.len) return;
      store_own<R, DW>(row, dk, a.scale, hi, W);
      store_own<R, DW>(row + v_from_k, dv, 1.f, hi, W);
    }
  };
  if (shares > 1)
    write(a.parts + (((int64_t)share * 2 * a.tokens + span.begin + key) * a.kv_heads + kv) * W, (int64_t)a.tokens * a.kv_heads * W);
  else
    write(static_cast<T*>(a.dqkv) + (int64_t)(span.begin + key) * (a.heads + 2 * a.kv_heads) * W + (a.heads + kv) * W, (int64_t)a.kv_heads * W);
}
template <typename T, int SW, bool SPLIT>
__global__ __launch_bounds__(256, (sizeof(T) == 2 && (SW <= 96 || !SPLIT)) || SW <= 32 ? 2 : 1)
void packed_bwd_kv_kernel(const PackedAttention a, const int shares) {
  __shared__ __attribute__((aligned(1024))) char memory[Tile<T, SW, SPLIT>::LDS];
  const unsigned smem = (unsigned)(uintptr_t)(lds_ptr)memory;
  bwd_kv<T, SW, SPLIT, false>(a, smem, blockIdx.x, shares);
}
// Both in one launch, for few rows: the workgroups past `queries` are those for keys.  bf16: P and dS in two planes, as there is time for it (0.1 of 7.7 us,
// 128 tokens, 8 heads of 64; 0.9 of 16.6, 512 tokens): their rounding is half of what a gradient is off (2.5e-3 of its norm, 2.0e-3 so; 1.7e-3 are its own).
template <typename T, int SW> __global__ __launch_bounds__(256, 1) void packed_bwd_both_kernel(const PackedAttention a, const unsigned queries) {
  __shared__ __attribute__((aligned(1024))) char memory[Tile<T, SW, true>::LDS];
  const unsigned smem = (unsigned)(uintptr_t)(lds_ptr)memory;
  if (blockIdx.x < queries) bwd_q<T, SW, true, true>(a, smem, blockIdx.x, queries, false);
  else bwd_kv<T, SW, true, true>(a, smem, blockIdx.x - queries, 1);
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

// Kernels for every 16 columns, as products along a row go, though across rows they go by 32 (us, forward and backward, at widths of whole 32 / so: fp32
// 2500 tokens in 5 sequences, 8 heads of 80 39 and 118 / 37 and 112, 4096 in 2 of 16 43 and 126 / 38 and 108; bf16 8192 in 2 of 48 80 and 228 / 77 and 215).
#define CDP_WIDTHS(CALL)                                     \
  do {                                                       \
    switch ((a.width + 15) / 16) {                       \
      case 1: { constexpr int SW = 16; CALL; } break;    \
      case 2: { constexpr int SW = 32; CALL; } break;    \
      case 3: { constexpr int SW = 48; CALL; } break;    \
      case 4: { constexpr int SW = 64; CALL; } break;    \
      case 5: { constexpr int SW = 80; CALL; } break;    \
      case 6: { constexpr int SW = 96; CALL; } break;    \
      case 7: { constexpr int SW = 112; CALL; } break;   \
      default: { constexpr int SW = 128; CALL; }         \
    }                                                    \
  } while (0)

int64_t workgroups(const PackedAttention& a, int own, int heads) { return ((int64_t)a.tokens / own + a.sequences) * heads; }

// Whether the wavefronts of a workgroup share 32 rows' other side (SPLIT) instead of having 32 rows each: a quarter of the way through the longest sequence
// for the few workgroups that there are, against filling LDS four times as often.  Worth it while the workgroups of 128 rows do not fill the chip; up to
// what count goes by the workgroups that a CU holds, which registers and LDS of wide heads and of fp32 keep down.  us, 128 rows / split, at so many
// workgroups of 128 rows:
//   forward, bf16 width 64: 272 28.9 / 19.5, 384 18.6 / 13.4, 528 59.7 / 64.0; 128: 272 41.7 / 33.4, 384 17.8 / 17.8, 528 94 / 111; fp32 64: 528 265 / 230,
//   792 345 / 345; 128: 264 408 / 271, 384 73 / 63, 528 463 / 531 (dq crosses at the same counts);
//   backward by its kernel for keys, bf16 64: 528 204 / 185, 768 57.6 / 53.2, 896 93 / 98; 96: 528 255 / 255; 128: 192 115 / 106, 272 152 / 153, 384 60 / 73;
//   fp32 64: 384 123 / 114, 528 889 / 927; 128: 264 1488 / 1441, 384 240 / 254.  Where query heads share a key head, 128 rows need their shares' fold too:
//   above width 96 that goes by the workgroups for keys of 32 rows: bf16 128, 16 heads over 2, 130 216 / 150, 168 (20 sequences) 73 / 56, 216 (30) 56 / 57, 258
//   462 / 417, 302 549 / 556, 402 762 / 901; fp32 158 1429 / 1003, 258 2494 / 2490, 302 3140 / 3523.  Up to width 96 by those of 128 rows again: bf16 96,
//   16 over 2, 528 337 / 234, 640 429 / 326, 80, 16 over 4, 640 301 / 304; fp32 64, 16 over 2, 528 1215 / 815, 640 1569 / 1239, 48, 16 over 4, 640
//   1083 / 1093 (with eight query heads to a key head still so at 752, bf16 538 / 440, fp32 1993 / 1724), and there 128 rows cost more than
//   the shorter way unless sequences are long: 8192 tokens in 24 sequences, 12 heads of 64 over 4 83 / 72, 32 of 96 over 8 219 / 198, fp32 32 of 32 over 8
//   311 / 262, in one sequence bf16 16 of 64 over 8 515 / 535.
template <typename T> bool split_wanted(const PackedAttention& a, bool kv) {
  int most;
  const bool shared = a.heads > a.kv_heads;
  if (!kv) most = sizeof(T) == 2 ? (a.width <= 64 ? 500 : 330) : (a.width <= 64 ? 800 : 400);
  else if (a.width > 96 && shared && workgroups(a, 32, a.kv_heads) <= 300) return a.tokens > 64;
  else if (a.width > 96) most = shared ? 380 : 240;
  else if (shared && a.tokens <= 2048 * (int64_t)a.sequences) return a.tokens > 64;
  else if (sizeof(T) == 2) most = a.width <= 64 ? 768 : shared ? 640 : 500;
  else most = a.width <= 32 ? 800 : shared ? 640 : 450;
  return a.tokens > 64 && workgroups(a, 128, a.heads) <= most;  // (one tile of 64 rows has nothing to share)
}
// Workgroups that share a key tile's query heads: as few as make 1024 workgroups, two rounds of two per CU (a causal launch's workgroups differ in
// length by as much as their tiles are many, and the longest, which start first, have to be short against the whole).  Not where sequences are
// shorter than a tile on average: there is nothing to share.  us, backward in bf16, unshared / at 512 / 1024 / 2048: 8192 tokens, 32 heads of 128 over 8
// 2150 / 2147 / 1785 / 1791; 4096 tokens, 16 heads of 64 over 4 215 / 215 / 175 / 178, in 16 sequences 65 / 65 / 57 / 62; 500 tokens in 60, 32 heads over 8
// 20 / 25 / 29 / 29.  Where wavefronts share the keys' rows (own == 32) it goes by the rows that a workgroup has left on average: LONG or more, of sequences
// that differ, 2048 workgroups for the longest one's sake (1024 / 2048: 16384 tokens in 20, 16 heads over 2, of 32 266 / 191, of 96 538 / 396), under
// SHORT, a few tiles a wavefront, 512 (1024 / 512: 4096
// tokens in 100, 12 heads of 64 over 4 44 / 29, fp32 16 of 96 over 2 199 / 166; in 40 of 32 over 2 72 / 89, 12 of 96 over 4 206 / 169).
int shares_of(const PackedAttention& a, int own) {
  constexpr int SHORT = 512, LONG = 3000;
  const int group = a.heads / a.kv_heads;
  const int64_t have = workgroups(a, own, a.kv_heads), mean = a.tokens / a.sequences;
  int shares = 1;
  if (mean < 32) return shares;
  for (int n = 2; n <= group && n <= a.max_parts; ++n) {
    const int64_t rows = mean * (group / shares);
    if (have * shares >= (own > 32 ? 1024 : rows < SHORT ? 512 : rows >= LONG && a.sequences > 1 ? 2048 : 1024)) break;
    if (group % n == 0) shares = n;
  }
  return shares;
}

template <typename T, bool SPLIT> hipError_t forward(const PackedAttention& a, hipStream_t stream) {
  const dim3 grid((unsigned)workgroups(a, SPLIT ? 32 : 128, a.heads));
  CDP_WIDTHS(hipLaunchKernelGGL((packed_fwd_kernel<T, SW, SPLIT>), grid, dim3(256), 0, stream, a));
  return hipGetLastError();
}
template <typename T, bool SPLIT> hipError_t backward_q(const PackedAttention& a, hipStream_t stream) {
  const dim3 grid((unsigned)workgroups(a, SPLIT ? 32 : 128, a.heads));
  CDP_WIDTHS(hipLaunchKernelGGL((packed_bwd_q_kernel<T, SW, SPLIT>), grid, dim3(256), 0, stream, a));
  return hipGetLastError();
}
template <typename T, bool SPLIT> hipError_t backward_kv(const PackedAttention& a, hipStream_t stream) {
  const int shares = shares_of(a, SPLIT ? 32 : 128);
  const dim3 grid((unsigned)workgroups(a, SPLIT ? 32 : 128, a.kv_heads) * shares);
  CDP_WIDTHS(hipLaunchKernelGGL((packed_bwd_kv_kernel<T, SW, SPLIT>), grid, dim3(256), 0, stream, a, shares));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || shares == 1) return e;
  const int64_t n = (int64_t)a.tokens * a.kv_heads * a.width / 8;
  hipLaunchKernelGGL((packed_bwd_fold_kernel<T>), dim3((unsigned)((n + 255) / 256), 2), dim3(256), 0, stream, a, shares);
  return hipGetLastError();
}
// One launch for queries and keys: where what it saves, a launch and a half-empty chip, is more than the deltas that every workgroup for keys makes for
// itself (us, two launches / one: bf16 width 64, 64 tokens, 4 heads over 2 11.4 / 6.7, 256 tokens, 8 heads 13.5 / 11.1, 128 tokens, 16 heads
// over 4 14.8 / 17.3; fp32 width 128, 512 tokens, 8 heads 82.6 / 57.9, 32 heads 119 / 137, 256 tokens in 8 sequences, 32 heads 62 / 60).
bool both_wanted(const PackedAttention& a) {
  const int64_t rows = (int64_t)a.tokens * (a.heads / a.kv_heads);
  return rows <= (a.heads == a.kv_heads ? OWN_ROWS : OWN_ROWS / 2) && workgroups(a, 32, a.heads + a.kv_heads) <= 512;
}
template <typename T> hipError_t backward_both(const PackedAttention& a, hipStream_t stream) {
  const unsigned queries = (unsigned)workgroups(a, 32, a.heads), keys = (unsigned)workgroups(a, 32, a.kv_heads);
  CDP_WIDTHS(hipLaunchKernelGGL((packed_bwd_both_kernel<T, SW>), dim3(queries + keys), dim3(256), 0, stream, a, queries));
  return hipGetLastError();
}
template <typename T> hipError_t backward(const PackedAttention& a, hipStream_t stream) {
  for (bool kv : {false, true})
    if (!launchable(workgroups(a, split_wanted<T>(a, kv) ? 32 : 128, kv ? a.kv_heads : a.heads), 256)) return hipErrorInvalidConfiguration;
  if (both_wanted(a)) return backward_both<T>(a, stream);
  const hipError_t e = split_wanted<T>(a, false) ? backward_q<T, true>(a, stream) : backward_q<T, false>(a, stream);
  if (e != hipSuccess) return e;
  return split_wanted<T>(a, true) ? backward_kv<T, true>(a, stream) : backward_kv<T, false>(a, stream);
}
template <typename T> hipError_t forward(const PackedAttention& a, hipStream_t stream) {
  if (!launchable(workgroups(a, split_wanted<T>(a, false) ? 32 : 128, a.heads), 256)) return hipErrorInvalidConfiguration;
  return split_wanted<T>(a, false) ? forward<T, true>(a, stream) : forward<T, false>(a, stream);
}

}  // namespace

hipError_t launch_packed_attention_fwd(const PackedAttention& a, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? forward<uint16_t>(a, stream) : forward<float>(a, stream);
}
hipError_t launch_packed_attention_bwd(const PackedAttention& a, int dtype, hipStream_t stream) {
  return dtype == DT_BF16 ? backward<uint16_t>(a, stream) : backward<float>(a, stream);
}

}  // namespace cdp
