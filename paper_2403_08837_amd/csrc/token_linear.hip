// Linear maps of tokens with what follows them in registers, and their gradients:
//   gated    h = act(g) u, g = x wg^T, u = x wu^T;   dg = dh u act'(g), du = dh act(g);   dx = dg wg + du wu,  dwg = dg^T x,  dwu = du^T x
//   linear   y = act(z) + residual, z = x w^T + bias;   dz = dy act'(z);   dx = dz w,  dw = dz^T x,  dbias = column sums of dz
//
// Long reductions over many rows are bound by the matrix cores.  One kernel makes all products: 32 x 32 x 16 bf16 matrix instructions, operands loaded straight
// into LDS as they lie in memory (16 bytes a lane).  An operand whose reduction index is the fast one (forward; dg, du, dz for dx) has tile rows of BK
// elements, read as 16-byte fragments; one whose reduction index is the slow one (weights for dx; both for the weights' gradients) has a tile row for every
// index, read by the transposing LDS loads: nothing is transposed in memory.  Both lie swizzled, so that a fragment read meets every bank once.
// Of a gated map a workgroup has as many columns of wg as of wu, dealt so that a wavefront holds both of the same columns, and the activation and the product
// happen in registers; g and u (z) are written beside h (y) where the backward is to follow.
//   fp32: an operand is cut into three bf16 planes (rounded: 2^-9, 2^-18 and 2^-27 of it are left), and the six products of planes of which more than 2^-26
// comes are segments of one reduction.
//   few tiles: the reduction is shared by `splits` workgroups, whose sums (fp32, in the workspace) are joined in order.
// Forward of up to 16 rows (single tokens): bound by reading the weights once (token_few_kernel).
#include "elem.h"
#include "gelu.h"
#include "kernels.h"

#include <algorithm>
#include <cstring>

namespace cdp {

namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float v4f_t;

// ---- activations ------------------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float sigmoid_of(float g, float& away) {
  float s;
  if constexpr (sizeof(T) == 2) {
    away = __expf(-g);
    s = __builtin_amdgcn_rcpf(1.f + away);
  } else {
    away = expf(-g);
    s = 1.f / (1.f + away);
  }
  away = fminf(away * s, 1.f);  // 1 - s, not as a difference (1 where that is inf * 0)
  return s;
}
template <typename T> __device__ __forceinline__ void act_both(int act, float g, float& a, float& da) {
  float away;
  if (act == TOKEN_SILU) {
    const float s = sigmoid_of<T>(g, away);
    a = g * s;
    da = s * fmaf(g, away, 1.f);
  } else if (act == TOKEN_GELU) {
    float Phi, phi;
    gauss<T>(g, Phi, phi);
    a = g * Phi;
    da = fmaf(g, phi, Phi);
  } else if (act == TOKEN_NONE) {
    a = g;
    da = 1.f;
  } else {
    a = sigmoid_of<T>(g, away);
    da = a * away;
  }
}

// (one branch for all values)
template <typename T, int N> __device__ __forceinline__ void act_all(int act, float (&v)[N]) {
  float away;
  if (act == TOKEN_SILU) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] *= sigmoid_of<T>(v[k], away);
  } else if (act == TOKEN_GELU) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = gelu_f<T>(v[k]);
  } else if (act == TOKEN_SIGMOID) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = sigmoid_of<T>(v[k], away);
  }
}

// ---- elementwise passes -----------------------------------------------------------------------------------------------
// Three bf16 planes of a float.
__device__ __forceinline__ void planes_of(float v, uint16_t (&p)[3]) {
  uint16_t h = f32_to_bf16(v);
  if ((h & 0x7fff) == 0x7f80 && fabsf(v) <= 3.402823466e38f) --h;  // rounded up to infinity
  p[0] = h;
  v -= bf16_to_f32(h);
  p[1] = f32_to_bf16(v);
  v -= bf16_to_f32(p[1]);
  p[2] = f32_to_bf16(v);
}
// Planes of up to three tensors, each [3][n]; n a multiple of 8.
struct Cut {
  const float* from[3];
  uint16_t* to[3];
  int64_t n[3];
  int64_t first[4];  // 8-element pieces of the tensors before
};
__global__ __launch_bounds__(256) void token_cut_kernel(const Cut c) {
  const int64_t piece = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (piece >= c.first[3]) return;
  const int t = (piece >= c.first[1]) + (piece >= c.first[2]);
  const int64_t i = (piece - c.first[t]) * 8;
  Chunk16<float> q[2];
  q[0].v = *reinterpret_cast<const uint4*>(c.from[t] + i);
  q[1].v = *reinterpret_cast<const uint4*>(c.from[t] + i + 4);
  Chunk16<uint16_t> o[3];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint16_t p[3];
    planes_of(q[e / 4].e[e % 4], p);
#pragma unroll
    for (int k = 0; k < 3; ++k) o[k].e[e] = p[k];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(c.to[t] + k * c.n[t] + i) = o[k].v;
}
// dg and du from g, u and dh.  bf16: rounded, as the operands of the products that follow; fp32: as planes.
template <typename T>
__global__ __launch_bounds__(256) void gated_grad_kernel(const T* g, const T* u, const T* dh, uint16_t* dg, uint16_t* du, int64_t n, int act) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  constexpr int Q = 8 / Elem<T>::VEC;
  Chunk16<T> a[Q], b[Q], d[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    a[q].v = *reinterpret_cast<const uint4*>(g + i + q * Elem<T>::VEC);
    b[q].v = *reinterpret_cast<const uint4*>(u + i + q * Elem<T>::VEC);
    d[q].v = *reinterpret_cast<const uint4*>(dh + i + q * Elem<T>::VEC);
  }
  Chunk16<uint16_t> og[sizeof(T) == 2 ? 1 : 3], ou[sizeof(T) == 2 ? 1 : 3];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    constexpr int V = Elem<T>::VEC;
    const float gv = Elem<T>::to_f32(a[e / V].e[e % V]), uv = Elem<T>::to_f32(b[e / V].e[e % V]), dv = Elem<T>::to_f32(d[e / V].e[e % V]);
    float f, df;
    act_both<T>(act, gv, f, df);
    const float x = dv * uv * df, y = dv * f;
    if constexpr (sizeof(T) == 2) {
      og[0].e[e] = f32_to_bf16(x);
      ou[0].e[e] = f32_to_bf16(y);
    } else {
      uint16_t p[3];
      planes_of(x, p);
#pragma unroll
      for (int k = 0; k < 3; ++k) og[k].e[e] = p[k];
      planes_of(y, p);
#pragma unroll
      for (int k = 0; k < 3; ++k) ou[k].e[e] = p[k];
    }
  }
#pragma unroll
  for (int k = 0; k < (sizeof(T) == 2 ? 1 : 3); ++k) {
    *reinterpret_cast<uint4*>(dg + k * n + i) = og[k].v;
    *reinterpret_cast<uint4*>(du + k * n + i) = ou[k].v;
  }
}

// dz from dy and z (act none: dy; dz null then in bf16), and its column sums: 256 columns of the rows blockIdx.y * share .. a workgroup, whose sums of dz as it
// is before it is rounded go to part[blockIdx.y][out] (null: not wanted), or, where there is one part, to dbias.
template <typename T>
__global__ __launch_bounds__(256) void linear_grad_kernel(const T* z, const T* dy, uint16_t* dz, float* part, T* dbias, int rows, int out, int share, int act) {
  constexpr int V = Elem<T>::VEC, Q = 8 / V;
  __shared__ float sums[8][256 + 8];
  const int lane = threadIdx.x & 31, strip = threadIdx.x >> 5, col = (blockIdx.x * 32 + lane) * 8;
  const int row0 = blockIdx.y * share, row1 = min(row0 + share, rows);
  const int64_t n = (int64_t)rows * out;
  float s[8] = {};
  if (col < out)
#pragma unroll 2
    for (int r = row0 + strip; r < row1; r += 8) {
      const int64_t i = (int64_t)r * out + col;
      Chunk16<T> a[Q], d[Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        d[q].v = *reinterpret_cast<const uint4*>(dy + i + q * V);
        a[q].v = act == TOKEN_NONE ? d[q].v : *reinterpret_cast<const uint4*>(z + i + q * V);
      }
      Chunk16<uint16_t> o[sizeof(T) == 2 ? 1 : 3];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float f, df, v = Elem<T>::to_f32(d[e / V].e[e % V]);
        act_both<T>(act, Elem<T>::to_f32(a[e / V].e[e % V]), f, df);
        v *= df;
        s[e] += v;
        if constexpr (sizeof(T) == 2) {
          o[0].e[e] = f32_to_bf16(v);
        } else {
          uint16_t p[3];
          planes_of(v, p);
#pragma unroll
          for (int k = 0; k < 3; ++k) o[k].e[e] = p[k];
        }
      }
      if (dz)
#pragma unroll
        for (int k = 0; k < (sizeof(T) == 2 ? 1 : 3); ++k) *reinterpret_cast<uint4*>(dz + k * n + i) = o[k].v;
    }
  if (!part && !dbias) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[strip][lane * 8 + e] = s[e];
  __syncthreads();
  const int c = threadIdx.x, at = blockIdx.x * 256 + c;
  if (at >= out) return;
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) v += sums[k][c];
  if (dbias) dbias[at] = Elem<T>::from_f32(v);
  else part[(int64_t)blockIdx.y * out + at] = v;
}
// 8 columns a workgroup, 32 lanes share the parts of a column.
template <typename T> __global__ __launch_bounds__(256) void linear_bias_kernel(const float* part, T* dbias, int parts, int out) {
  __shared__ float shares[32][8];
  const int c = threadIdx.x & 7, share = threadIdx.x >> 3, col = blockIdx.x * 8 + c;
  float s = 0.f;
#pragma unroll 8
  for (int k = share; k < parts; k += 32) s += part[(int64_t)k * out + col];
  shares[share][c] = s;
  __syncthreads();
  if (share) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) s += shares[k][c];
  dbias[col] = Elem<T>::from_f32(s);
}

// ---- the products -----------------------------------------------------------------------------------------------------
constexpr int MAX_SEGMENTS = 12;
// out[M][N] = sum over segments of A_s B_s, each over K.  A_s[m][k] at A[m * lda + k] (or A[k * lda + m]), B_s[n][k] likewise.
// GATED: the columns of B come from two matrices, B and B2, and the results are h (and g, u).  LINEAR: y (and z).  WGRAD with pair: two such products (dwg, dwu),
// the second of A2.
struct Product {
  const uint16_t *A[MAX_SEGMENTS], *B[MAX_SEGMENTS], *other[MAX_SEGMENTS / 2];  // other: B2 (GATED) or A2 (pair)
  int segments, K, M, N, lda, ldb;
  int tiles_m, tiles_n, tiles;  // of one product; of all
  int splits, slabs_per;        // parts of the reduction, slabs of each
  void *out, *out2, *out3;      // GATED: h, g, u (g, u may be null); LINEAR: y, z (or null); pair: dwg, dwu; else the result
  const void *bias, *residual;  // LINEAR: or null
  float* part;                  // splits > 1: sums [splits][results of all][M][N]
  int act, pair;
};
enum { GATED, LINEAR, DGRAD, WGRAD };

// One operand's slabs of BK on their way into LDS.  SLOW: its reduction index is the slow one in memory.
template <int TILE, int NWAVE, int BK, bool SLOW> struct Slabs {
  static constexpr int ROW = SLOW ? TILE * 2 : BK * 2, CPR = ROW / 16, RPB = 1024 / ROW;  // bytes and 16-byte chunks of a tile row, rows per 1 KB block
  static constexpr int BYTES = TILE * BK * 2, LP = BYTES / 1024 / NWAVE;                    // loads of a wavefront per slab
  static_assert(LP * 1024 * NWAVE == BYTES && CPR <= 64 && TILE >= 64, "tile rows are dealt to the wavefronts in 1 KB blocks");
  unsigned off[LP];  // byte offsets from the tile's first element in this slab, ~0: outside
  int chunk[2];      // !SLOW: first reduction index, in the slab, of the chunk of even and odd loads
  // chunk c of tile row r sits in slot c ^ swz(r)
  static __device__ __forceinline__ int swz(int r) { return SLOW ? 4 * piece(r) : (r >> 1) & 7; }
  static __device__ __forceinline__ int piece(int r) { return TILE >= 128 ? r & 3 : (r >> 1) & 1; }  // SLOW: 64-byte pieces of four rows on banks of their own
  // row_of: tile row -> row of the matrix, from the tile's first; `first` of `size` rows (SLOW: columns)
  template <typename F> __device__ __forceinline__ void start(int wave, int lane, int first, int size, int ld, F&& row_of) {
#pragma unroll
    for (int i = 0; i < LP; ++i) {
      const int r = (wave * LP + i) * RPB + lane / CPR, c = (lane % CPR) ^ swz(r);
      if (SLOW) off[i] = first + c * 8 < size ? 2u * ((unsigned)r * (unsigned)ld + c * 8) : ~0u;
      else off[i] = 2u * ((unsigned)min(row_of(r), size - 1 - first) * (unsigned)ld + c * 8);  // rows past the last repeat it
      if (!SLOW && i < 2) chunk[i] = c * 8;
    }
    static_assert(SLOW || (BK == 64 && LP % 2 == 0), "loads two apart have the same chunks");
  }
  // `left` reduction indices in the slab: what is past them reads as zero.  SLOW: they are rows, and the buffer ends there.
  __device__ __forceinline__ unsigned place(int i, int left) const { return SLOW || chunk[i & 1] < left ? off[i] : ~0u; }
  static __device__ __forceinline__ unsigned records(int left, int ld) { return SLOW ? 2u * (unsigned)left * (unsigned)ld : left > 0 ? 0xfffffff0u : 0u; }
};
__device__ __forceinline__ void load_lds(unsigned lds, unsigned off, const void* base, unsigned records) {
  typedef unsigned v4u __attribute__((ext_vector_type(4)));
  auto uniform = [](unsigned x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)x); };
  const uintptr_t p = (uintptr_t)base;
  const v4u buffer = {uniform((unsigned)p), uniform((unsigned)(p >> 32)), uniform(records), 0x00020000u};
  // The wait states are written out, the compiler does not look into assembly: one between the write of m0 and the load, five between a write of a
  // descriptor word by the vector unit and the load (s_mov_b32 is one, s_nop 3 four).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uniform(lds)), "v"(off), "s"(buffer) : "m0");
#pragma clang diagnostic pop
}
template <int N> __device__ __forceinline__ void wait_newest() {
  static_assert(N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}
__device__ __forceinline__ void slab_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Two groups of four values, of the columns n + 4 hi .. and n + 8 + 4 hi .. of a lane, as eight neighbouring columns n + 8 hi ..: 16 bytes of bf16.
__device__ __forceinline__ uint4 eight(const float* v) {
  auto two = [](float a, float b) { return (unsigned)f32_to_bf16(a) | (unsigned)f32_to_bf16(b) << 16; };
  const auto x = __builtin_amdgcn_permlane32_swap(two(v[0], v[1]), two(v[4], v[5]), false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(two(v[2], v[3]), two(v[6], v[7]), false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}
// A 32 x 32 block of results: row m, columns n ..; v[4 q + e] is column 8 q + 4 hi + e of it (q < 4, e < 4).
__device__ __forceinline__ void store_block(float* out, int64_t m, int n, int M, int N, int hi, const float (&v)[16]) {
  if (m >= M) return;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (n + 8 * q + 4 * hi < N) *reinterpret_cast<float4*>(out + m * N + n + 8 * q + 4 * hi) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
}
__device__ __forceinline__ void store_block(uint16_t* out, int64_t m, int n, int M, int N, int hi, const float (&v)[16]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const uint4 w = eight(v + 8 * q);
    if (m < M && n + 16 * q + 8 * hi < N) *reinterpret_cast<uint4*>(out + m * N + n + 16 * q + 8 * hi) = w;
  }
}
// Adds row m of a matrix to a block.
template <typename T> __device__ __forceinline__ void add_block(const T* from, int64_t m, int n, int M, int N, int hi, float (&v)[16]) {
  if (m >= M) return;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = n + 8 * q + 4 * hi;
    if (c >= N) continue;
    if constexpr (sizeof(T) == 4) {
      const float4 w = *reinterpret_cast<const float4*>(from + m * N + c);
      v[4 * q] += w.x;
      v[4 * q + 1] += w.y;
      v[4 * q + 2] += w.z;
      v[4 * q + 3] += w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(from + m * N + c);
      v[4 * q] += __uint_as_float(w.x << 16);
      v[4 * q + 1] += __uint_as_float(w.x & 0xffff0000u);
      v[4 * q + 2] += __uint_as_float(w.y << 16);
      v[4 * q + 3] += __uint_as_float(w.y & 0xffff0000u);
    }
  }
}

template <int WHAT, typename T, int BM, int BN, int WAVES_M, int WAVES_N, int BK, int STAGES, int WPS>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64, WPS) void token_product_kernel(const Product P) {
  constexpr int NWAVE = WAVES_M * WAVES_N, WTM = BM / WAVES_M, WTN = BN / WAVES_N, MI = WTM / 32, NI = WTN / 32, KK = BK / 16;
  constexpr bool DUAL = WHAT == GATED, ASLOW = WHAT == WGRAD, BSLOW = WHAT == DGRAD || WHAT == WGRAD;
  using SA = Slabs<BM, NWAVE, BK, ASLOW>;
  using SB = Slabs<BN, NWAVE, BK, BSLOW>;
  constexpr int STAGE_BYTES = SA::BYTES + SB::BYTES, LP = SA::LP + SB::LP, COLS = DUAL ? BN / 2 : BN;
  static_assert(!DUAL || NI % 2 == 0, "a wavefront has both of its columns");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[STAGES * STAGE_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WAVES_N, wn = wave % WAVES_N;
  const unsigned lds = (unsigned)(uintptr_t)(lds_ptr)smem;
  // tiles in panels of eight columns, row by row inside a panel; 32 neighbours in that order go to one XCD
  const int split = blockIdx.x / (unsigned)P.tiles;
  int tile = xcd_block_cyclic((int)(blockIdx.x - (unsigned)split * P.tiles), P.tiles, 32);
  const int one = P.tiles_m * P.tiles_n, second = WHAT == WGRAD && tile >= one;  // (of a pair)
  if (second) tile -= one;
  const int panel = tile / (P.tiles_m * 8), in = tile - panel * P.tiles_m * 8, pw = min(8, P.tiles_n - panel * 8), tm = in / pw;
  const int row0 = tm * BM, col0 = (panel * 8 + in - tm * pw) * COLS;

  // the slabs of this workgroup: `todo` from slab `split * slabs_per` of segment, slab order
  const int per_segment = (P.K + BK - 1) / BK, total = per_segment * P.segments;
  const int first_slab = split * P.slabs_per, todo = min(P.slabs_per, total - first_slab);
  SA sa;
  SB sb;
  const char *pa, *pb, *pb2;
  int seg = first_slab / per_segment, slab = first_slab - seg * per_segment, left = todo;
  int in_slab = min(BK, P.K - slab * BK);  // reduction indices in the next slab; 0 behind the last, and the loads that the counted waits expect read nothing
  auto b_row = [](int r) { return DUAL ? (r >> 6) * 32 + (r & 31) : r; };  // DUAL: 32 columns of B, 32 of B2, ..
  auto bases = [&] {
    const uint16_t* const a = (WHAT == WGRAD && second ? P.other[seg] : P.A[seg]);
    pa = reinterpret_cast<const char*>(ASLOW ? a + (int64_t)slab * BK * P.lda + row0 : a + (int64_t)row0 * P.lda + slab * BK);
    const uint16_t* const b = P.B[seg];
    pb = reinterpret_cast<const char*>(BSLOW ? b + (int64_t)slab * BK * P.ldb + col0 : b + (int64_t)col0 * P.ldb + slab * BK);
    if (DUAL) pb2 = reinterpret_cast<const char*>(P.other[seg] + (int64_t)col0 * P.ldb + slab * BK);
  };
  bases();
  sa.start(wave, lane, row0, P.M, P.lda, [](int r) { return r; });
  sb.start(wave, lane, col0, P.N, P.ldb, b_row);
  auto issue = [&](unsigned at, int e) {
    if (e < SA::LP) return load_lds(at + (wave * SA::LP + e) * 1024, sa.place(e, in_slab), pa, SA::records(in_slab, P.lda));
    const int i = e - SA::LP;
    const bool two = DUAL && (((wave * SB::LP + i) * SB::RPB >> 5) & 1);
    load_lds(at + SA::BYTES + (wave * SB::LP + i) * 1024, sb.place(i, in_slab), two ? pb2 : pb, SB::records(in_slab, P.ldb));
  };
  auto advance = [&] {
    if (--left <= 0) {
      in_slab = 0;
      return;
    }
    pa += ASLOW ? 2ll * BK * P.lda : 2ll * BK;
    pb += BSLOW ? 2ll * BK * P.ldb : 2ll * BK;
    if (DUAL) pb2 += 2 * BK;
    if (++slab == per_segment) {
      slab = 0;
      ++seg;
      bases();
    }
    in_slab = min(BK, P.K - slab * BK);
  };
#pragma unroll
  for (int q = 0; q < STAGES; ++q) {
#pragma unroll
    for (int e = 0; e < LP; ++e) issue(lds + q * STAGE_BYTES, e);
    advance();
  }
  v16f_t acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  // fragments.  fast index: row base + lane % 32, chunk 2 kk + lane / 32.  slow index: two transposing reads of rows k + 8 (lane / 32) + (lane % 16) / 4 (+ 4), four lanes
  // a row, 8 bytes each
  const int l31 = lane & 31, hi = lane >> 5, rho = lane & 15;
  auto slow_at = [&](int block, int row_bytes, int piece) {  // of 32 columns, number `block` of the tile
    return (8 * hi + (rho >> 2)) * row_bytes + (4 * (block ^ piece) + 2 * ((lane >> 4) & 1) + ((rho & 3) >> 1)) * 16 + 8 * (rho & 1);
  };
  unsigned xa[ASLOW ? MI : 1], xb[BSLOW ? NI : 1];
  if constexpr (ASLOW) {
#pragma unroll
    for (int i = 0; i < MI; ++i) xa[i] = slow_at(wm * MI + i, SA::ROW, SA::piece(rho >> 2));
  } else {
    xa[0] = (wm * WTM + l31) * SA::ROW;
  }
  if constexpr (BSLOW) {
#pragma unroll
    for (int j = 0; j < NI; ++j) xb[j] = SA::BYTES + slow_at(wn * NI + j, SB::ROW, SB::piece(rho >> 2));
  } else {
    xb[0] = SA::BYTES + (wn * WTN + l31) * SB::ROW;
  }
  uint4 fa[2][MI], fb[2][NI];
  auto slow = [&](unsigned at, int row_bytes) {
    union { v4s h[2]; uint4 u; } r;
    r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(smem + at));
    r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(smem + at + 4 * row_bytes));
    return r.u;
  };
  auto frag = [&](int q, int kk, int buf, int e) {
    if (e < MI) {
      if constexpr (ASLOW) fa[buf][e] = slow(q * STAGE_BYTES + xa[e] + kk * 16 * SA::ROW, SA::ROW);
      else fa[buf][e] = *reinterpret_cast<const uint4*>(smem + q * STAGE_BYTES + xa[0] + e * 32 * SA::ROW + (((kk * 2 + hi) ^ SA::swz(l31)) << 4));
    } else {
      if constexpr (BSLOW) fb[buf][e - MI] = slow(q * STAGE_BYTES + xb[e - MI] + kk * 16 * SB::ROW, SB::ROW);
      else fb[buf][e - MI] = *reinterpret_cast<const uint4*>(smem + q * STAGE_BYTES + xb[0] + (e - MI) * 32 * SB::ROW + (((kk * 2 + hi) ^ SB::swz(l31)) << 4));
    }
  };
  wait_newest<(STAGES - 1) * LP>();
  slab_barrier();
#pragma unroll
  for (int e = 0; e < MI + NI; ++e) frag(0, 0, 0, e);
  // a slab of stage q.  The barrier stands before its last step, whose fragments are in registers by then: the first fragments of the next slab are read and
  // the loads into the stage just freed requested between the products of that step
  auto step = [&](auto qc) {
    constexpr int q = decltype(qc)::value, next = (q + 1) % STAGES;
    constexpr int MN = MI * NI, RP = (MI + NI + MN - 1) / MN, IP = (LP + MN - 1) / MN;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const bool last = kk == KK - 1;
      if (last) {
        wait_newest<(STAGES - 2) * LP>();  // the next slab is whole, and every wavefront has read this one
        slab_barrier();
      }
#pragma unroll
      for (int e = 0; e < MN; ++e) {
        acc[e / NI][e % NI] = mfma_bf16(fb[kk & 1][e % NI], fa[kk & 1][e / NI], acc[e / NI][e % NI]);  // transposed: a lane has a row's neighbours
#pragma unroll
        for (int r = 0; r < RP; ++r)
          if (e * RP + r < MI + NI) frag(last ? next : q, last ? 0 : kk + 1, (kk + 1) & 1, e * RP + r);
#pragma unroll
        for (int r = 0; r < IP; ++r)
          if (last && e * IP + r < LP) issue(lds + q * STAGE_BYTES, e * IP + r);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    advance();
  };
  // whole rounds of the stages: slabs past the last are zeros, and one way out of the loop leaves the accumulators where they are
  for (int t = todo; t > 0; t -= STAGES) {
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    if constexpr (STAGES > 2) step(std::integral_constant<int, 2>{});
    if constexpr (STAGES > 3) step(std::integral_constant<int, 3>{});
  }
  wait_newest<0>();  // no load is left that writes LDS when this workgroup gives it back
  const int64_t MN = (int64_t)P.M * P.N;
  float* const part = P.part + (int64_t)split * (DUAL || P.pair ? 2 : 1) * MN;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t m = row0 + wm * WTM + i * 32 + l31;
#pragma unroll
    for (int j = 0; j < NI; j += DUAL ? 2 : 1) {
      const int n = DUAL ? col0 + (wn * NI + j) / 2 * 32 : col0 + wn * WTN + j * 32;
      float v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = acc[i][j][k];
      if (P.splits > 1) {
        store_block(part + (second ? MN : 0), m, n, P.M, P.N, hi, v);
        if constexpr (DUAL) {
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = acc[i][j + 1][k];
          store_block(part + MN, m, n, P.M, P.N, hi, v);
        }
      } else if constexpr (DUAL) {
        if (P.out2) {
          float u[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) u[k] = acc[i][j + 1][k];
          store_block(static_cast<T*>(P.out2), m, n, P.M, P.N, hi, v);
          store_block(static_cast<T*>(P.out3), m, n, P.M, P.N, hi, u);
        }
        act_all<T>(P.act, v);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] *= acc[i][j + 1][k];
        store_block(static_cast<T*>(P.out), m, n, P.M, P.N, hi, v);
      } else if constexpr (WHAT == LINEAR) {
        if (P.bias) add_block(static_cast<const T*>(P.bias), 0, n, 1, P.N, hi, v);
        if (P.out2) store_block(static_cast<T*>(P.out2), m, n, P.M, P.N, hi, v);
        act_all<T>(P.act, v);
        if (P.residual) add_block(static_cast<const T*>(P.residual), m, n, P.M, P.N, hi, v);
        store_block(static_cast<T*>(P.out), m, n, P.M, P.N, hi, v);
      } else {
        store_block(static_cast<T*>(second ? P.out2 : P.out), m, n, P.M, P.N, hi, v);
      }
      __builtin_amdgcn_sched_barrier(0);  // one block's values and addresses at a time
    }
  }
}
// Joins the sums of a shared reduction: eight neighbours a thread.
template <typename T> __global__ __launch_bounds__(256) void token_join_kernel(const Product P, int what) {
  const int64_t MN = (int64_t)P.M * P.N, stride = (what == GATED || P.pair ? 2 : 1) * MN, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= (what == GATED ? MN : stride)) return;
  auto sum = [&](int64_t at, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    for (int s = 0; s < P.splits; ++s) {
      Chunk16<float> q[2];
      q[0].v = *reinterpret_cast<const uint4*>(P.part + s * stride + at);
      q[1].v = *reinterpret_cast<const uint4*>(P.part + s * stride + at + 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += q[e / 4].e[e % 4];
    }
  };
  auto store = [&](void* out, int64_t at, const float (&v)[8]) {
    Chunk16<T> q[8 / Elem<T>::VEC];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e / Elem<T>::VEC].e[e % Elem<T>::VEC] = Elem<T>::from_f32(v[e]);
#pragma unroll
    for (int k = 0; k < 8 / Elem<T>::VEC; ++k) *reinterpret_cast<uint4*>(static_cast<T*>(out) + at + k * Elem<T>::VEC) = q[k].v;
  };
  auto add = [&](const void* from, int64_t at, float (&v)[8]) {
    Chunk16<T> q[8 / Elem<T>::VEC];
#pragma unroll
    for (int k = 0; k < 8 / Elem<T>::VEC; ++k) q[k].v = *reinterpret_cast<const uint4*>(static_cast<const T*>(from) + at + k * Elem<T>::VEC);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += Elem<T>::to_f32(q[e / Elem<T>::VEC].e[e % Elem<T>::VEC]);
  };
  float v[8];
  sum(i, v);
  if (what == LINEAR) {
    if (P.bias) add(P.bias, i % P.N, v);  // (N is a multiple of 8)
    if (P.out2) store(P.out2, i, v);
    act_all<T>(P.act, v);
    if (P.residual) add(P.residual, i, v);
    store(P.out, i, v);
  } else if (what == GATED) {
    float u[8];
    sum(MN + i, u);
    if (P.out2) {
      store(P.out2, i, v);
      store(P.out3, i, u);
    }
    act_all<T>(P.act, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= u[e];
    store(P.out, i, v);
  } else if (i < MN) {
    store(P.out, i, v);
  } else {
    store(P.out2, i - MN, v);
  }
}

// ---- few rows ---------------------------------------------------------------------------------------------------------
// Up to 16 rows of x: the 16 rows of one operand are eight columns of wg and of wu each, or 16 of w, those of the other the rows of x; the four wavefronts of a
// workgroup share the reduction.
struct Few {
  const void *x, *w, *w2;       // gated: wg, wu
  void *out, *out2, *out3;      // gated: h, g, u; else y, z
  const void *bias, *residual;
  int rows, in, cols, act;
};
template <typename T, bool DUAL> __global__ __launch_bounds__(256) void token_few_kernel(const Few a) {
  constexpr int V = Elem<T>::VEC, STEP = 4 * V, UNROLL = 8;  // reduction indices that the lanes of a wavefront have at once; such steps in flight
  __shared__ v4f_t shares[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, quarter = lane >> 4;
  const int col0 = blockIdx.x * (DUAL ? 8 : 16);  // (cols: a multiple of 8)
  const T* const w = static_cast<const T*>(DUAL && r >= 8 ? a.w2 : a.w) + (int64_t)(DUAL ? col0 + (r & 7) : min(col0 + r, a.cols - 1)) * a.in + quarter * V;
  const T* const x = static_cast<const T*>(a.x) + (int64_t)min(r, a.rows - 1) * a.in + quarter * V;
  v4f_t acc = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = wave * STEP * UNROLL; k0 < a.in; k0 += 4 * STEP * UNROLL) {
    uint4 p[UNROLL], q[UNROLL];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int k = k0 + i * STEP;
      const bool in = k + quarter * V < a.in;
      p[i] = in ? *reinterpret_cast<const uint4*>(w + k) : make_uint4(0, 0, 0, 0);
      q[i] = in ? *reinterpret_cast<const uint4*>(x + k) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf16_t, p[i]), __builtin_bit_cast(v8bf16_t, q[i]), acc, 0, 0, 0);
      } else {
        Chunk16<float> f, g;
        f.v = p[i];
        g.v = q[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(f.e[e], g.e[e], acc, 0, 0, 0);
      }
    }
  }
  shares[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
  // row of x lane % 16; columns 4 (lane / 16) .., gated: 4 (lane / 16 % 2) .. of wg (lanes below 32) or wu
  acc = (shares[0][lane] + shares[1][lane]) + (shares[2][lane] + shares[3][lane]);
  float u[4], v[4] = {acc[0], acc[1], acc[2], acc[3]};
  if constexpr (DUAL)
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __shfl(acc[e], lane + 32, 64);
  const int col = col0 + 4 * (DUAL ? quarter & 1 : quarter);
  if (r >= a.rows || col >= a.cols) return;
  const int64_t at = (int64_t)r * a.cols + col;
  auto store = [&](void* out) {
    if constexpr (sizeof(T) == 2) {
      Chunk16<T> c;
#pragma unroll
      for (int e = 0; e < 4; ++e) c.e[e] = Elem<T>::from_f32(v[e]);
      *reinterpret_cast<uint2*>(static_cast<T*>(out) + at) = c.h[0];
    } else {
      *reinterpret_cast<float4*>(static_cast<T*>(out) + at) = make_float4(v[0], v[1], v[2], v[3]);
    }
  };
  auto add = [&](const void* from, int64_t i) {
    if constexpr (sizeof(T) == 2) {
      Chunk16<T> c;
      c.h[0] = *reinterpret_cast<const uint2*>(static_cast<const T*>(from) + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += Elem<T>::to_f32(c.e[e]);
    } else {
      const float4 c = *reinterpret_cast<const float4*>(static_cast<const T*>(from) + i);
      v[0] += c.x;
      v[1] += c.y;
      v[2] += c.z;
      v[3] += c.w;
    }
  };
  if constexpr (DUAL) {
    if (a.out2) store(lane < 32 ? a.out2 : a.out3);
    if (lane >= 32) return;
    act_all<T>(a.act, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= u[e];
  } else {
    if (a.bias) add(a.bias, col);
    if (a.out2) store(a.out2);
    act_all<T>(a.act, v);
    if (a.residual) add(a.residual, at);
  }
  store(a.out);
}

// ---- launches ---------------------------------------------------------------------------------------------------------
template <int WHAT, typename T, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, int WPS> hipError_t launch_tiles(Product& p, int64_t room, hipStream_t stream) {
  constexpr int BK = 64, COLS = WHAT == GATED ? BN / 2 : BN;
  p.tiles_m = (p.M + BM - 1) / BM;
  p.tiles_n = (p.N + COLS - 1) / COLS;
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * (p.pair ? 2 : 1), slabs = (int64_t)(p.K + BK - 1) / BK * p.segments;
  if (!launchable(tiles, WAVES_M * WAVES_N * 64) || slabs > INT32_MAX) return hipErrorInvalidConfiguration;
  p.tiles = (int)tiles;
  // parts of at least 8 slabs while they all run at once
  const int64_t resident = 256 * (BM * BN >= 256 * 256 ? 1 : 2), MN = (int64_t)p.M * p.N * (WHAT == GATED || p.pair ? 2 : 1);
  int64_t splits = std::max<int64_t>(1, std::min({resident / tiles, slabs / 8, room / (4 * MN)}));
  p.slabs_per = (int)((slabs + splits - 1) / splits);
  p.splits = (int)((slabs + p.slabs_per - 1) / p.slabs_per);
  hipLaunchKernelGGL((token_product_kernel<WHAT, T, BM, BN, WAVES_M, WAVES_N, BK, STAGES, WPS>), dim3((unsigned)(tiles * p.splits)), dim3(WAVES_M * WAVES_N * 64), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const dim3 grid((unsigned)(((WHAT == GATED ? MN / 2 : MN) / 8 + 255) / 256));
  hipLaunchKernelGGL((token_join_kernel<T>), grid, dim3(256), 0, stream, p, (int)WHAT);
  return hipGetLastError();
}
template <int WHAT, typename T> hipError_t launch_tiled(Product& p, int64_t room, hipStream_t stream) {
  const int64_t cols = WHAT == GATED ? 2ll * p.N : p.N, pair = p.pair ? 2 : 1;
  if (((p.M + 255) / 256) * ((cols + 255) / 256) * pair >= 256) return launch_tiles<WHAT, T, 256, 256, 2, 4, 2, 2>(p, room, stream);
  if (p.M <= 64) return launch_tiles<WHAT, T, 64, 128, 2, 2, 3, 2>(p, room, stream);
  return launch_tiles<WHAT, T, 128, 128, 2, 2, 2, 2>(p, room, stream);
}

template <int WHAT> hipError_t launch_product(Product& p, int64_t room, bool f32, hipStream_t stream) {
  return f32 ? launch_tiled<WHAT, float>(p, room, stream) : launch_tiled<WHAT, uint16_t>(p, room, stream);
}

// The six products of planes, the smallest first.
constexpr int PLANE_A[6] = {2, 0, 1, 1, 0, 0}, PLANE_B[6] = {0, 2, 1, 0, 1, 0};

int64_t rounded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Tensors of n[i] floats in planes at `at`, and where what follows begins.
hipError_t cut(const void* const (&from)[3], const int64_t (&n)[3], char*& at, uint16_t* (&planes)[3], hipStream_t stream) {
  Cut c;
  c.first[0] = 0;
  for (int i = 0; i < 3; ++i) {
    c.from[i] = static_cast<const float*>(from[i]);
    c.to[i] = planes[i] = reinterpret_cast<uint16_t*>(at);
    c.n[i] = n[i];
    c.first[i + 1] = c.first[i] + n[i] / 8;
    at += rounded(6 * n[i]);
  }
  const int64_t groups = (c.first[3] + 255) / 256;
  if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(token_cut_kernel, dim3((unsigned)groups), dim3(256), 0, stream, c);
  return hipGetLastError();
}
template <bool DUAL> hipError_t launch_few(const Few& a, int dtype, hipStream_t stream) {
  const dim3 grid((a.cols + (DUAL ? 7 : 15)) / (DUAL ? 8 : 16));
  if (dtype == DT_BF16) hipLaunchKernelGGL((token_few_kernel<uint16_t, DUAL>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((token_few_kernel<float, DUAL>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}
constexpr int FEW_ROWS = 16;
// The segments of a product of planes: `n` elements of A and B a plane; in bf16 the one of A and B.
struct Segments {
  int count;
  int a[6], b[6];
  explicit Segments(bool f32) : count(f32 ? 6 : 1) {
    for (int s = 0; s < count; ++s) {
      a[s] = f32 ? PLANE_A[s] : 0;
      b[s] = f32 ? PLANE_B[s] : 0;
    }
  }
};

}  // namespace

// Bytes that the calls cannot do without.
int64_t gated_linear_workspace_bytes(bool backward, int rows, int in, int hidden, int dtype) {
  const int64_t planes = dtype == DT_F32 ? 6 * ((int64_t)rows * in + 2ll * hidden * in) + 1024 : 0;
  if (!backward) return planes;
  return planes + (dtype == DT_F32 ? 12 : 4) * (int64_t)rows * hidden + 1024;
}
int64_t token_linear_workspace_bytes(bool backward, int rows, int in, int out, int dtype) {
  const int64_t planes = dtype == DT_F32 ? 6 * ((int64_t)rows * in + (int64_t)out * in) + 1024 : 0;
  if (!backward) return planes;
  return planes + (dtype == DT_F32 ? 6 : 2) * (int64_t)rows * out + 4ll * out * std::min(rows, LINEAR_MAX_PARTS) + 1024;
}

hipError_t launch_gated_linear(const GatedLinear& a, int dtype, hipStream_t stream) {
  if (a.rows <= FEW_ROWS) return launch_few<true>({a.x, a.wg, a.wu, a.h, a.g, a.u, nullptr, nullptr, a.rows, a.in, a.hidden, a.act}, dtype, stream);
  Product p;
  memset(&p, 0, sizeof(p));
  p.K = a.in; p.M = a.rows; p.N = a.hidden; p.lda = p.ldb = a.in;
  p.out = a.h; p.out2 = a.g; p.out3 = a.u;
  p.act = a.act;
  const bool f32 = dtype == DT_F32;
  char *at = static_cast<char*>(a.workspace), *const end = at + a.workspace_bytes;
  const int64_t xn = (int64_t)a.rows * a.in, wn = (int64_t)a.hidden * a.in;
  const uint16_t *x = static_cast<const uint16_t*>(a.x), *wg = static_cast<const uint16_t*>(a.wg), *wu = static_cast<const uint16_t*>(a.wu);
  if (f32) {
    uint16_t* planes[3];
    const hipError_t e = cut({a.x, a.wg, a.wu}, {xn, wn, wn}, at, planes, stream);
    if (e != hipSuccess) return e;
    x = planes[0];
    wg = planes[1];
    wu = planes[2];
  }
  const Segments of(f32);
  p.segments = of.count;
  for (int s = 0; s < of.count; ++s) {
    p.A[s] = x + of.a[s] * xn;
    p.B[s] = wg + of.b[s] * wn;
    p.other[s] = wu + of.b[s] * wn;
  }
  p.part = reinterpret_cast<float*>(at);
  return launch_product<GATED>(p, std::max<int64_t>(0, end - at), f32, stream);
}

hipError_t launch_gated_linear_bwd(const GatedLinear& a, int dtype, hipStream_t stream) {
  char *at = static_cast<char*>(a.workspace), *const end = at + a.workspace_bytes;
  const int64_t n = (int64_t)a.rows * a.hidden, groups = (n / 8 + 255) / 256, xn = (int64_t)a.rows * a.in, wn = (int64_t)a.hidden * a.in;
  if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
  const bool f32 = dtype == DT_F32;
  const uint16_t *x = static_cast<const uint16_t*>(a.x), *wg = static_cast<const uint16_t*>(a.wg), *wu = static_cast<const uint16_t*>(a.wu);
  hipError_t e;
  if (f32) {
    uint16_t* planes[3];
    e = cut({a.x, a.wg, a.wu}, {xn, wn, wn}, at, planes, stream);
    if (e != hipSuccess) return e;
    x = planes[0];
    wg = planes[1];
    wu = planes[2];
  }
  uint16_t* const dg = reinterpret_cast<uint16_t*>(at);
  at += rounded((f32 ? 6 : 2) * n);
  uint16_t* const du = reinterpret_cast<uint16_t*>(at);
  at += rounded((f32 ? 6 : 2) * n);
  if (f32) {
    hipLaunchKernelGGL((gated_grad_kernel<float>), dim3((unsigned)groups), dim3(256), 0, stream, static_cast<const float*>(a.g), static_cast<const float*>(a.u),
                       static_cast<const float*>(a.dh), dg, du, n, a.act);
  } else {
    hipLaunchKernelGGL((gated_grad_kernel<uint16_t>), dim3((unsigned)groups), dim3(256), 0, stream, static_cast<const uint16_t*>(a.g),
                       static_cast<const uint16_t*>(a.u), static_cast<const uint16_t*>(a.dh), dg, du, n, a.act);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const Segments of(f32);
  Product p;
  if (a.dx) {
    memset(&p, 0, sizeof(p));
    p.segments = 2 * of.count;
    p.K = a.hidden; p.M = a.rows; p.N = a.in; p.lda = a.hidden; p.ldb = a.in;
    for (int s = 0; s < of.count; ++s) {
      p.A[2 * s] = dg + of.a[s] * n;
      p.A[2 * s + 1] = du + of.a[s] * n;
      p.B[2 * s] = wg + of.b[s] * wn;
      p.B[2 * s + 1] = wu + of.b[s] * wn;
    }
    p.out = a.dx; p.part = reinterpret_cast<float*>(at);
    e = launch_product<DGRAD>(p, std::max<int64_t>(0, end - at), f32, stream);
    if (e != hipSuccess) return e;
  }
  if (a.dwg) {
    memset(&p, 0, sizeof(p));
    p.segments = of.count;
    p.K = a.rows; p.M = a.hidden; p.N = a.in; p.lda = a.hidden; p.ldb = a.in;
    for (int s = 0; s < of.count; ++s) {
      p.A[s] = dg + of.a[s] * n;
      p.other[s] = du + of.a[s] * n;
      p.B[s] = x + of.b[s] * xn;
    }
    p.out = a.dwg; p.out2 = a.dwu; p.pair = 1; p.part = reinterpret_cast<float*>(at);
    e = launch_product<WGRAD>(p, std::max<int64_t>(0, end - at), f32, stream);
  }
  return e;
}

hipError_t launch_token_linear(const TokenLinear& a, int dtype, hipStream_t stream) {
  if (a.rows <= FEW_ROWS) return launch_few<false>({a.x, a.w, nullptr, a.y, a.z, nullptr, a.bias, a.residual, a.rows, a.in, a.out, a.act}, dtype, stream);
  Product p;
  memset(&p, 0, sizeof(p));
  p.K = a.in; p.M = a.rows; p.N = a.out; p.lda = p.ldb = a.in;
  p.out = a.y; p.out2 = a.z; p.bias = a.bias; p.residual = a.residual;
  p.act = a.act;
  const bool f32 = dtype == DT_F32;
  char *at = static_cast<char*>(a.workspace), *const end = at + a.workspace_bytes;
  const int64_t xn = (int64_t)a.rows * a.in, wn = (int64_t)a.out * a.in;
  const uint16_t *x = static_cast<const uint16_t*>(a.x), *w = static_cast<const uint16_t*>(a.w);
  if (f32) {
    uint16_t* planes[3];
    const hipError_t e = cut({a.x, a.w, nullptr}, {xn, wn, 0}, at, planes, stream);
    if (e != hipSuccess) return e;
    x = planes[0];
    w = planes[1];
  }
  const Segments of(f32);
  p.segments = of.count;
  for (int s = 0; s < of.count; ++s) {
    p.A[s] = x + of.a[s] * xn;
    p.B[s] = w + of.b[s] * wn;
  }
  p.part = reinterpret_cast<float*>(at);
  return launch_product<LINEAR>(p, std::max<int64_t>(0, end - at), f32, stream);
}

hipError_t launch_token_linear_bwd(const TokenLinear& a, int dtype, hipStream_t stream) {
  char *at = static_cast<char*>(a.workspace), *const end = at + a.workspace_bytes;
  const int64_t n = (int64_t)a.rows * a.out, xn = (int64_t)a.rows * a.in, wn = (int64_t)a.out * a.in;
  const bool f32 = dtype == DT_F32;
  const uint16_t *x = static_cast<const uint16_t*>(a.x), *w = static_cast<const uint16_t*>(a.w), *dz = static_cast<const uint16_t*>(a.dy);
  hipError_t e = hipSuccess;
  const bool products = a.dx || a.dw;
  if (f32 && products) {
    uint16_t* planes[3];
    e = cut({a.x, a.w, nullptr}, {xn, wn, 0}, at, planes, stream);
    if (e != hipSuccess) return e;
    x = planes[0];
    w = planes[1];
  }
  // places in the workspace, whatever is wanted: a result does not depend on which others are
  at = static_cast<char*>(a.workspace) + (f32 ? rounded(6 * xn) + rounded(6 * wn) : 0);
  uint16_t* to = nullptr;  // dz, where it is not dy
  if (products && (f32 || a.act != TOKEN_NONE)) dz = to = reinterpret_cast<uint16_t*>(at);
  at += rounded((f32 ? 6 : 2) * n);
  float* const sums = reinterpret_cast<float*>(at);
  at += rounded(4ll * a.out * std::min(a.rows, LINEAR_MAX_PARTS));
  if (to || a.dbias) {
    // strips of 32 rows at least, for as many workgroups as run at once
    const int columns = (a.out + 255) / 256;
    int share = std::max({32, (a.rows + LINEAR_MAX_PARTS - 1) / LINEAR_MAX_PARTS});
    const int parts = (a.rows + share - 1) / share;
    float* const part = a.dbias && parts > 1 ? sums : nullptr;
    const dim3 grid(columns, parts);
    if (f32) {
      hipLaunchKernelGGL((linear_grad_kernel<float>), grid, dim3(256), 0, stream, static_cast<const float*>(a.z), static_cast<const float*>(a.dy), to, part,
                         part ? nullptr : static_cast<float*>(a.dbias), a.rows, a.out, share, a.act);
    } else {
      hipLaunchKernelGGL((linear_grad_kernel<uint16_t>), grid, dim3(256), 0, stream, static_cast<const uint16_t*>(a.z), static_cast<const uint16_t*>(a.dy), to,
                         part, part ? nullptr : static_cast<uint16_t*>(a.dbias), a.rows, a.out, share, a.act);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (part) {
      if (f32) hipLaunchKernelGGL((linear_bias_kernel<float>), dim3(a.out / 8), dim3(256), 0, stream, part, static_cast<float*>(a.dbias), parts, a.out);
      else hipLaunchKernelGGL((linear_bias_kernel<uint16_t>), dim3(a.out / 8), dim3(256), 0, stream, part, static_cast<uint16_t*>(a.dbias), parts, a.out);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  const Segments of(f32);
  Product p;
  if (a.dx) {
    memset(&p, 0, sizeof(p));
    p.segments = of.count;
    p.K = a.out; p.M = a.rows; p.N = a.in; p.lda = a.out; p.ldb = a.in;
    for (int s = 0; s < of.count; ++s) {
      p.A[s] = dz + of.a[s] * n;
      p.B[s] = w + of.b[s] * wn;
    }
    p.out = a.dx; p.part = reinterpret_cast<float*>(at);
    e = launch_product<DGRAD>(p, std::max<int64_t>(0, end - at), f32, stream);
    if (e != hipSuccess) return e;
  }
  if (a.dw) {
    memset(&p, 0, sizeof(p));
    p.segments = of.count;
    p.K = a.rows; p.M = a.out; p.N = a.in; p.lda = a.out; p.ldb = a.in;
    for (int s = 0; s < of.count; ++s) {
      p.A[s] = dz + of.a[s] * n;
      p.B[s] = x + of.b[s] * xn;
    }
    p.out = a.dw; p.part = reinterpret_cast<float*>(at);
    e = launch_product<WGRAD>(p, std::max<int64_t>(0, end - at), f32, stream);
  }
  return e;
}

}  // namespace cdp
