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
//   fp32 (exact_body): operands pass through registers, where each is cut into three bf16 planes (rounded: 2^-9, 2^-18 and 2^-27 of it are left), which lie in LDS as
// the bf16 operands do; the six products of planes of which more than 2^-26 comes are added up, the smallest first.
//   few tiles: the reduction is shared by `splits` workgroups, whose sums (fp32, in the workspace) are joined in order.
// Forward of few rows (single tokens, up to 64): bound by reading the weights once and the rows from cache (token_few_kernel); backward of few outputs one launch (token_few_backward_kernel).
#include "elem.h"
#include "gelu.h"
#include "kernels.h"
#include "lane_sums.h"

#include <algorithm>
#include <climits>
#include <cmath>
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
// Eight neighbours.
template <typename T> struct Eight {
  static constexpr int V = Elem<T>::VEC, Q = 8 / V;
  Chunk16<T> q[Q];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int k = 0; k < Q; ++k) q[k].v = *reinterpret_cast<const uint4*>(p + k * V);
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int k = 0; k < Q; ++k) *reinterpret_cast<uint4*>(p + k * V) = q[k].v;
  }
  __device__ __forceinline__ float operator[](int e) const { return Elem<T>::to_f32(q[e / V].e[e % V]); }
  __device__ __forceinline__ void set(int e, float v) { q[e / V].e[e % V] = Elem<T>::from_f32(v); }
};
// dg and du from g, u and dh.  Memory: three read, two written: 8192 x 12288 in bf16 173 to 190 us (5.3 to 5.8 TB/s), 6272 x 2048 20.
// bf16: they are rounded, being operands of the products that follow, and so were g and u, being written: dx, dwg and dwu are 3.0e-3 of their norm off (6272 x 768 x 2048),
// 1.7e-3 of that their own rounding.  With two bf16 each for dg and du the products would take twice their time (8192 x 4096 x 12288 2.5 of 4.0 ms); with g and u made again
// from x, instead of read, half as much more.
template <typename T> __global__ __launch_bounds__(256) void gated_grad_kernel(const T* g, const T* u, const T* dh, T* dg, T* du, int64_t n, int act) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  Eight<T> a, b, d;
  a.load(g + i);
  b.load(u + i);
  d.load(dh + i);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float f, df;
    act_both<T>(act, a[e], f, df);
    const float x = d[e] * b[e] * df, y = d[e] * f;
    a.set(e, x);
    b.set(e, y);
  }
  a.store(dg + i);
  b.store(du + i);
}
// Memory: 1999 x 1368 in fp32 with its sums 9.6 us (3.4 TB/s; 1500 short workgroups).
// bf16: dz is rounded, as above: dx and dw are 2.4e-3 of their norm off (6272 x 768 x 2048, GELU), 1.7e-3 of that their own rounding; z as the forward rounded it is hardly any of it. The products
// would take twice their time with two bf16 for dz (413 to 450 us for 8192 x 4096 x 4096).
// dz from dy and z (null: not wanted, or it is dy), and its column sums: 256 columns of the rows blockIdx.y * share .. a workgroup, whose sums of dz as it
// is before it is rounded go to part[blockIdx.y][out] (null: not wanted), or, where there is one part, to dbias.
template <typename T>
__global__ __launch_bounds__(256) void linear_grad_kernel(const T* z, const T* dy, T* dz, float* part, T* dbias, int rows, int out, int share, int act) {
  __shared__ float sums[8][256 + 8];
  const int lane = threadIdx.x & 31, strip = threadIdx.x >> 5, col = (blockIdx.x * 32 + lane) * 8;
  const int row0 = blockIdx.y * share, row1 = min(row0 + share, rows);
  float s[8] = {};
  if (col < out)
#pragma unroll 4
    for (int r = row0 + strip; r < row1; r += 8) {
      const int64_t i = (int64_t)r * out + col;
      Eight<T> a, d;
      d.load(dy + i);
      if (act != TOKEN_NONE) a.load(z + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float f, df = 1.f;
        if (act != TOKEN_NONE) act_both<T>(act, a[e], f, df);
        const float v = d[e] * df;
        s[e] += v;
        d.set(e, v);
      }
      if (dz) d.store(dz + i);
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
// Sums of the parts of dbias: THREADS / 32 columns a workgroup, 32 lanes share the parts of a column.
struct BiasParts {
  const float* part;
  void* dbias;
  int parts, out;
};
template <typename T, int THREADS> __device__ __forceinline__ void bias_body(const BiasParts& a, int block, unsigned char* smem) {
  constexpr int C = THREADS / 32;
  float* const shares = reinterpret_cast<float*>(smem);
  const int c = threadIdx.x % C, share = threadIdx.x / C, col = block * C + c;
  float s = 0.f;
  if (col < a.out)
#pragma unroll 8
    for (int k = share; k < a.parts; k += 32) s += a.part[(int64_t)k * a.out + col];
  shares[share * C + c] = s;
  __syncthreads();
  if (share || col >= a.out) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) s += shares[k * C + c];
  static_cast<T*>(a.dbias)[col] = Elem<T>::from_f32(s);
}

// ---- the products -----------------------------------------------------------------------------------------------------
// out[M][N] = sum over segments of A_s B_s, each over K.  A_s[m][k] at A[m * lda + k] (WGRAD: A[k * lda + m]), B_s[n][k] likewise (DGRAD, WGRAD: B[k * ldb + n]).
// GATED: the columns of B come from two matrices, B and `other`, and the results are h (and g, u).  LINEAR: y (and z).  WGRAD with pair: two such products (dwg,
// dwu), the second of `other` for A.
struct Product {
  const void *A[2], *B[2], *other;
  int segments, K, M, N, lda, ldb;
  int tiles_m, tiles_n, tiles;  // of one product; of all
  int splits, slabs_per;        // parts of the reduction, slabs of each
  void *out, *out2, *out3;      // GATED: h, g, u (g, u may be null); LINEAR: y, z (or null); pair: dwg, dwu; else the result
  const void *bias, *residual;  // LINEAR: or null
  float* part;                  // splits > 1: sums [splits][results of all][M][N]
  int act, pair;
  int workgroups() const { return tiles * splits; }
};
enum { GATED, LINEAR, DGRAD, WGRAD };

// One operand's slabs of BK on their way into LDS.  SLOW: its reduction index is the slow one in memory.
template <int TILE, int NWAVE, int BK, bool SLOW> struct Slabs {
  static constexpr int ROW = SLOW ? TILE * 2 : BK * 2, CPR = ROW / 16, RPB = 1024 / ROW;  // bytes and 16-byte chunks of a tile row, rows per 1 KB block
  static constexpr int BYTES = TILE * BK * 2, LP = BYTES / 1024 / NWAVE;                    // loads of a wavefront per slab
  static_assert(LP * 1024 * NWAVE == BYTES && CPR <= 64 && TILE >= 64, "tile rows are dealt to the wavefronts in 1 KB blocks");
  unsigned off[LP];  // byte offsets from the tile's first element in this slab, ~0: outside
  static constexpr int KINDS = BK == 32 ? 1 : BK == 64 ? 2 : 4;
  int chunk[KINDS];  // !SLOW: first reduction index, in the slab, of the chunk of load i: the same for loads KINDS apart
  // chunk c of tile row r sits in slot c ^ swz(r)
  static __device__ __forceinline__ int swz(int r) { return SLOW ? 4 * piece(r) : BK == 32 ? (r >> 2) & 3 : BK == 64 ? (r >> 1) & 7 : r & 15; }
  static __device__ __forceinline__ int piece(int r) { return TILE >= 128 ? r & 3 : (r >> 1) & 1; }  // SLOW: 64-byte pieces of four rows on banks of their own
  // row_of: tile row -> row of the matrix, from the tile's first; `first` of `size` rows (SLOW: columns)
  template <typename F> __device__ __forceinline__ void start(int wave, int lane, int first, int size, int ld, F&& row_of) {
#pragma unroll
    for (int i = 0; i < LP; ++i) {
      const int r = (wave * LP + i) * RPB + lane / CPR, c = (lane % CPR) ^ swz(r);
      if (SLOW) off[i] = first + c * 8 < size ? 2u * ((unsigned)r * (unsigned)ld + c * 8) : ~0u;
      else off[i] = 2u * ((unsigned)min(row_of(r), size - 1 - first) * (unsigned)ld + c * 8);  // rows past the last repeat it
      if (!SLOW && i < KINDS) chunk[i] = c * 8;
    }
    static_assert(SLOW || ((BK == 32 || BK == 64 || BK == 128) && LP % KINDS == 0), "rows of a load and of the one KINDS on swizzle alike");
  }
  // `left` reduction indices in the slab: what is past them reads as zero.  SLOW: they are rows, and the buffer ends there.
  __device__ __forceinline__ unsigned place(int i, int left) const { return SLOW || chunk[i & (KINDS - 1)] < left ? off[i] : ~0u; }
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

__device__ __forceinline__ unsigned two_bf16(float a, float b) {  // (one instruction)
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  typedef float v2f __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((v2f){a, b}, v2bf));
}
// Two groups of four values, of the columns n + 4 hi .. and n + 8 + 4 hi .. of a lane, as eight neighbouring columns n + 8 hi ..: 16 bytes of bf16.
__device__ __forceinline__ uint4 eight(const float* v) {
  const auto x = __builtin_amdgcn_permlane32_swap(two_bf16(v[0], v[1]), two_bf16(v[4], v[5]), false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(two_bf16(v[2], v[3]), two_bf16(v[6], v[7]), false, false);
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

// What a workgroup makes of a product: its tile, its part of the reduction.
template <int WHAT, int BM, int BN, int BK> struct Share {
  int row0, col0, split, todo;  // slabs of BK to do
  bool second;                  // of a pair
  int seg, slab, per_segment;   // the first of them
  __device__ __forceinline__ Share(const Product& P, int block) {
    constexpr int COLS = WHAT == GATED ? BN / 2 : BN;
    split = block / P.tiles;
    // tiles in panels of eight columns, row by row inside a panel; 32 neighbours in that order go to one XCD
    int tile = xcd_block_cyclic(block - split * P.tiles, P.tiles, 32);
    const int one = P.tiles_m * P.tiles_n;
    second = WHAT == WGRAD && tile >= one;
    if (second) tile -= one;
    const int panel = tile / (P.tiles_m * 8), in = tile - panel * P.tiles_m * 8, pw = min(8, P.tiles_n - panel * 8), tm = in / pw;
    row0 = tm * BM;
    col0 = (panel * 8 + in - tm * pw) * COLS;
    per_segment = (int)(((unsigned)P.K + BK - 1) / BK);
    const int first = split * P.slabs_per;
    todo = min(P.slabs_per, per_segment * P.segments - first);
    seg = first / per_segment;
    slab = first - seg * per_segment;
  }
};
// A barrier for what is in LDS: loads into registers stay on their way (__syncthreads waits for them).
__device__ __forceinline__ void lds_barrier() {
  wait_newest<63>();
  slab_barrier();
}
// From the accumulators: block (i, j) of a wavefront, transposed (a lane has neighbouring columns of one row), of rows m0 + 32 i and columns n0 + 32 j; GATED: the
// columns n0 + 16 j of both, at j and j + 1.
template <int WHAT, typename T, int MI, int NI>
__device__ __forceinline__ void leave(const Product& P, const v16f_t (&acc)[MI][NI], int m0, int n0, int split, bool second, int lane) {
  constexpr bool DUAL = WHAT == GATED;
  const int l31 = lane & 31, hi = lane >> 5;
  const int64_t MN = (int64_t)P.M * P.N;
  float* const part = P.part + (int64_t)split * (DUAL || P.pair ? 2 : 1) * MN;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t m = m0 + i * 32 + l31;
#pragma unroll
    for (int j = 0; j < NI; j += DUAL ? 2 : 1) {
      const int n = n0 + j * (DUAL ? 16 : 32);
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

template <int WHAT, typename T, int BM, int BN, int WAVES_M, int WAVES_N, int BK, int STAGES>
__device__ __forceinline__ void product_body(const Product& P, int block, unsigned char* smem) {
  constexpr int NWAVE = WAVES_M * WAVES_N, WTM = BM / WAVES_M, WTN = BN / WAVES_N, MI = WTM / 32, NI = WTN / 32, KK = BK / 16;
  constexpr bool DUAL = WHAT == GATED, ASLOW = WHAT == WGRAD, BSLOW = WHAT == DGRAD || WHAT == WGRAD;
  using SA = Slabs<BM, NWAVE, BK, ASLOW>;
  using SB = Slabs<BN, NWAVE, BK, BSLOW>;
  constexpr int STAGE_BYTES = SA::BYTES + SB::BYTES, LP = SA::LP + SB::LP;
  static_assert(!DUAL || NI % 2 == 0, "a wavefront has both of its columns");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WAVES_N, wn = wave % WAVES_N;
  const unsigned lds = (unsigned)(uintptr_t)(lds_ptr)smem;
  const Share<WHAT, BM, BN, BK> at(P, block);
  const int row0 = at.row0, col0 = at.col0, per_segment = at.per_segment;
  SA sa;
  SB sb;
  const char *pa, *pb, *pb2;
  int seg = at.seg, slab = at.slab, left = at.todo;
  int in_slab = min(BK, P.K - slab * BK);  // reduction indices in the next slab; 0 behind the last, and the loads that the counted waits expect read nothing
  auto b_row = [](int r) { return DUAL ? (r >> 6) * 32 + (r & 31) : r; };  // DUAL: 32 columns of B, 32 of B2, ..
  auto bases = [&] {
    const uint16_t* const a = static_cast<const uint16_t*>(at.second ? P.other : P.A[seg]);
    pa = reinterpret_cast<const char*>(ASLOW ? a + (int64_t)slab * BK * P.lda + row0 : a + (int64_t)row0 * P.lda + slab * BK);
    const uint16_t* const b = static_cast<const uint16_t*>(P.B[seg]);
    pb = reinterpret_cast<const char*>(BSLOW ? b + (int64_t)slab * BK * P.ldb + col0 : b + (int64_t)col0 * P.ldb + slab * BK);
    if (DUAL) pb2 = reinterpret_cast<const char*>(static_cast<const uint16_t*>(P.other) + (int64_t)col0 * P.ldb + slab * BK);
  };
  bases();
  sa.start(wave, lane, row0, P.M, P.lda, [](int r) { return r; });
  sb.start(wave, lane, col0, P.N, P.ldb, b_row);
  auto issue = [&](unsigned to, int e) {
    if (e < SA::LP) return load_lds(to + (wave * SA::LP + e) * 1024, sa.place(e, in_slab), pa, SA::records(in_slab, P.lda));
    const int i = e - SA::LP;
    const bool two = DUAL && (((wave * SB::LP + i) * SB::RPB >> 5) & 1);
    load_lds(to + SA::BYTES + (wave * SB::LP + i) * 1024, sb.place(i, in_slab), two ? pb2 : pb, SB::records(in_slab, P.ldb));
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
  auto slow = [&](unsigned from, int row_bytes) {
    union { v4s h[2]; uint4 u; } r;
    r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(smem + from));
    r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(smem + from + 4 * row_bytes));
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
  // Large tiles: whole rounds of the stages, slabs past the last are zeros; one way out of the loop leaves the accumulators where they are (with a way out
  // behind every step they are copied, and spilled: 8192 x 4096 x 4096 1080 us instead of 216).
  constexpr bool ROUNDS = MI * NI > 2;
  for (int t = at.todo; t > 0; t -= STAGES) {
    step(std::integral_constant<int, 0>{});
    if (!ROUNDS && t == 1) break;
    step(std::integral_constant<int, 1>{});
    if constexpr (STAGES > 2) {
      if (!ROUNDS && t == 2) break;
      step(std::integral_constant<int, 2>{});
    }
    if constexpr (STAGES > 3) {
      if (!ROUNDS && t == 3) break;
      step(std::integral_constant<int, 3>{});
    }
  }
  wait_newest<0>();  // no load is left that writes LDS when this workgroup gives it back
  leave<WHAT, T>(P, acc, at.row0 + wm * WTM, at.col0 + wn * (DUAL ? WTN / 2 : WTN), at.split, at.second, lane);
}
// ---- fp32 -------------------------------------------------------------------------------------------------------------
// An fp32 operand's slab of 32 on its way into three planes of bf16 in LDS.  Loads are in flight while the slab before is contracted.
template <int TILE, bool SLOW> struct Planes {
  static constexpr int BK = 32, LP = TILE * BK / 4 / 256, PER_ROW = SLOW ? TILE / 4 : BK / 4;  // 16-byte loads of a thread; of a tile row
  static constexpr int ROW = SLOW ? TILE * 2 : BK * 2, BYTES = TILE * BK * 2;                    // of a plane
  unsigned off[LP];
  int k0;  // !SLOW: first reduction index, in the slab, of every load
  struct Held { uint4 v[LP]; };
  static __device__ __forceinline__ int swz(int r) { return SLOW ? 4 * piece(r) : (r >> 2) & 3; }
  static __device__ __forceinline__ int piece(int r) { return TILE >= 128 ? r & 3 : (r >> 1) & 1; }
  template <typename F> __device__ __forceinline__ void start(int first, int size, int ld, F&& row_of) {
#pragma unroll
    for (int i = 0; i < LP; ++i) {
      const int id = i * 256 + threadIdx.x, r = id / PER_ROW, c = id % PER_ROW;
      if (SLOW) off[i] = first + c * 4 < size ? 4u * ((unsigned)r * (unsigned)ld + c * 4) : ~0u;
      else off[i] = 4u * ((unsigned)min(row_of(r), size - 1 - first) * (unsigned)ld + c * 4);
    }
    k0 = threadIdx.x % PER_ROW * 4;
  }
  // `left` reduction indices in the slab, what is past them reads as zero; b2: for the odd groups of 32 tile rows, or null
  __device__ __forceinline__ void load(Held& held, const char* base, const char* b2, int left, int ld) const {
    typedef __attribute__((ext_vector_type(4))) unsigned v4u;
#pragma unroll
    for (int i = 0; i < LP; ++i) {
      const bool two = b2 && ((i * 256 / PER_ROW + (int)__builtin_amdgcn_readfirstlane(threadIdx.x / PER_ROW)) >> 5 & 1);  // (uniform: a wavefront has 8 rows)
      const __amdgpu_buffer_rsrc_t b = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(two ? b2 : base), 0, SLOW ? 4u * (unsigned)left * (unsigned)ld : 0xfffffff0u, 0x00020000);
      held.v[i] = __builtin_bit_cast(uint4, (v4u)__builtin_amdgcn_raw_buffer_load_b128(b, SLOW || k0 < left ? off[i] : ~0u, 0, 0));
    }
  }
  // A float is the sum of its planes to 2^-27 of it; the largest finite ones, which would round up to infinity, through the largest bf16.
  __device__ __forceinline__ void cut(const Held& held, unsigned char* planes) const {
    auto low = [](unsigned p) { return __uint_as_float(p << 16); };
    auto high = [](unsigned p) { return __uint_as_float(p & 0xffff0000u); };
    auto most = [](float v) { return __builtin_amdgcn_fmed3f(v, -3.3895313892515355e38f, 3.3895313892515355e38f); };
#pragma unroll
    for (int i = 0; i < LP; ++i) {
      const int id = i * 256 + threadIdx.x, r = id / PER_ROW, c = id % PER_ROW;
      unsigned char* const to = planes + r * ROW + (((c >> 1) ^ swz(r)) << 4) + (c & 1) * 8;
      float v[4] = {__uint_as_float(held.v[i].x), __uint_as_float(held.v[i].y), __uint_as_float(held.v[i].z), __uint_as_float(held.v[i].w)};
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        uint2 w;
        if (p == 0) w = make_uint2(two_bf16(most(v[0]), most(v[1])), two_bf16(most(v[2]), most(v[3])));
        else w = make_uint2(two_bf16(v[0], v[1]), two_bf16(v[2], v[3]));
        *reinterpret_cast<uint2*>(to + p * BYTES) = w;
        if (p == 2) break;
        v[0] -= low(w.x);
        v[1] -= high(w.x);
        v[2] -= low(w.y);
        v[3] -= high(w.y);
      }
    }
  }
};
// AHEAD slabs are on their way in registers.  While one is contracted out of one half of LDS the next is cut into the other.  A chain of slabs is bound by LDS
// (three planes of either operand are written once and read by two wavefronts) and by the 7 instructions a float takes to cut: 0.53 us a slab of a 64 x 64 tile, on
// its own in a CU; four slabs ahead or a fixed order of matrix and other instructions change nothing.  4096^3 184 TFLOP/s.
template <int WHAT, int BM, int BN, int WAVES_M, int WAVES_N, int AHEAD>
__device__ __forceinline__ void exact_body(const Product& P, int block, unsigned char* smem) {
  constexpr int BK = 32, WTM = BM / WAVES_M, WTN = BN / WAVES_N, MI = WTM / 32, NI = WTN / 32;
  constexpr bool DUAL = WHAT == GATED, ASLOW = WHAT == WGRAD, BSLOW = WHAT == DGRAD || WHAT == WGRAD;
  using PA = Planes<BM, ASLOW>;
  using PB = Planes<BN, BSLOW>;
  static_assert(WAVES_M * WAVES_N == 4 && (!DUAL || NI % 2 == 0), "");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WAVES_N, wn = wave % WAVES_N;
  const Share<WHAT, BM, BN, BK> at(P, block);
  constexpr int BUFFER = 3 * (PA::BYTES + PB::BYTES);
  PA sa;
  PB sb;
  sa.start(at.row0, P.M, P.lda, [](int r) { return r; });
  sb.start(at.col0, P.N, P.ldb, [](int r) { return DUAL ? (r >> 6) * 32 + (r & 31) : r; });
  // where the slabs of either segment begin
  const char *a0[2], *b0[2], *other = reinterpret_cast<const char*>(static_cast<const float*>(P.other) + (int64_t)at.col0 * P.ldb);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float *const a = static_cast<const float*>(at.second ? P.other : P.A[i]), *const b = static_cast<const float*>(P.B[i]);
    a0[i] = reinterpret_cast<const char*>(ASLOW ? a + at.row0 : a + (int64_t)at.row0 * P.lda);
    b0[i] = reinterpret_cast<const char*>(BSLOW ? b + at.col0 : b + (int64_t)at.col0 * P.ldb);
  }
  int seg = at.seg, slab = at.slab, left_to_ask = at.todo;
  typename PA::Held ha[AHEAD];
  typename PB::Held hb[AHEAD];
  auto request = [&](auto w) {  // (past the last slab: zeros)
    constexpr int h = decltype(w)::value;
    const int left = left_to_ask > 0 ? min(BK, P.K - slab * BK) : 0;
    const int64_t k = (int64_t)slab * (4 * BK);
    sa.load(ha[h], (seg ? a0[1] : a0[0]) + (ASLOW ? k * P.lda : k), nullptr, left, P.lda);
    sb.load(hb[h], (seg ? b0[1] : b0[0]) + (BSLOW ? k * P.ldb : k), DUAL ? other + k : nullptr, left, P.ldb);
    --left_to_ask;
    const bool end = ++slab == at.per_segment;
    slab = end ? 0 : slab;
    seg += end;
  };
  static_for<AHEAD>(request);
  v16f_t acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  const int l31 = lane & 31, hi = lane >> 5, rho = lane & 15;
  auto fragment = [&](const unsigned char* plane, int block, int kk, auto side) {
    using S = decltype(side);
    if constexpr (S::ROW == 64) {
      return *reinterpret_cast<const uint4*>(plane + (block * 32 + l31) * 64 + (((kk * 2 + hi) ^ S::swz(l31)) << 4));
    } else {
      const unsigned char* const q = plane + (kk * 16 + 8 * hi + (rho >> 2)) * S::ROW + (4 * (block ^ S::piece(rho >> 2)) + 2 * ((lane >> 4) & 1) + ((rho & 3) >> 1)) * 16 + 8 * (rho & 1);
      union { v4s h[2]; uint4 u; } r;
      r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(q));
      r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(q + 4 * S::ROW));
      return r.u;
    }
  };
  auto contract = [&](const unsigned char* la) {
    const unsigned char* const lb = la + 3 * PA::BYTES;
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      uint4 fa[3][MI], fb[3][NI];
#pragma unroll
      for (int p = 0; p < 3; ++p) {
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[p][i] = fragment(la + p * PA::BYTES, wm * MI + i, kk, PA{});
#pragma unroll
        for (int j = 0; j < NI; ++j) fb[p][j] = fragment(lb + p * PB::BYTES, wn * NI + j, kk, PB{});
      }
      constexpr int OF_A[6] = {2, 0, 1, 1, 0, 0}, OF_B[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
      for (int s = 0; s < 6; ++s)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j) acc[i][j] = mfma_bf16(fb[OF_B[s]][j], fa[OF_A[s]][i], acc[i][j]);
    }
  };
  auto cut = [&](auto w) {
    constexpr int h = decltype(w)::value;
    unsigned char* const la = smem + h % 2 * BUFFER;
    sa.cut(ha[h], la);
    sb.cut(hb[h], la + 3 * PA::BYTES);
    request(w);
  };
  static_assert(AHEAD % 2 == 0, "");
  cut(std::integral_constant<int, 0>{});
  lds_barrier();
  for (int t = at.todo; t > 0; t -= AHEAD) {
    static_for<AHEAD>([&](auto w) {
      constexpr int h = decltype(w)::value;
      contract(smem + h % 2 * BUFFER);
      cut(std::integral_constant<int, (h + 1) % AHEAD>{});
      lds_barrier();
    });
  }
  leave<WHAT, float>(P, acc, at.row0 + wm * WTM, at.col0 + wn * (DUAL ? WTN / 2 : WTN), at.split, at.second, lane);
}

// ---- kernels ----------------------------------------------------------------------------------------------------------
// Tiles by size: 0 64 x 64 in slabs of 128, 1 64 x 128, 2 128 x 128, 4 the same in slabs of 32, four of them on their way, for tiles that have a CU to themselves, all with two
// workgroups a CU, 3 256 x 256, one a CU.  A gated map's wavefronts have 64 columns or more.
// us, size 2 / 4: fewer tiles than CUs, forward 512 x 4096 x 4096 41 / 33, backward 1500 x 1536 x 6144 129 / 114; more, backward of 6272 x 768 x 2048, gated, 85 / 92.
// us, products of 8192 x 4096 x 12288: 256 x 256 with two slabs of 64 / four of 32, gated forward 1357 / 1420, both backward 2563 / 2504; with four wavefronts of 128 x 128
// instead of eight of 128 x 64 1418 / 2664 (and they spill).
constexpr int threads_of(int what, int size) { return size == 3 ? 512 : size == 0 && what == GATED ? 128 : 256; }
template <int WHAT, typename T, int SIZE> struct Tile {
  static constexpr bool EXACT = sizeof(T) == 4, DUAL = WHAT == GATED, BACK = WHAT == DGRAD || WHAT == WGRAD;
  static constexpr int BM = SIZE == 3 ? 256 : SIZE >= 2 ? 128 : 64, BN = SIZE == 3 ? 256 : SIZE >= 1 ? 128 : 64;
  static constexpr int WAVES_M = 2, WAVES_N = SIZE == 3 ? 4 : SIZE == 0 && DUAL ? 1 : 2, THREADS = WAVES_M * WAVES_N * 64;
  static_assert(THREADS == threads_of(WHAT, SIZE), "");
  static constexpr int BK = EXACT || SIZE == 4 || (SIZE == 3 && BACK) ? 32 : SIZE == 0 ? 128 : 64, STAGES = SIZE == 4 || (SIZE == 3 && BACK) ? 4 : SIZE == 1 ? 3 : 2;
  static constexpr int AHEAD = 2;  // EXACT
  static constexpr int LDS = EXACT ? (BM + BN) * BK * 6 * 2 : (BM + BN) * BK * 2 * STAGES;
  static constexpr int WAVES = LDS > 80 * 1024 || THREADS < 256 ? (THREADS + 255) / 256 : 2;  // a SIMD, as LDS allows: registers for them
  static __device__ __forceinline__ void body(const Product& P, int block, unsigned char* smem) {
    if constexpr (EXACT) exact_body<WHAT, BM, BN, WAVES_M, WAVES_N, AHEAD>(P, block, smem);
    else product_body<WHAT, T, BM, BN, WAVES_M, WAVES_N, BK, STAGES>(P, block, smem);
  }
};
template <int WHAT, typename T, int SIZE>
__global__ __launch_bounds__((Tile<WHAT, T, SIZE>::THREADS), (Tile<WHAT, T, SIZE>::WAVES)) void token_product_kernel(const Product P) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[Tile<WHAT, T, SIZE>::LDS];
  Tile<WHAT, T, SIZE>::body(P, blockIdx.x, smem);
}
// Both products of a backward pass and the last sums of dbias, in the order dw, dx, dbias of workgroups (the first two of no tiles: not wanted).
template <typename T, int SIZE>
__global__ __launch_bounds__((Tile<WGRAD, T, SIZE>::THREADS), (Tile<WGRAD, T, SIZE>::WAVES)) void token_backward_kernel(const Product dw, const Product dx, const BiasParts bias) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[Tile<WGRAD, T, SIZE>::LDS];
  const int weights = dw.tiles * dw.splits, all = weights + dx.tiles * dx.splits, block = blockIdx.x;
  if (block < weights) Tile<WGRAD, T, SIZE>::body(dw, block, smem);
  else if (block < all) Tile<DGRAD, T, SIZE>::body(dx, block - weights, smem);
  else bias_body<T, Tile<WGRAD, T, SIZE>::THREADS>(bias, block - all, smem);
}
// Joins the sums of a shared reduction: eight neighbours a thread.  Memory, and a launch of 3 to 5 us, which is why reductions are shared only where that is less than it gains.
template <typename T> __device__ __forceinline__ void join_body(const Product& P, int what, int64_t block) {
  const int64_t MN = (int64_t)P.M * P.N, stride = (what == GATED || P.pair ? 2 : 1) * MN, i = (block * 256 + threadIdx.x) * 8;
  if (i >= (what == GATED ? MN : stride)) return;
  auto sum = [&](int64_t at, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll 8
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
template <typename T> __global__ __launch_bounds__(256) void token_join_kernel(const Product P, int what) { join_body<T>(P, what, blockIdx.x); }
// Workgroups dw_groups are those of dw.
template <typename T> __global__ __launch_bounds__(256) void token_backward_join_kernel(const Product dw, const Product dx, int dw_groups) {
  if ((int)blockIdx.x < dw_groups) join_body<T>(dw, WGRAD, blockIdx.x);
  else join_body<T>(dx, DGRAD, blockIdx.x - dw_groups);
}

// ---- few rows ---------------------------------------------------------------------------------------------------------
// Memory: 1 x 4096 x 12288 in bf16, gated, reads 201 MB in 29.6 to 37 us (5.4 to 6.8 TB/s, part of it from cache).
// Up to 64 rows of x: the 16 rows of one operand are eight columns of wg and of wu each, or 16 of w, those of the other 16 rows of x; RG groups of rows, CG of columns; the
// wavefronts of a workgroup share the reduction.
struct Few {
  const void *x, *w, *w2;       // gated: wg, wu
  void *out, *out2, *out3;      // gated: h, g, u; else y, z
  const void *bias, *residual;
  int rows, in, cols, act;
};
template <typename T, bool DUAL, int RG, int CG, int WAVES> __global__ __launch_bounds__(WAVES * 64) void token_few_kernel(const Few a) {
  constexpr int V = Elem<T>::VEC, STEP = 4 * V, UNROLL = RG * CG == 1 ? 8 : 4;  // reduction indices that the lanes of a wavefront have at once; such steps in flight
  __shared__ v4f_t shares[WAVES][RG * CG][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, quarter = lane >> 4;
  const int col0 = blockIdx.x * (DUAL ? 8 : 16) * CG;
  const T *w[CG], *x[RG];
#pragma unroll
  for (int g = 0; g < CG; ++g)
    w[g] = static_cast<const T*>(DUAL && r >= 8 ? a.w2 : a.w) + (int64_t)min(col0 + (DUAL ? g * 8 + (r & 7) : g * 16 + r), a.cols - 1) * a.in + quarter * V;
#pragma unroll
  for (int g = 0; g < RG; ++g) x[g] = static_cast<const T*>(a.x) + (int64_t)min(g * 16 + r, a.rows - 1) * a.in + quarter * V;
  v4f_t acc[RG][CG] = {};
  for (int k0 = wave * STEP * UNROLL; k0 < a.in; k0 += WAVES * STEP * UNROLL) {
    uint4 p[UNROLL][CG], q[UNROLL][RG];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int k = k0 + i * STEP;
      const bool in = k + quarter * V < a.in;
#pragma unroll
      for (int g = 0; g < CG; ++g) p[i][g] = in ? *reinterpret_cast<const uint4*>(w[g] + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int g = 0; g < RG; ++g) q[i][g] = in ? *reinterpret_cast<const uint4*>(x[g] + k) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < UNROLL; ++i)
#pragma unroll
      for (int m = 0; m < RG; ++m)
#pragma unroll
        for (int n = 0; n < CG; ++n) {
          if constexpr (sizeof(T) == 2) {
            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf16_t, p[i][n]), __builtin_bit_cast(v8bf16_t, q[i][m]), acc[m][n], 0, 0, 0);
          } else {
            Chunk16<float> f, g;
            f.v = p[i][n];
            g.v = q[i][m];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.e[e], g.e[e], acc[m][n], 0, 0, 0);
          }
        }
  }
#pragma unroll
  for (int m = 0; m < RG; ++m)
#pragma unroll
    for (int n = 0; n < CG; ++n) shares[wave][m * CG + n][lane] = acc[m][n];
  __syncthreads();
  for (int which = wave; which < RG * CG; which += WAVES) {
    // row of x lane % 16; columns 4 (lane / 16) .., gated: 4 (lane / 16 % 2) .. of wg (lanes below 32) or wu
    v4f_t sum = shares[0][which][lane];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) sum += shares[i][which][lane];
    float u[4], v[4] = {sum[0], sum[1], sum[2], sum[3]};
    if constexpr (DUAL)
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = __shfl(sum[e], lane + 32, 64);
    const int row = which / CG * 16 + r, col = col0 + which % CG * (DUAL ? 8 : 16) + 4 * (DUAL ? quarter & 1 : quarter);
    if (row >= a.rows || col >= a.cols) continue;
    const int64_t at = (int64_t)row * a.cols + col;
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
      if (lane >= 32) continue;
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
}

// Backward of up to 16 rows and few outputs: bound by launches and round trips, so that it is one launch.  dz (dg, du) is made again by every workgroup that has it for a factor,
// and stays fp32; products are of 16 x 16 x 4.
struct FewBack {
  const void *x, *w, *w2, *z, *u, *dy;  // gated: wg, wu, g, u, dh
  void *dx, *dw, *dw2, *dbias;          // gated: dx, dwg, dwu; each may be null (dw and dw2 together)
  int rows, in, out, act;
  int dx_groups;
};
constexpr int FEW_BACK_WAVES = 8;
template <typename T> struct alignas(4 * sizeof(T)) Four {
  T e[4];
  __device__ __forceinline__ float operator[](int i) const { return Elem<T>::to_f32(e[i]); }
};
template <typename T, bool DUAL> __global__ __launch_bounds__(FEW_BACK_WAVES * 64) void token_few_backward_kernel(const FewBack a) {
  constexpr int STEPS = 8, SLAB = FEW_BACK_WAVES * 4 * STEPS;  // reduction indices that the wavefronts have at once
  __shared__ v4f_t shares[FEW_BACK_WAVES][4][64];
  __shared__ __attribute__((aligned(16))) float factors[DUAL ? 2 : 1][16][SLAB + 4];  // (rows on banks of their own)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, quarter = lane >> 4;
  const T *const z = static_cast<const T*>(a.z), *const u = static_cast<const T*>(a.u), *const dy = static_cast<const T*>(a.dy);
  auto gradient = [&](float z, float u, float dy, float& p, float& q) {  // dg and du, or dz
    float f = z, df = 1.f;
    if (a.act != TOKEN_NONE) act_both<T>(a.act, z, f, df);
    p = DUAL ? dy * u * df : dy * df;
    q = dy * f;
  };
  if ((int)blockIdx.x < a.dx_groups) {
    // 64 columns of dx; the wavefronts share the reduction.  lane: row c of dz, index `quarter` of four; columns 4 c .. of w
    static_assert(FEW_BACK_WAVES * 64 == 16 * SLAB / 8, "eight values of a slab of dz a thread");
    const int col = blockIdx.x * 64 + c * 4;
    v4f_t acc[4] = {};
    for (int o0 = 0; o0 < a.out; o0 += SLAB) {
      Four<T> w[STEPS], w2[STEPS];
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int o = o0 + (wave * STEPS + i) * 4 + quarter;
        const bool there = o < a.out && col < a.in;
        const int64_t at = there ? (int64_t)o * a.in + col : 0;
        w[i] = there ? *reinterpret_cast<const Four<T>*>(static_cast<const T*>(a.w) + at) : Four<T>{};
        if (DUAL) w2[i] = there ? *reinterpret_cast<const Four<T>*>(static_cast<const T*>(a.w2) + at) : Four<T>{};
      }
      const int r = threadIdx.x / (SLAB / 8), o = threadIdx.x % (SLAB / 8) * 8;
      float p[8] = {}, q[8] = {};
      if (r < a.rows && o0 + o < a.out) {  // (out: a multiple of 8)
        const int64_t at = (int64_t)r * a.out + o0 + o;
        Eight<T> vz, vu, vd;
        vd.load(dy + at);
        if (DUAL || a.act != TOKEN_NONE) vz.load(z + at);
        if (DUAL) vu.load(u + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) gradient(DUAL || a.act != TOKEN_NONE ? vz[e] : 0.f, DUAL ? vu[e] : 0.f, vd[e], p[e], q[e]);
      }
      if (o0) __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        *reinterpret_cast<float4*>(&factors[0][r][o + e]) = make_float4(p[e], p[e + 1], p[e + 2], p[e + 3]);
        if (DUAL) *reinterpret_cast<float4*>(&factors[DUAL ? 1 : 0][r][o + e]) = make_float4(q[e], q[e + 1], q[e + 2], q[e + 3]);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int k = (wave * STEPS + i) * 4 + quarter;
        const float dg = factors[0][c][k], du = DUAL ? factors[DUAL ? 1 : 0][c][k] : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(dg, w[i][e], acc[e], 0, 0, 0);
          if (DUAL) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(du, w2[i][e], acc[e], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) shares[wave][e][lane] = acc[e];
    __syncthreads();
    // row 4 (lane / 16) + k, columns 4 c ..
    const int k = wave, r = 4 * quarter + k;
    if (k >= 4 || r >= a.rows || col >= a.in) return;
    Four<T> res;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < FEW_BACK_WAVES; ++i) s += shares[i][e][lane][k];
      res.e[e] = Elem<T>::from_f32(s);
    }
    *reinterpret_cast<Four<T>*>(static_cast<T*>(a.dx) + (int64_t)r * a.in + col) = res;
    return;
  }
  // 16 rows of dw a wavefront, 64 columns.  lane: row c of them, rows of x quarter, quarter + 4, ..
  const int columns = a.dw ? (a.in + 63) / 64 : 1, tile = (blockIdx.x - a.dx_groups) * FEW_BACK_WAVES + wave, o0 = tile / columns * 16, strip = tile % columns, col = strip * 64 + c * 4;
  if (o0 >= a.out) return;
  float p[4], q[4], sum = 0.f;
  Four<T> x[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int r = quarter + 4 * s;
    const bool there = r < a.rows && o0 + c < a.out;
    const int64_t at = there ? (int64_t)r * a.out + o0 + c : 0;
    gradient(there && (DUAL || a.act != TOKEN_NONE) ? Elem<T>::to_f32(z[at]) : 0.f, DUAL && there ? Elem<T>::to_f32(u[at]) : 0.f, there ? Elem<T>::to_f32(dy[at]) : 0.f, p[s],
             q[s]);
    sum += p[s];
    x[s] = a.dw && r < a.rows && col < a.in ? *reinterpret_cast<const Four<T>*>(static_cast<const T*>(a.x) + (int64_t)r * a.in + col) : Four<T>{};
  }
  if (!DUAL && a.dbias && strip == 0) {
    sum = lanes_swap32(lanes_swap16(sum));
    if (lane < 16 && o0 + c < a.out) static_cast<T*>(a.dbias)[o0 + c] = Elem<T>::from_f32(sum);
  }
  if (!a.dw) return;
#pragma unroll
  for (int which = 0; which < (DUAL ? 2 : 1); ++which) {
    v4f_t acc[4] = {};
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(which ? q[s] : p[s], x[s][e], acc[e], 0, 0, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int o = o0 + 4 * quarter + k;
      if (o >= a.out || col >= a.in) continue;
      Four<T> res;
#pragma unroll
      for (int e = 0; e < 4; ++e) res.e[e] = Elem<T>::from_f32(acc[e][k]);
      *reinterpret_cast<Four<T>*>(static_cast<T*>(which ? a.dw2 : a.dw) + (int64_t)o * a.in + col) = res;
    }
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------
int slab_of(int what, int size, bool f32) { return f32 || size == 4 || (size == 3 && (what == DGRAD || what == WGRAD)) ? 32 : size == 0 ? 128 : 64; }
int rows_of(int size) { return size == 3 ? 256 : size >= 2 ? 128 : 64; }
int columns_of(int what, int size) { return (size == 3 ? 256 : size >= 1 ? 128 : 64) / (what == GATED ? 2 : 1); }
// Tiles of a product by size.
int64_t tiles_of(const Product& p, int what, int size) {
  const int bm = rows_of(size), bn = columns_of(what, size);
  return (((int64_t)p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn) * (p.pair ? 2 : 1);
}
// Tiles and parts of a product; `slabs_each`: slabs that a workgroup should have at least.
bool plan(Product& p, int what, int size, bool f32, int64_t slabs_each, int64_t room) {
  const int bm = rows_of(size), bn = columns_of(what, size), bk = slab_of(what, size, f32);
  p.tiles_m = (int)(((int64_t)p.M + bm - 1) / bm);
  p.tiles_n = (p.N + bn - 1) / bn;
  const int64_t tiles = tiles_of(p, what, size), slabs = ((int64_t)p.K + bk - 1) / bk * p.segments, results = (int64_t)p.M * p.N * (what == GATED || p.pair ? 2 : 1);
  const int threads = threads_of(what, size);
  if (!launchable(tiles, threads) || slabs > INT32_MAX) return false;
  p.tiles = (int)tiles;
  const int64_t splits = std::max<int64_t>(1, std::min(slabs / slabs_each, room / (4 * results)));
  p.slabs_per = (int)((slabs + splits - 1) / splits);
  p.splits = (int)((slabs + p.slabs_per - 1) / p.slabs_per);
  return launchable((int64_t)p.tiles * p.splits, threads);
}
// Tiles and slabs a workgroup for products of one launch: the least of the times that the following gives.  A CU takes `slab` us for a slab of a tile (`alone`: where it has one), and
// `tile` us for what else there is to one (for those that it has at a time); `resident` tiles run at once.  Joining costs a launch and its memory.  The figures are fitted to products of 14
// shapes at every size; of 20 others, of short and long sums, the tile taken is 3 % off the best of the five on average, 20 at most (3546 x 1312 x 2368 bf16 43 for 36 us).
// Only what can be launched is taken, with `others` workgroups beside it: 2^29 rows are too many tiles of 64.
struct Choice {
  int size;
  int64_t each;
  double time;
};
template <int N> Choice choose(const Product* const (&p)[N], const int (&what)[N], bool f32, int64_t room, int64_t others) {
  struct Cost { double slab, alone, tile; int resident; };
  static constexpr Cost BF16[5] = {{0.40, 0.43, 1.0, 512}, {0.30, 0.36, 1.6, 512}, {0.49, 0.68, 2.0, 512}, {1.60, 1.60, 5.0, 256}, {0.57, 0.46, 2.0, 512}},
                        F32[3] = {{0.45, 0.53, 1.5, 768}, {0.78, 0.85, 2.0, 512}, {1.47, 1.47, 7.0, 256}};
  const int first = f32 && what[0] == GATED ? 1 : 0;  // (64 x 64 of a gated map in fp32 would be two wavefronts)
  Choice best = {first, INT32_MAX, 0};
  double least = 1e30;
  for (int size = first; size < (f32 ? 3 : 5); ++size) {
    const Cost& cost = f32 ? F32[size] : BF16[size];
    int64_t tiles[N], slabs[N], most = 1;
    double unit[N];  // of a slab
    for (int i = 0; i < N; ++i) {
      const int bk = slab_of(what[i], size, f32);
      tiles[i] = p[i]->K ? tiles_of(*p[i], what[i], size) : 0;
      slabs[i] = p[i]->K ? ((int64_t)p[i]->K + bk - 1) / bk * p[i]->segments : 0;
      // (of 64 x 64 tiles whose reduction is the slow index of both operands the time a slab is twice that: 136 x 680 x 5273 0.8 us)
      unit[i] = cost.slab * bk / (f32 ? 32 : size ? 64 : 128) * (what[i] == WGRAD && size == 0 && !f32 ? 2 : 1);
      most = std::max(most, slabs[i]);
    }
    for (int64_t parts = 1; parts <= 32; parts += parts < 4 ? 1 : parts / 2) {
      const int64_t each = (most + parts - 1) / parts;
      if (parts > 1 && each * slab_of(what[0], size, f32) < (f32 ? 128 : 256)) break;
      double work = 0, longest = 0, join = 0, groups = 0, left = (double)room;
      for (int i = 0; i < N; ++i) {
        if (!tiles[i]) continue;
        const double results = (double)p[i]->M * p[i]->N * (what[i] == GATED || p[i]->pair ? 2 : 1);
        const double splits = std::max(1.0, std::min<double>(parts > 1 ? (double)(slabs[i] / each) : 1.0, std::floor(left / (4 * results))));
        if (splits > 1) {
          join = std::max(join, 4.0) + 8e-6 / 4.5 * results * splits;
          left -= 4 * results * splits;
        }
        work += (double)tiles[i] * slabs[i] * unit[i];
        longest = std::max(longest, slabs[i] / splits * unit[i] * cost.alone / cost.slab);
        groups += tiles[i] * splits;
      }
      if (!launchable((int64_t)groups + others, threads_of(what[0], size))) break;
      // whole rounds of what is resident, then a last one of fewer a CU
      const double whole = std::floor(groups / cost.resident), last = std::ceil((groups - whole * cost.resident) / 256);
      const double tiles_a_cu = whole * (cost.resident / 256) + (last == 1 ? cost.alone / cost.slab : last);
      const double time = std::max(tiles_a_cu * work / groups, longest) + std::ceil(groups / cost.resident) * cost.tile + join;
      if (time < least) {
        least = time;
        best = {size, parts > 1 ? each : (int64_t)INT32_MAX, time};
      }
    }
  }
  return best;
}
int64_t join_groups(const Product& p, int what) {
  return p.splits > 1 ? ((int64_t)p.M * p.N * (what != GATED && p.pair ? 2 : 1) / 8 + 255) / 256 : 0;
}

template <int WHAT, typename T, int SIZE> void start_product(const Product& p, hipStream_t stream) {
  hipLaunchKernelGGL((token_product_kernel<WHAT, T, SIZE>), dim3(p.workgroups()), dim3(Tile<WHAT, T, SIZE>::THREADS), 0, stream, p);
}
// Few rows.  A CU reads 37 KB a us of weights and rows out of the caches, all of them 5 MB of weights out of memory.  Two groups of columns a workgroup read the rows half as
// often (only of gated maps, whose groups have 8 of either matrix: us, 16 x 4096 x 12288 44 / 35, 32 x 1024 x 2816 7.4 / 5.8); of plain maps that are no more workgroups
// than CUs those have eight wavefronts (1 x 4096 x 4096 7.7 / 6.9).
struct FewChoice {
  int groups;  // of columns
  double time;
};
FewChoice choose_few(const Few& a, bool dual, bool f32) {
  const double bytes = (f32 ? 4.0 : 2.0) * a.in, least = (dual ? 2 : 1) * bytes * a.cols / 5e6;
  FewChoice best = {1, 1e30};
  for (int groups = 1; groups <= (dual ? 2 : 1); ++groups) {
    const int columns = (dual ? 8 : 16) * groups;
    const double time = std::max(least, ((a.cols + columns - 1) / columns + 255) / 256 * bytes * (16 * groups + a.rows) / 37e3 * (groups == 2 ? 1.2 : 1.0));
    if (time < best.time) best = {groups, time};
  }
  best.time *= !f32 ? 1.0 : a.rows <= 32 ? 1.25 : 1.6;
  return best;
}
template <typename T, bool DUAL, int RG, int CG, int WAVES> void start_few(const Few& a, hipStream_t stream) {
  constexpr int COLS = (DUAL ? 8 : 16) * CG;
  hipLaunchKernelGGL((token_few_kernel<T, DUAL, RG, CG, WAVES>), dim3((a.cols + COLS - 1) / COLS), dim3(WAVES * 64), 0, stream, a);
}
template <typename T, bool DUAL, int RG> void start_few(const Few& a, int groups, hipStream_t stream) {
  if constexpr (DUAL) {
    if (groups == 2) return start_few<T, true, RG, 2, 4>(a, stream);
  } else if constexpr (sizeof(T) == 2) {
    if (a.cols <= 16 * 256) return start_few<T, false, RG, 1, 8>(a, stream);
  }
  start_few<T, DUAL, RG, 1, 4>(a, stream);
}
template <typename T, bool DUAL> hipError_t launch_few(const Few& a, int groups, hipStream_t stream) {
  if (a.rows <= 16) start_few<T, DUAL, 1>(a, groups, stream);
  else if (a.rows <= 32) start_few<T, DUAL, 2>(a, groups, stream);
  else start_few<T, DUAL, 4>(a, groups, stream);
  return hipGetLastError();
}
constexpr int FEW_ROWS = 16, FEW_MOST = 64;

// A forward product, on tiles or, up to 16 rows and where its estimate is less, as one of few rows (us so / on tiles, bf16: 32 x 4096 x 4096 13.3 / 21.6, 64 x 12288 x 4096 55 / 64,
// 32 x 4096 x 12288, which stays on tiles, 34 / 24; fp32: gated 32 x 1024 x 2816 12.8 / 17.4, 64 x 520 x 1000 7.7 / 13.8, 64 x 4096 x 4096, which stays, 41 / 25).  What tiles take
// beside the estimate, at so few rows 1.1 (fp32) to 1.3 (bf16) of it, and a launch either way, are left out there.
template <int WHAT, typename T> hipError_t launch_forward(Product& p, const Few& few, int64_t room, hipStream_t stream) {
  constexpr bool F32 = sizeof(T) == 4, DUAL = WHAT == GATED;
  FewChoice rows = {1, 1e30};
  if (p.M <= FEW_MOST) rows = choose_few(few, DUAL, F32);
  if (p.M <= FEW_ROWS) return launch_few<T, DUAL>(few, rows.groups, stream);
  const Product* const all[1] = {&p};
  const int what[1] = {WHAT};
  const Choice of = choose(all, what, F32, room, 0);
  if (rows.time < std::max((F32 ? 1.1 : 1.3) * of.time, (double)sizeof(T) * (DUAL ? 2 : 1) * p.K * p.N / 5e6)) return launch_few<T, DUAL>(few, rows.groups, stream);
  const int size = of.size;
  if (!plan(p, WHAT, size, F32, of.each, room)) return hipErrorInvalidConfiguration;
  if (size == 1) start_product<WHAT, T, 1>(p, stream);
  else if (size == 2) start_product<WHAT, T, 2>(p, stream);
  else if constexpr (!F32 || WHAT != GATED)
    if (size == 0) start_product<WHAT, T, 0>(p, stream);
  if constexpr (!F32)
    if (size >= 3) size == 3 ? start_product<WHAT, T, 3>(p, stream) : start_product<WHAT, T, 4>(p, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL((token_join_kernel<T>), dim3((unsigned)join_groups(p, WHAT)), dim3(256), 0, stream, p, (int)WHAT);
  return hipGetLastError();
}
template <typename T, int SIZE> void start_backward(const Product& dw, const Product& dx, const BiasParts& bias, hipStream_t stream) {
  constexpr int THREADS = Tile<WGRAD, T, SIZE>::THREADS, C = THREADS / 32;
  const int groups = dw.workgroups() + dx.workgroups() + (bias.dbias ? (bias.out + C - 1) / C : 0);
  hipLaunchKernelGGL((token_backward_kernel<T, SIZE>), dim3(groups), dim3(THREADS), 0, stream, dw, dx, bias);
}
// The products of a backward pass (K 0: not wanted) in one launch, with the last sums of dbias: planned, so that what is refused is refused before anything runs ..
template <typename T> int plan_backward(Product& dw, Product& dx, const BiasParts& bias, char* at, int64_t room) {  // their size of tiles, or -1
  constexpr bool F32 = sizeof(T) == 4;
  const Product* const all[2] = {&dw, &dx};
  const int what[2] = {WGRAD, DGRAD};
  const Choice of = choose(all, what, F32, room, bias.out);
  const int size = of.size;
  const int64_t each = of.each;
  dw.part = reinterpret_cast<float*>(at);
  if (dw.K) {
    if (!plan(dw, WGRAD, size, F32, each, room)) return -1;
    const int64_t used = dw.splits > 1 ? 4ll * dw.splits * dw.M * dw.N * (dw.pair ? 2 : 1) : 0;
    at += used;
    room -= used;
  }
  dx.part = reinterpret_cast<float*>(at);
  if (dx.K && !plan(dx, DGRAD, size, F32, each, room)) return -1;
  return launchable((int64_t)dw.workgroups() + dx.workgroups() + bias.out, threads_of(WGRAD, size)) ? size : -1;
}
// .. and launched.
template <typename T> hipError_t launch_backward(const Product& dw, const Product& dx, const BiasParts& bias, int size, hipStream_t stream) {
  if (size == 0) start_backward<T, 0>(dw, dx, bias, stream);
  else if (size == 1) start_backward<T, 1>(dw, dx, bias, stream);
  else if (size == 2) start_backward<T, 2>(dw, dx, bias, stream);
  else if constexpr (sizeof(T) == 2) size == 3 ? start_backward<T, 3>(dw, dx, bias, stream) : start_backward<T, 4>(dw, dx, bias, stream);
  const hipError_t e = hipGetLastError();
  const int64_t first = join_groups(dw, WGRAD), groups = first + join_groups(dx, DGRAD);
  if (e != hipSuccess || !groups) return e;
  hipLaunchKernelGGL((token_backward_join_kernel<T>), dim3((unsigned)groups), dim3(256), 0, stream, dw, dx, (int)first);
  return hipGetLastError();
}

int64_t rounded(int64_t bytes) { return (bytes + 255) / 256 * 256; }
// Whether a backward pass is one launch: while dx is one slab or two behind each other.  us so / in the launches of more rows, of rows x inputs x outputs: bf16 16 x 256 x 256 4.8 / 7.8,
// gated 6.4 / 8.2, 16 x 4096 x 256 5.3 / 7.9, 7.1 / 10.0; 16 x 512 x 512, which is not, 7.7 / 8.2, 11.0 / 9.8, 16 x 512 x 1024 13.0 / 10.0, 20.0 / 12.5; fp32 16 x 512 x 512 8.1 / 13.2,
// 11.3 / 12.8, 16 x 4096 x 512 10.5 / 16.2, 14.5 / 20.8; 16 x 512 x 1024, which is not, 14.2 / 13.1, 22.0 / 14.8, 16 x 512 x 12288 161 / 31.
bool few_backward(int rows, int out, int dtype) { return rows <= FEW_ROWS && out <= (dtype == DT_F32 ? 512 : 256); }
template <bool DUAL> hipError_t launch_few_backward(FewBack a, int dtype, hipStream_t stream) {
  a.dx_groups = a.dx ? (a.in + 63) / 64 : 0;
  const int64_t tiles = (int64_t)((a.out + 15) / 16) * (a.dw ? (a.in + 63) / 64 : 1);
  const int64_t groups = a.dx_groups + (a.dw || a.dbias ? (tiles + FEW_BACK_WAVES - 1) / FEW_BACK_WAVES : 0);
  if (!launchable(groups, FEW_BACK_WAVES * 64)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)groups), block(FEW_BACK_WAVES * 64);
  if (dtype == DT_BF16) hipLaunchKernelGGL((token_few_backward_kernel<uint16_t, DUAL>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((token_few_backward_kernel<float, DUAL>), grid, block, 0, stream, a);
  return hipGetLastError();
}

template <typename T> hipError_t gated_backward(const GatedLinear& a, hipStream_t stream) {
  char* at = static_cast<char*>(a.workspace);
  const int64_t n = (int64_t)a.rows * a.hidden, groups = (n / 8 + 255) / 256;
  if (!launchable(groups, 256)) return hipErrorInvalidConfiguration;
  T *const dg = reinterpret_cast<T*>(at), *const du = reinterpret_cast<T*>(at + rounded((int)sizeof(T) * n));
  at += 2 * rounded((int)sizeof(T) * n);
  Product dw, dx;
  memset(&dw, 0, sizeof(dw));
  memset(&dx, 0, sizeof(dx));
  if (a.dwg) {
    dw.segments = 1;
    dw.K = a.rows; dw.M = a.hidden; dw.N = a.in; dw.lda = a.hidden; dw.ldb = a.in;
    dw.A[0] = dg; dw.other = du; dw.B[0] = a.x;
    dw.out = a.dwg; dw.out2 = a.dwu; dw.pair = 1;
  }
  if (a.dx) {
    dx.segments = 2;
    dx.K = a.hidden; dx.M = a.rows; dx.N = a.in; dx.lda = a.hidden; dx.ldb = a.in;
    dx.A[0] = dg; dx.A[1] = du; dx.B[0] = a.wg; dx.B[1] = a.wu;
    dx.out = a.dx;
  }
  const BiasParts none = {nullptr, nullptr, 0, 0};
  const int size = plan_backward<T>(dw, dx, none, at, static_cast<char*>(a.workspace) + a.workspace_bytes - at);
  if (size < 0) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((gated_grad_kernel<T>), dim3((unsigned)groups), dim3(256), 0, stream, static_cast<const T*>(a.g), static_cast<const T*>(a.u),
                     static_cast<const T*>(a.dh), dg, du, n, a.act);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_backward<T>(dw, dx, none, size, stream);
}
template <typename T> hipError_t linear_backward(const TokenLinear& a, hipStream_t stream) {
  char* at = static_cast<char*>(a.workspace);
  const int64_t n = (int64_t)a.rows * a.out;
  T* const to = (a.dx || a.dw) && a.act != TOKEN_NONE ? reinterpret_cast<T*>(at) : nullptr;  // dz, where it is not dy
  at += rounded((int)sizeof(T) * n);
  float* const sums = reinterpret_cast<float*>(at);
  at += rounded(4ll * a.out * std::min(a.rows, LINEAR_MAX_PARTS));
  const int share = (int)(((int64_t)a.rows + 8 * LINEAR_MAX_PARTS - 1) / (8 * LINEAR_MAX_PARTS) * 8), parts = (int)(((int64_t)a.rows + share - 1) / share);  // strips of whole eights of rows
  BiasParts bias = {nullptr, nullptr, 0, 0};
  if (a.dbias && parts > 1) bias = {sums, a.dbias, parts, a.out};
  Product dw, dx;
  memset(&dw, 0, sizeof(dw));
  memset(&dx, 0, sizeof(dx));
  const void* const dz = to ? to : a.dy;
  if (a.dw) {
    dw.segments = 1;
    dw.K = a.rows; dw.M = a.out; dw.N = a.in; dw.lda = a.out; dw.ldb = a.in;
    dw.A[0] = dz; dw.B[0] = a.x; dw.out = a.dw;
  }
  if (a.dx) {
    dx.segments = 1;
    dx.K = a.out; dx.M = a.rows; dx.N = a.in; dx.lda = a.out; dx.ldb = a.in;
    dx.A[0] = dz; dx.B[0] = a.w; dx.out = a.dx;
  }
  const int size = plan_backward<T>(dw, dx, bias, at, static_cast<char*>(a.workspace) + a.workspace_bytes - at);
  if (size < 0) return hipErrorInvalidConfiguration;
  if (to || a.dbias) {
    hipLaunchKernelGGL((linear_grad_kernel<T>), dim3((a.out + 255) / 256, parts), dim3(256), 0, stream, static_cast<const T*>(a.z), static_cast<const T*>(a.dy), to,
                       bias.dbias ? sums : nullptr, bias.dbias ? nullptr : static_cast<T*>(a.dbias), a.rows, a.out, share, a.act);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.dx && !a.dw && !bias.dbias)) return e;
  }
  return launch_backward<T>(dw, dx, bias, size, stream);
}

}  // namespace

// Bytes that the calls cannot do without.
int64_t gated_linear_bwd_workspace_bytes(int rows, int hidden, int dtype) { return (dtype == DT_F32 ? 8 : 4) * (int64_t)rows * hidden + 1024; }
int64_t token_linear_bwd_workspace_bytes(int rows, int out, int dtype) {
  return (dtype == DT_F32 ? 4 : 2) * (int64_t)rows * out + 4ll * out * std::min(rows, LINEAR_MAX_PARTS) + 1024;
}

hipError_t launch_gated_linear(const GatedLinear& a, int dtype, hipStream_t stream) {
  const Few few = {a.x, a.wg, a.wu, a.h, a.g, a.u, nullptr, nullptr, a.rows, a.in, a.hidden, a.act};
  Product p;
  memset(&p, 0, sizeof(p));
  p.segments = 1;
  p.K = a.in; p.M = a.rows; p.N = a.hidden; p.lda = p.ldb = a.in;
  p.A[0] = a.x; p.B[0] = a.wg; p.other = a.wu;
  p.out = a.h; p.out2 = a.g; p.out3 = a.u;
  p.act = a.act;
  p.part = static_cast<float*>(a.workspace);
  return dtype == DT_BF16 ? launch_forward<GATED, uint16_t>(p, few, a.workspace_bytes, stream) : launch_forward<GATED, float>(p, few, a.workspace_bytes, stream);
}
hipError_t launch_gated_linear_bwd(const GatedLinear& a, int dtype, hipStream_t stream) {
  if (few_backward(a.rows, a.hidden, dtype))
    return launch_few_backward<true>({a.x, a.wg, a.wu, a.g, a.u, a.dh, a.dx, a.dwg, a.dwu, nullptr, a.rows, a.in, a.hidden, a.act, 0}, dtype, stream);
  return dtype == DT_BF16 ? gated_backward<uint16_t>(a, stream) : gated_backward<float>(a, stream);
}
hipError_t launch_token_linear(const TokenLinear& a, int dtype, hipStream_t stream) {
  const Few few = {a.x, a.w, nullptr, a.y, a.z, nullptr, a.bias, a.residual, a.rows, a.in, a.out, a.act};
  Product p;
  memset(&p, 0, sizeof(p));
  p.segments = 1;
  p.K = a.in; p.M = a.rows; p.N = a.out; p.lda = p.ldb = a.in;
  p.A[0] = a.x; p.B[0] = a.w;
  p.out = a.y; p.out2 = a.z; p.bias = a.bias; p.residual = a.residual;
  p.act = a.act;
  p.part = static_cast<float*>(a.workspace);
  return dtype == DT_BF16 ? launch_forward<LINEAR, uint16_t>(p, few, a.workspace_bytes, stream) : launch_forward<LINEAR, float>(p, few, a.workspace_bytes, stream);
}
hipError_t launch_token_linear_bwd(const TokenLinear& a, int dtype, hipStream_t stream) {
  if (few_backward(a.rows, a.out, dtype))
    return launch_few_backward<false>({a.x, a.w, nullptr, a.z, nullptr, a.dy, a.dx, a.dw, nullptr, a.dbias, a.rows, a.in, a.out, a.act, 0}, dtype, stream);
  return dtype == DT_BF16 ? linear_backward<uint16_t>(a, stream) : linear_backward<float>(a, stream);
}

}  // namespace cdp
