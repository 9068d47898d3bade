// The products of tile.h for few rows (single tokens and small batches): C[m][n] = sum_k A[m][k] B[n][k] with at most 32 rows m.  Bound by reading B once,
// so B goes from memory to registers and from there to the matrix core, past LDS: no barrier stands between a wave's loads, and any alignment will do.
//
// OP_K (a column's elements side by side): a workgroup takes 16 columns, its waves take the contraction in turns of four matrix-core operands.
// OP_T (a row of B, one k, side by side; float32): a wave takes 64 columns.  The waves of a workgroup take the contraction in turns; where the column blocks do
// not fill the chip, it is also cut into parts of a workgroup each, whose sums a second launch adds in order.
// Taken where it beats the tiles, which read B as fast from 64 or 128 of their rows used (both sides measured): float32 up to 16 rows (the float32 instruction
// has no pieces to make; 7168 x 14336, 16 rows 159 us, in tiles of 64 rows 220) and up to 32 of small matrices (2048 x 8192 40 to 44 us and 45 to 50, 1365 x
// 3001 f x d 21 and 36; 7168 x 14336 225 to 275 and 220), bf16 OP_K up to 16 rows of small matrices (2048 x 5461 13 us, tiles in two launches 15; 7168 x 14336
// 82 and 76; nothing between was measured) and of those that tiles need copied (7161 x 14333, one row 143 and 240, 16 rows 205 and 243), int8 up to 16 rows
// (14336 x 7168 22 and 26; 24 rows 27 and 27).
#pragma once
#include "ops.h"
#include "tile.h"

namespace osscar {
namespace thin {

using tile::OP_K;
using tile::OP_T;
using tile::v4f;
using tile::v4i;
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int WIDE_FROM = 6144;    // columns from which on 32 of them a workgroup fill three quarters of the compute units
enum { BF16 = 0, F32 = 1, I8 = 2 };

// Packet: 16 bytes of one row or column.  ELEMS of them; a matrix-core step contracts STEP elements, OPS instructions.
template <int KIND> struct Num;
template <> struct Num<BF16> {
  typedef v4f acc; typedef float val; typedef uint16_t el;
  static constexpr int ELEMS = 8, STEP = 32;
  static __device__ __forceinline__ void mma(v4i b, v4i a, acc& c) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b), __builtin_bit_cast(v8bf, a), c, 0, 0, 0);
  }
};
template <> struct Num<F32> {      // lane group g contracts k = 4 g + e in instruction e
  typedef v4f acc; typedef float val; typedef uint32_t el;
  static constexpr int ELEMS = 4, STEP = 16;
  static __device__ __forceinline__ void mma(v4i b, v4i a, acc& c) {
#pragma unroll
    for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(b[e]), __int_as_float(a[e]), c, 0, 0, 0);
  }
};
template <> struct Num<I8> {
  typedef v4i acc; typedef int val; typedef uint8_t el;
  static constexpr int ELEMS = 16, STEP = 64;
  static __device__ __forceinline__ void mma(v4i b, v4i a, acc& c) { c = __builtin_amdgcn_mfma_i32_16x16x64_i8(b, a, c, 0, 0, 0); }
};

typedef v4i v4i_any __attribute__((aligned(1)));
// The packet at element k of a row of `K` elements; zeros past its end
template <int KIND>
__device__ __forceinline__ v4i packet(const char* row, int k, int K) {
  typedef typename Num<KIND>::el el;
  constexpr int E = Num<KIND>::ELEMS;
  const el* p = reinterpret_cast<const el*>(row) + k;
  if (k + E <= K) return *reinterpret_cast<const v4i_any*>(p);
  el w[E];
#pragma unroll
  for (int e = 0; e < E; e++) {
    w[e] = 0;
    if (k + e < K) w[e] = p[e];
  }
  return __builtin_bit_cast(v4i, w);
}

template <int NB>
struct Product {
  const char *a, *b[NB];
  int64_t lda, ldb;          // bytes
  int M, N, K;
  int parts;                 // of the contraction, a workgroup each (blockIdx.y)
  void* sums;                // parts > 1: [part][matrix][m][n], 4 bytes each
};

// WIDE: OP_K with 32 columns a wave and turns of two operands, so that the rows of A are read half as often (14336 x 7168 int8, 16 rows: 28 us without, 23 with);
// taken where the chip is full with it.
template <int LAYOUT, int KIND, int NB, int RT, bool WIDE> struct Wave;
// OP_K
template <int KIND, int NB, int RT, bool WIDE>
struct Wave<OP_K, KIND, NB, RT, WIDE> {
  typedef Num<KIND> T;
  static constexpr int TILES = WIDE ? 2 : 1, U = WIDE ? 2 : 4, COLS = 16 * TILES, WAVES = 8, TURN = U * T::STEP;
  static __device__ __forceinline__ int column(int t, int i) { return t * 16 + i; }
  const char *rb[NB][TILES], *ra[RT];
  int koff;
  __device__ __forceinline__ void open(const Product<NB>& q, int n0, int lane) {
    const int i = lane & 15;
    koff = (lane >> 4) * T::ELEMS;
#pragma unroll
    for (int z = 0; z < NB; z++)
#pragma unroll
      for (int t = 0; t < TILES; t++) rb[z][t] = q.b[z] + (int64_t)min(n0 + t * 16 + i, q.N - 1) * q.ldb;      // (past the end: the last one again, not used)
#pragma unroll
    for (int r = 0; r < RT; r++) ra[r] = q.a + (int64_t)min(r * 16 + i, q.M - 1) * q.lda;
  }
  struct Regs { v4i b[NB][TILES][U], a[RT][U]; };
  __device__ __forceinline__ void load(const Product<NB>& q, int k0, Regs& w) const {
    if (k0 + TURN <= q.K) {
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int64_t at = (int64_t)(k0 + u * T::STEP + koff) * sizeof(typename T::el);
#pragma unroll
        for (int z = 0; z < NB; z++)
#pragma unroll
          for (int t = 0; t < TILES; t++) w.b[z][t][u] = *reinterpret_cast<const v4i_any*>(rb[z][t] + at);
#pragma unroll
        for (int r = 0; r < RT; r++) w.a[r][u] = *reinterpret_cast<const v4i_any*>(ra[r] + at);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int k = k0 + u * T::STEP + koff;
#pragma unroll
        for (int z = 0; z < NB; z++)
#pragma unroll
          for (int t = 0; t < TILES; t++) w.b[z][t][u] = packet<KIND>(rb[z][t], k, q.K);
#pragma unroll
        for (int r = 0; r < RT; r++) w.a[r][u] = packet<KIND>(ra[r], k, q.K);
      }
    }
  }
  __device__ __forceinline__ void multiply(const Regs& w, typename T::acc (&acc)[RT][NB][TILES]) const {
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int z = 0; z < NB; z++)
#pragma unroll
        for (int t = 0; t < TILES; t++)
#pragma unroll
          for (int r = 0; r < RT; r++) T::mma(w.b[z][t][u], w.a[r][u], acc[r][z][t]);
  }
};
// OP_T (float32): four columns of four rows k per lane, 64 columns a wave; the instruction that contracts k = 4 g + e of tile t takes column t of row e
// as it is.
template <int NB, int RT>
struct Wave<OP_T, F32, NB, RT, false> {
  typedef Num<F32> T;
  static constexpr int E = 4, COLS = 64, TILES = 4, WAVES = 4, TURN = T::STEP;
  static __device__ __forceinline__ int column(int t, int i) { return i * 4 + t; }
  const char *cb[NB], *ra[RT];
  int koff, left;      // columns of the lane's packet that exist
  __device__ __forceinline__ void open(const Product<NB>& q, int n0, int lane) {
    const int i = lane & 15, n = n0 + i * 4;
    koff = (lane >> 4) * E;
    left = min(4, q.N - n);
#pragma unroll
    for (int z = 0; z < NB; z++) cb[z] = q.b[z] + (int64_t)min(n, q.N - 1) * 4;
#pragma unroll
    for (int r = 0; r < RT; r++) ra[r] = q.a + (int64_t)min(r * 16 + i, q.M - 1) * q.lda;
  }
  struct Regs { v4i b[NB][E], a[RT]; };
  __device__ __forceinline__ void load(const Product<NB>& q, int k0, Regs& w) const {
    const int k = k0 + koff;
    if (k0 + TURN <= q.K) {
#pragma unroll
      for (int r = 0; r < RT; r++) w.a[r] = *reinterpret_cast<const v4i_any*>(ra[r] + (int64_t)k * 4);
    } else {
#pragma unroll
      for (int r = 0; r < RT; r++) w.a[r] = packet<F32>(ra[r], k, q.K);
    }
    if (k0 + TURN <= q.K && left == 4) {
#pragma unroll
      for (int z = 0; z < NB; z++)
#pragma unroll
        for (int e = 0; e < E; e++) w.b[z][e] = *reinterpret_cast<const v4i_any*>(cb[z] + (int64_t)(k + e) * q.ldb);
    } else {
#pragma unroll
      for (int z = 0; z < NB; z++)
#pragma unroll
        for (int e = 0; e < E; e++) {
          const int* p = reinterpret_cast<const int*>(cb[z] + (int64_t)min(k + e, q.K - 1) * q.ldb);
#pragma unroll
          for (int c = 0; c < 4; c++) {
            w.b[z][e][c] = 0;
            if (c < left && k + e < q.K) w.b[z][e][c] = p[c];
          }
        }
    }
  }
  __device__ __forceinline__ void multiply(const Regs& w, typename T::acc (&acc)[RT][NB][TILES]) const {
#pragma unroll
    for (int z = 0; z < NB; z++)
#pragma unroll
      for (int t = 0; t < TILES; t++) {
        const v4i b{w.b[z][0][t], w.b[z][1][t], w.b[z][2][t], w.b[z][3][t]};
#pragma unroll
        for (int r = 0; r < RT; r++) T::mma(b, w.a[r], acc[r][z][t]);
      }
  }
};

// Epi::one(f) calls f(put) once, put(m, n, val (&v)[NB])
template <int LAYOUT, int KIND, int NB, int RT, bool WIDE, class Epi>
__device__ __forceinline__ void product(const Product<NB>& q, const Epi& epi) {
  typedef Wave<LAYOUT, KIND, NB, RT, WIDE> W;
  typedef typename W::T T;
  typedef typename T::val val;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * W::COLS;
  W w;
  w.open(q, n0, lane);
  typename T::acc acc[RT][NB][W::TILES];
#pragma unroll
  for (int r = 0; r < RT; r++)
#pragma unroll
    for (int z = 0; z < NB; z++)
#pragma unroll
      for (int t = 0; t < W::TILES; t++)
#pragma unroll
        for (int e = 0; e < 4; e++) acc[r][z][t][e] = 0;
  // turns of this part, one wave after the other; the next turn's loads are on their way while one is multiplied
  const int turns = (q.K + W::TURN - 1) / W::TURN, per = (turns + q.parts - 1) / q.parts;
  const int first = blockIdx.y * per + wave, last = min(turns, (int)(blockIdx.y + 1) * per);
  if (first < last) {
    typename W::Regs x[2];
    w.load(q, first * W::TURN, x[0]);
    for (int t = first; t < last; t += 2 * W::WAVES) {
      if (t + W::WAVES < last) w.load(q, (t + W::WAVES) * W::TURN, x[1]);
      w.multiply(x[0], acc);
      if (t + W::WAVES >= last) break;
      if (t + 2 * W::WAVES < last) w.load(q, (t + 2 * W::WAVES) * W::TURN, x[0]);
      w.multiply(x[1], acc);
    }
  }
  // the waves' sums, added in order: [wave][row tile][matrix][column][16 rows + 1]
  constexpr int PER = W::TILES * 16 * 17, ALL = RT * NB * PER;
  __shared__ val sums[W::WAVES / 2][ALL];
  const int g = lane >> 4, i = lane & 15;
  auto each = [&](auto f) {      // f(place, value): the new value
    if (i >= q.M && RT == 1) return;
#pragma unroll
    for (int r = 0; r < RT; r++)
#pragma unroll
      for (int z = 0; z < NB; z++)
#pragma unroll
        for (int t = 0; t < W::TILES; t++)
#pragma unroll
          for (int e = 0; e < 4; e++) acc[r][z][t][e] = f((r * NB + z) * PER + W::column(t, g * 4 + e) * 17 + i, acc[r][z][t][e]);
  };
#pragma unroll
  for (int half = W::WAVES / 2; half > 0; half /= 2) {
    if (wave >= half && wave < 2 * half) each([&](int at, val v) { return sums[wave - half][at] = v; });
    __syncthreads();
    if (wave < half) each([&](int at, val v) { return v + sums[wave][at]; });
    __syncthreads();
  }
  if (wave == 0) each([&](int at, val v) { return sums[0][at] = v; });
  __syncthreads();
  const int rows = q.M, cols = min(W::COLS, q.N - n0);
  if (q.parts > 1) {
    val* out = reinterpret_cast<val*>(q.sums) + (int64_t)blockIdx.y * NB * q.M * q.N;
    for (int j = threadIdx.x; j < NB * rows * W::COLS; j += W::WAVES * 64) {
      const int c = j % W::COLS, m = j / W::COLS % rows, z = j / W::COLS / rows;
      if (c < cols) out[((int64_t)z * q.M + m) * q.N + n0 + c] = sums[0][((m >> 4) * NB + z) * PER + c * 17 + (m & 15)];
    }
    return;
  }
  epi.one([&](auto put) {
    for (int j = threadIdx.x; j < rows * W::COLS; j += W::WAVES * 64) {
      const int c = j % W::COLS, m = j / W::COLS;
      if (c >= cols) continue;
      val v[NB];
#pragma unroll
      for (int z = 0; z < NB; z++) v[z] = sums[0][((m >> 4) * NB + z) * PER + c * 17 + (m & 15)];
      put(m, n0 + c, v, q.N);
    }
  });
}
// How a product is dealt out: column blocks, wide or not, and parts of the contraction, enough for about two workgroups of four waves (OP_T) or half a
// workgroup of eight (OP_K) per compute unit, each wave with at least two turns.
struct Deal { unsigned blocks; int parts; bool wide; int threads; };
template <int LAYOUT, int KIND>
Deal deal(int64_t M, int64_t N, int64_t K) {
  typedef Wave<LAYOUT, KIND, 1, 1, false> W;
  Deal d{(unsigned)((N + W::COLS - 1) / W::COLS), 1, LAYOUT == OP_K && KIND != BF16 && M > 1 && N >= WIDE_FROM, W::WAVES * 64};
  if (d.wide) { d.blocks = (unsigned)((N + 31) / 32); return d; }
  const int64_t turns = (K + W::TURN - 1) / W::TURN, want = LAYOUT == OP_K ? 128 : 512, most = turns / (W::WAVES * 2);
  int64_t parts = want / d.blocks;
  if (parts > most) parts = most;
  if (parts > 16) parts = 16;
  d.parts = parts < 1 ? 1 : (int)parts;
  return d;
}

}  // namespace thin
}  // namespace osscar
