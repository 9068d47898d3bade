// Low-rank adapters of many requests beside a shared projection: y_i = base_i + s_e B_e^T (A_e x_i) with e the adapter of row i, and the gradients.
// A (count x rank x d) and B (count x rank x m) both hold a component's numbers side by side, so that three kernels do it all:
//   contract  T[i][j] = sum_k Z[i][k] V_e[j][k]        (T from X and A; dT from dY and B)
//   expand    Y[i][c] = base[i][c] + sum_j T[i][j] V_e[j][c]      (y from T and B; dX from dT and A)
//   outer     dV_e[j][c] = sum over the rows i of e of T[i][j] Z[i][c]      (dA from dT and X; dB from T and dY)
// Rows go through in tiles, a tile once for each adapter in it, each time with the results of that adapter's rows kept: as they lie, or in the order of their adapters (places alone, no row is moved) from 8
// adapters and 512 rows on, and wherever dA and dB are made of more than 256 rows.  Up to 64 rows (256 with an index) take kernels that read V once per row instead.  All are bound by reading and writing Z, base
// and Y, or A and B where rows are few: 2 rank operations for each of their elements.
#include "ops.h"
#include <algorithm>
#include <type_traits>

using namespace osscar;

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// Which adapter each row has, and what it says of itself.  index NULL: every row has the first.
struct Pick {
  const int64_t* index;
  const float* scale;
  const int32_t* ranks;
  int count, rank;
  const int2* order;      // which row, of which adapter, lies at which place of the tiles (NULL: as they are)
  __device__ __forceinline__ int of(int64_t row) const {      // -1: none; -2: there is no such adapter
    if (!index) return 0;
    const int64_t e = index[row];
    return e < 0 ? -1 : e < count ? (int)e : -2;
  }
  __device__ __forceinline__ float scale_of(int e) const { return scale ? scale[e] : 1.f; }
  __device__ __forceinline__ int rank_of(int e) const { return ranks ? min(max(ranks[e], 0), rank) : rank; }
};
// f(e, which rows of the tile) for each adapter that some of the lanes' rows have, every `slots`-th of them.
template <class F>
__device__ __forceinline__ void each_adapter(int mine, int slot, int slots, F f) {
  uint64_t left = __ballot(mine >= 0);
  for (int k = 0; left; k++) {
    const int e = __builtin_amdgcn_readlane(mine, __ffsll((unsigned long long)left) - 1);
    const uint64_t rows = __ballot(mine == e);
    left &= ~rows;
    if (k % slots == slot) f(e, rows);
  }
}

struct Mat { const void* p; int64_t ld; };                  // rows of elements
struct Adapters { const void* p; int64_t ld, next; };       // of one component, of one adapter

// 16 bytes of a row and the matrix instruction that contracts them: lane (i, g) = (lane % 16, lane / 16) holds elements g E .. g E + E - 1 of row i.
template <bool F32> struct Num;
template <> struct Num<false> {
  static constexpr int E = 8, STEP = 32, ES = 2;
  static __device__ __forceinline__ v4f mma(u32x4 a, u32x4 b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  }
};
template <> struct Num<true> {
  static constexpr int E = 4, STEP = 16, ES = 4;
  static __device__ __forceinline__ v4f mma(u32x4 a, u32x4 b, v4f c) {
#pragma unroll
    for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
};
template <bool F32>
__device__ __forceinline__ u32x4 packet(const char* row, int k) { return *reinterpret_cast<const u32x4_any*>(row + (int64_t)k * Num<F32>::ES); }
// The same where the row ends: zeros from K on; read from a packet before the end on and moved to their places, but for rows of fewer elements
template <bool F32>
__device__ __forceinline__ u32x4 packet_some(const char* row, int k, int K) {
  constexpr int E = Num<F32>::E;
  u32x4 x;
  if (K >= E) {
    const int at = min(k, K - E), s = k - at;
    x = packet<F32>(row, at);
    const int words = F32 ? s : s >> 1;
    if (words & 2) x = u32x4{x[2], x[3], 0, 0};
    if (words & 1) x = u32x4{x[1], x[2], x[3], 0};
    if (!F32 && (s & 1)) x = u32x4{x[0] >> 16 | x[1] << 16, x[1] >> 16 | x[2] << 16, x[2] >> 16 | x[3] << 16, x[3] >> 16};
    return s >= E ? u32x4{0, 0, 0, 0} : x;
  }
  if constexpr (F32) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + k;
#pragma unroll
    for (int e = 0; e < 4; e++) { x[e] = 0; if (k + e < K) x[e] = p[e]; }
  } else {
    x = __builtin_bit_cast(u32x4, Eight<false>::load(row, k, K - k));
  }
  return x;
}

// --------------------------------------------------------------------------------------------------
// contract
// --------------------------------------------------------------------------------------------------
// A workgroup takes 16 RT rows and 16 CT components; its waves take the contraction in turns, parts of it are a workgroup's each (their sums are added where T is
// read).  Operands go from memory to registers, the next turn's while one is multiplied.  The instruction wants 64 bytes of each of 16 rows in a packet of its lanes, which memory
// answers in requests of 64 bytes: rows of Z are fetched 128 bytes at a time and change lanes through LDS, a piece of it for every wave (8192 x 14336, rank 32: 83 us without, 72 with).
constexpr int FW = 4;      // waves of the kernel for few rows
struct Contract {
  Mat z;
  Adapters v;
  int64_t n;
  int K, parts, slots, scaled;      // scaled: times the adapter's scale
  float* t;                         // [part][n][rank]
};
constexpr int CW = 8;      // waves
constexpr int RT = 2;      // row tiles of 16 in a workgroup (with four, half as many reads of V, it takes as long: 75 us instead of 74 at rank 32; with rank 64 they do not fit the registers)
constexpr int U = 2;       // instructions' worth of a row in a turn (four, rows 256 bytes at a time: with bf16 and two column tiles 24 registers too many, 6000 x 2048 x 8192 rank 32 forward 52 us instead of 48; with one no difference)
template <bool F32, int CT, bool SORTED>
__global__ __launch_bounds__(CW * 64) void contract_kernel(Contract q, Pick pick) {
  typedef Num<F32> N;
  constexpr int TURN = U * N::STEP, ROWS = RT * 16, COLS = CT * 16;
  constexpr int NC = U * 4, PER = 64 / NC, ROW = NC * 16;      // packets of a row in a turn, rows of one load, bytes of a row
  constexpr int SUMS = CW / 2 * ROWS * (COLS + 1) * 4, TURNS = CW * ROWS * ROW;
  __shared__ __align__(16) char lds[SUMS > TURNS ? SUMS : TURNS];
  float(*sums)[ROWS * (COLS + 1)] = reinterpret_cast<float(*)[ROWS * (COLS + 1)]>(lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const int64_t tiles = (q.n + ROWS - 1) / ROWS, row0 = (blockIdx.x % tiles) * ROWS;
  const int slot = (int)(blockIdx.x / tiles), part = blockIdx.y, j0 = blockIdx.z * COLS;
  const int have = (int)std::min<int64_t>(ROWS, q.n - row0);
  const int2 at = SORTED && lane < have ? pick.order[row0 + lane] : int2{0, -1};
  const int line = at.x;
  auto row_of = [&](int r) -> int64_t { return SORTED ? __shfl(line, r, 64) : row0 + r; };      // (by all lanes)
  const int mine = SORTED ? at.y : lane < have ? pick.of(row0 + lane) : -1;
  float* t = q.t + (int64_t)part * q.n * pick.rank;
  if (slot == q.slots - 1) {      // rows without an adapter (by the slot that is likeliest to have none itself)
    const uint64_t none = __ballot(mine < 0);
    for (int k = threadIdx.x; k < have * COLS; k += CW * 64) {
      const int r = k / COLS, j = j0 + k % COLS;
      if ((none >> r & 1) && j < pick.rank) t[(SORTED ? pick.order[row0 + r].x : row0 + r) * pick.rank + j] = 0.f;
    }
  }
  each_adapter(mine, slot, q.slots, [&](int e, uint64_t rows) {
    const int rank = pick.rank_of(e), first = __ffsll((unsigned long long)rows) - 1;
    const char *zr[RT][U], *vr[CT];
#pragma unroll
    for (int r = 0; r < RT; r++)
#pragma unroll
      for (int u = 0; u < U; u++) {      // (rows of other adapters: one of this one's again, not used)
        const int row = r * 16 + u * PER + lane / NC, at = rows >> row & 1 ? row : first;
        zr[r][u] = reinterpret_cast<const char*>(q.z.p) + row_of(at) * q.z.ld * N::ES;
      }
    const int zk = lane % NC * N::E;
    char* mine_lds = lds + wave * ROWS * ROW;
#pragma unroll
    for (int c = 0; c < CT; c++) vr[c] = reinterpret_cast<const char*>(q.v.p) + (e * q.v.next + (int64_t)std::max(0, std::min(j0 + c * 16 + i, rank - 1)) * q.v.ld) * N::ES;
    struct Regs { u32x4 z[RT][U], v[CT][U]; };
    auto load = [&](int k0, Regs& w) {
      if (k0 + TURN <= q.K) {
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int k = k0 + u * N::STEP + g * N::E;
#pragma unroll
          for (int r = 0; r < RT; r++) w.z[r][u] = packet<F32>(zr[r][u], k0 + zk);
#pragma unroll
          for (int c = 0; c < CT; c++) w.v[c][u] = packet<F32>(vr[c], k);
        }
      } else {
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int k = k0 + u * N::STEP + g * N::E;
#pragma unroll
          for (int r = 0; r < RT; r++) w.z[r][u] = packet_some<F32>(zr[r][u], k0 + zk, q.K);
#pragma unroll
          for (int c = 0; c < CT; c++) w.v[c][u] = packet_some<F32>(vr[c], k, q.K);
        }
      }
    };
    v4f acc[RT][CT];
#pragma unroll
    for (int r = 0; r < RT; r++)
#pragma unroll
      for (int c = 0; c < CT; c++) acc[r][c] = v4f{0, 0, 0, 0};
    auto multiply = [&](const Regs& w) {      // (packets of a row change places, so that the lanes of one access meet the banks evenly)
#pragma unroll
      for (int r = 0; r < RT; r++)
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int row = u * PER + lane / NC;
          *reinterpret_cast<u32x4*>(mine_lds + (r * 16 + row) * ROW + ((lane % NC) ^ (row & (NC - 1))) * 16) = w.z[r][u];
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int r = 0; r < RT; r++) {
          const u32x4 z = *reinterpret_cast<const u32x4*>(mine_lds + (r * 16 + i) * ROW + ((u * 4 + g) ^ (i & (NC - 1))) * 16);
#pragma unroll
          for (int c = 0; c < CT; c++) acc[r][c] = N::mma(z, w.v[c][u], acc[r][c]);
        }
      __builtin_amdgcn_wave_barrier();
    };
    const int turns = (q.K + TURN - 1) / TURN, per = (turns + q.parts - 1) / q.parts;
    const int begin = part * per + wave, end = std::min(turns, (part + 1) * per);
    if (j0 < rank && begin < end) {
      Regs x[2];
      load(begin * TURN, x[0]);
      for (int k = begin; k < end; k += 2 * CW) {
        if (k + CW < end) load((k + CW) * TURN, x[1]);
        multiply(x[0]);
        if (k + CW >= end) break;
        if (k + 2 * CW < end) load((k + 2 * CW) * TURN, x[0]);
        multiply(x[1]);
      }
    }
    // the waves' sums, added in a fixed order
    auto each = [&](auto f) {
#pragma unroll
      for (int r = 0; r < RT; r++)
#pragma unroll
        for (int c = 0; c < CT; c++)
#pragma unroll
          for (int d = 0; d < 4; d++) acc[r][c][d] = f((r * 16 + g * 4 + d) * (COLS + 1) + c * 16 + i, acc[r][c][d]);
    };
#pragma unroll
    for (int half = CW / 2; half > 0; half /= 2) {
      __syncthreads();
      if (wave >= half && wave < 2 * half) each([&](int at, float s) { return sums[wave - half][at] = s; });
      __syncthreads();
      if (wave < half) each([&](int at, float s) { return s + sums[wave][at]; });
    }
    __syncthreads();      // (the next adapter's operands take the same place)
    if (wave == 0) {
      const float s = q.scaled ? pick.scale_of(e) : 1.f;
#pragma unroll
      for (int r = 0; r < RT; r++)
#pragma unroll
        for (int d = 0; d < 4; d++) {
          const int row = r * 16 + g * 4 + d;
          const int64_t to = row_of(row);
          if (rows >> row & 1) {
#pragma unroll
            for (int c = 0; c < CT; c++) {
              const int j = j0 + c * 16 + i;
              if (j < pick.rank) t[to * pick.rank + j] = j < rank ? acc[r][c][d] * s : 0.f;
            }
          }
        }
    }
  });
}

// --------------------------------------------------------------------------------------------------
// expand
// --------------------------------------------------------------------------------------------------
// float32 factors of a bf16 product go in as two pieces of bf16 each (16 bits: what is left out is 2^-16 of a term at most, the rounding of a bf16 result 2^-8 of its), or three (24 bits).
template <int PIECES>
__device__ __forceinline__ void pieces(const float (&x)[8], u32x4 (&p)[PIECES]) {
  float left[8];
#pragma unroll
  for (int e = 0; e < 8; e++) left[e] = x[e];
#pragma unroll
  for (int k = 0; k < PIECES; k++) {
    v8bf w;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      w[e] = (__bf16)left[e];
      left[e] -= (float)w[e];
    }
    p[k] = __builtin_bit_cast(u32x4, w);
  }
}
// Eight rows of eight bf16 columns, turned: operand t holds column t of all eight.
__device__ __forceinline__ void turned(const u16x8 (&w)[8], u32x4 (&p)[8]) {
#pragma unroll
  for (int t = 0; t < 8; t++) {
    u16x8 c;
#pragma unroll
    for (int e = 0; e < 8; e++) c[e] = w[e][t];
    p[t] = __builtin_bit_cast(u32x4, c);
  }
}

struct Expand {
  const float* t;      // [part][n][rank]
  int parts, slots, scaled, subs;
  Adapters v;
  Mat base;            // (p may be NULL, or y)
  int64_t n;
  int C;
  void* y;
  int64_t ldy;
  float* t_out;        // the parts' sum, or NULL
};
constexpr int EW = 4, ECOLS = 128, PARTS_MOST = 4;      // waves, columns of each; parts of T
// The components j .. of eight columns from c, as the matrix instruction takes them; zeros from `rank` on.
template <bool F32> struct Columns;
template <> struct Columns<false> {
  static constexpr int STEP = 32, E = 8;
  u32x4 w[8];      // column c + t of eight components
  __device__ __forceinline__ void load(const char* v, int64_t ld, int j, int rank, int c, bool whole, int C) {
    u16x8 x[E];
#pragma unroll
    for (int k = 0; k < E; k++) {
      const int64_t row = (int64_t)std::min(j + k, rank - 1) * ld;
      x[k] = whole ? Eight<false>::load(v, row + c) : edge_load<false>(v, row, c, C);
    }
#pragma unroll
    for (int k = 0; k < E; k++)
      if (j + k >= rank) x[k] = u16x8{};
    turned(x, w);
  }
  __device__ __forceinline__ void multiply(const float (&x)[E], v4f (&acc)[8]) const {
    u32x4 p[2];
    pieces<2>(x, p);
#pragma unroll
    for (int k = 1; k >= 0; k--)
#pragma unroll
      for (int t = 0; t < 8; t++) acc[t] = Num<false>::mma(p[k], w[t], acc[t]);
  }
};
template <> struct Columns<true> {
  static constexpr int STEP = 16, E = 4;
  float w[E][8];
  __device__ __forceinline__ void load(const char* v, int64_t ld, int j, int rank, int c, bool whole, int C) {
    Eight<true>::type x[E];
#pragma unroll
    for (int k = 0; k < E; k++) {
      const int64_t row = (int64_t)std::min(j + k, rank - 1) * ld;
      x[k] = whole ? Eight<true>::load(v, row + c) : edge_load<true>(v, row, c, C);
    }
#pragma unroll
    for (int k = 0; k < E; k++) {
      Eight<true>::values(x[k], w[k]);
#pragma unroll
      for (int t = 0; t < 8; t++) w[k][t] = j + k < rank ? w[k][t] : 0.f;
    }
  }
  __device__ __forceinline__ void multiply(const float (&x)[E], v4f (&acc)[8]) const {
#pragma unroll
    for (int k = 0; k < E; k++)
#pragma unroll
      for (int t = 0; t < 8; t++) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k], w[k][t], acc[t], 0, 0, 0);
  }
};
// E numbers of a row of T, from its j-th of `rank`
template <int E>
__device__ __forceinline__ void t_values(const float* t, int j, int rank, float (&x)[E]) {
  if (j + E <= rank) {
#pragma unroll
    for (int k = 0; k < E; k += 4) {
      const f32x4 w = *reinterpret_cast<const f32x4_any*>(t + j + k);
#pragma unroll
      for (int e = 0; e < 4; e++) x[k + e] = w[e];
    }
  } else {
#pragma unroll
    for (int k = 0; k < E; k++) { x[k] = 0.f; if (j + k < rank) x[k] = t[j + k]; }
  }
}
// A wave takes 128 columns of up to 64 rows, 16 at a time: lane (i, g) reads eight columns c0 + 8 i .. of components 8 g .. and turns them in its registers, so that
// the instruction for tile t has columns c0 + 8 i + t; the results of a lane are then eight neighbouring columns of four rows.  The columns stay in registers for all rows of their
// adapter (KS steps of components; 0: more than that, read again for each 16 rows), the next 16 rows' base and T are on their way while those before are multiplied (AHEAD).
// Float32 of up to 16 components without AHEAD takes 165 registers instead of 192, so that a third wave fits: better where a workgroup has one or two tiles of 16 rows (777 rows of three adapters,
// 1365 x 5461, rank 12: 28.6 us instead of 32.3 forward, 2000 41.7 instead of 44.7), worse with four (6000 sorted rows 97.6 instead of 91.7); bf16 gains nothing by it.
// 8192 x 14336 bf16, rank 32: 90 us (base and y 470 MB, 5.2 TB/s; 16 and 32 rows at a time without that: 193); 6000 x 8192, rank 64: 52 us (3.8 TB/s).
template <bool F32, int KS, bool PARTS, bool AHEAD, bool SORTED>
__global__ __launch_bounds__(EW * 64, AHEAD ? 2 : 3) void expand_kernel(Expand q, Pick pick) {
  typedef Eight<F32> E8;
  typedef Columns<F32> Cols;
  constexpr int STEP = Cols::STEP, E = Cols::E, HELD = KS > 0 ? KS : 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4, rows_a_tile = q.subs * 16;
  const int blocks = (q.C + EW * ECOLS - 1) / (EW * ECOLS);
  const int64_t row0 = (int64_t)(blockIdx.x / blocks) * rows_a_tile;
  const int c0 = (blockIdx.x % blocks) * (EW * ECOLS) + wave * ECOLS, slot = blockIdx.y, c = c0 + i * 8;
  if (c0 >= q.C) return;
  const int have = (int)std::min<int64_t>(rows_a_tile, q.n - row0), most = q.C - c;
  const int2 at = SORTED && lane < have ? pick.order[row0 + lane] : int2{0, -1};
  const int line = at.x;
  auto row_of = [&](int r) -> int64_t { return SORTED ? __shfl(line, r, 64) : row0 + r; };      // (by all lanes)
  auto line_of = [&](int r) -> int64_t { return SORTED ? pick.order[row0 + r].x : row0 + r; };    // (by any)
  const int mine = SORTED ? at.y : lane < have ? pick.of(row0 + lane) : -1;
  const bool whole = c0 + ECOLS <= q.C, keeps = q.t_out && c0 == 0;
  constexpr size_t ES = F32 ? 4 : 2;
  if (slot == q.slots - 1) {      // rows without an adapter (by the slot that is likeliest to have none itself)
    uint64_t none = __ballot(mine < 0 && lane < have);
    const uint64_t wrong = __ballot(mine == -2);
    if (keeps)
      for (int k = lane; k < have * pick.rank; k += 64)
        if (none >> (k / pick.rank) & 1) q.t_out[line_of(k / pick.rank) * pick.rank + k % pick.rank] = 0.f;
    if (q.y == q.base.p) none = wrong;
    while (none) {      // four at a time, one for each group of lanes
      int r = -1;
      for (int k = 0; k < 4 && none; k++, none &= none - 1)
        if (g == k) r = __ffsll((unsigned long long)none) - 1;
      if (r >= 0 && most > 0) {
        const int64_t row = line_of(r);
        float y[8];
        if (q.base.p) E8::values(E8::load(q.base.p, row * q.base.ld + c, most), y);
#pragma unroll
        for (int t = 0; t < 8; t++) y[t] = wrong >> r & 1 ? NAN : q.base.p ? y[t] : 0.f;
        E8::store(q.y, row * q.ldy + c, y, most);
      }
    }
  }
  each_adapter(mine, slot, q.slots, [&](int e, uint64_t rows) {
    const int rank = pick.rank_of(e);
    const float s = q.scaled ? pick.scale_of(e) : 1.f;
    const char* v = reinterpret_cast<const char*>(q.v.p) + e * q.v.next * ES;
    struct Rows16 { typename E8::type base[4]; float x[HELD][E]; };
    auto next = [&](int sub) {      // the first from there on with rows of this adapter
      while (sub < q.subs && !(rows >> (sub * 16) & 0xFFFF)) sub++;
      return sub;
    };
    auto fetch = [&](int sub, Rows16& w) {
      if (q.base.p) {
#pragma unroll
        for (int d = 0; d < 4; d++) {
          const int row = sub * 16 + g * 4 + d;
          const int64_t from = row_of(row);
          if (rows >> row & 1) w.base[d] = whole ? E8::load(q.base.p, from * q.base.ld + c) : edge_load<F32>(q.base.p, from * q.base.ld, c, q.C);
        }
      }
      const int row = sub * 16 + i;
      const int64_t from = row_of(row);
#pragma unroll
      for (int k = 0; k < KS; k++) {
#pragma unroll
        for (int x = 0; x < E; x++) w.x[k][x] = 0.f;
        if (rows >> row & 1) t_values<E>(q.t + from * pick.rank, k * STEP + g * E, pick.rank, w.x[k]);
      }
    };
    // T of a row: the other parts, kept where that is asked for, components past the rank left out, scaled
    auto finish = [&](int sub, int j, float (&x)[E]) {
      const int row = sub * 16 + i;
      const int64_t from = row_of(row);
      if (rows >> row & 1) {
        if constexpr (PARTS) {      // (all on their way together: few rows wait for each load)
          float more[PARTS_MOST - 1][E];
#pragma unroll
          for (int p = 1; p < PARTS_MOST; p++) t_values<E>(q.t + ((int64_t)std::min(p, q.parts - 1) * q.n + from) * pick.rank, j, pick.rank, more[p - 1]);
#pragma unroll
          for (int p = 1; p < PARTS_MOST; p++)
#pragma unroll
            for (int k = 0; k < E; k++) x[k] += p < q.parts ? more[p - 1][k] : 0.f;
        }
        if (keeps) {
#pragma unroll
          for (int k = 0; k < E; k++)
            if (j + k < pick.rank) q.t_out[from * pick.rank + j + k] = x[k];
        }
      }
#pragma unroll
      for (int k = 0; k < E; k++) x[k] = j + k < rank ? x[k] * s : 0.f;
    };
    Rows16 now, then;
    int sub = next(0);
    fetch(sub, now);
    Cols cols[HELD];
    if (rank > 0) {
#pragma unroll
      for (int k = 0; k < KS; k++) cols[k].load(v, q.v.ld, k * STEP + g * E, rank, c, whole, q.C);
    }
    while (sub < q.subs) {
      const int after = next(sub + 1);
      if (AHEAD && after < q.subs) fetch(after, then);
      v4f acc[8];
#pragma unroll
      for (int t = 0; t < 8; t++) acc[t] = v4f{0, 0, 0, 0};
      if constexpr (KS > 0) {
#pragma unroll
        for (int k = 0; k < KS; k++) {
          finish(sub, k * STEP + g * E, now.x[k]);
          if (k * STEP < rank) cols[k].multiply(now.x[k], acc);
        }
      } else {
        const int row = sub * 16 + i;
        const int64_t from = row_of(row);
        for (int j0 = 0; j0 < (keeps ? pick.rank : rank); j0 += STEP) {
          float x[E];
#pragma unroll
          for (int k = 0; k < E; k++) x[k] = 0.f;
          if (rows >> row & 1) t_values<E>(q.t + from * pick.rank, j0 + g * E, pick.rank, x);
          finish(sub, j0 + g * E, x);
          if (j0 < rank) {
            cols[0].load(v, q.v.ld, j0 + g * E, rank, c, whole, q.C);
            cols[0].multiply(x, acc);
          }
        }
      }
#pragma unroll
      for (int d = 0; d < 4; d++) {
        const int row = sub * 16 + g * 4 + d;
        const int64_t to = row_of(row);
        if (rows >> row & 1) {
          float y[8];
          if (q.base.p) E8::values(now.base[d], y);
#pragma unroll
          for (int t = 0; t < 8; t++) y[t] = q.base.p ? y[t] + acc[t][d] : acc[t][d];
          if (whole) E8::store(q.y, to * q.ldy + c, y);
          else E8::store(q.y, to * q.ldy + c, y, most);
        }
      }
      if (AHEAD) now = then;
      else if (after < q.subs) fetch(after, now);
      sub = after;
    }
  });
}

// Few rows wait for one load after the other; these two kernels have few of them in a row, and read V once per row.  16 rows of any of 32 adapters of rank 16, 7168 x 14336: 10 us for both
// (12 MB, 2.5 us at the rate of a copy), 9.4 with one row: two launches of 4 us, most of it waiting for index, operands and T one behind the other.
// A workgroup takes 16 components of one row and a part of the contraction, a wave 512 numbers of it at a time.
template <bool F32>
__global__ __launch_bounds__(FW * 64) void contract_few_kernel(Contract q, Pick pick) {
  typedef Eight<F32> E8;
  constexpr size_t ES = F32 ? 4 : 2;
  constexpr int SPAN = 512;
  __shared__ float sums[FW][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = blockIdx.x, j0 = blockIdx.z * 16;
  const int64_t row = blockIdx.y;
  const int e = pick.of(row), rank = e < 0 ? 0 : pick.rank_of(e);
  const float s = e >= 0 && q.scaled ? pick.scale_of(e) : 1.f;
  float acc[16];
#pragma unroll
  for (int j = 0; j < 16; j++) acc[j] = 0.f;
  if (j0 < rank) {
    const char* v = reinterpret_cast<const char*>(q.v.p) + (e * q.v.next + (int64_t)j0 * q.v.ld) * ES;
    for (int b = (part * FW + wave) * SPAN; b < q.K; b += q.parts * FW * SPAN) {
      const int k = b + lane * 8, most = q.K - k;
      typename E8::type z, w[16];
      if (b + SPAN <= q.K) {
        z = E8::load(q.z.p, row * q.z.ld + k);
#pragma unroll
        for (int j = 0; j < 16; j++) w[j] = E8::load(v, std::min(j, rank - 1 - j0) * q.v.ld + k);
      } else {
        z = E8::load(q.z.p, row * q.z.ld + k, most);
#pragma unroll
        for (int j = 0; j < 16; j++) w[j] = E8::load(v, std::min(j, rank - 1 - j0) * q.v.ld + k, most);
      }
      float x[8];
      E8::values(z, x);
#pragma unroll
      for (int j = 0; j < 16; j++) {
        float y[8];
        E8::values(w[j], y);
#pragma unroll
        for (int d = 0; d < 8; d++) acc[j] = fmaf(x[d], y[d], acc[j]);
      }
    }
  }
  // sums over the lanes: in each step a lane keeps half of its numbers and gets its partner's share of them
#pragma unroll
  for (int half = 8; half > 0; half /= 2) {
    const int o = half * 4;      // partners 32, 16, 8, 4 lanes away
    const bool upper = lane & o;
#pragma unroll
    for (int j = 0; j < half; j++) {
      const float mine = upper ? acc[j + half] : acc[j], other = upper ? acc[j] : acc[j + half];
      acc[j] = mine + __shfl_xor(other, o, 64);
    }
  }
  acc[0] += __shfl_xor(acc[0], 2, 64);
  acc[0] += __shfl_xor(acc[0], 1, 64);
  if ((lane & 3) == 0) sums[wave][lane >> 2] = acc[0];
  __syncthreads();
  const int j = j0 + threadIdx.x;
  if (threadIdx.x < 16 && j < pick.rank) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < FW; w++) t += sums[w][threadIdx.x];
    q.t[((int64_t)part * q.n + row) * pick.rank + j] = j < rank ? t * s : 0.f;
  }
}
// A workgroup takes 512 columns of one row, its waves (one for each 16 components, up to four) the components in turns; a component's number goes to all lanes as a scalar.
template <bool F32>
__global__ __launch_bounds__(256) void expand_few_kernel(Expand q, Pick pick) {
  typedef Eight<F32> E8;
  constexpr size_t ES = F32 ? 4 : 2;
  __shared__ __align__(16) float sums[3][64][8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, c = (blockIdx.x * 64 + lane) * 8, most = q.C - c;
  const bool whole = ((int)blockIdx.x + 1) * 512 <= q.C;
  const int64_t row = blockIdx.y;
  const int e = pick.of(row);
  typename E8::type base{};
  if (q.base.p && wave == 0) base = whole ? E8::load(q.base.p, row * q.base.ld + c) : edge_load<F32>(q.base.p, row * q.base.ld, c, q.C);
  const int rank = e < 0 ? 0 : pick.rank_of(e);
  const float s = e >= 0 && q.scaled ? pick.scale_of(e) : 1.f;
  const char* v = reinterpret_cast<const char*>(q.v.p) + std::max(e, 0) * q.v.next * ES;
  float y[8];
#pragma unroll
  for (int t = 0; t < 8; t++) y[t] = 0.f;
  for (int j0 = wave * 16; j0 < pick.rank; j0 += waves * 16) {
    const int j = j0 + (lane & 15);
    float t = 0.f, part[PARTS_MOST];
    typename E8::type w[16];
    if (j0 < rank) {
#pragma unroll
      for (int k = 0; k < 16; k++) w[k] = whole ? E8::load(v, std::min(j0 + k, rank - 1) * q.v.ld + c) : edge_load<F32>(v, std::min(j0 + k, rank - 1) * q.v.ld, c, q.C);
#pragma unroll
      for (int p = 0; p < PARTS_MOST; p++) part[p] = q.t[((int64_t)std::min(p, q.parts - 1) * q.n + row) * pick.rank + std::min(j, rank - 1)];
#pragma unroll
      for (int p = 0; p < PARTS_MOST; p++) t += p < q.parts && j < rank ? part[p] : 0.f;
    }
    if (q.t_out && blockIdx.x == 0 && lane < 16 && j < pick.rank) q.t_out[row * pick.rank + j] = t;
    if (j0 >= rank) continue;
    t *= s;
#pragma unroll
    for (int k = 0; k < 16; k++) {
      if (j0 + k < rank) {
        float x[8];
        E8::values(w[k], x);
        const float a = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(t), k));
#pragma unroll
        for (int d = 0; d < 8; d++) y[d] = fmaf(a, x[d], y[d]);
      }
    }
  }
  if (waves > 1) {
    if (wave > 0) {
#pragma unroll
      for (int d = 0; d < 8; d++) sums[wave - 1][lane][d] = y[d];
    }
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < waves; w++) {
#pragma unroll
      for (int d = 0; d < 8; d++) y[d] += sums[w - 1][lane][d];
    }
  }
  if (most <= 0 || (e == -1 && q.y == q.base.p)) return;
  float x[8];
  E8::values(base, x);
#pragma unroll
  for (int t = 0; t < 8; t++) y[t] = e == -2 ? NAN : q.base.p ? x[t] + y[t] : y[t];
  E8::store(q.y, row * q.ldy + c, y, most);
}

// T's parts added, in the order that expand adds them in: where dX takes the place of dY or X, the outer products come before it and want T whole (n rank numbers, a few us at most).
__global__ __launch_bounds__(256) void add_parts_kernel(const float* part, int parts, int64_t size, float* t) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= size) return;
  float s = part[i];
  for (int p = 1; p < parts; p++) s += part[p * size + i];
  t[i] = s;
}

// --------------------------------------------------------------------------------------------------
// outer
// --------------------------------------------------------------------------------------------------
// The rows in the order of their adapters, and pieces of at most `chunk` rows of one adapter.
struct Chunk { int e, begin, end; };
struct Plan {
  const int* order;            // (NULL: as they lie)
  const Chunk* chunks;
  const int* first;            // count + 1: an adapter's first chunk
  int64_t n;
  int total, chunk;            // order NULL: how many; rows of one at most
  __device__ __forceinline__ Chunk at(int c) const {
    if (!order) return Chunk{0, c * chunk, (int)min(n, ((int64_t)c + 1) * chunk)};
    return chunks[c];
  }
  __device__ __forceinline__ int chunks_of(int e) const { return order ? first[e + 1] - first[e] : e == 0 ? total : 0; }
  __device__ __forceinline__ int first_of(int e) const { return order ? first[e] : 0; }
  __device__ __forceinline__ int all(int count) const { return order ? first[count] : total; }
};
// One workgroup; waves take the rows in spans, in order, so that an adapter's rows keep theirs.  Each wave counts its span by adapter; after sums over waves
// and adapters it goes over the span again, 64 rows at a time, and gives rows of one adapter their places together.  Rows without one come last (in `places` alone).  A lane finds the
// others with its adapter by the bits of the number: with a turn for each adapter, and sums in LDS by atomics, 16384 rows of 1000 adapters took 89 us more.  One compute unit, bound by its vector instructions at about 1 ns a row from there on: 6000 rows in runs of 8 adapters 9 us, 16384 16 (12 and 24 without the shortcut for 64 rows of one adapter
// and with the masks made twice); 777 rows of 3 mixed adapters 6 us.
constexpr int PLAN_WORDS = 32768;      // of LDS: counts by wave and adapter
static_assert(OSSCAR_ADAPTERS_MAX * 2 <= PLAN_WORDS, "");
__global__ __launch_bounds__(1024) void plan_kernel(Pick pick, int n, int waves, uint32_t rows_a_chunk, int2* places, int* order, Chunk* chunks, int* first) {
  __shared__ uint32_t counts[PLAN_WORDS];
  __shared__ uint32_t wave_rows[16], wave_chunks[16], wave_none[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, count = pick.count;
  for (int k = threadIdx.x; k < waves * count; k += 1024) counts[k] = 0;
  __syncthreads();
  const int span = ((n + waves - 1) / waves + 63) / 64 * 64;
  const int64_t begin = (int64_t)wave * span, end = std::min<int64_t>(n, begin + span);
  const int bits = 32 - __clz(count);
  auto same = [&](int mine) {      // the lanes whose rows have this one's adapter (one bit of its number after the other; -1 and -2 are none)
    uint64_t rows = __ballot(mine >= 0);
    if (!__ballot(mine != __builtin_amdgcn_readfirstlane(mine))) return rows;      // (in runs most often: all the same)
    for (int b = 0; b < bits; b++) {
      const uint64_t set = __ballot(mine >> b & 1);
      rows &= mine >> b & 1 ? set : ~set;
    }
    return rows;
  };
  const uint64_t below = (1ull << lane) - 1;
  constexpr int AT_ONCE = 8;      // times 64 rows, of which the reads are on their way together; those that a wave begins with stay for the second time
  auto read = [&](int64_t r0, int (&mine)[AT_ONCE]) {
#pragma unroll
    for (int b = 0; b < AT_ONCE; b++) mine[b] = pick.of(std::min<int64_t>(r0 + b * 64 + lane, n - 1));
  };
  uint32_t none = 0;
  int kept[AT_ONCE];
  uint64_t kept_rows[AT_ONCE];
  read(begin, kept);
  if (wave < waves)
    for (int64_t r0 = begin; r0 < end; r0 += AT_ONCE * 64) {
      int some[AT_ONCE];
      if (r0 > begin) read(r0, some);
#pragma unroll
      for (int b = 0; b < AT_ONCE; b++) {
        if (r0 + b * 64 >= end) break;
        const bool is = r0 + b * 64 + lane < end;
        const int mine = !is ? -1 : r0 > begin ? some[b] : kept[b];
        const uint64_t rows = same(mine);
        if (r0 == begin) kept_rows[b] = rows;
        if (mine >= 0 && !(rows & below)) counts[wave * count + mine] += __popcll(rows);      // (this wave's own word)
        if (mine < 0 && is) none++;
        __builtin_amdgcn_wave_barrier();
      }
    }
  for (int o = 32; o > 0; o >>= 1) none += __shfl_xor(none, o, 64);
  if (lane == 0) wave_none[wave] = none;
  __syncthreads();
  // places of adapters, `each` of them a thread: rows before, chunks before
  const int each = (count + 1023) / 1024;
  uint32_t rows = 0, parts = 0;
  for (int k = 0; k < each; k++) {
    const int e = threadIdx.x * each + k;
    if (e >= count) break;
    uint32_t s = 0;
    for (int w = 0; w < waves; w++) s += counts[w * count + e];
    rows += s;
    parts += (s + rows_a_chunk - 1) / rows_a_chunk;
  }
  uint32_t rows_to = rows, parts_to = parts;      // sums up to this thread, itself included
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t a = __shfl_up(rows_to, o, 64), b = __shfl_up(parts_to, o, 64);
    if (lane >= o) { rows_to += a; parts_to += b; }
  }
  if (lane == 63) { wave_rows[wave] = rows_to; wave_chunks[wave] = parts_to; }
  __syncthreads();
  uint32_t at = rows_to - rows, chunk = parts_to - parts;
  for (int w = 0; w < wave; w++) { at += wave_rows[w]; chunk += wave_chunks[w]; }
  for (int k = 0; k < each; k++) {
    const int e = threadIdx.x * each + k;
    if (e >= count) break;
    if (first) first[e] = (int)chunk;
    const uint32_t from = at;
    for (int w = 0; w < waves; w++) {
      const uint32_t s = counts[w * count + e];
      counts[w * count + e] = at;
      at += s;
    }
    for (uint32_t b = from; first && b < at; b += rows_a_chunk) chunks[chunk++] = Chunk{e, (int)b, (int)min(at, b + rows_a_chunk)};
    if (first && e == count - 1) first[count] = (int)chunk;
  }
  __syncthreads();
  if (wave >= waves) return;
  uint32_t last = 0;      // rows without an adapter lie behind all others
  for (int w = 0; w < 16; w++) last += wave_rows[w] + (w < wave ? wave_none[w] : 0);
  for (int64_t r0 = begin; r0 < end; r0 += AT_ONCE * 64) {
    int some[AT_ONCE];
    if (r0 > begin) read(r0, some);
#pragma unroll
    for (int b = 0; b < AT_ONCE; b++) {
      const int64_t r = r0 + b * 64 + lane;
      if (r0 + b * 64 >= end) break;
      const int mine = r >= end ? -1 : r0 > begin ? some[b] : kept[b];
      const uint64_t without = __ballot(mine < 0 && r < end), rows = r0 > begin ? same(mine) : kept_rows[b];
      if (places && (without >> lane & 1)) places[last + __popcll(without & below)] = int2{(int)r, mine};
      last += __popcll(without);
      const uint32_t base = mine >= 0 ? counts[wave * count + mine] : 0;
      __builtin_amdgcn_wave_barrier();
      if (mine >= 0) {
        const uint32_t to = base + __popcll(rows & below);
        if (places) places[to] = int2{(int)r, mine};
        if (order) order[to] = (int)r;
        if (!(rows & below)) counts[wave * count + mine] = base + __popcll(rows);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// A workgroup takes 16 CT components and 128 columns of a chunk, 32 columns a wave.  Rows go through LDS, STAGE of them at a time (the next ones on their way in registers while
// one stage is multiplied): Z as it is, T cut into its pieces once for all waves.  The contraction runs across the rows of both, so bf16 operands come through the transposing
// read of four 16-bit elements, float32 ones word by word.  8192 rows, 7168 and 14336 columns of bf16, rank 32: 110 us (3.6 TB/s with the chunks' sums); with the columns turned in
// registers 188, with two stages' rows on their way 134.
struct Outer {
  const float* t;      // [n][rank]
  Mat z;
  int C, scaled;
  float* part;         // [chunk][rank][C]
};
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;
constexpr int OW = 4, OCOLS = 128;
template <bool F32, int CT, int PIECES> struct Stage;
template <int CT, int PIECES>
struct Stage<false, CT, PIECES> {
  static constexpr int ROWS = 64, ZROW = OCOLS * 2, TROW = CT * 32 + 16, ZBYTES = ROWS * ZROW, BYTES = ZBYTES + PIECES * ROWS * TROW;
  // packets of a row change places, so that the four rows that sixteen lanes read at once meet other banks
  static __device__ __forceinline__ int swizzle(int row) { return ((row & 3) | ((row >> 3) & 1) << 2) << 1; }
  static __device__ __forceinline__ void put_z(char* lds, int row, int packet, const u16x8& w) {
    *reinterpret_cast<u16x8*>(lds + row * ZROW + ((packet ^ swizzle(row)) * 16)) = w;
  }
  static __device__ __forceinline__ void put_t(char* lds, int row, int j, const float (&x)[4]) {
    float left[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int p = 0; p < PIECES; p++) {
      typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
      v4bf w;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        w[e] = (__bf16)left[e];
        left[e] -= (float)w[e];
      }
      *reinterpret_cast<v4bf*>(lds + ZBYTES + (p * ROWS + row) * TROW + j * 2) = w;
    }
  }
  static __device__ __forceinline__ u32x4 turned_read(const char* q, int below) {
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)q), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(q + below));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // sixteen lanes read four rows of four quads of neighbouring elements each and get a column of them
  static __device__ __forceinline__ void multiply(const char* lds, int wave, int lane, v4f (&acc)[CT][2]) {
    const int i = lane & 15, g = lane >> 4, k = g * 8 + (i >> 2), q = i & 3;
#pragma unroll
    for (int half = 0; half < ROWS / 32; half++) {
      u32x4 z[2];
#pragma unroll
      for (int t = 0; t < 2; t++) {
        const int row = half * 32 + k, col = wave * 32 + t * 16 + q * 4;
        z[t] = turned_read(lds + row * ZROW + (((col >> 3) ^ swizzle(row)) * 16) + ((col >> 2) & 1) * 8, 4 * ZROW);      // (rows + 4: the same swizzle)
      }
#pragma unroll
      for (int a = 0; a < CT; a++)
#pragma unroll
        for (int p = PIECES - 1; p >= 0; p--) {
          const u32x4 w = turned_read(lds + ZBYTES + (p * ROWS + half * 32 + k) * TROW + a * 32 + q * 8, 4 * TROW);
#pragma unroll
          for (int t = 0; t < 2; t++) acc[a][t] = Num<false>::mma(w, z[t], acc[a][t]);
        }
    }
  }
};
template <int CT, int PIECES>
struct Stage<true, CT, PIECES> {
  static constexpr int ROWS = 32, ZROW = (OCOLS + 16) * 4, TROW = (CT == 1 ? 16 : CT * 16 + 16) * 4, ZBYTES = ROWS * ZROW, BYTES = ZBYTES + ROWS * TROW;      // (four rows meet other banks)
  static __device__ __forceinline__ void put_z(char* lds, int row, int packet, const Eight<true>::type& w) {
    f32x4* q = reinterpret_cast<f32x4*>(lds + row * ZROW + packet * 32);
    q[0] = w.a;
    q[1] = w.b;
  }
  static __device__ __forceinline__ void put_t(char* lds, int row, int j, const float (&x)[4]) {
    *reinterpret_cast<f32x4*>(lds + ZBYTES + row * TROW + j * 4) = f32x4{x[0], x[1], x[2], x[3]};
  }
  static __device__ __forceinline__ void multiply(const char* lds, int wave, int lane, v4f (&acc)[CT][2]) {
    const int i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int k = 0; k < ROWS; k += 4) {
      float z[2];
#pragma unroll
      for (int t = 0; t < 2; t++) z[t] = *reinterpret_cast<const float*>(lds + (k + g) * ZROW + (wave * 32 + t * 16 + i) * 4);
#pragma unroll
      for (int a = 0; a < CT; a++) {
        const float w = *reinterpret_cast<const float*>(lds + ZBYTES + (k + g) * TROW + (a * 16 + i) * 4);
#pragma unroll
        for (int t = 0; t < 2; t++) acc[a][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w, z[t], acc[a][t], 0, 0, 0);
      }
    }
  }
};
struct Outers { Outer a, b; int blocks_a; };      // dA and dB in one launch: that many column blocks are of dA
template <bool F32, int CT, int PIECES>
__global__ __launch_bounds__(OW * 64) void outer_kernel(Outers both, Plan plan, Pick pick) {
  typedef Eight<F32> E8;
  typedef Stage<F32, CT, PIECES> S;
  constexpr int NZ = S::ROWS * (OCOLS / 8) / (OW * 64), TPR = OW * 64 / S::ROWS, NT = CT * 16 / (TPR * 4) > 0 ? CT * 16 / (TPR * 4) : 1;      // packets of Z, quads of T a thread
  __shared__ __align__(16) char lds[S::BYTES];
  const int chunk = blockIdx.y;
  if (chunk >= plan.all(pick.count)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool first = (int)blockIdx.x < both.blocks_a;
  const Outer q = first ? both.a : both.b;
  const int c0 = ((int)blockIdx.x - (first ? 0 : both.blocks_a)) * OCOLS, j0 = blockIdx.z * CT * 16;
  const bool whole = c0 + OCOLS <= q.C;
  const Chunk h = plan.at(chunk);
  const float s = q.scaled ? pick.scale_of(h.e) : 1.f;
  typename E8::type z[NZ];
  float t[NT][4];
  const int zc = tid % (OCOLS / 8), zr = tid / (OCOLS / 8), tr = tid / TPR, tq = tid % TPR;
  auto fetch = [&](int b) {
#pragma unroll
    for (int k = 0; k < NZ; k++) {
      const int at = b + zr + k * (OW * 64 / (OCOLS / 8)), c = c0 + zc * 8;
      const int64_t row = plan.order ? plan.order[min(at, h.end - 1)] : min(at, h.end - 1);
      z[k] = whole ? E8::load(q.z.p, row * q.z.ld + c) : edge_load<F32>(q.z.p, row * q.z.ld, c, q.C);
      if (at >= h.end) z[k] = typename E8::type{};
    }
    const int at = b + tr;
    const float* from = q.t + (int64_t)(plan.order ? plan.order[min(at, h.end - 1)] : min(at, h.end - 1)) * pick.rank;
#pragma unroll
    for (int k = 0; k < NT; k++) {
      const int j = j0 + (tq + k * TPR) * 4;
      t_values<4>(from, j, pick.rank, t[k]);
#pragma unroll
      for (int e = 0; e < 4; e++) t[k][e] = at < h.end ? t[k][e] * s : 0.f;
    }
  };
  v4f acc[CT][2];
#pragma unroll
  for (int a = 0; a < CT; a++)
#pragma unroll
    for (int c = 0; c < 2; c++) acc[a][c] = v4f{0, 0, 0, 0};
  fetch(h.begin);
  for (int b = h.begin; b < h.end; b += S::ROWS) {      // (two buffers and one barrier a stage leave fewer workgroups on a compute unit: 62 and 92 us instead of 39 and 74)
#pragma unroll
    for (int k = 0; k < NZ; k++) S::put_z(lds, zr + k * (OW * 64 / (OCOLS / 8)), zc, z[k]);
#pragma unroll
    for (int k = 0; k < NT; k++)
      if ((tq + k * TPR) * 4 < CT * 16) S::put_t(lds, tr, (tq + k * TPR) * 4, t[k]);
    __syncthreads();
    if (b + S::ROWS < h.end) fetch(b + S::ROWS);
    S::multiply(lds, wave, lane, acc);
    __syncthreads();
  }
#pragma unroll
  for (int a = 0; a < CT; a++)
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
      for (int d = 0; d < 4; d++) {
        const int j = j0 + a * 16 + (lane >> 4) * 4 + d, col = c0 + wave * 32 + c * 16 + (lane & 15);
        if (j < pick.rank && col < q.C) q.part[((int64_t)chunk * pick.rank + j) * q.C + col] = acc[a][c][d];
      }
}
// The chunks' sums of an adapter's component, added in order; zeros for what has no rows.
struct Join { const float* part; int C; void* out; };
__global__ __launch_bounds__(256) void join_kernel(Join a, Join b, int blocks_a, Plan plan, Pick pick, int f32) {
  const int64_t rows = (int64_t)pick.count * pick.rank;
  const bool first_half = (int)blockIdx.x < blocks_a;
  const Join q = first_half ? a : b;
  const int c = (((int)blockIdx.x - (first_half ? 0 : blocks_a)) * 256 + threadIdx.x) * 4;
  if (c >= q.C) return;
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    const int e = (int)(row / pick.rank), j = (int)(row % pick.rank), first = plan.first_of(e), chunks = j < pick.rank_of(e) ? plan.chunks_of(e) : 0;
    float s[4] = {};
#pragma unroll 4
    for (int k = 0; k < chunks; k++) {
      float v[4];
      t_values<4>(q.part + ((int64_t)(first + k) * pick.rank + j) * q.C, c, q.C, v);
#pragma unroll
      for (int t = 0; t < 4; t++) s[t] += v[t];
    }
#pragma unroll
    for (int t = 0; t < 4; t++)
      if (c + t < q.C) {
        if (f32) reinterpret_cast<float*>(q.out)[row * q.C + c + t] = s[t];
        else reinterpret_cast<uint16_t*>(q.out)[row * q.C + c + t] = bf16_nearest(s[t]);
      }
  }
}

// --------------------------------------------------------------------------------------------------
// host
// --------------------------------------------------------------------------------------------------
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Rows that go through the kernels for few.  7168 x 14336 bf16, forward, these and the tiles: rows of 32 adapters, rank 16: 16 rows 10 and 13 us, 64 rows 12 and 25, 256 rows 24 and 52 (rank 64: 128 rows
// 50 and 74); of two adapters, sorted: 128 rows 14 and 18 (rank 64: 35 and 35), 256 rows 21 and 24; without an index 64 rows 11 and 13 (20 and 23), 128 rows 14 and 14 (34 and 23).
int64_t few_of(bool index) { return index ? 256 : 64; }
// Rows of many adapters are put in their order first, by a launch of one workgroup: where they are mixed, a tile has most adapters among its rows and is taken once for each; where they
// lie together already, that launch is lost.  bf16, forward, rank 16, as they lie and in order: 6000 rows, 2048 x 8192, mixed of 3 adapters 86 and 59 us, of 8 172 and 63, of 32 359 and 66; in runs
// of 2 49 and 59, of 8 51 and 61.  777 rows, 1365 x 5461, mixed of 8 42 and 28, in runs 23 and 28; 300 rows, 2048 x 2048, of 8, mixed or not, 13 and 18.  The gradients of A and B need the order
// in any case, so that their pass goes by it whenever there are more than few rows.
constexpr int SORT_FROM = 8, SORT_ROWS = 512;
bool sorts(int64_t n, int count, bool index) { return index && n >= SORT_ROWS && count >= SORT_FROM; }
static_assert(SORT_ROWS > 256, "");      // (more than few)
// Row tiles of 16 in a workgroup, and how its work is dealt out: parts of the contraction and slots of adapters to fill the chip where rows are few.
struct Deal { bool few; int ct, parts, slots; int64_t tiles; };
Deal deal(int64_t n, int64_t K, int count, int rank, bool f32, bool index, bool sorted) {
  if (n <= few_of(index)) return Deal{true, 0, (int)std::min<int64_t>(PARTS_MOST, up(K, FW * 512)), 1, n};
  Deal d{false, rank <= 16 ? 1 : rank <= 32 ? 2 : 4, 1, 1, up(n, 16 * RT)};
  if (index) d.slots = (int)std::max<int64_t>(1, std::min<int64_t>({256 / d.tiles, 16 * RT, count, sorted ? up(d.tiles + count, d.tiles) : count}));
  const int64_t turns = up(K, U * (f32 ? 16 : 32)), blocks = d.tiles * d.slots * up(rank, 16 * d.ct);
  d.parts = (int)std::max<int64_t>(1, std::min<int64_t>({256 / blocks, up(turns, 2 * CW), PARTS_MOST}));
  return d;
}

template <bool F32>
void contract(const Contract& all, const Pick& pick, const Deal& d, hipStream_t s) {
  if (d.few) {
    hipLaunchKernelGGL(contract_few_kernel<F32>, dim3((unsigned)all.parts, (unsigned)all.n, (unsigned)up(pick.rank, 16)), dim3(FW * 64), 0, s, all, pick);
    return;
  }
  const dim3 grid((unsigned)(d.tiles * d.slots), (unsigned)all.parts, (unsigned)up(pick.rank, 16 * d.ct)), block(CW * 64);
  auto go = [&](auto sorted) {
    constexpr bool SORTED = decltype(sorted)::value;
    if (d.ct == 1) hipLaunchKernelGGL((contract_kernel<F32, 1, SORTED>), grid, block, 0, s, all, pick);
    else if (d.ct == 2) hipLaunchKernelGGL((contract_kernel<F32, 2, SORTED>), grid, block, 0, s, all, pick);
    else hipLaunchKernelGGL((contract_kernel<F32, 4, SORTED>), grid, block, 0, s, all, pick);
  };
  if (pick.order) go(std::true_type{});
  else go(std::false_type{});
}
void order_rows(const Pick& pick, int64_t n, int rows_a_chunk, int2* places, int* order, Chunk* chunks, int* first, hipStream_t s) {
  const int waves = (int)std::min<int64_t>({16, PLAN_WORDS / pick.count, up(n, 64)});
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(1024), 0, s, pick, (int)n, waves, (uint32_t)rows_a_chunk, places, order, chunks, first);
}
template <bool F32>
void expand(const Expand& q, const Pick& pick, hipStream_t s) {
  if (q.n <= few_of(pick.index != nullptr)) {
    hipLaunchKernelGGL(expand_few_kernel<F32>, dim3((unsigned)up(q.C, 512), (unsigned)q.n), dim3((unsigned)(64 * std::min<int64_t>(4, up(pick.rank, 16)))), 0, s, q, pick);
    return;
  }
  const int64_t blocks = up(q.C, EW * ECOLS);
  Expand a = q;
  a.subs = 4;
  while (a.subs > 1 && up(q.n, a.subs * 16) * blocks < 512) a.subs /= 2;
  const int64_t tiles = up(q.n, 16 * a.subs);
  a.slots = pick.index ? (int)std::max<int64_t>(1, std::min<int64_t>({2048 / (tiles * blocks), 16 * a.subs, q.n, pick.order ? up(tiles + pick.count, tiles) : pick.count})) : 1;
  const dim3 grid((unsigned)(tiles * blocks), (unsigned)a.slots), block(EW * 64);
  auto go = [&](auto parts, auto sorted) {
    constexpr bool PARTS = decltype(parts)::value, SORTED = decltype(sorted)::value;
    if (pick.rank <= Columns<F32>::STEP) {
      if (F32 && a.subs < 4) hipLaunchKernelGGL((expand_kernel<F32, 1, PARTS, !F32, SORTED>), grid, block, 0, s, a, pick);
      else hipLaunchKernelGGL((expand_kernel<F32, 1, PARTS, true, SORTED>), grid, block, 0, s, a, pick);
    } else if (pick.rank <= 2 * Columns<F32>::STEP) hipLaunchKernelGGL((expand_kernel<F32, 2, PARTS, true, SORTED>), grid, block, 0, s, a, pick);
    else hipLaunchKernelGGL((expand_kernel<F32, 0, PARTS, true, SORTED>), grid, block, 0, s, a, pick);
  };
  if (a.parts > 1) pick.order ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
  else pick.order ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
}
template <bool F32, int PIECES>
void outer(const Outers& q, const Plan& plan, const Pick& pick, int64_t chunks, hipStream_t s) {
  const int ct = pick.rank <= 16 ? 1 : pick.rank <= 32 ? 2 : 4;
  const dim3 grid((unsigned)(q.blocks_a + up(q.b.C, OCOLS)), (unsigned)chunks, (unsigned)up(pick.rank, 16 * ct)), block(OW * 64);
  if (ct == 1) hipLaunchKernelGGL((outer_kernel<F32, 1, PIECES>), grid, block, 0, s, q, plan, pick);
  else if (ct == 2) hipLaunchKernelGGL((outer_kernel<F32, 2, PIECES>), grid, block, 0, s, q, plan, pick);
  else hipLaunchKernelGGL((outer_kernel<F32, 4, PIECES>), grid, block, 0, s, q, plan, pick);
}

// Rows of a chunk: 512, of many rows as many as leave 64 chunks (their sums are written and read again: as much as 2 rank rows of bf16 each), and half of that again and again, down to 65, while the
// narrower width's workgroups are fewer than 512.  So a narrow width has up to 1023 chunks: 2^20 rows of 256 x 14336, rank 64, have 256 of them, 956 MB of sums.
int chunk_of(const osscar_adapters_desc& d) {
  int chunk = (int)std::max<int64_t>(512, up(up(d.n, 64), 64) * 64);
  while (chunk > 128 && up(d.n, chunk) * up(std::min(d.d, d.m), OCOLS) * up(d.rank, 64) < 512) chunk /= 2;
  return chunk;
}
int64_t chunks_of(const osscar_adapters_desc& d) { return up(d.n, chunk_of(d)) + (d.index ? std::min<int64_t>(d.n, d.count) : 0); }

const char* bad_desc(const osscar_adapters_desc* d) {
  if (!d) return "osscar_adapters: NULL description";
  if (!a_size(d->n, 0) || !a_size(d->d, 1) || !a_size(d->m, 1)) return "osscar_adapters: n >= 0, d and m must be positive, none above 2^30";
  if (d->count < 1 || d->count > OSSCAR_ADAPTERS_MAX) return "osscar_adapters: 1 to OSSCAR_ADAPTERS_MAX adapters";
  if (d->rank < 1 || d->rank > OSSCAR_ADAPTER_MAX_RANK) return "osscar_adapters: ranks are 1 to OSSCAR_ADAPTER_MAX_RANK";
  if (!real_dtype(d->dtype)) return "osscar_adapters: unknown dtype";
  if (d->ldx < d->d || d->lda < d->d || d->ldb < d->m) return "osscar_adapters: leading dimension below the row length";
  if (d->next_a < 0 || d->next_b < 0) return "osscar_adapters: negative stride of adapters";
  // (of the launches' grids, which one row tile times the column blocks fill)
  if (d->n > (int64_t)1 << 22) return "osscar_adapters: more than 2^22 rows in one call";
  if (up(d->n, 16) * up(std::max(d->d, d->m), EW * ECOLS) >= (int64_t)1 << 23) return "osscar_adapters: too large";
  return nullptr;
}
// (of the outer products' launch, which has the column blocks of both widths in one row of its grid)
const char* bad_gradients(const osscar_adapters_desc& d) {
  return launchable(up(d.d, OCOLS) + up(d.m, OCOLS), OW * 64) ? nullptr : "osscar_adapters_backward: d and m are too large together for dA and dB";
}
bool misaligned(const void* p, int32_t dtype) { return (uintptr_t)p % (dtype == OSSCAR_F32 ? 4 : 2) != 0; }
// Whether rows of one matrix reach into the memory of another's (n > 0 rows)
bool meet(const void* a, int64_t lda, int64_t d, const void* b, int64_t ldb, int64_t m, int64_t n, int32_t dtype) {
  const uintptr_t size = dtype == OSSCAR_F32 ? 4 : 2, p = (uintptr_t)a, q = (uintptr_t)b;
  return p < q + ((n - 1) * ldb + m) * size && q < p + ((n - 1) * lda + d) * size;
}
size_t t_bytes(const osscar_adapters_desc& d, int parts) { return (size_t)parts * d.n * d.rank * 4; }

// (the gradients of A and B need the order in any case)
bool sorts_backward(const osscar_adapters_desc& d, bool grads) { return d.index && d.n > few_of(true) && (grads || sorts(d.n, d.count, true)); }
struct BackwardSpace { float *dt_parts, *dt, *t; int2* places; int* order; Chunk* table; int* first; float *part_a, *part_b; };
BackwardSpace backward_space(Carve& c, const osscar_adapters_desc& d, bool grads, int parts) {
  BackwardSpace w{};
  w.dt_parts = reinterpret_cast<float*>(c.take(t_bytes(d, parts)));
  if (sorts_backward(d, grads)) w.places = reinterpret_cast<int2*>(c.take((size_t)d.n * 8));
  if (!grads) return w;
  const int64_t chunks = chunks_of(d);
  w.dt = reinterpret_cast<float*>(c.take(t_bytes(d, 1)));
  w.t = reinterpret_cast<float*>(c.take(t_bytes(d, 1)));      // where T is not given
  if (d.index) {
    w.order = reinterpret_cast<int*>(c.take((size_t)d.n * 4));
    w.table = reinterpret_cast<Chunk*>(c.take((size_t)chunks * sizeof(Chunk)));
    w.first = reinterpret_cast<int*>(c.take((size_t)(d.count + 1) * 4));
  }
  w.part_a = reinterpret_cast<float*>(c.take((size_t)chunks * d.rank * d.d * 4));
  w.part_b = reinterpret_cast<float*>(c.take((size_t)chunks * d.rank * d.m * 4));
  return w;
}

}  // namespace

extern "C" size_t osscar_adapters_workspace_bytes(const osscar_adapters_desc* d, int32_t backward) {
  if (bad_desc(d)) return 0;
  Carve c(nullptr);
  if (d->n == 0 && !backward) return 256;
  const bool f32 = d->dtype == OSSCAR_F32;
  if (!backward) {
    const bool sorted = sorts(d->n, d->count, d->index != 0);
    c.take(t_bytes(*d, deal(std::max<int64_t>(d->n, 1), d->d, d->count, d->rank, f32, d->index != 0, sorted).parts));
    if (sorted) c.take((size_t)d->n * 8);
  } else {
    const bool grads = backward != 2;
    if (grads && bad_gradients(*d)) return 0;
    backward_space(c, *d, grads, deal(std::max<int64_t>(d->n, 1), d->m, d->count, d->rank, f32, d->index != 0, sorts_backward(*d, grads)).parts);
  }
  return c.used + 256;
}

extern "C" osscar_status osscar_adapters_forward(const osscar_adapters_desc* d, const void* X_dev, const void* A_dev, const void* B_dev, const int64_t* index_dev,
                                                 const float* scale_dev, const int32_t* ranks_dev, const void* base_dev, int64_t ldbase, void* Y_dev, int64_t ldy, float* T_dev,
                                                 void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* bad = bad_desc(d);
  if (!bad && (ldy < d->m || (base_dev && ldbase < d->m))) bad = "osscar_adapters_forward: leading dimension below the row length";
  if (!bad && d->n > 0 && (d->index != 0) != (index_dev != nullptr)) bad = "osscar_adapters_forward: the description says whether there is an index";
  if (!bad && (!A_dev || !B_dev || (d->n > 0 && (!X_dev || !Y_dev)))) bad = "osscar_adapters_forward: NULL pointer";
  if (!bad && (misaligned(X_dev, d->dtype) || misaligned(A_dev, d->dtype) || misaligned(B_dev, d->dtype) || misaligned(base_dev, d->dtype) || misaligned(Y_dev, d->dtype) ||
               misaligned(T_dev, OSSCAR_F32) || misaligned(scale_dev, OSSCAR_F32) || misaligned(ranks_dev, OSSCAR_F32) || ((uintptr_t)index_dev & 7)))
    bad = "osscar_adapters_forward: a buffer is not aligned to its elements";
  if (!bad && base_dev && base_dev == Y_dev && ldbase != ldy && d->n > 1) bad = "osscar_adapters_forward: in place, both leading dimensions are the same";
  if (!bad && ((uintptr_t)workspace_dev & 255)) bad = "osscar_adapters_forward: the workspace must begin at a 256-byte boundary";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if (d->n == 0) return OSSCAR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const bool f32 = d->dtype == OSSCAR_F32;
  const bool sorted = sorts(d->n, d->count, d->index != 0);
  const Deal deal1 = deal(d->n, d->d, d->count, d->rank, f32, d->index != 0, sorted);
  Carve c(workspace_dev);
  float* t = reinterpret_cast<float*>(c.take(t_bytes(*d, deal1.parts)));
  int2* places = sorted ? reinterpret_cast<int2*>(c.take((size_t)d->n * 8)) : nullptr;
  const Pick pick{index_dev, scale_dev, ranks_dev, d->count, d->rank, places};
  if (!workspace_dev || c.used > workspace_bytes) return refuse_call(OSSCAR_ENOMEM, "osscar_adapters_forward: workspace too small");
  const bool direct = T_dev && deal1.parts == 1;
  if (direct) t = T_dev;
  const Contract k{Mat{X_dev, d->ldx}, Adapters{A_dev, d->lda, d->next_a}, d->n, (int)d->d, deal1.parts, deal1.slots, 0, t};
  const Expand x{t, deal1.parts, 1, 1, 1, Adapters{B_dev, d->ldb, d->next_b}, Mat{base_dev, ldbase}, d->n, (int)d->m, Y_dev, ldy, direct ? nullptr : T_dev};
  if (sorted) order_rows(pick, d->n, 1, places, nullptr, nullptr, nullptr, s);
  if (f32) {
    contract<true>(k, pick, deal1, s);
    expand<true>(x, pick, s);
  } else {
    contract<false>(k, pick, deal1, s);
    expand<false>(x, pick, s);
  }
  return launched();
}

extern "C" osscar_status osscar_adapters_backward(const osscar_adapters_desc* d, const void* X_dev, const void* A_dev, const void* B_dev, const int64_t* index_dev,
                                                  const float* scale_dev, const int32_t* ranks_dev, const void* dY_dev, int64_t lddy, const float* T_dev, const void* base_dev,
                                                  int64_t ldbase, void* dX_dev, int64_t lddx, void* dA_dev, void* dB_dev, int32_t dw_dtype, void* workspace_dev,
                                                  size_t workspace_bytes, void* hip_stream) {
  const char* bad = bad_desc(d);
  const bool grads = dA_dev || dB_dev;
  if (!bad && (lddy < d->m || (dX_dev && lddx < d->d) || (base_dev && ldbase < d->d))) bad = "osscar_adapters_backward: leading dimension below the row length";
  if (!bad && d->n > 0 && (d->index != 0) != (index_dev != nullptr)) bad = "osscar_adapters_backward: the description says whether there is an index";
  if (!bad && (!A_dev || !B_dev || (d->n > 0 && (!X_dev || !dY_dev)))) bad = "osscar_adapters_backward: NULL pointer";
  if (!bad && (!dA_dev != !dB_dev)) bad = "osscar_adapters_backward: dA and dB are given together or not at all";
  if (!bad && base_dev && !dX_dev) bad = "osscar_adapters_backward: base goes with dX";
  if (!bad && grads && !real_dtype(dw_dtype)) bad = "osscar_adapters_backward: unknown dtype";
  if (!bad && grads) bad = bad_gradients(*d);
  if (!bad && (misaligned(X_dev, d->dtype) || misaligned(A_dev, d->dtype) || misaligned(B_dev, d->dtype) || misaligned(base_dev, d->dtype) || misaligned(dY_dev, d->dtype) ||
               misaligned(dX_dev, d->dtype) || misaligned(T_dev, OSSCAR_F32) || misaligned(scale_dev, OSSCAR_F32) || misaligned(ranks_dev, OSSCAR_F32) || ((uintptr_t)index_dev & 7) ||
               (grads && (misaligned(dA_dev, dw_dtype) || misaligned(dB_dev, dw_dtype)))))
    bad = "osscar_adapters_backward: a buffer is not aligned to its elements";
  if (!bad && base_dev && base_dev == dX_dev && ldbase != lddx && d->n > 1) bad = "osscar_adapters_backward: in place, both leading dimensions are the same";
  if (!bad && ((uintptr_t)workspace_dev & 255)) bad = "osscar_adapters_backward: the workspace must begin at a 256-byte boundary";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if ((!grads && !dX_dev) || (d->n == 0 && !grads)) return OSSCAR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const bool f32 = d->dtype == OSSCAR_F32, index = d->index != 0;
  const int64_t chunks = chunks_of(*d);
  const bool sorted = sorts_backward(*d, grads);
  Deal dy = deal(std::max<int64_t>(d->n, 1), d->m, d->count, d->rank, f32, index, sorted), dx = deal(std::max<int64_t>(d->n, 1), d->d, d->count, d->rank, f32, index, sorted);
  Carve c(workspace_dev);
  const BackwardSpace w = backward_space(c, *d, grads, dy.parts);
  if (c.used > 0 && (!workspace_dev || c.used > workspace_bytes)) return refuse_call(OSSCAR_ENOMEM, "osscar_adapters_backward: workspace too small");
  float *dt_parts = w.dt_parts, *const dt = w.dt;      // (dt, whole, is wanted by the outer products alone)
  const Pick pick{index_dev, scale_dev, ranks_dev, d->count, d->rank, w.places};
  // The outer products read X and dY: where dX takes the place of one of them, it comes behind
  const bool late = grads && dX_dev && d->n > 0 && (meet(dX_dev, lddx, d->d, dY_dev, lddy, d->m, d->n, d->dtype) || meet(dX_dev, lddx, d->d, X_dev, d->ldx, d->d, d->n, d->dtype));
  auto make_dx = [&] {
    const Expand x{dt_parts, dy.parts, 1, 0, 1, Adapters{A_dev, d->lda, d->next_a}, Mat{base_dev, ldbase}, d->n, (int)d->d, dX_dev, lddx, dy.parts > 1 ? dt : nullptr};
    if (f32) expand<true>(x, pick, s);
    else expand<false>(x, pick, s);
  };
  if (d->n > 0) {
    if (index && (grads || sorted)) order_rows(pick, d->n, chunk_of(*d), w.places, w.order, w.table, w.first, s);
    if (!dX_dev) dy.parts = 1;      // (the parts are added where dX is made)
    if (dy.parts == 1 && grads) dt_parts = dt;
    const Contract k{Mat{dY_dev, lddy}, Adapters{B_dev, d->ldb, d->next_b}, d->n, (int)d->m, dy.parts, dy.slots, 1, dt_parts};
    if (f32) contract<true>(k, pick, dy, s);
    else contract<false>(k, pick, dy, s);
    if (late && dy.parts > 1) {      // (few rows: 2^12 at most)
      const int64_t size = d->n * d->rank;
      hipLaunchKernelGGL(add_parts_kernel, dim3((unsigned)up(size, 256)), dim3(256), 0, s, dt_parts, dy.parts, size, dt);
      dt_parts = dt;
      dy.parts = 1;
    }
    if (dX_dev && !late) make_dx();
    if (!grads) return launched();
    if (!T_dev) {
      dx.parts = 1;
      const Contract k2{Mat{X_dev, d->ldx}, Adapters{A_dev, d->lda, d->next_a}, d->n, (int)d->d, 1, dx.slots, 0, w.t};
      if (f32) contract<true>(k2, pick, dx, s);
      else contract<false>(k2, pick, dx, s);
      T_dev = w.t;
    }
  }
  const bool listed = index && d->n > 0;
  const Plan plan{listed ? w.order : nullptr, w.table, w.first, d->n, listed ? 0 : (int)chunks, chunk_of(*d)};
  const Outers both{Outer{dt, Mat{X_dev, d->ldx}, (int)d->d, 0, w.part_a}, Outer{T_dev, Mat{dY_dev, lddy}, (int)d->m, 1, w.part_b}, (int)up(d->d, OCOLS)};
  if (d->n > 0) {
    if (f32) outer<true, 1>(both, plan, pick, chunks, s);
    else if (dw_dtype == OSSCAR_F32) outer<false, 3>(both, plan, pick, chunks, s);
    else outer<false, 2>(both, plan, pick, chunks, s);
  }
  if (late) make_dx();
  const int blocks_a = (int)up(d->d, 1024);
  hipLaunchKernelGGL(join_kernel, dim3((unsigned)(blocks_a + up(d->m, 1024)), (unsigned)std::min<int64_t>((int64_t)d->count * d->rank, 65535)), dim3(256), 0, s,
                     Join{w.part_a, (int)d->d, dA_dev}, Join{w.part_b, (int)d->m, dB_dev}, blocks_a, plan, pick, dw_dtype == OSSCAR_F32);
  return launched();
}
