// One matrix product for the operators of gated.hip and intprod.hip: C[m][n] = sum over segments and k of A[m][k] B[n][k], in bf16
// (v_mfma_f32_16x16x32_bf16, float32 sums) or int8 (v_mfma_i32_16x16x64_i8, exact int32 sums), with an epilogue of the caller's.
//
// An operand is stored with the contraction along its rows (OP_K: element (row, k), k side by side) or across them (OP_T: element (k, row),
// rows of the result side by side).  Both go from global memory straight into LDS in packets of 16 bytes.  OP_K operands are read
// from there a packet per lane, OP_T operands through the transposing read of four 16-bit elements (ds_read_b64_tr_b16), so that no
// pass over an operand is needed for any of the three products of a layer's forward and backward pass.
// A segment is one pair of operands of the same shapes; several are summed: the two products of dX, and the six products of bf16 pieces that
// make a float32 product (x = x1 + x2 + x3 of 8 bits each; all products of weight 2^-16 and more).
//
// Every packet is read through a buffer descriptor that ends where the operand ends, and a lane whose packet lies beyond the end of a
// row gets an offset past that end: what is outside an operand reads as zero.  Rows and packets begin at 16-byte boundaries and the
// contiguous length is a multiple of a packet; the callers copy operands of other alignments first.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace osscar {
namespace tile {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;

enum { OP_K = 0, OP_T = 1 };
constexpr int SEGS = 12;                        // two products of float32 operands
constexpr int STEP_BYTES = 128;                 // contraction per stage and row: 64 bf16 or 128 int8
constexpr int64_t MAX_LD_BYTES = 1 << 22;       // 256 rows stay below the 2^30 bytes that an offset may take

struct Operand {
  const char* p[SEGS];
  int64_t ldb;               // bytes from one row to the next
  int rows, cols;            // stored rows, stored elements of a row
};
// element sizes and stages
inline bool operand_fits(const void* p, int64_t ld, int64_t cols, int es) {
  return ((uintptr_t)p & 15) == 0 && (ld * es) % 16 == 0 && (cols * es) % 16 == 0 && ld * es <= MAX_LD_BYTES;
}

template <bool I8> struct Num;
template <> struct Num<false> {
  typedef v4f acc; typedef float val;
  static constexpr int ES = 2;
  static __device__ __forceinline__ acc mma(v4i a, v4i b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  }
};
template <> struct Num<true> {
  typedef v4i acc; typedef int val;
  static constexpr int ES = 1;
  static __device__ __forceinline__ acc mma(v4i a, v4i b, acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

// The shape of a workgroup: WM x WN waves, each of FM x (NB FN) tiles of 16 x 16.  NB: matrices on the B side whose columns a wave takes
// alike (gate and up projection), FN tiles of each.
template <int WM_, int WN_, int FM_, int FN_, int NB_>
struct Shape {
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, NB = NB_, WAVES = WM * WN, BM = WM * FM * 16, BN = WN * FN * 16;
};

// One side's way into LDS and out of it.  EXT: rows of the result that the workgroup takes of it; PER: tiles of 16 per wave.  A-side tiles
// lie one behind the other.  On the B side (PERM) lane group g holds PER x 4 neighbouring columns: tile j, matrix-core row i is column
// (i / 4) 4 PER + 4 j + i % 4 of the wave's, so that a lane's results are 4 PER neighbours in memory.
// Packets are permuted inside an LDS row so that the lanes of one access meet all banks once.
template <int MODE, int ES, int EXT, int PER, bool PERM, int WAVES>
struct Side {
  static constexpr int ROW = MODE == OP_K ? STEP_BYTES : EXT * ES;      // bytes of an LDS row
  static constexpr int PK = ROW / 16;                                   // its packets
  static constexpr int BYTES = EXT * STEP_BYTES;
  static constexpr int NJ = BYTES / 1024 / WAVES;                       // loads of a wave per stage
  static_assert(BYTES % (1024 * WAVES) == 0, "every wave issues the same number of loads");
  static constexpr int RPI = 64 / PK;                                   // LDS rows per load
  static __device__ __forceinline__ int swizzle(int row) {
    if (MODE == OP_K) return PERM ? (row & 3) | (((row / (4 * PER)) & 1) << 2) : row & 7;
    if (!PERM) return (((row & 3) | (((row >> 3) & 1) << 2)) << 1) & (PK - 1);
    if (PK == 8) return ((row >> 1) & 1) << 2;
    return PER >= 4 ? (row & 1) | ((row & 2) << 2) : (row & 3) << 2;
  }
  int voff[NJ], vcol[NJ];      // byte offset of the lane's packet from the stage's corner; first element of it along the row
  int seg_row0;                // result rows before the workgroup's
  __device__ __forceinline__ void open(const Operand& o, int row0, int wave, int lane) {
    seg_row0 = row0;
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const int r = (wave + WAVES * j) * RPI + lane / PK, c = (lane % PK) ^ swizzle(r);
      vcol[j] = c * (16 / ES);
      voff[j] = (lane / PK) * (int)o.ldb + c * 16;
      if (MODE == OP_T && row0 + vcol[j] >= o.cols) voff[j] = 0x7FFFFFF0;
    }
  }
  // requests the stage that begins at k of segment seg
  __device__ __forceinline__ void load(const Operand& o, int seg, int k, char* lds, int wave) const {
    const int r0 = MODE == OP_K ? seg_row0 : k, c0 = MODE == OP_K ? k : seg_row0;
    const int64_t at = (int64_t)r0 * o.ldb + (int64_t)c0 * ES;
    int64_t left = (int64_t)(o.rows - r0 - 1) * o.ldb + (int64_t)(o.cols - c0) * ES;      // bytes from here to the end of the operand
    left = left < 0 || r0 >= o.rows || c0 >= o.cols ? 0 : (left > 0x7FFFFFF0 ? 0x7FFFFFF0 : left);
    __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)(o.p[seg] + at), 0, (int)left, 0x00020000);
    const bool tail = MODE == OP_K && k + STEP_BYTES / ES > o.cols;
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const int i = wave + WAVES * j;
      const int v = tail && k + vcol[j] >= o.cols ? 0x7FFFFFF0 : voff[j];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(lds + i * 1024), 16, v, i * RPI * (int)o.ldb, 0, 0);
    }
  }
  // the wave's PER operands of half stage `sub`, wpos: its place among the waves along this side
  int raddr[MODE == OP_K ? 1 : PER];
  __device__ __forceinline__ void open_read(int wpos, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if (MODE == OP_K) {
      const int row = wpos * PER * 16 + (PERM ? (i >> 2) * 4 * PER + (i & 3) : i);
      raddr[0] = row * ROW + ((g ^ swizzle(row)) * 16);
    } else {
#pragma unroll
      for (int t = 0; t < PER; t++) {
        const int col = wpos * PER * 16 + (PERM ? (i & 3) * 4 * PER + t * 4 : t * 16 + (i & 3) * 4), k = g * 8 + (i >> 2);
        raddr[t] = k * ROW + (((col >> 3) ^ swizzle(k)) * 16) + ((col >> 2) & 1) * 8;
      }
    }
  }
  __device__ __forceinline__ v4i read(const char* lds, int t, int sub) const {
    if (MODE == OP_K) return *reinterpret_cast<const v4i*>(lds + (raddr[0] ^ (sub * 64)) + t * (PERM ? 4 : 16) * ROW);
    typedef __attribute__((address_space(3))) v4s lds_v4s;
    const char* q = lds + raddr[MODE == OP_K ? 0 : t] + sub * 32 * ROW;
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)q), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(q + 4 * ROW));
    return __builtin_bit_cast(v4i, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

template <int NB>
struct Product {
  Operand a, b[NB];
  int nseg, k;               // segments, contraction of each in elements
  int M, N;
};

// Workgroup b runs on XCD b % 8: every XCD gets a contiguous range of the tiles, which go down eight rows of tiles before the next column, so
// that what an XCD works on together shares operands in its L2.
__device__ __forceinline__ void tile_of(int b, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int n = tiles_m * tiles_n, q = n / 8, r = n % 8, x = b % 8;
  const int id = x * q + (x < r ? x : r) + b / 8;
  const int group = id / (8 * tiles_n), first = group * 8, rows = tiles_m - first < 8 ? tiles_m - first : 8;
  const int in = id - group * 8 * tiles_n;
  tm = first + in % rows;
  tn = in / rows;
}

// Epi: __device__ void put(int m, int n, const val (&v)[NB][4 * FN], int M, int N), 4 FN neighbouring columns of row m from n on; m < M, but columns may pass N.
template <bool I8, int AM, int BMODE, class S, class Epi>
__device__ __forceinline__ void product_tile(const Product<S::NB>& q, const Epi& epi) {
  typedef Num<I8> T;
  constexpr int ES = T::ES, KS = STEP_BYTES / ES;
  typedef Side<AM, ES, S::BM, S::FM, false, S::WAVES> SA;
  typedef Side<BMODE, ES, S::BN, S::FN, true, S::WAVES> SB;
  // Two stages, each in arrays of its own: with one array the compiler waits before every read of LDS for all requests under way.
  __shared__ __align__(1024) char a0[SA::BYTES], a1[SA::BYTES], b0[S::NB][SB::BYTES], b1[S::NB][SB::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
  int tm, tn;
  tile_of(blockIdx.x, (q.M + S::BM - 1) / S::BM, (q.N + S::BN - 1) / S::BN, tm, tn);
  SA sa;
  SB sb;
  sa.open(q.a, tm * S::BM, wave, lane);
  sb.open(q.b[0], tn * S::BN, wave, lane);
  sa.open_read(wm, lane);
  sb.open_read(wn, lane);
  typename T::acc acc[S::FM][S::NB][S::FN];
#pragma unroll
  for (int i = 0; i < S::FM; i++)
#pragma unroll
    for (int z = 0; z < S::NB; z++)
#pragma unroll
      for (int j = 0; j < S::FN; j++)
#pragma unroll
        for (int r = 0; r < 4; r++) acc[i][z][j][r] = 0;
  int seg = 0, k = 0;      // of the next stage to be requested
  const int per = (q.k + KS - 1) / KS, total = per * q.nseg;
  auto request = [&](char* a, char (*b)[SB::BYTES]) {
    sa.load(q.a, seg, k, a, wave);
#pragma unroll
    for (int z = 0; z < S::NB; z++) sb.load(q.b[z], seg, k, b[z], wave);
    k += KS;
    if (k >= q.k) { k = 0; seg++; }
  };
  auto multiply = [&](const char* a, const char (*b)[SB::BYTES]) {
#pragma unroll
    for (int sub = 0; sub < 2; sub++) {
      v4i fa[S::FM], fb[S::NB][S::FN];
#pragma unroll
      for (int z = 0; z < S::NB; z++)
#pragma unroll
        for (int j = 0; j < S::FN; j++) fb[z][j] = sb.read(b[z], j, sub);
#pragma unroll
      for (int i = 0; i < S::FM; i++) fa[i] = sa.read(a, i, sub);
#pragma unroll
      for (int i = 0; i < S::FM; i++)
#pragma unroll
        for (int z = 0; z < S::NB; z++)
#pragma unroll
          for (int j = 0; j < S::FN; j++) acc[i][z][j] = T::mma(fb[z][j], fa[i], acc[i][z][j]);      // rows of the result tile: columns n
    }
  };
  request(a0, b0);
  for (int st = 0; st < total; st += 2) {
    __syncthreads();      // the stage has landed (every wave waits for its requests) and the other one's readers are done
    if (st + 1 < total) request(a1, b1);
    multiply(a0, b0);
    if (st + 1 >= total) break;
    __syncthreads();
    if (st + 2 < total) request(a0, b0);
    multiply(a1, b1);
  }
  const int i = lane & 15, g = lane >> 4;
#pragma unroll
  for (int f = 0; f < S::FM; f++) {
    const int m = tm * S::BM + (wm * S::FM + f) * 16 + i, n = tn * S::BN + wn * S::FN * 16 + g * 4 * S::FN;
    typename T::val v[S::NB][4 * S::FN];
#pragma unroll
    for (int z = 0; z < S::NB; z++)
#pragma unroll
      for (int j = 0; j < S::FN; j++)
#pragma unroll
        for (int r = 0; r < 4; r++) v[z][4 * j + r] = acc[f][z][j][r];
    if (m < q.M && n < q.N) epi.put(m, n, v, q.M, q.N);
  }
}

}  // namespace tile
}  // namespace osscar
