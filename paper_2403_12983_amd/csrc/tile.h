// One matrix product for the operators of gated.hip and intprod.hip: C[m][n] = sum over segments and k of A[m][k] B[n][k], in bf16
// (v_mfma_f32_16x16x32_bf16, float32 sums) or int8 (v_mfma_i32_16x16x64_i8, exact int32 sums), with an epilogue of the caller's.
//
// An operand is stored with the contraction along its rows (OP_K: element (row, k), k side by side) or across them (OP_T: element (k, row),
// rows of the result side by side).  Both go from global memory straight into LDS in packets of 16 bytes.  OP_K operands are read
// from there a packet per lane, OP_T operands through the transposing read of four 16-bit elements (ds_read_b64_tr_b16), so that no
// pass over an operand is needed for any of the three products of a layer's forward and backward pass.
// A segment is one pair of operands of the same shapes; two are summed for dX.
//
// Every packet is read through a buffer descriptor that ends where the operand ends, and a lane whose packet lies beyond the end of a row gets an offset past
// that end: what is outside an operand reads as zero.  Rows and packets begin at 16-byte boundaries and the contiguous length is a multiple of a packet; the
// callers copy operands of other alignments first (any alignment by way of registers, without the copy: half the rate from 256 rows on).
// Bound by the matrix cores and the chip's power (8192 x 8192 x 8192 on random operands: bf16 1470 to 1520 TFLOP/s in each order of the operands, the library
// 1200 to 1620; the clock falls to 1.7 to 2.1 GHz); few rows, by reading B (16 x 7168 x 14336, both projections 77 us, 5.3 TB/s).
#pragma once
#include "ops.h"

namespace osscar {
namespace tile {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;

enum { OP_K = 0, OP_T = 1 };
constexpr int SEGS = 2;                         // the two products of dX
constexpr int STEP_BYTES = 128;                 // contraction per stage and row: 64 bf16 or 128 int8, two matrix-core operands
constexpr int64_t MAX_LD_BYTES = 1 << 22;       // of an operand in place: 256 rows stay below 2^30 bytes
// of any operand: what a tile (OP_K, 256 rows) or a stage (OP_T, 64) spans stays below the 0x7FFFFFF0 bytes that stand for an offset past every end
constexpr int64_t MAX_K_BYTES = 0x7FFFFFF0 / 256 / 16 * 16, MAX_T_BYTES = 0x7FFFFFF0 / 64 / 16 * 16;

struct Operand {
  const char* p[SEGS];
  int64_t ldb;               // bytes from one row to the next
  int rows, cols;            // stored rows, stored elements of a row
};
// whether an operand of elements of es bytes is read in place
inline bool operand_fits(const void* p, int64_t ld, int64_t cols, int es) {
  return ((uintptr_t)p & 15) == 0 && (ld * es) % 16 == 0 && (cols * es) % 16 == 0 && ld * es <= MAX_LD_BYTES;
}

// vmcnt <= N; lgkmcnt = 0, then the barrier: builtins, which the compiler takes into account where it places waits of its own
template <int N>
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14)); }
__device__ __forceinline__ void stage_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// D = A B + D with the sums in the accumulation registers.  Written out so that the sums stay where they are: the compiler's own form gives D
// other registers than it reads, which four tiles' worth of copies per product pay for where 256 registers of sums are all there are.
// Of the two shapes of the instruction the 16 x 16 one moves less between registers per operation: on random operands, where the chip's power
// sets its clock, 2.1 PFLOP/s alone against 1.8.
template <bool I8> struct Num;
template <> struct Num<false> {
  typedef v4f acc; typedef float val;
  static constexpr int ES = 2;
  static __device__ __forceinline__ void mma(v4i a, v4i b, acc& c) { asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};
template <> struct Num<true> {
  typedef v4i acc; typedef int val;
  static constexpr int ES = 1;
  static __device__ __forceinline__ void mma(v4i a, v4i b, acc& c) { asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};
// The matrix core has written the sums when this has passed (16 wait states cover its longest result).  The compiler does not see matrix instructions there,
// and without settled() it reads sums before the wait, and all 256 of them at once, which it then moves about between registers and memory.
__device__ __forceinline__ void sums_written() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
template <class V>
__device__ __forceinline__ void settled(V& c) { asm volatile("" : "+a"(c)); }

// The shape of a workgroup: WM x WN waves, each of FM x (NB FN) tiles of 16 x 16.  NB: matrices on the B side whose columns a wave takes
// alike (gate and up projection), FN tiles of each.
template <int WM_, int WN_, int FM_, int FN_, int NB_>
struct Shape {
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, NB = NB_, WAVES = WM * WN, BM = WM * FM * 16, BN = WN * FN * 16;
};

// One side's way into LDS and out of it.  EXT: rows of the result that the workgroup takes of it; PER: tiles of 16 per wave.  A-side tiles
// lie one behind the other.  Lane group g (16 lanes) of the matrix core's result holds rows 4 g + b of a tile, b < 4; on the B side (PERM) that row of
// tile t is column 32 (t / 2) + 8 g + 4 (t % 2) + b of the wave's: a lane holds eight neighbours of a pair of tiles, and the four groups together 32, 64
// bytes of bf16, which a write to memory takes as one (with 32 or 64 neighbours in one lane, four times the writes: 7 % of a product of
// contraction 2048).
// Packets are permuted inside an LDS row so that the lanes of one access meet the banks evenly.
template <int MODE, int ES, int EXT, int PER, bool PERM, int WAVES>
struct Side {
  static constexpr int ROW = MODE == OP_K ? STEP_BYTES : EXT * ES;      // bytes of an LDS row
  static constexpr int PK = ROW / 16;                                   // its packets
  static constexpr int BYTES = EXT * STEP_BYTES;
  static constexpr int NJ = BYTES / 1024 / WAVES;                       // loads of a wave per stage
  static constexpr int READS = MODE == OP_K ? 1 : 2;                    // reads of LDS per operand
  static_assert(BYTES % (1024 * WAVES) == 0, "every wave issues the same number of loads");
  static constexpr int RPI = 64 / PK;                                   // LDS rows per load
  static __device__ __forceinline__ int swizzle(int row) {
    if (MODE == OP_K) return PERM ? ((row >> 1) & 1) | (((row >> 3) & 3) << 1) : (row >> 1) & 7;
    if (PERM) return PK == 8 ? (row & 2) << 1 : (row & 3) << 2;
    return (((row & 3) | (((row >> 3) & 1) << 2)) << 1) & (PK - 1);
  }
  // Load j of a wave begins at LDS row (wave + WAVES j) RPI: its lanes' packets are permuted like those of load j % NV
  static constexpr int NV = MODE == OP_T && !PERM && NJ > 1 ? 2 : 1;
  static_assert(WAVES == 4, "");
  int voff[NV], vcol[MODE == OP_K ? NV : 1];      // byte offset of the lane's packet from the load's corner; first element of it along the row
  int seg_row0;                                   // result rows before the workgroup's
  __device__ __forceinline__ void open(const Operand& o, int row0, int wave, int lane) {
    seg_row0 = row0;
#pragma unroll
    for (int j = 0; j < NV; j++) {
      const int r = (wave + WAVES * j) * RPI + lane / PK, c = (lane % PK) ^ swizzle(r);
      voff[j] = (lane / PK) * (int)o.ldb + c * 16;
      if (MODE == OP_K) vcol[j] = c * (16 / ES);
      else if (row0 + c * (16 / ES) >= o.cols) voff[j] = 0x7FFFFFF0;
    }
  }
  // Where the requests of a stage begin, kept from stage to stage so that a new one costs few scalar instructions: a wave has no time to spare
  // for them between two matrix instructions.  OP_K: the corner of the segment, the stage's k is in the offsets; OP_T: the stage's row.
  struct Stage { const char* cur; int num; __amdgpu_buffer_rsrc_t rs; int v[NV]; };
  __device__ __forceinline__ void place(const Operand& o, const char* p, int k, Stage& st) const {
    st.cur = p + (MODE == OP_K ? (int64_t)seg_row0 * o.ldb : (int64_t)k * o.ldb + (int64_t)seg_row0 * ES);
    if (MODE == OP_K) {      // bytes from there to the end of the operand
      const int64_t left = (int64_t)(o.rows - seg_row0 - 1) * o.ldb + (int64_t)o.cols * ES;
      st.num = seg_row0 >= o.rows ? 0 : (left > 0x7FFFFFF0 ? 0x7FFFFFF0 : (int)left);
    }
  }
  __device__ __forceinline__ void advance(const Operand& o, Stage& st) const {
    if (MODE == OP_T) st.cur += o.ldb * (STEP_BYTES / ES);
  }
  __device__ __forceinline__ void prepare(const Operand& o, int k, bool there, Stage& st) const {
    if (MODE == OP_T) {      // rows of the stage that exist; columns that do not have offsets past any end
      const int n = o.rows - k;
      st.num = n <= 0 ? 0 : (n >= STEP_BYTES / ES ? 0x7FFFFFF0 : (n - 1) * (int)o.ldb + (o.cols - seg_row0) * ES);
    }
    st.rs = __builtin_amdgcn_make_buffer_rsrc((void*)st.cur, 0, there ? st.num : 0, 0x00020000);      // (zeros if there is no such stage)
#pragma unroll
    for (int j = 0; j < NV; j++) st.v[j] = MODE == OP_T ? voff[j] : (k + vcol[MODE == OP_K ? j : 0] >= o.cols ? 0x7FFFFFF0 : voff[j] + k * ES);
  }
  __device__ __forceinline__ void load(const Operand& o, const Stage& st, int j, char* lds, int wave) const {
    const int i = wave + WAVES * j;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(st.rs, (lds_void*)(lds + i * 1024), 16, st.v[j % NV], i * RPI * (int)o.ldb, 0, 0);
  }
  // the wave's operands of a stage: tile t < PER, half `sub` of the contraction; wpos: the wave's place among those along this side
  int raddr[MODE == OP_K ? 2 : PER];
  __device__ __forceinline__ void open_read(int wpos, int lane) {
    const int i = lane & 15, g = lane >> 4, first = wpos * PER * 16;
    if (MODE == OP_K) {
      const int row = first + (PERM ? (i >> 2) * 8 + (i & 3) : i);
#pragma unroll
      for (int sub = 0; sub < 2; sub++) raddr[sub] = row * ROW + (((sub * 4 + g) ^ swizzle(row)) * 16);
    } else {
      // sixteen lanes read four rows k of four quads of neighbouring elements each and get a column of them
      const int k = g * 8 + (i >> 2), q = i & 3;      // the quad that this lane fetches
#pragma unroll
      for (int t = 0; t < PER; t++) {
        const int col = first + (PERM ? (t >> 1) * 32 + q * 8 + (t & 1) * 4 : t * 16 + q * 4);
        raddr[t] = k * ROW + (((col >> 3) ^ swizzle(k)) * 16) + ((col >> 2) & 1) * 8;
      }
    }
  }
  __device__ __forceinline__ v4i read(const char* lds, int t, int sub) const {
    if (MODE == OP_K) return *reinterpret_cast<const v4i*>(lds + raddr[MODE == OP_K ? sub : 0] + (PERM ? (t >> 1) * 32 + (t & 1) * 4 : t * 16) * ROW);
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
  int whole, parts;          // tiles from `whole` on have their stages dealt out in parts, a workgroup each
  void* sums;                // of those: [part][tile][matrix][row][column], 4 bytes each, for join_tiles()
};
// What workgroup b does: part `part` of `parts` of tile t, whose sums are the slot-th of all parts'
struct Share { int t, part, parts, slot; };
__device__ __forceinline__ Share share_of(int b, int tiles, int whole, int parts) {
  if (b < whole) return Share{b, 0, 1, 0};
  const int j = b - whole, rest = tiles - whole;
  return Share{whole + j % rest, j / rest, parts, j};
}
__device__ __forceinline__ void put_sums(float* p, const float (&v)[8]) { put_f32(p, v, 8); }
__device__ __forceinline__ void put_sums(int* p, const int (&v)[8]) {
  *reinterpret_cast<v4i*>(p) = v4i{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<v4i*>(p + 4) = v4i{v[4], v[5], v[6], v[7]};
}
// Adds the parts' sums [part][matrix][m][n] in order and goes on with them.  Epi::one(f) calls f(put) once, put(m, n, V (&v)[NB], N).
template <int NB, class V, class Epi>
__device__ __forceinline__ void join(const V* sums, int parts, int M, int N, const Epi& epi) {
  epi.one([&](auto put) {
    for (int64_t j = blockIdx.x * (int64_t)256 + threadIdx.x; j < (int64_t)M * N; j += (int64_t)gridDim.x * 256) {
      V v[NB];
#pragma unroll
      for (int z = 0; z < NB; z++) {
        V t = 0;
        for (int p = 0; p < parts; p++) t += sums[((int64_t)p * NB + z) * M * N + j];
        v[z] = t;
      }
      put((int)(j / N), (int)(j % N), v, N);
    }
  });
}
inline unsigned join_grid(int64_t M, int64_t N) {
  const int64_t n = (M * N + 255) / 256;
  return (unsigned)(n > 4096 ? 4096 : n);
}

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

// Epi::each(f) calls f(put) once, put(m, n, val (&v)[NB][8], N): eight neighbouring columns of row m from n on; n < N, but columns may pass N.
template <bool I8, int AM, int BMODE, class S, class Epi>
__device__ __forceinline__ void product_tile(const Product<S::NB>& q, const Epi& epi) {
  typedef Num<I8> T;
  constexpr int ES = T::ES, KS = STEP_BYTES / ES;
  typedef Side<AM, ES, S::BM, S::FM, false, S::WAVES> SA;
  typedef Side<BMODE, ES, S::BN, S::FN, true, S::WAVES> SB;
  // An array per stage: with one array the compiler waits before every read of LDS for all requests under way.
  __shared__ __align__(1024) char a0[SA::BYTES], a1[SA::BYTES], b0[S::NB][SB::BYTES], b1[S::NB][SB::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
  const int tiles_m = (q.M + S::BM - 1) / S::BM, tiles_n = (q.N + S::BN - 1) / S::BN;
  const Share share = share_of(blockIdx.x, tiles_m * tiles_n, q.whole, q.parts);
  int tm, tn;
  tile_of(share.t, tiles_m, tiles_n, tm, tn);
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
  const int parts = share.parts;
  const int per = (q.k + KS - 1) / KS, all = per * q.nseg, span = (all + parts - 1) / parts;      // stages of a segment, of all, of a part
  const int begin = min(all, share.part * span), total = min(all - begin, span);
  // Workgroups begin at stages of their own, so that rows whose distance is a power of two do not all ask one memory channel at a time (contraction 2048: 7 %;
  // int8, 14336: 5 %).
  const int k0 = per > 0 && parts == 1 ? (tm + tn) % per * KS : 0;
  int seg = per > 0 ? begin / per : 0, k = per > 0 && parts > 1 ? begin % per * KS : k0;      // of the stage that is prepared
  int left = total;                                                                             // stages from there on
  constexpr int NL = SA::NJ + S::NB * SB::NJ;      // loads of a wave per stage
  typename SA::Stage qa;
  typename SB::Stage qb[S::NB];
  auto place = [&]() {
    const int at = seg < q.nseg ? seg : 0;
    sa.place(q.a, q.a.p[at], k, qa);
#pragma unroll
    for (int z = 0; z < S::NB; z++) sb.place(q.b[0], q.b[z].p[at], k, qb[z]);
  };
  auto step = [&]() {      // to the next stage
    bool anew = false;
    left--;
    k += KS;
    if (k >= q.k) { k = 0; anew = true; }
    if (k == k0) { seg++; anew = true; }
    if (anew) { place(); return; }
    sa.advance(q.a, qa);
#pragma unroll
    for (int z = 0; z < S::NB; z++) sb.advance(q.b[0], qb[z]);
  };
  auto prepare = [&](int part) {      // 0: A, 1 + z: B
    if (part == 0) sa.prepare(q.a, k, left > 0, qa);
    else sb.prepare(q.b[0], k, left > 0, qb[part - 1]);
  };
  auto request = [&](int l, char* a, char (*b)[SB::BYTES]) {      // load l < NL of a stage
    if (l < SA::NJ) sa.load(q.a, qa, l, a, wave);
    else sb.load(q.b[0], qb[(l - SA::NJ) / SB::NJ], (l - SA::NJ) % SB::NJ, b[(l - SA::NJ) / SB::NJ], wave);
  };
  constexpr int NF = S::NB * S::FN + S::FM, NM = S::FM * S::NB * S::FN;      // operands and products of half a stage
  v4i fa[2][S::FM], fb[2][S::NB][S::FN];
  auto read = [&](int set, int l, const char* a, const char (*b)[SB::BYTES]) {      // operand l < NF of half `set` of a stage, into register set `set`
    if (l < S::NB * S::FN) fb[set][l / S::FN][l % S::FN] = sb.read(b[l / S::FN], l % S::FN, set);
    else fa[set][l - S::NB * S::FN] = sa.read(a, l - S::NB * S::FN, set);
  };
  // Half `set` is multiplied; meanwhile half 1 - set of (ra, rb) is read and, for set = 1, the stage prepared in qa, qb requested into (la, lb), evenly spread;
  // for set = 0 that stage is prepared.
  auto half = [&](int set, const char* ra, const char (*rb)[SB::BYTES], char* la, char (*lb)[SB::BYTES]) {
#pragma unroll
    for (int n = 0; n < NM; n++) {
#pragma unroll
      for (int l = n * NF / NM; l < (n + 1) * NF / NM; l++) read(1 - set, l, ra, rb);
      if (set == 1) {
#pragma unroll
        for (int l = n * NL / NM; l < (n + 1) * NL / NM; l++) request(l, la, lb);
      } else {
        if (n == NM / 8) step();
#pragma unroll
        for (int part = 0; part <= S::NB; part++)
          if (n == (part + 2) * NM / 8) prepare(part);
      }
      T::mma(fb[set][(n / S::FN) % S::NB][n % S::FN], fa[set][n / (S::NB * S::FN)], acc[n / (S::NB * S::FN)][(n / S::FN) % S::NB][n % S::FN]);      // rows of the result tile: columns n
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // The first half of a stage is in registers when its turn comes.  While it is multiplied the second half is read; then every wave has read all
  // of the stage, which the barrier establishes together with the arrival of the next one, its buffer takes the stage after that, and
  // the next stage's first half is read while the second half is multiplied.
#define OSSCAR_TILE_STAGE(a_, b_, an_, bn_) \
  half(0, a_, b_, nullptr, nullptr);        \
  wait_loads<0>();                          \
  stage_barrier();                          \
  half(1, an_, bn_, a_, b_);
  place();
#pragma unroll
  for (int part = 0; part <= S::NB; part++) prepare(part);
#pragma unroll
  for (int l = 0; l < NL; l++) request(l, a0, b0);
  step();
#pragma unroll
  for (int part = 0; part <= S::NB; part++) prepare(part);
#pragma unroll
  for (int l = 0; l < NL; l++) request(l, a1, b1);
  wait_loads<NL>();
  stage_barrier();
#pragma unroll
  for (int l = 0; l < NF; l++) read(0, l, a0, b0);
  for (int st = 0; st < total; st += 2) {      // (stages past the last one are zeros)
    OSSCAR_TILE_STAGE(a0, b0, a1, b1)
    OSSCAR_TILE_STAGE(a1, b1, a0, b0)
  }
#undef OSSCAR_TILE_STAGE
  sums_written();
  const int i = lane & 15, g = lane >> 4;
  auto each = [&](auto put) {
#pragma unroll
    for (int f = 0; f < S::FM; f++) {
      const int m = tm * S::BM + (wm * S::FM + f) * 16 + i;
#pragma unroll
      for (int t = 0; t < S::FN; t += 2) {
        const int n = tn * S::BN + wn * S::FN * 16 + t * 16 + g * 8;
#pragma unroll
        for (int z = 0; z < S::NB; z++) { settled(acc[f][z][t]); settled(acc[f][z][t + 1]); }
        typename T::val v[S::NB][8];
#pragma unroll
        for (int z = 0; z < S::NB; z++)
#pragma unroll
          for (int e = 0; e < 8; e++) v[z][e] = acc[f][z][t + e / 4][e % 4];
        if (m < q.M && n < q.N) put(m, n, v, q.N);
      }
    }
  };
  if (parts == 1) {
    epi.each(each);
  } else {
    typename T::val* sums = reinterpret_cast<typename T::val*>(q.sums) + (int64_t)share.slot * S::NB * S::BM * S::BN;
    each([&](int m, int n, const typename T::val (&v)[S::NB][8], int) {
#pragma unroll
      for (int z = 0; z < S::NB; z++) put_sums(sums + (z * S::BM + m - tm * S::BM) * S::BN + n - tn * S::BN, v[z]);
    });
  }
}

// Adds the sums of the tiles that were dealt out in parts and goes on with them, eight columns a thread: G groups of threads take the parts in turn, and their sums
// are added in order.  Where there are many parts one thread would wait for all of them one after the other (32 parts of five tiles 21 us, in four groups 4.8).
constexpr int JOIN_GROUPS_FROM = 8;      // parts
template <class S, class V, int G, class Epi>
__device__ __forceinline__ void join_tiles(const Product<S::NB>& q, const Epi& epi) {
  constexpr int L = 256 / G, PER = S::BM * S::BN / (8 * L);      // threads of a group; workgroups of a tile
  typedef V v4 __attribute__((ext_vector_type(4)));
  const int tiles_m = (q.M + S::BM - 1) / S::BM, tiles_n = (q.N + S::BN - 1) / S::BN, rest = tiles_m * tiles_n - q.whole;
  const int t = blockIdx.x / PER, group = threadIdx.x / L, mine = threadIdx.x % L, i = blockIdx.x % PER * L + mine, row = i / (S::BN / 8), col = i % (S::BN / 8) * 8;
  int tm, tn;
  tile_of(q.whole + t, tiles_m, tiles_n, tm, tn);
  const int m = tm * S::BM + row, n = tn * S::BN + col;
  const bool in = m < q.M && n < q.N;
  V v[S::NB][8];
#pragma unroll
  for (int z = 0; z < S::NB; z++)
#pragma unroll
    for (int e = 0; e < 8; e++) v[z][e] = 0;
  for (int p = group; p < q.parts && in; p += G) {
#pragma unroll
    for (int z = 0; z < S::NB; z++) {
      const v4* w = reinterpret_cast<const v4*>(reinterpret_cast<const V*>(q.sums) + (((int64_t)p * rest + t) * S::NB + z) * (S::BM * S::BN) + row * S::BN + col);
      const v4 a = w[0], b = w[1];
#pragma unroll
      for (int e = 0; e < 4; e++) { v[z][e] += a[e]; v[z][4 + e] += b[e]; }
    }
  }
  if constexpr (G > 1) {
    __shared__ V sh[G - 1][S::NB * 8][L];
    if (group > 0)
#pragma unroll
      for (int e = 0; e < S::NB * 8; e++) sh[group - 1][e][mine] = v[e / 8][e % 8];
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 0; g < G - 1; g++)
#pragma unroll
      for (int e = 0; e < S::NB * 8; e++) v[e / 8][e % 8] += sh[g][e][mine];
  }
  if (in) epi.each([&](auto put) { put(m, n, v, q.N); });
}

// How a product of `stages` stages is dealt out, one of `count` in a launch.  The chip takes 256 big tiles at a time or 512 small ones, a big one, four times a
// small one, in BIG times its time (8192 x 8192 x 8192 bf16: 1500 TFLOP/s and 1200).  Tiles past the last full 256 or 512 would keep part of the chip busy for
// as long as all: their stages are dealt out in parts of at least `least` (eight; float32, whose stages take three times as long, three), so many that they
// fill it once, twice or three times, where that makes up for the launch that adds the sums and their way through memory (as long as about `launch` stages, and
// `sums` for a chip full of tiles).  The shape that takes less time is taken.
constexpr double BIG = 1.6;
struct Plan { double time; int64_t whole, parts, blocks; };      // time: rounds of the chip
inline Plan plan(int64_t tiles, int64_t slots, int64_t stages, int64_t least, double alone, double launch, double sums) {
  const int64_t rest = tiles % slots;
  auto rounds = [&](int64_t n) { return n / slots + (2 * (n % slots) > slots ? 1 : n % slots > 0 ? alone : 0); };
  Plan best{rounds(tiles), tiles, 1, tiles};
  for (int r = 1; r <= 3 && rest > 0; r++) {
    int64_t p = r * slots / rest;
    if (p > stages / least) p = stages / least;
    if (p > 32) p = 32;
    if (p < 2) continue;
    const double time = tiles / slots + rounds(rest * p) / p + (launch + sums * rest * p / slots) / stages;
    if (time < best.time) best = Plan{time, tiles - rest, p, tiles - rest + rest * p};
  }
  return best;
}
enum Pick { SMALL, BIG_TILE, FLAT };
struct Deal { Pick pick; int whole, parts; unsigned blocks; size_t sums, join; };      // sums: bytes of a product's; join: workgroups that add them
template <class S>
Deal deal_of_plan(Pick pick, int64_t tiles, const Plan& p) {
  const int64_t rest = p.parts > 1 ? tiles - p.whole : 0, area = S::BM * S::BN;
  return Deal{pick, (int)p.whole, (int)p.parts, (unsigned)p.blocks, (size_t)(rest * p.parts * S::NB * area * 4), (size_t)(rest * (area / 2048) * (p.parts >= JOIN_GROUPS_FROM ? 4 : 1))};
}
template <class S> int64_t tiles_of(int64_t M, int64_t N) { return (M + S::BM - 1) / S::BM * ((N + S::BN - 1) / S::BN); }
template <class SB, class SS>
Deal deal(int64_t M, int64_t N, int64_t stages, int count) {
  const int64_t big = tiles_of<SB>(M, N), small = tiles_of<SS>(M, N);
  // (a small tile alone on its compute unit takes less time than one of two)
  const Plan s = plan(small, 512 / count, stages, 8, 0.75, 2, 15), b = plan(big, 256 / count, stages, 8, 1, 1.2, 18);
  return b.time * BIG <= s.time ? deal_of_plan<SB>(BIG_TILE, big, b) : deal_of_plan<SS>(SMALL, small, s);
}
// float32 (split.h): flat tiles, 64 rows instead of 128 and twice the columns, more of which are cut per product.  7168 x 14336, 64 rows 340 us in tiles of 128
// rows and 230 in flat ones, 150 rows 700 and 560; tiles of either count (100 rows) 335 and 375.
constexpr double FLAT_TIME = 1.1;
template <class SF, class SS>
Deal deal_split(int64_t M, int64_t N, int64_t stages, int count, bool flat_too) {
  const int64_t flat = tiles_of<SF>(M, N), small = tiles_of<SS>(M, N);
  const Plan s = plan(small, 512 / count, stages, 3, 0.75, 1, 2.5), f = plan(flat, 512 / count, stages, 3, 0.75, 1, 2.5);
  return flat_too && f.time * FLAT_TIME < s.time ? deal_of_plan<SF>(FLAT, flat, f) : deal_of_plan<SS>(SMALL, small, s);
}

}  // namespace tile
}  // namespace osscar
